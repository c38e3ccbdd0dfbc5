"""MXFP4 rows and the product of two such matrices on the GPU against the fp64 oracle.

Codes, scales and values are exact: equal to the last bit.  Logits: every product of two elements and their scales is exact in
fp32, so what is left is the fp32 sum of `width` terms, |error| <= width 2^-24 sum |a w| (any order), and the rounding of the
result, 2^-24 of it.  bf16 logits are the fp32 ones rounded to nearest even, to the last bit."""
import numpy as np
import pytest
import torch

import oracle.rollout_oracle as O
from paper_2605_13907_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = B.AisContext()
    yield c
    c.close()


def host(t):
    return t.float().cpu().numpy().astype(np.float64)


def check_quantize(ctx, x):
    codes, scales, values = ctx.mxfp4_quantize_rows(x, want_values=True)
    want_codes, want_scales, want_values = O.mxfp4_quantize(host(x))
    assert scales.stride(0) % 16 == 0 or scales.shape[0] == 1
    np.testing.assert_array_equal(scales.cpu().numpy(), want_scales)
    got, finite = codes.cpu().numpy(), np.repeat(want_scales != 255, 16, axis=1)
    np.testing.assert_array_equal(got[finite], want_codes[finite])
    np.testing.assert_array_equal(host(values), want_values)
    assert values.dtype == x.dtype and values.is_contiguous()
    again = ctx.mxfp4_quantize_rows(x)
    assert torch.equal(again[0], codes) and torch.equal(again[1], scales)
    return codes, scales


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,width", [(1, 1), (1, 7), (3, 31), (2, 32), (5, 33), (4, 64), (17, 100), (9, 1000), (3, 4096), (300, 40)])
def test_quantize_sizes(ctx, dtype, rows, width):
    gen = torch.Generator(device="cuda").manual_seed(rows * 10_000 + width)
    x = torch.randn(rows, width, generator=gen, device="cuda") * torch.exp(3 * torch.randn(rows, 1, generator=gen, device="cuda"))
    check_quantize(ctx, x.to(dtype))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_quantize_every_rounding(ctx, dtype):
    """Multiples of 1/32 up to 8 of either sign, at several scales: every midpoint and what lies beside it."""
    grid = torch.arange(-256, 257, device="cuda") / 32.0
    x = torch.zeros(513 * 4, 32, device="cuda")
    x[:, 5] = grid.repeat(4)
    x[:, 0] = 6.0                             # holds the block's scale at 1
    x *= torch.tensor([1.0, 2.0 ** 60, 2.0 ** -60, 2.0 ** -120], device="cuda").repeat_interleave(513).unsqueeze(1)
    check_quantize(ctx, x.to(dtype))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_quantize_extremes(ctx, dtype):
    x = torch.zeros(12, 64, device="cuda")
    x[0, 3] = float("nan")
    x[1, 40] = float("inf")
    x[2, 40] = -float("inf")
    x[3, :32] = 3.3e38
    x[4, 0], x[4, 1] = 1e-38, 1e-40           # the scale's lowest exponents, subnormal elements
    x[5, 0] = 2.0 ** -126
    x[6, 0], x[6, 1] = 2.0 ** -128, 2.0 ** -130
    x[7, 10] = -0.0
    x[8, 0], x[8, 1] = 2.0 ** -127, -(2.0 ** -129)
    x[9, 0], x[9, 31] = 2.0 ** -124, 2.0 ** -128
    x[10, 0], x[10, 1] = -1.0, -0.05          # rounds to -0
    x = x.to(dtype)
    codes, scales = check_quantize(ctx, x)
    assert scales[0, 0] == 255 and scales[0, 1] == 0 and scales[1, 1] == 255 and scales[2, 1] == 255


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("offset", [0, 1, 3, 8])
def test_quantize_strides_and_in_place(ctx, dtype, offset):
    gen = torch.Generator(device="cuda").manual_seed(offset)
    wide = torch.randn(7, 130, generator=gen, device="cuda").to(dtype)
    x = wide[:, offset:offset + 101]
    check_quantize(ctx, x)
    want = O.mxfp4_quantize(host(x))[2]
    lib = B._lib()
    codes = torch.empty(7, 64, dtype=torch.uint8, device="cuda")
    scales = torch.empty(7, 4, dtype=torch.uint8, device="cuda")
    keep = wide.clone()
    ctx._sync_stream()
    rc = lib.ais_mxfp4_quantize_rows(ctx._h, x.data_ptr(), B._dtype_code(x), 7, 101, 130, codes.data_ptr(), 64,
                                     scales.data_ptr(), 4, x.data_ptr(), 130)
    assert rc == 0
    np.testing.assert_array_equal(host(x), want)
    torch.cuda.synchronize()
    keep[:, offset:offset + 101] = x
    assert torch.equal(keep, wide)             # nothing beside the row's elements was written


def operand(rows, width, seed, dtype=torch.bfloat16):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(rows, width, generator=gen, device="cuda")
            * torch.exp(torch.randn(rows, 1, generator=gen, device="cuda"))).to(dtype)


def check_product(ctx, hidden, weight, dtype):
    got = ctx.mxfp4_logits(*hidden, *weight, dtype=torch.float32)
    h = O.mxfp4_values(hidden[0].cpu().numpy(), hidden[1].cpu().numpy())
    w = O.mxfp4_values(weight[0].cpu().numpy(), weight[1].cpu().numpy())
    want, size = h @ w.T, np.abs(h) @ np.abs(w).T
    bound = (h.shape[1] * 2.0 ** -24) * size + 2.0 ** -24 * np.abs(want) * 1.01
    assert got.dtype == torch.float32 and got.shape == want.shape
    assert (np.abs(host(got) - want) <= bound)[~np.isnan(want)].all()
    assert (np.isnan(host(got)) == np.isnan(want)).all()
    if dtype == torch.bfloat16:
        half = ctx.mxfp4_logits(*hidden, *weight)
        assert half.dtype == dtype
        assert torch.equal(torch.nan_to_num(half, nan=0.125), torch.nan_to_num(got.bfloat16(), nan=0.125))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,vocab,width", [
    (1, 1, 1), (1, 64, 32), (2, 17, 33), (16, 64, 512), (15, 63, 480), (17, 65, 544), (1, 1000, 4096), (33, 515, 100),
    (64, 256, 1024), (65, 300, 2000), (128, 257, 160), (129, 511, 1100), (200, 1030, 96), (256, 256, 256), (300, 777, 640),
    (513, 1025, 64), (31, 4097, 4096)])
def test_product_sizes(ctx, dtype, rows, vocab, width):
    hidden = ctx.mxfp4_quantize_rows(operand(rows, width, rows))
    weight = ctx.mxfp4_quantize_rows(operand(vocab, width, vocab + 1))
    check_product(ctx, hidden, weight, dtype)


@pytest.mark.parametrize("rows,vocab,width", [
    (5, 700, 2048), (20, 900, 2000), (20, 333, 2080), (13, 5003, 3100), (40, 500, 4096), (64, 1000, 3000), (16, 300, 5120),
    (30, 300, 6200), (32, 270, 8192), (9, 17, 8180), (33, 4100, 2100)])
def test_product_of_few_long_rows(ctx, rows, vocab, width):
    """Contractions of 64 to 256 blocks, whole and with a rest, that wavefronts share."""
    hidden = ctx.mxfp4_quantize_rows(operand(rows, width, rows))
    weight = ctx.mxfp4_quantize_rows(operand(vocab, width, vocab + 1))
    check_product(ctx, hidden, weight, torch.bfloat16)


@pytest.mark.parametrize("rows,vocab,width", [
    (65, 33_500, 40), (128, 40_001, 512), (200, 33_100, 70), (256, 33_281, 1024), (700, 30_000, 96), (1, 70_001, 33),
    (129, 66_000, 600), (300, 33_000, 1100), (40, 70_000, 800)])
def test_product_of_more_tiles_than_compute_units(ctx, rows, vocab, width):
    hidden = ctx.mxfp4_quantize_rows(operand(rows, width, rows))
    weight = ctx.mxfp4_quantize_rows(operand(vocab, width, vocab + 1))
    check_product(ctx, hidden, weight, torch.bfloat16)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,vocab,width", [(5, 333, 2048), (70, 333, 100), (90, 34_000, 40)])
@pytest.mark.parametrize("offset,beside", [(1, 0), (3, 2), (0, 5)])
def test_product_into_rows_that_begin_anywhere(ctx, dtype, rows, vocab, width, offset, beside):
    hidden = ctx.mxfp4_quantize_rows(operand(rows, width, rows))
    weight = ctx.mxfp4_quantize_rows(operand(vocab, width, vocab + 1))
    want = ctx.mxfp4_logits(*hidden, *weight, dtype=dtype)
    stride = vocab + beside
    room = torch.full((rows * stride + 16,), 7.0, device="cuda", dtype=dtype)
    out = room[offset:offset + rows * stride].view(rows, stride)
    ctx._sync_stream()
    rc = B._lib().ais_mxfp4_logits(ctx._h, hidden[0].data_ptr(), hidden[0].stride(0), hidden[1].data_ptr(), hidden[1].stride(0),
                                   rows, weight[0].data_ptr(), weight[0].stride(0), weight[1].data_ptr(), weight[1].stride(0),
                                   vocab, width, out.data_ptr(), B._dtype_code(out), stride)
    assert rc == 0
    torch.cuda.synchronize()
    assert torch.equal(out[:, :vocab], want)
    out[:, :vocab] = 7.0
    assert bool((room == 7.0).all())           # nothing beside the logits was written


@pytest.mark.parametrize("rows", [1, 20, 130])
def test_product_of_views(ctx, rows):
    """Rows of a larger matrix, every other row, and a column range of whole blocks."""
    hidden = ctx.mxfp4_quantize_rows(operand(2 * rows, 640, 1))
    weight = ctx.mxfp4_quantize_rows(operand(500, 640, 2))
    h = hidden[0][::2], hidden[1][::2]
    w = weight[0][77:330], weight[1][77:330]
    check_product(ctx, h, w, torch.float32)
    cut = [t[:, 4 * 16:13 * 16] if t.shape[1] > 100 else t[:, 4:13] for t in (*h, *w)]
    check_product(ctx, cut[:2], cut[2:], torch.bfloat16)


@pytest.mark.parametrize("rows", [3, 150])
def test_product_of_blocks_without_a_value(ctx, rows):
    x, y = operand(rows, 300, 5), operand(400, 300, 6)
    x[1, 37] = float("nan")
    y[200, 299] = float("inf")
    check_product(ctx, ctx.mxfp4_quantize_rows(x), ctx.mxfp4_quantize_rows(y), torch.float32)


@pytest.mark.parametrize("rows", [2, 140])
def test_product_of_extreme_scales(ctx, rows):
    x, y = operand(rows, 128, 7, torch.float32), operand(300, 128, 8, torch.float32)
    x[0] *= 2.0 ** 60
    x[1] *= 2.0 ** -60
    y[:100] *= 2.0 ** 50
    y[100:200] *= 2.0 ** -50
    y[200] = 0
    check_product(ctx, ctx.mxfp4_quantize_rows(x), ctx.mxfp4_quantize_rows(y), torch.float32)


def test_rows_alone_and_together(ctx):
    """A row's logits do not depend on how many rows are beside it by more than the order of its sum allows."""
    weight = ctx.mxfp4_quantize_rows(operand(1500, 960, 9))
    codes, scales = ctx.mxfp4_quantize_rows(operand(700, 960, 10))
    for dtype in (torch.float32, torch.bfloat16):
        for n in (1, 16, 40, 200, 700):
            check_product(ctx, (codes[:n], scales[:n]), weight, dtype)


def test_empty_and_own_stream(ctx):
    weight = ctx.mxfp4_quantize_rows(operand(50, 64, 1))
    none = ctx.mxfp4_quantize_rows(torch.empty(0, 64, device="cuda"))
    assert ctx.mxfp4_logits(*none, *weight).shape == (0, 50)
    side = torch.cuda.Stream()
    x = operand(8, 64, 3)
    want = ctx.mxfp4_logits(*ctx.mxfp4_quantize_rows(x), *weight)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = ctx.mxfp4_logits(*ctx.mxfp4_quantize_rows(x), *weight)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)


def test_recorded_into_a_graph(ctx):
    weight = ctx.mxfp4_quantize_rows(operand(3000, 512, 1))
    x = operand(24, 512, 2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        ctx.mxfp4_logits(*ctx.mxfp4_quantize_rows(x), *weight)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = ctx.mxfp4_logits(*ctx.mxfp4_quantize_rows(x), *weight)
    for seed in range(4):
        x.copy_(operand(24, 512, 20 + seed))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, ctx.mxfp4_logits(*ctx.mxfp4_quantize_rows(x), *weight))


def test_refusals(ctx):
    x = operand(4, 64, 1)
    codes, scales = ctx.mxfp4_quantize_rows(x)
    with pytest.raises(TypeError):
        ctx.mxfp4_quantize_rows(x.half())
    with pytest.raises(ValueError):
        ctx.mxfp4_quantize_rows(x.t())
    with pytest.raises(ValueError):
        ctx.mxfp4_quantize_rows(x.cpu())
    with pytest.raises(ValueError):
        ctx.mxfp4_logits(codes[:, :16], scales, codes, scales)
    with pytest.raises(ValueError):
        ctx.mxfp4_logits(codes, scales, codes[:, :16], scales[:, :1])
    with pytest.raises(ValueError):
        ctx.mxfp4_logits(codes.cpu(), scales, codes, scales)
    with pytest.raises(TypeError):
        ctx.mxfp4_logits(codes.int(), scales, codes, scales)
    with pytest.raises(TypeError):
        ctx.mxfp4_logits(codes, scales, codes, scales, dtype=torch.float16)
    shifted = torch.empty(4 * 32 + 1, dtype=torch.uint8, device="cuda")[1:].view(4, 32)
    with pytest.raises(B.AisError) as e:
        ctx.mxfp4_logits(shifted, scales, codes, scales)
    assert e.value.code == -4
    with pytest.raises(B.AisError) as e:
        ctx.mxfp4_logits(codes, scales.contiguous(), codes, scales)     # a row of scales does not begin at a word
    assert e.value.code == -4
