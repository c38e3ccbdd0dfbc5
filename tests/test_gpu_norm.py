"""Normalised rows and their gradient against their 64-bit forms: widths around every class of rows, types, strides, rows that begin
anywhere, masks.

Tolerances, in units of u = 2^-24.  A sum over a row goes through at most `depth` additions one after the other: a lane's groups of
eight (3 and the number of groups), the wavefront (6), its workgroup (16).  The mean is off by (depth + 2) u mean |x|, a deviation by that and
u of itself, the mean square by (depth + 3) u of itself, so the reciprocal deviation by half of that and 4 u; each product and the last rounding add u,
the type's rounding half of its step."""
import numpy as np
import pytest
import torch

import oracle.training_oracle as O
from paper_2605_13907_amd import binding as B

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}          # eps / 2
WIDTHS = [1, 2, 7, 8, 9, 63, 64, 255, 256, 257, 511, 512, 513, 767, 769, 1_023, 1_024, 1_025, 1_100, 1_280, 1_281, 1_536, 1_537, 2_047, 2_048,
          2_049, 4_095, 4_096, 4_097, 5_120, 5_123, 6_143, 6_145, 8_191, 8_192, 8_193, 10_240, 10_243, 12_288, 12_290, 16_384, 16_385, 32_768,
          32_769, 70_001]


@pytest.fixture(scope="module")
def ctx():
    c = B.AisContext()
    yield c
    c.close()


def depth(width):
    return 3 + -(-width // (8 * 64)) + 6 + 16


def rows(n, width, dtype, seed, offset=0, pitch=None):
    """[n, width] that begins `offset` elements into a buffer and has its own pitch."""
    pitch = pitch or width
    gen = torch.Generator(device="cuda").manual_seed(seed)
    flat = torch.full((offset + n * pitch + 8,), float("nan"), dtype=dtype, device="cuda")
    x = flat[offset:offset + n * pitch].view(n, pitch)[:, :width] if n else flat[:0].view(0, width)
    x.copy_(torch.randn(n, width, generator=gen, device="cuda") * torch.exp(torch.randn(n, 1, generator=gen, device="cuda")) + 0.3)
    return x


def numbers(t):
    return None if t is None else t.double().cpu().numpy()


def check_norm(ctx, x, weight, bias, centered, valid=None, eps=1e-5):
    y, mean, rstd = ctx.norm_rows(x, weight, bias, eps=eps, centered=centered, valid=valid)
    assert y.shape == x.shape and y.dtype == x.dtype and (mean is None) == (not centered)
    live = np.ones(len(x), bool) if valid is None else numbers(valid) != 0
    a, w, b = np.where(live[:, None], numbers(x), 0.0), numbers(weight), numbers(bias)
    want, want_mean, want_rstd = O.norm(a, w, b, float(np.float32(eps)), centered, live)
    d = depth(x.shape[1])
    size = np.abs(a).mean(axis=1)
    off = (d + 2) * U * size if centered else 0 * size
    # a deviation's error e adds e^2 to the mean square, and to its own part of the sum 2 |deviation| e, which the deviations' zero sum cancels but for e u
    loose = ((d + 3) / 2 + 6) * U + (off * want_rstd) ** 2
    assert (np.abs(numbers(rstd) - want_rstd) <= want_rstd * loose).all()
    if centered:
        assert (np.abs(numbers(mean) - np.where(live, want_mean, 0.0)) <= off + 1e-45).all()
    scale = 1.0 if w is None else np.abs(w)
    rest = np.abs(a - (want_mean[:, None] if centered else 0.0))
    tol = scale * want_rstd[:, None] * (rest * (loose[:, None] + 4 * U) + off[:, None]) + U * np.abs(want) + (0.0 if b is None else np.abs(b) * U)
    tol = tol * (1 + HALF[x.dtype]) + HALF[x.dtype] * np.abs(want) + 2.0 ** -133
    assert (np.abs(numbers(y) - want) <= tol).all()
    assert (numbers(y)[~live] == 0).all() and (numbers(rstd)[~live] == 0).all()
    return mean, rstd


def check_grad(ctx, dy, x, weight, mean, rstd, valid=None, want_bias=True):
    dx, dw, db = ctx.norm_rows_grad(dy, x, weight, mean, rstd, valid=valid, want_bias=want_bias)
    assert dx.shape == x.shape and dx.dtype == x.dtype and (dw is None) == (weight is None) and (db is None) == (not want_bias)
    live = np.ones(len(x), bool) if valid is None else numbers(valid) != 0
    a, g, w = np.where(live[:, None], numbers(x), 0.0), np.where(live[:, None], numbers(dy), 0.0), numbers(weight)
    want, want_w, want_b = O.norm_grad(g, a, w, numbers(mean), numbers(rstd), live)
    rs = np.where(live, numbers(rstd), 0.0)[:, None]
    n = np.abs((a - (0.0 if mean is None else np.where(live, numbers(mean), 0.0)[:, None])) * rs)
    u = np.abs(g * (1.0 if w is None else w))
    d = depth(x.shape[1])
    tol = rs * (4 * U * u + n * (u * n).mean(axis=1, keepdims=True) * (d + 10) * U + (u.mean(axis=1, keepdims=True) * (d + 6) * U))
    tol = tol * (1 + HALF[x.dtype]) + HALF[x.dtype] * np.abs(want) + 2.0 ** -133
    assert (np.abs(numbers(dx) - want) <= tol).all()
    assert (numbers(dx)[~live] == 0).all()
    # a column's sum: at most as many additions as there are rows, and those of the partials
    k = len(x) + 40
    if dw is not None:
        assert (np.abs(numbers(dw) - want_w) <= (k + 3) * U * (np.abs(g) * n).sum(axis=0) + 1e-45).all()
    if db is not None:
        assert (np.abs(numbers(db) - want_b) <= k * U * np.abs(g).sum(axis=0) + 1e-45).all()
    return dx, dw, db


def params(width, dtype, seed=5):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return ((1.0 + 0.2 * torch.randn(width, generator=gen, device="cuda")).to(dtype), torch.randn(width, generator=gen, device="cuda").to(dtype))


@pytest.mark.parametrize("centered", [True, False])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("width", WIDTHS)
def test_widths(ctx, width, dtype, centered):
    x = rows(5, width, dtype, width)
    weight, bias = params(width, dtype)
    mean, rstd = check_norm(ctx, x, weight, bias, centered)
    for dy_dtype in (torch.bfloat16, torch.float32):
        check_grad(ctx, rows(5, width, dy_dtype, width + 1), x, weight, mean, rstd)


@pytest.mark.parametrize("n", [0, 1, 2, 255, 257, 1_030, 3_001])
@pytest.mark.parametrize("width", [40, 1_100, 4_096])
def test_numbers_of_rows(ctx, n, width):
    x = rows(n, width, torch.bfloat16, n)
    weight, bias = params(width, torch.float32)
    mean, rstd = check_norm(ctx, x, weight, bias, True)
    check_grad(ctx, rows(n, width, torch.float32, n + 1), x, weight, mean, rstd)


@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("width", [1_601, 2_048, 2_049, 2_237, 3_001, 3_500, 5_001, 7_001, 8_192, 8_193])
def test_several_rows_to_a_workgroup(ctx, width, dtype, offset):
    """Rows of one workgroup that begin at a whole word and in the middle of one, and masked ones among them."""
    n = 1_603
    x, valid = rows(n, width, torch.bfloat16, width, offset), (torch.arange(n, device="cuda") % 7 != 3).to(torch.uint8)
    weight, bias = params(width, torch.float32)
    mean, rstd = check_norm(ctx, x, weight, bias, True, valid)
    check_grad(ctx, rows(n, width, dtype, width + 1, offset), x, weight, mean, rstd, valid)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("width", [5, 100, 1_101, 4_096, 20_001, 40_003])
def test_rows_that_begin_anywhere(ctx, width, dtype):
    for offset, extra in ((1, 0), (3, 5), (0, 1)):
        x = rows(4, width, dtype, 3, offset, width + extra)
        weight = rows(1, width, dtype, 4, offset)[0]
        bias = rows(1, width, dtype, 6, offset + 1)[0]
        mean, rstd = check_norm(ctx, x, weight, bias, True)
        check_grad(ctx, rows(4, width, torch.float32, 5, offset, width + extra), x, weight, mean, rstd)


@pytest.mark.parametrize("width", [64, 1_100, 4_096, 20_000, 40_000])
@pytest.mark.parametrize("live", [0.0, 0.3])
def test_masked_rows_are_not_looked_at(ctx, width, live):
    n = 60
    x, dy = rows(n, width, torch.bfloat16, 1), rows(n, width, torch.float32, 2)
    valid = (torch.rand(n, generator=torch.Generator().manual_seed(1)) < live).to(torch.uint8).cuda()
    x[valid == 0], dy[valid == 0] = float("nan"), float("inf")
    weight, bias = params(width, torch.bfloat16)
    for centered in (True, False):
        mean, rstd = check_norm(ctx, x, weight, bias, centered, valid)
        check_grad(ctx, dy, x, weight, mean, rstd, valid)


@pytest.mark.parametrize("width", [7, 1_100, 40_000])
def test_without_weight_or_bias(ctx, width):
    x, dy = rows(9, width, torch.float32, 1), rows(9, width, torch.float32, 2)
    for weight, bias in ((None, None), (params(width, torch.bfloat16)[0], None), (None, params(width, torch.bfloat16)[1])):
        mean, rstd = check_norm(ctx, x, weight, bias, True)
        check_grad(ctx, dy, x, weight, mean, rstd, want_bias=bias is not None)


def test_far_from_zero(ctx):
    """Rows whose mean is a thousand deviations: the variance is of deviations, not a difference of squares."""
    x = rows(8, 1_100, torch.float32, 1) * 0.01 + 10.0
    check_norm(ctx, x, None, None, True)


def test_a_constant_row_is_all_bias(ctx):
    x = torch.full((3, 100), 2.5, device="cuda")
    bias = torch.arange(100, device="cuda", dtype=torch.float32)
    y, mean, rstd = ctx.norm_rows(x, None, bias, eps=1e-5)
    assert torch.equal(y, bias.expand(3, 100)) and (mean == 2.5).all()
    assert torch.allclose(rstd, torch.full_like(rstd, 1e-5 ** -0.5), rtol=4 * U)


@pytest.mark.parametrize("width", [64, 1_100, 40_000])
def test_what_is_not_finite_stays_in_its_row(ctx, width):
    x = rows(6, width, torch.float32, 1)
    want, _, _ = ctx.norm_rows(x)
    x[2, width // 2], x[4, 0] = float("nan"), float("inf")
    y, _, _ = ctx.norm_rows(x)
    keep = [0, 1, 3, 5]
    assert torch.equal(y[keep], want[keep]) and torch.isnan(y[2]).all() and torch.isnan(y[4]).any()


@pytest.mark.parametrize("width", [64, 1_100, 4_096, 40_000])
def test_in_place(ctx, width):
    """Through the C entry points: y over x, dx over dy or over x."""
    x, dy = rows(6, width, torch.float32, 1), rows(6, width, torch.float32, 2)
    weight, bias = params(width, torch.float32)
    y, mean, rstd = ctx.norm_rows(x, weight, bias)
    dx, dw, db = ctx.norm_rows_grad(dy, x, weight, mean, rstd)
    lib, h = ctx._lib, ctx._h
    for target in ("dy", "x"):
        a, b = x.clone(), dy.clone()
        out = b if target == "dy" else a
        dw2 = torch.empty_like(dw)
        rc = lib.ais_norm_rows_grad(h, b.data_ptr(), B.AIS_F32, width, a.data_ptr(), B.AIS_F32, 6, width, width, None, weight.data_ptr(),
                                    B.AIS_F32, mean.data_ptr(), rstd.data_ptr(), out.data_ptr(), width, dw2.data_ptr(), None)
        assert rc == 0 and torch.equal(out, dx) and torch.equal(dw2, dw)
    a = x.clone()
    rc = lib.ais_norm_rows(h, a.data_ptr(), B.AIS_F32, 6, width, width, None, weight.data_ptr(), bias.data_ptr(), B.AIS_F32, 1e-5, 1, a.data_ptr(),
                           width, mean.data_ptr(), rstd.data_ptr())
    assert rc == 0 and torch.equal(a, y)


def test_columns_behind_the_rows_stay(ctx):
    x = rows(5, 100, torch.float32, 1, 0, 104)
    out = torch.full((5, 104), 7.0, device="cuda")
    rstd = torch.empty(5, device="cuda")
    rc = ctx._lib.ais_norm_rows(ctx._h, x.data_ptr(), B.AIS_F32, 5, 100, 104, None, None, None, B.AIS_F32, 1e-5, 0, out.data_ptr(), 104, None,
                                rstd.data_ptr())
    assert rc == 0 and (out[:, 100:] == 7.0).all() and torch.equal(out[:, :100], ctx.norm_rows(x, centered=False)[0])


@pytest.mark.parametrize("width", [100, 4_097, 20_000])
def test_offsets_beyond_32_bits(ctx, width):
    """Rows 2^29 + 1 elements apart, the last of them beyond 2^32 elements into its buffer: the same as rows beside one another."""
    n, pitch = 9, (1 << 29) + 1
    flat = torch.empty((n - 1) * pitch + width, dtype=torch.bfloat16, device="cuda")
    far = flat.as_strided((n, width), (pitch, 1))
    x, dy = rows(n, width, torch.bfloat16, 1), rows(n, width, torch.float32, 2)
    far.copy_(x)
    weight, bias = params(width, torch.bfloat16)
    want = ctx.norm_rows(x, weight, bias)
    for a, b in zip(want, ctx.norm_rows(far, weight, bias)):
        assert torch.equal(a, b)
    for a, b in zip(ctx.norm_rows_grad(dy, x, weight, *want[1:]), ctx.norm_rows_grad(dy, far, weight, *want[1:])):
        assert torch.equal(a, b)


def test_runs_alike(ctx):
    x, dy = rows(3_000, 1_100, torch.bfloat16, 1), rows(3_000, 1_100, torch.float32, 2)
    weight, _ = params(1_100, torch.bfloat16)
    _, mean, rstd = ctx.norm_rows(x, weight)
    first = ctx.norm_rows_grad(dy, x, weight, mean, rstd)
    for _ in range(5):
        for a, b in zip(first, ctx.norm_rows_grad(dy, x, weight, mean, rstd)):
            assert torch.equal(a, b)
