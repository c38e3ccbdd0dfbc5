"""Masked rows between live ones of the same workgroup, whose wavefronts meet at a live row's barrier alone: results are those of calls in
which no row is masked, to the bit."""
import pytest
import torch

from paper_2605_13907_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = B.AisContext()
    yield c
    c.close()


def batch(n, width, dtype, dy_dtype):
    gen = torch.Generator(device="cuda").manual_seed(width)
    randn = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    return randn(n, width).to(dtype), randn(n, width).to(dy_dtype), (1.0 + 0.1 * randn(width)).to(dtype), randn(width).to(dtype)


def masks(n):
    """Live, masked, live at the distances that workgroups' rows have (as many as compute units, and small multiples), and at every row."""
    units = torch.cuda.get_device_properties(0).multi_processor_count
    row = torch.arange(n, device="cuda")
    for apart in (1, units, 2 * units, 3 * units):
        for start in (0, 1):
            yield ((row // apart + start) % 2 == 0).to(torch.uint8)
    yield ((row // units) % 4 != 1).to(torch.uint8)
    yield ((row // units) % 4 == 0).to(torch.uint8)


TYPES = [(torch.bfloat16, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.float32, torch.float32), (torch.float32, torch.bfloat16)]


@pytest.mark.parametrize("centered", [True, False])
@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("width", [512, 1_500, 2_000, 2_237, 4_096, 5_120, 8_192, 8_200])
def test_gradient(ctx, width, types, centered):
    n = 1_533
    x, dy, weight, bias = batch(n, width, *types)
    _, mean, rstd = ctx.norm_rows(x, weight, bias, centered=centered)
    dx, _, _ = ctx.norm_rows_grad(dy, x, weight, mean, rstd)
    for valid in masks(n):
        live = valid != 0
        rest = torch.where(live[:, None], dy, torch.zeros_like(dy))
        _, dw, db = ctx.norm_rows_grad(rest, x, weight, mean, rstd)
        got = ctx.norm_rows_grad(dy, x, weight, mean, rstd, valid=valid)
        assert torch.equal(got[0], torch.where(live[:, None], dx, torch.zeros_like(dx)))
        assert torch.equal(got[1], dw) and torch.equal(got[2], db)


@pytest.mark.parametrize("centered", [True, False])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("width", [64, 2_237, 4_096, 16_384, 16_392])
def test_rows(ctx, width, dtype, centered):
    n = 3_001 if width < 10_000 else 2_100
    x, _, weight, bias = batch(n, width, dtype, dtype)
    want = ctx.norm_rows(x, weight, bias, centered=centered)
    for valid in masks(n):
        live = valid != 0
        for a, b in zip(ctx.norm_rows(x, weight, bias, centered=centered, valid=valid), want):
            if b is None:
                assert a is None
                continue
            assert torch.equal(a, torch.where(live.view(-1, *[1] * (b.dim() - 1)), b, torch.zeros_like(b)))
