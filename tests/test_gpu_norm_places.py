"""Outputs of the normalised rows and of their gradient that begin anywhere in memory, through the C entry points: rows of every class in the
middle of a word, all of them or every second one, and what lies between the rows left as it was."""
import pytest
import torch

from paper_2605_13907_amd import binding as B
from tests.test_gpu_norm import check_grad, check_norm, params, rows

pytestmark = pytest.mark.gpu

GUARD = 3.0


class Placed:
    """A context whose rows leave `offset` elements into a buffer, `gap` elements apart."""

    def __init__(self, ctx, offset, gap):
        self.ctx, self.offset, self.gap = ctx, offset, gap

    def out(self, n, width, dtype):
        pitch = width + self.gap
        flat = torch.full((self.offset + n * pitch + 16,), GUARD, dtype=dtype, device="cuda")
        return flat, flat[self.offset:self.offset + n * pitch].view(n, pitch)[:, :width], pitch

    def untouched(self, flat, view):
        view = view.clone(), view
        view[1].fill_(GUARD)
        assert (flat == GUARD).all()
        return view[0]

    def norm_rows(self, x, weight, bias, eps=1e-5, centered=True, valid=None):
        n, width = x.shape
        flat, y, pitch = self.out(n, width, x.dtype)
        mean, rstd = (torch.empty(n, device="cuda") for _ in range(2))
        at = lambda t: None if t is None else t.data_ptr()
        rc = self.ctx._lib.ais_norm_rows(self.ctx._h, x.data_ptr(), B._dtype_code(x), n, width, x.stride(0), at(valid), at(weight), at(bias),
                                         B._dtype_code(weight), eps, int(centered), y.data_ptr(), pitch, mean.data_ptr() if centered else None,
                                         rstd.data_ptr())
        assert rc == 0
        return self.untouched(flat, y), mean if centered else None, rstd

    def norm_rows_grad(self, dy, x, weight, mean, rstd, valid=None, want_bias=True):
        n, width = x.shape
        flat, dx, pitch = self.out(n, width, x.dtype)
        dw, db = (torch.empty(width, device="cuda") for _ in range(2))
        at = lambda t: None if t is None else t.data_ptr()
        rc = self.ctx._lib.ais_norm_rows_grad(self.ctx._h, dy.data_ptr(), B._dtype_code(dy), dy.stride(0), x.data_ptr(), B._dtype_code(x), n, width,
                                              x.stride(0), at(valid), at(weight), B._dtype_code(weight), at(mean), rstd.data_ptr(),
                                              dx.data_ptr(), pitch, dw.data_ptr(), db.data_ptr())
        assert rc == 0
        return self.untouched(flat, dx), dw, db


@pytest.fixture(scope="module")
def ctx():
    c = B.AisContext()
    yield c
    c.close()


@pytest.mark.parametrize("types", [(torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32), (torch.float32, torch.float32)])
@pytest.mark.parametrize("offset,gap", [(1, 0), (0, 1), (1, 1), (3, 8)])
@pytest.mark.parametrize("width", [1, 7, 64, 513, 1_100, 2_048, 2_237, 4_096, 8_192, 8_193, 16_385])
def test_places(ctx, width, offset, gap, types):
    n = 1_603 if width < 3_000 else 601
    placed = Placed(ctx, offset, gap)
    x, valid = rows(n, width, types[0], width), (torch.arange(n, device="cuda") % 5 != 3).to(torch.uint8)
    weight, bias = params(width, torch.float32)
    mean, rstd = check_norm(placed, x, weight, bias, True, valid)
    check_grad(placed, rows(n, width, types[1], width + 1), x, weight, mean, rstd, valid)
