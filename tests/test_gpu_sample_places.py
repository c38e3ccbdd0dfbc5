"""Rows whose cut lies among values that the count of bf16 values does not tell apart (beyond 2^31 below zero, and within 2^-32 of
zero), with the bound on the candidates between them: what is collected is what was counted, not every token of the place."""
import pytest
import torch

from paper_2605_13907_amd import binding as B
from tests.test_gpu_sample import check

pytestmark = pytest.mark.gpu

ORDINARY = 2_500


@pytest.fixture(scope="module")
def ctx():
    c = B.AisContext()
    yield c
    c.close()


def row(vocab, upper, rest, centre, masked, dtype, seed):
    """ORDINARY tokens around `centre`, `masked` at `upper` and all others at `rest`, in any order; the indices of the former two."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    order = torch.randperm(vocab, generator=gen, device="cuda")
    z = torch.full((1, vocab), rest, device="cuda")
    z[0, order[:ORDINARY]] = centre + torch.randn(ORDINARY, generator=gen, device="cuda")
    at = order[ORDINARY:ORDINARY + masked].sort().values
    z[0, at] = upper
    e = torch.empty(1, vocab, device="cuda").exponential_(generator=gen)
    return z.to(dtype), e, at


# k lies between the threads' parts that hold an ordinary token (about 1,870 of 4,096) and those that hold one of either (2,730): the
# bound is looked for below the ordinary ones, and is right as soon as it has passed the upper value
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("masked", [2_000, 3_000])
@pytest.mark.parametrize("upper,rest", [(-1e30, None), (-3e9, -1e20), (-1e20, -1e30)])
def test_two_masks_far_below(ctx, dtype, masked, upper, rest):
    z, e, _ = row(151_936, upper, torch.finfo(dtype).min if rest is None else rest, 0.0, masked, dtype, 1)
    for limits in (dict(top_k=2_600), dict(top_k=2_600, top_p=0.9999), dict(top_k=2_600, min_p=1e-6), dict(top_k=2_510)):
        check(ctx, z, e, **limits)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("masked", [2_000, 3_000])
@pytest.mark.parametrize("upper,rest", [(1e-11, 0.0), (-1e-20, -1e-11), (1e-20, -1e-20), (0.0, -1e-30)])
def test_values_next_to_zero(ctx, dtype, masked, upper, rest):
    """The random numbers make up for 40 units of logit: the last kept token of the cut's value is drawn, not the first that is cut."""
    z, e, at = row(151_936, upper, rest, 40.0, masked, dtype, 2)
    for k in (2_600, 2_550, 2_699):
        last = int(at[k - ORDINARY - 1])
        noise = torch.where(z == z[0, last], torch.full_like(e, 1.2e-38), e)
        noise[0, at[:k - ORDINARY]] = 1.0
        noise[0, last] = 1e-37
        assert check(ctx, z, noise, top_k=k).tolist() == [last]
