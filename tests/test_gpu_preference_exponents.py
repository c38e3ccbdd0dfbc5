"""The log-probabilities that the preference loss adds up, whose exponents are formed with a scale that fp32 rounds: the error that every row
has from it, in the same direction, is taken out again.

Tolerances.  A reward over 512 rows less the same rows' sum in 64 bits, divided by 512, is the mean error of a log-probability.  60,000 of a row's
logits are 12 below the largest and have 60,000 e^-12 = 0.37 of its probability, or 0.44 with their spread.  What is left of errors that differ from term to term: an exponent's rounding of
2^-20, 4e-7 of a term on the average, is 7e-11 of 3e7 of them; a batch's sums, 16 times 2^-24, less.  What may be the same in many terms is the exponential's
own error, one step at most, 2^-23, a quarter of which is left on the average over exponents that are spread: 2^-25.  The largest logit's term is the
same in every row.  It is 1, exactly, where that logit is 0; elsewhere its exponent is what the largest one's own rounding leaves, and its term is off by
up to a step, 2^-23, times its share of at most 1 / 1.37 of the sum: 0.75 * 2^-23."""
import numpy as np
import pytest
import torch

from paper_2605_13907_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = B.AisContext()
    yield c
    c.close()


def exact_of(z, ids, inv_t):
    return torch.log_softmax(z.double() * float(np.float32(inv_t)), dim=1).gather(1, ids.long()[:, None])[:, 0]


@pytest.mark.parametrize("inv_t", [1.0, 0.9, 0.7, 1.3, 0.83, 1 / 0.6])
@pytest.mark.parametrize("shift", [0.0, 40.0, -300.0])
@pytest.mark.parametrize("vocab", [60_001, 60_008])
def test_no_row_is_off_in_the_same_direction(ctx, vocab, shift, inv_t):
    rows = 512
    gen = torch.Generator(device="cuda").manual_seed(1)
    z = -12.0 / inv_t + 0.5 * torch.randn(rows, vocab, generator=gen, device="cuda")
    z[:, 0] = 0.0
    z += shift
    ids = torch.ones(rows, dtype=torch.int32, device="cuda")
    exact = exact_of(z, ids, inv_t)
    ref = exact.float()
    cu = torch.tensor([0, rows, rows], device="cuda")
    p = B.default_preference_params(beta=1.0, inv_temperature=inv_t)
    reward = ctx.preference_loss_grad(z, ids, None, cu, ref, p, want_grad=False)[1][0].item()
    tol = 2.0 ** -25 + (0.75 * 2.0 ** -23 if shift else 0.0)
    assert abs(reward - float((exact - ref.double()).sum())) / rows <= tol


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("inv_t", [1.0, 0.7])
@pytest.mark.parametrize("vocab", [300, 4_096, 33_001])
def test_masked_logits(ctx, vocab, inv_t, dtype):
    """Infinite ones here and there, in whole stretches, and everywhere but at the token; lowest values of the type.  2^-20 of the others'
    share, as for rows without any, and 2^-24 of the log-prob."""
    rows = 24
    gen = torch.Generator(device="cuda").manual_seed(vocab)
    z = (3 * torch.randn(rows, vocab, generator=gen, device="cuda")).to(dtype)
    for r in range(0, 8):
        z[r, torch.rand(vocab, generator=gen, device="cuda") < 0.3] = -float("inf")
    for r in range(8, 12):
        z[r, : vocab * (r - 7) // 5] = -float("inf")
    z[12:14, torch.rand(vocab, generator=gen, device="cuda") < 0.5] = torch.finfo(dtype).min
    z[14] = -float("inf")
    z[15] = torch.finfo(dtype).min
    ids = torch.full((rows,), vocab - 1, dtype=torch.int32, device="cuda")
    z[:, -1] = 0.5
    exact = exact_of(z, ids, inv_t)
    cu = torch.tensor([0, rows // 2, rows], device="cuda")
    p = B.default_preference_params(inv_temperature=inv_t)
    loss, reward, logp, dz = ctx.preference_loss_grad(z, ids, None, cu, exact.float(), p)
    assert ((logp.double() - exact).abs() <= 2.0 ** -20 * -torch.expm1(exact) + 2.0 ** -24 * exact.abs()).all()
    assert torch.isfinite(loss).all() and torch.isfinite(reward).all() and torch.isfinite(dz).all()
    assert (dz[torch.isinf(z)] == 0).all()


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_what_is_not_finite_stays_in_its_row(ctx, bad):
    z = torch.randn(8, 5_000, device="cuda")
    ids = torch.zeros(8, dtype=torch.int32, device="cuda")
    cu = torch.tensor([0, 4, 8], device="cuda")
    want = ctx.preference_loss_grad(z, ids, None, cu, None)[2]
    z[3, 2_500] = bad
    got = ctx.preference_loss_grad(z, ids, None, cu, None)[2]
    keep = torch.arange(8, device="cuda") != 3
    assert torch.equal(got[keep], want[keep]) and not torch.isfinite(got[3])
