"""How exactly the soft-max sums of long rows are taken, in rows that are read twice (wide ones with their gradient, any for the loss
alone).  u = 2^-24, an fp32 rounding."""
import math

import numpy as np
import pytest
import torch

import oracle.rollout_oracle as O
from paper_2605_13907_amd import binding as B

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.fixture(scope="module")
def ctx():
    c = B.AisContext()
    yield c
    c.close()


@pytest.mark.parametrize("dtype,vocab,want_grad", [(torch.float32, 300_000, True), (torch.bfloat16, 300_000, True),
                                                   (torch.float32, 140_000, False), (torch.bfloat16, 151_936, False),
                                                   (torch.bfloat16, 600_001, False)])
def test_many_small_terms_beside_a_large_one(ctx, dtype, vocab, want_grad):
    """Each of 256 threads has one term of 1 first and then some hundred of 2^-24.2, every one less than half a unit in the last place
    of a sum that holds the 1.  The list is one token: kl = log(256 + (vocab - 256) e^-16.75).  The terms of 1 are exact and the
    small ones' errors vanish beside them; each thread's sum is rounded (u), sums of two are added 8 times (8 u) and kl, of about
    5.55, is stored (4 u)."""
    z = torch.full((3, vocab), -16.75, dtype=dtype, device="cuda")
    per_vector = 8 if dtype == torch.bfloat16 else 4
    z[:, :256 * per_vector:per_vector] = 0.0
    ids = torch.zeros(3, 1, dtype=torch.int32, device="cuda")
    teacher = torch.zeros(3, 1, device="cuda")
    kl = ctx.distill_topk(z, ids, teacher, want_grad=want_grad)[1].double().cpu().numpy()
    assert np.abs(kl - math.log(256 + (vocab - 256) * math.exp(-16.75))).max() <= 13 * U


@pytest.mark.parametrize("dtype,vocab,want_grad", [(torch.float32, 150_001, True), (torch.float32, 260_000, True),
                                                   (torch.bfloat16, 280_000, True), (torch.bfloat16, 151_936, False),
                                                   (torch.float32, 50_257, False)])
def test_rows_whose_probabilities_fall_with_a_power_of_the_rank(ctx, dtype, vocab, want_grad):
    """Errors are independent from row to row: the exponents' (each term's own, they average out), the threads' sums (u / 2), their
    eight additions (u / 2 each), q's and the stored kl's, some u together.  Their root mean square is held to 8 u."""
    gen = torch.Generator(device="cuda").manual_seed(vocab)
    rows = 24
    z = torch.empty(rows, vocab, device="cuda").exponential_(generator=gen)
    z = (z * (1.2 + 1.8 * torch.rand(rows, 1, generator=gen, device="cuda")) - 6.0).to(dtype)
    top = torch.topk(z.float() + 0.5 * torch.randn(rows, vocab, generator=gen, device="cuda"), 20, dim=1)
    ids, teacher = top.indices.int(), top.values.contiguous()
    weight = torch.full((rows,), 1.0 / rows, device="cuda")
    loss, kl, _ = ctx.distill_topk(z, ids, teacher, weight, want_grad=want_grad)
    want_loss, want, _ = O.distill(z.double().cpu().numpy(), ids.cpu().numpy(), teacher.double().cpu().numpy(),
                                   weight.double().cpu().numpy())
    off = kl.double().cpu().numpy() - want
    assert math.sqrt((off ** 2).mean()) <= 8 * U, off / U
    assert abs(loss.item() - want_loss) <= 8 * U
