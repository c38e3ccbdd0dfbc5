"""Lists of a teacher's logits that are padded or far from zero: a finite mask counts as what it is, next to other logits (nothing) and
alone (all alike).  Bounds as test_gpu_distill.py states them: 2e-6 of the terms of kl and loss, which are at most 60 + |kl|; 1e-5
of weight inv_temperature (p + q) for the gradient and half a unit in the last place of its type (2^-8, 2^-23)."""
import math

import numpy as np
import pytest
import torch

import oracle.rollout_oracle as O
from paper_2605_13907_amd import binding as B
from tests.test_gpu_distill import case

pytestmark = pytest.mark.gpu

MASKS = [-1e10, -1e20, -1e30, torch.finfo(torch.bfloat16).min, torch.finfo(torch.float32).min]


@pytest.fixture(scope="module")
def ctx():
    c = B.AisContext()
    yield c
    c.close()


def check(ctx, z, ids, teacher, weight, inv_t=1.0, want_grad=True):
    loss, kl, grad = ctx.distill_topk(z, ids, teacher, weight, inv_temperature=inv_t, want_grad=want_grad)
    w, idn = weight.double().cpu().numpy(), ids.cpu().numpy()
    want_loss, want_kl, want = O.distill(z.double().cpu().numpy(), idn, teacher.double().cpu().numpy(), w, inv_t)
    assert np.isfinite(want_kl).all() and np.isfinite(want).all()
    size = 60.0 + np.abs(want_kl)
    off = np.abs(kl.double().cpu().numpy() - want_kl)
    assert (off <= 2e-6 * size).all(), off
    assert abs(loss.item() - want_loss) <= 2e-6 * (w * size).sum()
    if not want_grad:
        assert grad is None
        return
    p_and_q = want.copy()                      # want = weight inv_temperature (p - q)
    for r in range(z.shape[0]):
        t = teacher[r].double().cpu().numpy()
        if np.isneginf(t).all():               # no entry counts: loss and gradient are 0
            continue
        q = np.exp((t - t.max()) * inv_t)
        np.add.at(p_and_q[r], idn[r], 2.0 * w[r] * inv_t * q / q.sum())
    bound = 1e-5 * p_and_q + (2.0 ** -8 if z.dtype == torch.bfloat16 else 2.0 ** -23) * np.abs(want) + 2.0 ** -126
    off = np.abs(grad.double().cpu().numpy() - want)
    assert (off <= bound).all(), [(r, off[r].max()) for r in range(z.shape[0]) if (off[r] > bound[r]).any()]


def padded(vocab, top, dtype, mask):
    z, ids, teacher, weight = case(9, vocab, top, dtype, vocab + top)
    teacher[0, 1:] = mask                     # one logit, the others padding
    teacher[1, (top + 1) // 2:] = mask
    teacher[2] = mask                         # nothing but padding
    teacher[3, ::2] = mask
    teacher[4] = mask
    teacher[4, 0] = -math.inf
    teacher[5] = -mask                        # as far above zero
    teacher[6, top // 2] = -mask
    teacher[7, :top - 1] = mask
    ids[7, :top - 1] = ids[7, 0].item()       # padded with one and the same token
    return z, ids, teacher, weight


# rows of one wavefront, of several, of a compute unit and of those that are read twice; lists shorter and longer than its threads
@pytest.mark.parametrize("mask", MASKS)
@pytest.mark.parametrize("inv_t", [0.001, 0.3, 0.5, 1.0, 2.0])
@pytest.mark.parametrize("dtype,vocab,top", [(torch.bfloat16, 1000, 64), (torch.float32, 1000, 200), (torch.float32, 40, 1),
                                             (torch.bfloat16, 9001, 33), (torch.bfloat16, 152_000, 64), (torch.float32, 152_000, 700)])
def test_finite_masks(ctx, dtype, vocab, top, inv_t, mask):
    z, ids, teacher, weight = padded(vocab, top, dtype, mask)
    check(ctx, z, ids, teacher, weight, inv_t=inv_t)
    check(ctx, z, ids, teacher, weight, inv_t=inv_t, want_grad=False)


@pytest.mark.parametrize("mask", MASKS)
def test_the_longest_lists(ctx, mask):
    z, ids, teacher, weight = padded(2050, 1024, torch.float32, mask)
    check(ctx, z, ids, teacher, weight)
    check(ctx, z, ids, teacher, weight, inv_t=0.25)


@pytest.mark.parametrize("offset", [1e4, -1e6, 1e8, -1e10, 1e20])
def test_lists_far_from_zero(ctx, offset):
    """Logits relative to each other decide, as far as they are told apart there."""
    z, ids, teacher, weight = case(6, 5000, 40, torch.float32, 3)
    teacher = teacher * max(1.0, abs(offset) * 2.0 ** -22) + offset
    for inv_t in (1.0, 0.3, 1e-4):
        check(ctx, z, ids, teacher, weight, inv_t=inv_t)
