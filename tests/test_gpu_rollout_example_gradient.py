"""The example's distillation steps along the gradient of the loss that it reports: the logits are a product with the quantised hidden
states, so those are what the gradient with respect to the weights holds."""
import numpy as np
import pytest
import torch

import oracle.rollout_oracle as O
from examples import mxfp4_rollout
from paper_2605_13907_amd import binding as B

pytestmark = pytest.mark.gpu


def test_the_step_is_the_gradient_of_the_reported_loss():
    ctx = B.AisContext()
    gen = torch.Generator(device="cuda").manual_seed(3)
    rows, vocab, width, top, rate = 60, 777, 96, 20, 0.25
    weight = (0.3 * torch.randn(vocab, width, generator=gen, device="cuda")).bfloat16()
    student = weight.float() + 0.05 * torch.randn(vocab, width, generator=gen, device="cuda")
    hidden = torch.randn(rows, width, generator=gen, device="cuda").bfloat16()
    valid = (torch.arange(rows, device="cuda") % 4 != 1).to(torch.uint8)
    before = student.clone()
    losses = mxfp4_rollout.distill(ctx, student, weight, hidden, valid, top, rate, 1)
    h4, w4 = ctx.mxfp4_quantize_rows(hidden), ctx.mxfp4_quantize_rows(before)
    z = ctx.mxfp4_logits(*h4, *w4).double().cpu().numpy()
    best = torch.topk(hidden.float() @ weight.float().T, top, dim=1)
    loss, _, dz = O.distill(z, best.indices.cpu().numpy(), best.values.double().cpu().numpy(), np.full(rows, 1.0 / rows),
                            valid=valid.cpu().numpy())
    assert losses[0] == pytest.approx(loss, rel=1e-5)
    want = dz.T @ O.mxfp4_values(*[t.cpu().numpy() for t in h4])
    got = (before - student).double().cpu().numpy() / rate
    # gradients of the logits are bf16 numbers, 2^-8 off at most and less than 2^-9 in the root mean square, each by itself; the step is
    # rounded to the weights' fp32
    assert np.linalg.norm(got - want) <= (2.0 ** -9 + 1e-4) * np.linalg.norm(want)
    ctx.close()
