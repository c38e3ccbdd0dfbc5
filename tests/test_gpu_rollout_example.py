"""The example of a 4-bit rollout policy runs its operators together, at sizes that are no multiple of a tile (widths are one of 32, as
the gradient of the read-out wants them)."""
import numpy as np
import pytest
import torch

import oracle.rollout_oracle as O
from examples import mxfp4_rollout
from paper_2605_13907_amd import binding as B

pytestmark = pytest.mark.gpu


def test_iterations():
    out = mxfp4_rollout.main(["--vocab", "5003", "--width", "224", "--prompts", "3", "--length", "9", "--iterations", "2"])
    assert len(out) == 2
    for r in out:
        assert 0.0 <= r["alpha"] <= 1.0 and np.isfinite(r["loss"])
        assert r["n_valid"] == int(r["valid"].sum())
        assert len(r["kl"]) == 9 and r["kl"][-1] < 0.9 * r["kl"][0]
        ended = r["valid"] == 0
        assert not r["logp_roll"][ended].any() and bool((r["logp_roll"][~ended] < 0).all())


def test_log_probabilities_are_those_of_the_four_bit_policy():
    ctx = B.AisContext()
    gen = torch.Generator(device="cuda").manual_seed(1)
    weight = torch.randn(777, 96, generator=gen, device="cuda")
    embedding = torch.randn(777, 96, generator=gen, device="cuda").bfloat16()
    weight4 = ctx.mxfp4_quantize_rows(weight * 0.3)
    start = mxfp4_rollout.normalised(torch.randn(10, 96, generator=gen, device="cuda")).bfloat16()
    hidden, tokens, logp, valid = mxfp4_rollout.Rollouts(ctx, embedding, 7, gen).run(weight4, start)
    codes, scales = ctx.mxfp4_quantize_rows(hidden)
    # bf16 logits as the rollout had them: the policy is their softmax
    z = ctx.mxfp4_logits(codes, scales, *weight4).double().cpu().numpy()
    exact = O.mxfp4_values(codes.cpu().numpy(), scales.cpu().numpy()) @ O.mxfp4_values(*[t.cpu().numpy() for t in weight4]).T
    # fp32 sum of 96 terms, rounded to bf16's 8 bits
    assert (np.abs(z - exact) <= 2.0 ** -8 * np.abs(exact) + 1e-4).all()
    want = z - np.log(np.exp(z - z.max(axis=1, keepdims=True)).sum(axis=1, keepdims=True)) - z.max(axis=1, keepdims=True)
    ids = tokens.cpu().numpy()
    live = valid.cpu().numpy() != 0
    got = logp.double().cpu().numpy()
    # 2e-5: the operator's own bound at logits of this size
    assert np.abs(got - want[np.arange(ids.size), ids])[live].max() <= 2e-5
    ctx.close()
