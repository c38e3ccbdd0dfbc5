"""The preference loss through logits for callers that hold token_logprob's outputs: the same numbers to the bit as without them, rewards as
near to 64 bits, and the refusals of either array."""
import numpy as np
import pytest
import torch

from paper_2605_13907_amd import binding as B
from tests.test_gpu_native_calls import bad_forms, both, same  # noqa: F401 (both: a fixture)

pytestmark = pytest.mark.gpu


def inputs(rows=96, vocab=1_003, dtype=torch.float32, seed=5):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    z = (2 * torch.randn(rows, vocab, generator=gen, device="cuda")).to(dtype)
    ids = torch.randint(0, vocab, (rows,), generator=gen, device="cuda", dtype=torch.int32)
    valid = (torch.rand(rows, generator=gen, device="cuda") < 0.8).to(torch.uint8)
    cu = torch.tensor([0, rows // 3, rows // 2, rows // 2, rows], device="cuda")
    exact = torch.log_softmax(z.double(), dim=1).gather(1, ids.long()[:, None])[:, 0]
    ref = (exact + 0.1 * torch.randn(rows, generator=gen, device="cuda")).float()
    return z, ids, valid, cu, ref, torch.rand(2, generator=gen, device="cuda"), exact


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows", [1, 96, 1_500])
def test_the_same_numbers(both, rows, dtype):  # noqa: F811
    z, ids, valid, cu, ref, weight, _ = inputs(rows, dtype=dtype)
    for ctx in both:
        for mask in (valid, None):
            logp, lse = ctx.token_logprob(z, ids, mask)
            for p in (None, B.default_preference_params(kind=2, beta=0.5, mean_logp=1)):
                want = ctx.preference_loss_grad(z, ids, mask, cu, ref, p, weight=weight)
                got = ctx.preference_loss_grad(z, ids, mask, cu, logp, lse, ref, p, weight=weight)
                assert len(got) == 3
                same(got, (want[0], want[1], want[3]))
                same(ctx.preference_loss_grad(z, ids, mask, cu, logp, lse, ref, p, weight), got)
                same(ctx.preference_loss_grad(logits=z, token_ids=ids, valid=mask, cu_rows=cu, logp_train=logp, lse=lse, logp_ref=ref,
                                              params=p, weight=weight), got)
        same(ctx.preference_loss_grad(z, ids, None, cu, logp, lse, None), tuple(ctx.preference_loss_grad(z, ids, None, cu, None)[i] for i in (0, 1, 3)))
        over = z.clone()
        got = ctx.preference_loss_grad(over, ids, valid, cu, logp, lse, ref, dlogits=over)[2]
        assert got.data_ptr() == over.data_ptr()
        same(got, ctx.preference_loss_grad(z, ids, valid, cu, ref)[3])


def test_rewards_are_those_of_64_bits():
    """A row of a large and 60,000 small terms, all rows alike: what 32-bit sums of the terms lose does not average out over a response.
    15 log2(e) in fp32 is off by 2^-25 times 22 as the terms' common exponent, a term by 2^-23, a batch of 16 by 16 of 2^-25."""
    rows, vocab = 512, 60_001
    z = torch.full((rows, vocab), -15.0, device="cuda")
    z[:, 0] = 0.0
    ids = torch.ones(rows, dtype=torch.int32, device="cuda")
    exact = torch.log_softmax(z[:1].double(), dim=1)[0, 1].item()
    ref = torch.full((rows,), float(np.float32(exact)), device="cuda")
    cu = torch.tensor([0, rows, rows], device="cuda")
    ctx = B.AisContext()
    logp, lse = ctx.token_logprob(z, ids)
    reward = ctx.preference_loss_grad(z, ids, None, cu, logp, lse, ref, B.default_preference_params(beta=1.0))[1]
    share = 60_000 * np.exp(-15.0) / (1 + 60_000 * np.exp(-15.0))
    assert abs(reward[0].item() - rows * (exact - float(np.float32(exact)))) <= rows * (share * (22 + 4 + 16) * 2.0 ** -25 + 15 * 2.0 ** -50)


def test_refusals(both):  # noqa: F811
    z, ids, valid, cu, ref, weight, _ = inputs(8, 70)
    for ctx in both:
        logp, lse = ctx.token_logprob(z, ids, valid)
        args = dict(logits=z, token_ids=ids, valid=valid, cu_rows=cu, logp_train=logp, lse=lse, logp_ref=ref)
        for name in ("logp_train", "lse"):
            for wrong in (*bad_forms(args[name]), None):
                with pytest.raises((TypeError, ValueError), match=name):
                    ctx.preference_loss_grad(**{**args, name: wrong})
        for name in ("logits", "token_ids", "valid", "logp_ref"):
            for wrong in bad_forms(args[name]):
                with pytest.raises((TypeError, ValueError)):
                    ctx.preference_loss_grad(**{**args, name: wrong})
        with pytest.raises(TypeError):
            ctx.preference_loss_grad(z, ids, valid, cu, logp, lse)           # no reference: it is given as None
        with pytest.raises(TypeError):
            ctx.preference_loss_grad(**args, want_grad=False)
        with pytest.raises(B.AisError):
            ctx.preference_loss_grad(**args, params=B.default_preference_params(beta=-1.0))


def test_recorded():
    z, ids, valid, cu, ref, weight, _ = inputs(700, 1_501)
    ctx = B.AisContext()
    step = lambda: ctx.preference_loss_grad(z, ids, valid, cu, *ctx.token_logprob(z, ids, valid), ref, weight=weight)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for k in range(3):
        z.copy_(inputs(700, 1_501, seed=20 + k)[0])
        graph.replay()
        torch.cuda.synchronize()
        same(out, step())
