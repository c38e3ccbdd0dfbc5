"""The operators of a training step as they are used together: normalised hidden states, the read-out without logits, the preference
loss, the gradients back through both, the step of the weights; against automatic differentiation in 64 bits, on streams, and
recorded."""
import numpy as np
import pytest
import torch

from paper_2605_13907_amd import binding as B

pytestmark = pytest.mark.gpu

ROWS, WIDTH, VOCAB = 300, 128, 1_000
P = dict(beta=0.5)


class Model:
    def __init__(self, bits, seed=0, step=0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        randn = lambda *s: torch.randn(*s, generator=gen, device="cuda")
        self.head, self.scale = 0.3 * randn(VOCAB, WIDTH), 1.0 + 0.1 * randn(WIDTH)
        self.copies = [self.head.bfloat16(), self.scale.bfloat16()]
        self.opt = B.AdamWState([self.head, self.scale], bits=bits, copies=self.copies, seed=7, step=step)


class Data:
    def __init__(self, seed=1):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.x = (2 * torch.randn(ROWS, WIDTH, generator=gen, device="cuda")).bfloat16()
        self.tokens = torch.randint(0, VOCAB, (ROWS,), generator=gen, device="cuda", dtype=torch.int32)
        self.valid = (torch.rand(ROWS, generator=gen, device="cuda") < 0.8).to(torch.uint8)
        self.cu = torch.tensor([0, 60, 130, 130, 200, 260, 300], device="cuda")
        self.ref = -7.0 + 0.2 * torch.randn(ROWS, generator=gen, device="cuda")


def train(ctx, model, d, lr=1e-2):
    head, scale = model.copies
    y, _, rstd = ctx.norm_rows(d.x, scale, centered=False, valid=d.valid)
    logp, lse = ctx.lm_head_logprob(y, head, d.tokens, d.valid)
    loss, reward, g = ctx.preference_row_scale(logp, d.ref, d.valid, d.cu, B.default_preference_params(**P))
    dy, dhead = ctx.lm_head_grad(y, head, d.tokens, lse, logp, g)
    dx, dscale, _ = ctx.norm_rows_grad(dy, d.x, scale, None, rstd, d.valid, want_bias=False)
    ctx.adamw_step(model.opt, [dhead, dscale], lr=lr)
    return dict(loss=loss, reward=reward, y=y, dx=dx, dhead=dhead, dscale=dscale)


def near(got, want, share):
    got, want = got.double().cpu(), want.double().cpu()
    assert (got - want).norm() <= share * want.norm(), float((got - want).norm() / want.norm())


def test_against_automatic_differentiation():
    """The read-out forms dlogits in bf16, off by 2^-9 of themselves in the root mean square at most, each by itself; dx is rounded to bf16
    once more.  Rounded hidden states are taken as they are, with the gradient of what they were rounded from."""
    ctx, model, d = B.AisContext(), Model(32), Data()
    head, scale = (c.double().cpu().requires_grad_() for c in model.copies)
    x = d.x.double().cpu().requires_grad_()
    out = train(ctx, model, d)
    live, cu = d.valid.cpu().bool(), d.cu.tolist()
    n = x * torch.rsqrt(x.square().mean(dim=1, keepdim=True) + 1e-5) * scale
    y = n + (torch.where(live[:, None], out["y"].double().cpu(), n.detach()) - n.detach())
    logp = torch.log_softmax(y @ head.T, dim=1)[torch.arange(ROWS), d.tokens.long().cpu()]
    delta = torch.where(live, logp - d.ref.double().cpu(), 0.0)
    sums = torch.stack([delta[a:b].sum() for a, b in zip(cu, cu[1:])])
    loss = -torch.nn.functional.logsigmoid(P["beta"] * (sums[0::2] - sums[1::2])).mean()
    loss.backward()
    # log-probs are fp32 numbers of size 7: 2^-24 of each, under beta and the sums of 2 * 50 of them
    assert out["loss"].item() == pytest.approx(loss.item(), rel=1e-6, abs=P["beta"] * 100 * 7 * 2.0 ** -23)
    near(out["reward"], P["beta"] * sums.detach(), 1e-5)
    for name, want, share in (("dhead", head.grad, 2.0 ** -8), ("dscale", scale.grad, 2.0 ** -8), ("dx", x.grad, 2.0 ** -7)):
        near(out[name], want, share)
    assert ctx.status() == 0
    ctx.close()


@pytest.mark.parametrize("bits", [32, 8])
def test_steps_against_the_gradient(bits):
    """The loss after a small step is what its gradient says: AdamW's first step is lr times the gradient's sign (its own rounding
    and eps aside), so the loss falls by lr times the gradient's absolute sum, to first order."""
    ctx, model, d = B.AisContext(), Model(bits), Data()
    model.copies[0].copy_(model.head)
    out = train(ctx, model, d, lr=0.0)
    want = [out["dhead"].abs().sum(), out["dscale"].abs().sum()]
    model = Model(bits)
    before = [model.head.clone(), model.scale.clone()]
    train(ctx, model, d, lr=1e-3)
    for p, b, g in zip((model.head, model.scale), before, (out["dhead"], out["dscale"])):
        moved, clear = p - b * (1 - 1e-3 * 0.01), g.abs() > 1e-6
        assert torch.allclose(moved[clear], -1e-3 * torch.sign(g[clear]), rtol=0.02)
    assert all(float(w) > 0 for w in want)
    ctx.close()


@pytest.mark.parametrize("bits", [32, 8])
def test_recorded_steps_match_eager_ones(bits):
    ctx = B.AisContext()
    count = lambda: torch.zeros(1, dtype=torch.int64, device="cuda")
    recorded, eager, d = Model(bits, step=count()), Model(bits, step=count()), Data()
    for m in (recorded, eager):
        train(ctx, m, d)                                         # sizes the workspace outside the capture
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    rate = torch.full((1,), 1e-2, device="cuda")
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            out = train(ctx, recorded, d, lr=rate)
    torch.cuda.synchronize()
    for it in range(4):
        rate.fill_(1e-2 / (it + 1))
        d.x.mul_(1.0 + 0.02 * it)
        d.valid.copy_((torch.rand(ROWS, device="cuda") < 0.9 - 0.2 * it).to(torch.uint8))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = {k: v.clone() for k, v in out.items()}
        want = train(ctx, eager, d, lr=rate)
        torch.cuda.synchronize()
        for k in want:
            assert torch.equal(got[k], want[k]), (it, k)
        for a, b in zip((recorded.head, recorded.scale, *recorded.copies, recorded.opt.m, recorded.opt.v, recorded.opt.step),
                        (eager.head, eager.scale, *eager.copies, eager.opt.m, eager.opt.v, eager.opt.step)):
            assert torch.equal(a, b), it
    assert recorded.opt.step.item() == 5 and ctx.status() == 0
    ctx.close()


def test_a_count_on_the_host_is_not_recorded():
    ctx = B.AisContext()
    state, grad = B.AdamWState([torch.ones(100, device="cuda")]), [torch.ones(100, device="cuda")]
    ctx.adamw_step(state, grad)
    want = state.params[0].clone()
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            other = grad[0] * 2
            with pytest.raises(ValueError, match="step"):
                ctx.adamw_step(state, grad)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(state.params[0], want) and state.step == 1 and bool((other == 2).all())
    ctx.close()


def test_two_graphs_share_a_workspace():
    """Two recorded calls of different sizes, replayed one after the other in either order."""
    ctx = B.AisContext()
    gen = torch.Generator(device="cuda").manual_seed(3)
    sizes = [(5_000, 12), (700, 40)]
    cases = []
    for rows, pairs in sizes:
        cu = torch.linspace(0, rows, 2 * pairs + 1, device="cuda").long()
        logp = -torch.rand(rows, generator=gen, device="cuda")
        x, dy = (torch.randn(rows, 257, generator=gen, device="cuda") for _ in range(2))
        cases.append((logp, cu, x, dy))

    def calls(logp, cu, x, dy):
        y, mean, rstd = ctx.norm_rows(x, x[0])
        return (*ctx.preference_row_scale(logp, None, None, cu), *ctx.norm_rows_grad(dy, x, x[0], mean, rstd))

    want = [[t.clone() for t in calls(*c)] for c in cases]
    torch.cuda.synchronize()
    graphs, outs = [], []
    for c in cases:
        side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        with torch.cuda.stream(side):
            with torch.cuda.graph(graph, stream=side):
                outs.append(calls(*c))
        graphs.append(graph)
        torch.cuda.synchronize()
    for order in ((0, 1), (1, 0), (1, 1, 0)):
        for k in order:
            graphs[k].replay()
        torch.cuda.synchronize()
        for out, w in zip(outs, want):
            for a, b in zip(out, w):
                assert torch.equal(a, b)
    ctx.close()


def test_other_streams():
    contexts, d = [B.AisContext(), B.AisContext()], Data()
    want = Model(8)
    ref = train(contexts[0], want, d)
    torch.cuda.synchronize()
    streams, models, outs = [torch.cuda.Stream() for _ in range(2)], [Model(8), Model(8)], [None, None]
    torch.cuda.synchronize()
    for k in range(2):
        with torch.cuda.stream(streams[k]):
            outs[k] = train(contexts[k], models[k], d)
    for s in streams:
        s.synchronize()
    for k in range(2):
        for name in ref:
            assert torch.equal(outs[k][name], ref[name]), (k, name)
        assert torch.equal(models[k].head, want.head) and torch.equal(models[k].opt.m, want.opt.m)
        assert contexts[k].status() == 0
        contexts[k].close()


def test_a_tiling_in_the_workspace_is_not_taken_for_theirs():
    """The diagnostics of many responses leave a tiling behind that the loss after them uses, unless another call has written there."""
    ctx = B.AisContext()
    n, per = 1_200, 3
    rows = n * per
    gen = torch.Generator(device="cuda").manual_seed(5)
    logp, roll = (-torch.rand(rows, generator=gen, device="cuda") for _ in range(2))
    cu = torch.arange(n + 1, device="cuda") * per
    rewards = torch.rand(n, generator=gen, device="cuda")
    x = torch.randn(rows, 64, generator=gen, device="cuda")
    adv, count, diag = ctx.diagnostics(logp, roll, None, cu, rewards, 8)
    want = [t.clone() for t in ctx.grpo_row_scale(logp, roll, None, cu, adv, count, diag)]
    for between in (lambda: ctx.preference_row_scale(logp, roll, None, cu),
                    lambda: ctx.norm_rows_grad(x, x, None, None, torch.ones(rows, device="cuda"))):
        adv, count, diag = ctx.diagnostics(logp, roll, None, cu, rewards, 8)
        between()
        for a, b in zip(ctx.grpo_row_scale(logp, roll, None, cu, adv, count, diag), want):
            assert torch.equal(a, b)
    ctx.close()


def test_kernel_times_can_be_read():
    ctx, model, d = B.AisContext(), Model(8), Data()
    train(ctx, model, d)
    ctx.profile(True)
    train(ctx, model, d)
    for which in (B.AIS_K_PREFERENCE, B.AIS_K_NORM, B.AIS_K_NORM_GRAD, B.AIS_K_ADAMW):
        ms, n = ctx.profile_read(which)
        assert n == 1 and 0.0 < ms < 1_000.0, which
    ctx.profile(False)
    ctx.close()


def test_no_memory_is_kept():
    d, model = Data(), Model(8)

    def one():
        ctx = B.AisContext()
        train(ctx, model, d)
        ctx.close()

    for _ in range(3):
        one()
    torch.cuda.synchronize()
    free, held = torch.cuda.mem_get_info()[0], torch.cuda.memory_reserved()
    for _ in range(50):
        one()
    torch.cuda.synchronize()
    assert (free - torch.cuda.mem_get_info()[0]) - (torch.cuda.memory_reserved() - held) < 32 << 20
