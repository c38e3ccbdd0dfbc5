"""A 4-bit rollout policy, its AIS-corrected update, and its distillation, on one GPU.

    python examples/mxfp4_rollout.py [--vocab 32000] [--width 1024] [--prompts 4] [--length 32] [--iterations 3]

A toy policy: the hidden state of a position is a function of the state before and of the token drawn there, and the read-out
is an output embedding W [V, D].  The trainer's W is bf16; the rollout engine has an MXFP4 copy.  An iteration is

1. rollout: quantise the hidden states, 4-bit logits, draw a token of every live response and keep the log-probability it was
   drawn with (Alg. 1, "sample a group of responses");
2. update: the trainer's log-probabilities from hidden states and W, the diagnostics and the mixing coefficient, the gradient
   of the AIS-GRPO loss with respect to W, a step;
3. distillation: the rollout's copy is pulled towards the trainer's most likely tokens; the gradient passes through the
   quantisation as if it were the identity, to fp32 weights that are quantised again after each step.

The rows of responses are padded to one length; `valid` says which of them exist.
"""
from __future__ import annotations

import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

from paper_2605_13907_amd import binding as B

GROUP = 8                      # responses to a prompt
STOP = 0                       # the token that ends a response


def normalised(h):
    return h * torch.rsqrt(h.float().pow(2).mean(dim=1, keepdim=True) + 1e-6)


class Rollouts:
    """Decodes with the 4-bit read-out; rows lie response after response."""

    def __init__(self, ctx, embedding, length, generator):
        self.ctx, self.embedding, self.length, self.generator = ctx, embedding, length, generator

    def run(self, weight4, start):
        """weight4: what mxfp4_quantize_rows returns for W; start [N, D] -> hidden [N L, D] bf16, tokens, logp, valid [N L]."""
        ctx, n = self.ctx, start.shape[0]
        hidden = torch.zeros(n, self.length, start.shape[1], dtype=torch.bfloat16, device=start.device)
        tokens = torch.zeros(n, self.length, dtype=torch.int32, device=start.device)
        logp = torch.zeros(n, self.length, device=start.device)
        valid = torch.zeros(n, self.length, dtype=torch.uint8, device=start.device)
        h, live = start, torch.ones(n, dtype=torch.uint8, device=start.device)
        noise = torch.empty(n, self.embedding.shape[0], device=start.device)
        for t in range(self.length):
            logits = ctx.mxfp4_logits(*ctx.mxfp4_quantize_rows(h), *weight4)
            drawn, drawn_logp, _ = ctx.sample_tokens(logits, noise.exponential_(generator=self.generator), valid=live)
            hidden[:, t], valid[:, t], logp[:, t] = h, live, drawn_logp
            tokens[:, t] = drawn.clamp(min=0)                # -1 where a response has ended
            live = live * (drawn != STOP)
            h = normalised(0.5 * h.float() + self.embedding[tokens[:, t].long()].float()).bfloat16()
        return hidden.view(n * self.length, -1), tokens.view(-1), logp.view(-1), valid.view(-1)


def update(ctx, weight, hidden, tokens, logp_roll, valid, cu_rows, rewards, rate):
    """One AIS-corrected step of the trainer's read-out, in place -> the diagnostics."""
    params = B.default_params()
    logp, lse = ctx.lm_head_logprob(hidden, weight, tokens, valid)
    adv, count, diag = ctx.diagnostics(logp, logp_roll, valid, cu_rows, rewards, GROUP, params)
    loss, _, g = ctx.grpo_row_scale(logp, logp_roll, valid, cu_rows, adv, count, diag, params)
    _, dweight = ctx.lm_head_grad(hidden, weight, tokens, lse, logp, g)
    weight.copy_(weight.float() - rate * dweight)
    return dict(ctx.read_diag(diag), loss=loss.item())


def distill(ctx, student, weight, hidden, valid, n_top, rate, steps):
    """`steps` steps of the fp32 weights behind the 4-bit read-out, in place -> the divergence before each, and after the last."""
    best = torch.topk(hidden.float() @ weight.float().T, n_top, dim=1)
    ids, teacher = best.indices.int(), best.values.contiguous()
    *hidden4, values = ctx.mxfp4_quantize_rows(hidden, want_values=True)     # the logits' gradient is taken at the values
    losses = []
    for step in range(steps + 1):
        logits = ctx.mxfp4_logits(*hidden4, *ctx.mxfp4_quantize_rows(student))
        last = step == steps
        loss, _, dlogits = ctx.distill_topk(logits, ids, teacher, valid=valid, want_grad=not last,
                                            dlogits=None if last else logits)
        losses.append(loss)
        if not last:
            student -= rate * (dlogits.float().T @ values.float())
    return torch.cat(losses).tolist()


def main(argv=None):
    parser = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    parser.add_argument("--vocab", type=int, default=32_000)
    parser.add_argument("--width", type=int, default=1_024, help="a multiple of 32")
    parser.add_argument("--prompts", type=int, default=4)
    parser.add_argument("--length", type=int, default=32)
    parser.add_argument("--iterations", type=int, default=3)
    parser.add_argument("--steps", type=int, default=8, help="of the distillation in each iteration")
    parser.add_argument("--top", type=int, default=64, help="tokens of the trainer that the rollout's copy is pulled towards")
    args = parser.parse_args(argv)

    gen = torch.Generator(device="cuda").manual_seed(0)
    randn = lambda *size: torch.randn(*size, generator=gen, device="cuda")
    weight = (3.0 / args.width ** 0.5 * randn(args.vocab, args.width)).bfloat16()
    student = weight.float()
    embedding = randn(args.vocab, args.width).bfloat16()
    n = args.prompts * GROUP
    cu_rows = torch.arange(n + 1, dtype=torch.int64, device="cuda") * args.length
    start = normalised(randn(args.prompts, args.width).repeat_interleave(GROUP, dim=0)).bfloat16()

    ctx = B.AisContext()
    rollouts = Rollouts(ctx, embedding, args.length, gen)
    out = []
    for r in range(args.iterations):
        hidden, tokens, logp_roll, valid = rollouts.run(ctx.mxfp4_quantize_rows(student), start)
        # a reward that any policy can learn: for even tokens
        even = ((tokens % 2 == 0).float() * valid).view(n, -1).sum(dim=1) / valid.view(n, -1).sum(dim=1)
        diag = update(ctx, weight, hidden, tokens, logp_roll, valid, cu_rows, (even > 0.5).float(), rate=10.0)
        rows = int(valid.sum())
        kl = distill(ctx, student, weight, hidden, valid, min(args.top, args.vocab), rate=0.5 * rows / args.width,
                     steps=args.steps)
        out.append(dict(diag, kl=kl, hidden=hidden, tokens=tokens, logp_roll=logp_roll, valid=valid))
        print(f"iteration {r}: {rows} tokens, alpha {diag['alpha']:.4f}, loss {diag['loss']:+.4e}, "
              f"divergence {kl[0]:.4f} -> {kl[-1]:.4f}", flush=True)
    status = ctx.status()
    ctx.close()
    if status:
        raise RuntimeError(f"the library reports status {status}")
    return out


if __name__ == "__main__":
    main()
