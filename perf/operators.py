"""The operators of a 4-bit rollout and of the distillation that brings the 4-bit policy back to its teacher: timed cases,
a generator of more of the same kinds, and each operator written in elementary operations.

A rollout engine that holds the output embedding in microscaled 4-bit floating point quantises the last hidden states,
multiplies them with the embedding's codes and draws each next token from the logits, together with the log-probability that
the importance ratio of the trainer divides by.  The distillation loss draws the student's logits to a teacher's top logits.

Kinds (the `kind` of a case):
  quantize  rows -> MXFP4 (blocks of 32 E2M1 elements under one E8M0 scale); the values that the codes stand for are returned
  head      hidden states, quantised on the way, times an MXFP4 output embedding -> logits
  sample    logits, given exponential noise, temperature, top-k, top-p and min-p of each row -> token and its log-probabilities
  distill   student logits and a teacher's top logits -> loss, divergence of each row, gradient of the logits

`own` False computes them in plain torch operations, `own` True through `paper_2605_13907_amd.binding.AisContext`.
"""
import functools
import math

import torch

own = False

BLOCK = 32                    # elements under one scale
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def listed():
    return [
        # The smallest rollout step: the hidden states of a decode batch of 64 sequences.
        dict(name="quantize-hidden-bf16", kind="quantize", rows=64, width=4_096, dtype="bf16"),
        # What the engine does after each weight update: the output embedding of the flagship workload.
        dict(name="quantize-embedding-bf16", kind="quantize", rows=151_936, width=4_096, dtype="bf16"),
        # fp32 master weights whose width is no multiple of a block.
        dict(name="quantize-odd-f32", kind="quantize", rows=5_001, width=1_100, dtype="f32"),
        # One decode step of 16 sequences: the embedding's codes are nearly all that is read.
        dict(name="head-decode-bf16", kind="head", rows=16, vocab=151_936, width=4_096, dtype="bf16"),
        # Scoring a chunk of 2,048 prompt tokens: a large product.
        dict(name="head-chunk-bf16", kind="head", rows=2_048, vocab=151_936, width=4_096, dtype="bf16"),
        # A ragged batch on a model of odd sizes, fp32 logits.
        dict(name="head-odd-f32", kind="head", rows=333, vocab=50_257, width=1_100, dtype="f32"),
        # A serving batch: every request has its own temperature, top-k, top-p and min-p, some none of them.
        dict(name="sample-served-bf16", kind="sample", rows=64, vocab=151_936, dtype="bf16", limits="mixed", live=1.0),
        # Rollouts for training: temperature 0.9 over the whole vocabulary.
        dict(name="sample-rollout-bf16", kind="sample", rows=256, vocab=151_936, dtype="bf16", limits="none", live=1.0),
        # fp32 logits of an odd vocabulary under top-p, a part of the sequences finished.
        dict(name="sample-nucleus-f32", kind="sample", rows=33, vocab=50_257, dtype="f32", limits="top_p", live=0.8),
        # Launch latency: the tiny workload of the benchmark.
        dict(name="distill-tiny-f32", kind="distill", rows=512, vocab=1_024, dtype="f32", top=8, live=1.0),
        # One training step over 8,192 token rows of the flagship vocabulary.
        dict(name="distill-step-bf16", kind="distill", rows=8_192, vocab=151_936, dtype="bf16", top=64, live=1.0),
        # An odd vocabulary, many teacher tokens, a part of the rows masked.
        dict(name="distill-odd-bf16", kind="distill", rows=3_001, vocab=50_257, dtype="bf16", top=200, live=0.6),
    ]


def draw(rng):
    def log_int(lo, hi):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    def vocabulary():
        # from a byte-level model's to the widest; most are padded to a multiple of 64, some are what they are
        v = log_int(1_000, 262_144)
        return max(64, v // 64 * 64) if rng.random() < 0.6 else v

    kind = rng.choice(["quantize", "head", "head", "sample", "sample", "distill", "distill"])
    if kind in ("quantize", "head"):
        width = 64 * log_int(8, 80) if rng.random() < 0.7 else log_int(200, 5_000)
        width += 64 * (width == 48 * 64)
    if kind == "quantize":
        dtype = rng.choice(["bf16", "f32"])
        rows = log_int(1, 200_000)
        return dict(kind=kind, rows=min(rows, 300_000_000 // width), width=width, dtype=dtype)
    vocab = vocabulary()
    if kind == "head":
        rows = log_int(1, 2_048)
        return dict(kind=kind, rows=max(1, min(rows, 300_000_000 // vocab)), vocab=vocab, width=width,
                    dtype=rng.choice(["bf16", "bf16", "f32"]))
    dtype = rng.choice(["bf16", "bf16", "f32"])
    live = rng.choice([1.0, 1.0, 0.7])
    if kind == "sample":
        return dict(kind=kind, rows=min(log_int(1, 512), 40_000_000 // vocab), vocab=vocab, dtype=dtype,
                    limits=rng.choice(["mixed", "mixed", "none", "top_k", "top_p", "min_p"]), live=live)
    rows = min(log_int(16, 20_000), 600_000_000 // vocab)
    return dict(kind=kind, rows=rows, vocab=vocab, dtype=dtype, top=log_int(1, 256), live=live)


# ---- inputs ----------------------------------------------------------------------------------------------------------

def type_of(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def blocks_of(width):
    return -(-width // BLOCK)


def zipf_logits(rows, vocab, dtype, gen, lo=1.2, hi=3.0):
    """Logits whose ranked probabilities fall as a power of the rank, an exponent for each row: from rows of which the nucleus
    of 95 % is a few tokens to rows where it is some ten thousand."""
    z = torch.empty(rows, vocab, device="cuda").exponential_(generator=gen)
    z *= lo + (hi - lo) * torch.rand(rows, 1, generator=gen, device="cuda")
    return (z - 6.0).to(dtype)


def live_rows(case, gen):
    if case["live"] >= 1.0:
        return None
    return (torch.rand(case["rows"], generator=gen, device="cuda") < case["live"]).to(torch.uint8)


def embedding_codes(weight):
    """(codes, scales) of a weight matrix, as the engine keeps them: 16 bytes of codes a block, the first element in the low
    half of the first byte; a byte of scale a block, rows padded to whole groups of 16 blocks."""
    values, exponent = rounded(weight)
    rows, blocks = exponent.shape
    a = values.abs()
    code = torch.where(a <= 2.0, 2.0 * a, torch.where(a <= 4.0, a + 2.0, torch.full_like(a, 7.0))).to(torch.uint8)
    code |= (values < 0).to(torch.uint8) << 3
    code = code.view(rows, blocks * 16, 2)
    scales = torch.zeros(rows, -(-blocks // 16) * 16, dtype=torch.uint8, device=weight.device)
    scales[:, :blocks] = (exponent + 127).to(torch.uint8)
    return code[..., 0] | code[..., 1] << 4, scales[:, :blocks]


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    kind, dtype = case["kind"], type_of(case)
    if kind == "quantize":
        x = torch.randn(case["rows"], case["width"], generator=gen, device="cuda")
        # rows of different magnitudes, a few channels that stand out, as hidden states and embeddings have them
        x *= torch.exp(0.5 * torch.randn(case["rows"], 1, generator=gen, device="cuda"))
        x[:, :: 97] *= 8.0
        return dict(case=case, x=x.to(dtype))
    if kind == "head":
        rows, vocab, width = case["rows"], case["vocab"], case["width"]
        weight = torch.randn(vocab, width, generator=gen, device="cuda") / math.sqrt(width)
        # every row has a preferred token, whose logit stands out by up to 12
        mode = torch.randint(0, vocab, (rows,), generator=gen, device="cuda")
        sharp = 12.0 * torch.rand(rows, 1, generator=gen, device="cuda")
        hidden = weight[mode] * sharp + torch.randn(rows, width, generator=gen, device="cuda")
        codes, scales = embedding_codes(weight)
        return dict(case=case, hidden=hidden.to(torch.bfloat16), codes=codes, scales=scales)
    rows, vocab = case["rows"], case["vocab"]
    if kind == "sample":
        def pick(values, kind_of):
            v = torch.tensor(values, dtype=kind_of, device="cuda")
            return v[torch.randint(0, len(values), (rows,), generator=gen, device="cuda")]

        limits = case["limits"]
        state = dict(case=case, logits=zipf_logits(rows, vocab, dtype, gen), valid=live_rows(case, gen),
                     noise=torch.empty(rows, vocab, device="cuda").exponential_(generator=gen),
                     temperature=torch.full((rows,), 0.9, device="cuda"), top_k=None, top_p=None, min_p=None)
        if limits == "mixed":
            state.update(temperature=pick([0.6, 0.7, 1.0, 1.2, 0.0], torch.float32), top_k=pick([20, 50, 0, 1], torch.int32),
                         top_p=pick([0.8, 0.95, 1.0], torch.float32), min_p=pick([0.0, 0.0, 0.05], torch.float32))
        elif limits == "top_k":
            state.update(top_k=pick([1, 5, 20, 50, 100, 1_000], torch.int32))
        elif limits == "top_p":
            state.update(top_p=pick([0.5, 0.8, 0.9, 0.95, 0.99], torch.float32))
        elif limits == "min_p":
            state.update(min_p=pick([0.02, 0.05, 0.1, 0.3], torch.float32))
        return state
    logits = zipf_logits(rows, vocab, dtype, gen)
    top, ids = case["top"], []
    values = []
    for r in range(0, rows, 1024):
        part = logits[r:r + 1024].float()
        t = torch.topk(part + 0.5 * torch.randn(part.shape, generator=gen, device="cuda"), min(top, vocab), dim=1)
        ids.append(t.indices.to(torch.int32))
        values.append(t.values)
    return dict(case=case, logits=logits, ids=torch.cat(ids), teacher=torch.cat(values), valid=live_rows(case, gen),
                weight=torch.rand(rows, generator=gen, device="cuda") / rows)


# ---- the plain forms -------------------------------------------------------------------------------------------------

def power_of_two(e):
    """2^e in fp32 for whole -127 <= e <= 127, exactly (2^-127 is a subnormal number)."""
    bits = torch.where(e > -127, (e + 127) << 23, torch.full_like(e, 1 << 22))
    return bits.to(torch.int32).view(torch.float32)


def rounded(x):
    """(E2M1 values [rows, blocks * 32], shared exponents [rows, blocks]) of x: the exponent of a block is that of its largest
    magnitude less two, elements are rounded to nearest, ties to even, and saturate at 6."""
    rows, width = x.shape
    blocks = blocks_of(width)
    x = torch.nn.functional.pad(x.float(), (0, blocks * BLOCK - width)).view(rows, blocks, BLOCK)
    largest = x.abs().amax(dim=2)
    exponent = torch.frexp(largest).exponent - 3
    exponent = torch.where(largest > 0, exponent, torch.full_like(exponent, -127)).clamp(min=-127)
    y = x * power_of_two(-exponent).unsqueeze(2)
    a = y.abs()
    step = torch.where(a < 2.0, torch.full_like(a, 0.5), torch.where(a < 4.0, torch.ones_like(a), torch.full_like(a, 2.0)))
    q = torch.minimum(torch.round(a / step) * step, torch.full_like(a, 6.0))
    return torch.where(y < 0, -q, q).view(rows, blocks * BLOCK), exponent


def plain_quantize(s):
    x = s["x"]
    q, exponent = rounded(x)
    values = q.view(*exponent.shape, BLOCK) * power_of_two(exponent).unsqueeze(2)
    return dict(values=values.view(x.shape[0], -1)[:, :x.shape[1]].to(x.dtype))


def plain_head(s):
    q, exponent = rounded(s["hidden"])
    hidden = (q.view(*exponent.shape, BLOCK) * power_of_two(exponent).unsqueeze(2)).view(q.shape)
    codes, scales = s["codes"], s["scales"]
    grid = torch.tensor(GRID + tuple(-g for g in GRID), device=codes.device)
    weight = torch.stack((grid[(codes & 15).int()], grid[(codes >> 4).int()]), dim=2).view(*scales.shape, BLOCK)
    weight = weight * power_of_two(scales.to(torch.int32) - 127).unsqueeze(2)
    return dict(logits=(hidden @ weight.view(codes.shape[0], -1).t()).to(type_of(s["case"])))


def plain_sample(s):
    z, vocab, rows = s["logits"].float(), s["case"]["vocab"], s["case"]["rows"]
    temperature = s["temperature"].unsqueeze(1)
    greedy = temperature == 0
    ranked, order = torch.sort(z, dim=1, descending=True, stable=True)
    t = (ranked - ranked[:, :1]) / torch.where(greedy, torch.ones_like(temperature), temperature)
    p = torch.exp(t)
    total = p.sum(dim=1, keepdim=True)
    rank = torch.arange(vocab, device=z.device).expand(rows, vocab)
    kept = torch.where(greedy, rank < 1, rank >= 0)
    if s["top_k"] is not None:
        k = s["top_k"].unsqueeze(1)
        kept = kept & ((rank < k) | (k == 0))
    if s["top_p"] is not None:
        below = p * kept
        top_p = s["top_p"].unsqueeze(1)
        mass = below.sum(dim=1, keepdim=True)
        kept = kept & ((below.cumsum(dim=1) - below < top_p * mass) | (top_p >= 1))
    if s["min_p"] is not None:
        kept = kept & (p >= s["min_p"].unsqueeze(1))
    score = t - torch.log(s["noise"].gather(1, order))
    score = torch.where(kept, score, torch.full_like(score, -math.inf))
    best = score.amax(dim=1, keepdim=True)
    token = torch.where(score == best, order, torch.full_like(order, vocab)).amin(dim=1, keepdim=True)
    at = (z.gather(1, token) - ranked[:, :1]) / torch.where(greedy, torch.ones_like(temperature), temperature)
    logp = at - torch.log((p * kept).sum(dim=1, keepdim=True))
    full = torch.where(greedy, torch.zeros_like(at), at - torch.log(total))
    token, logp, full = token.squeeze(1).to(torch.int32), logp.squeeze(1), full.squeeze(1)
    if s["valid"] is not None:
        live = s["valid"] != 0
        token = torch.where(live, token, torch.full_like(token, -1))
        logp, full = logp * live, full * live
    return dict(token=token, logp=logp, logp_full=full)


def plain_distill(s):
    z, ids, weight = s["logits"].float(), s["ids"].long(), s["weight"]
    if s["valid"] is not None:
        weight = weight * (s["valid"] != 0)
    top = z.amax(dim=1, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(dim=1, keepdim=True)
    t = s["teacher"] - s["teacher"].amax(dim=1, keepdim=True)
    q = torch.exp(t)
    mass = q.sum(dim=1, keepdim=True)
    q = q / mass
    logp = z.gather(1, ids) - top - torch.log(total)
    kl = (q * (t - torch.log(mass) - logp)).sum(dim=1)
    if s["valid"] is not None:
        kl = kl * (s["valid"] != 0)
    grad = (e / total).scatter_add_(1, ids, -q) * weight.unsqueeze(1)
    return dict(loss=(weight * kl).sum().reshape(1), kl=kl, dlogits=grad.to(s["logits"].dtype))


# ---- one pass --------------------------------------------------------------------------------------------------------

@functools.lru_cache(maxsize=None)
def context():
    """The one context that a program keeps."""
    from paper_2605_13907_amd import binding
    return binding.AisContext()


def run(state):
    case = state["case"]
    kind = case["kind"]
    if not own:
        return dict(quantize=plain_quantize, head=plain_head, sample=plain_sample, distill=plain_distill)[kind](state)
    ctx = context()
    if kind == "quantize":
        codes, scales, values = ctx.mxfp4_quantize_rows(state["x"], want_values=True)
        return dict(values=values)
    if kind == "head":
        codes, scales = ctx.mxfp4_quantize_rows(state["hidden"])
        return dict(logits=ctx.mxfp4_logits(codes, scales, state["codes"], state["scales"], dtype=type_of(case)))
    if kind == "sample":
        token, logp, full = ctx.sample_tokens(state["logits"], state["noise"], state["valid"], state["temperature"],
                                              state["top_k"], state["top_p"], state["min_p"])
        return dict(token=token, logp=logp, logp_full=full)
    loss, kl, dlogits = ctx.distill_topk(state["logits"], state["ids"], state["teacher"], state["weight"], state["valid"])
    return dict(loss=loss, kl=kl, dlogits=dlogits)


def work(case):
    kind, e = case["kind"], 2 if case["dtype"] == "bf16" else 4
    rows = case["rows"]
    if kind == "quantize":
        return dict(bytes=rows * (2 * e * case["width"] + 17 * blocks_of(case["width"])), flops=4 * rows * case["width"])
    vocab = case["vocab"]
    if kind == "head":
        width = case["width"]
        return dict(bytes=2 * rows * width + 17 * vocab * blocks_of(width) + e * rows * vocab, flops=2 * rows * vocab * width)
    live = case["live"] * rows
    if kind == "sample":
        # rows without a limit need a random number for every logit; the others for the few that are kept
        share = {"none": 1.0, "mixed": 0.2 / 3}.get(case["limits"], 0.0)
        return dict(bytes=int(live * vocab * (e + 4 * share)) + 24 * rows, flops=int(4 * live * vocab))
    return dict(bytes=int(e * vocab * (live + rows)) + 8 * int(live) * case["top"] + 8 * rows, flops=int(8 * live * vocab))


# ---- the definitions in 64 bits --------------------------------------------------------------------------------------

def e2m1_blocks(x):
    """x [rows, width] in 64 bits, each block of 32 replaced by the nearest values of its E2M1 grid."""
    rows, width = x.shape
    blocks = blocks_of(width)
    full = torch.zeros(rows, blocks * BLOCK, dtype=torch.float64, device=x.device)
    full[:, :width] = x
    b = full.view(rows, blocks, BLOCK)
    largest = b.abs().max(dim=2, keepdim=True).values
    unit = torch.where(largest > 0, torch.exp2(torch.floor(torch.log2(largest)) - 2.0), torch.ones_like(largest))
    r = b.abs() / unit
    out = torch.zeros_like(r)
    # a magnitude passes a grid value's midpoint below; on the midpoint itself it goes to the even one of the two
    for i in range(1, len(GRID)):
        middle = (GRID[i - 1] + GRID[i]) / 2.0
        out = torch.where(r >= middle if i % 2 == 0 else r > middle, torch.full_like(out, GRID[i]), out)
    return (torch.sign(b) * out * unit).view(rows, blocks * BLOCK)[:, :width]


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "quantize":
        return dict(values=torch.cat([e2m1_blocks(x.double()) for x in s["x"].split(16_384)]))
    if kind == "head":
        hidden = e2m1_blocks(s["hidden"].double())
        width = hidden.shape[1]
        parts = []
        for codes, scales in zip(s["codes"].split(16_384), s["scales"].split(16_384)):
            nibble = torch.stack((codes % 16, codes // 16), dim=2).view(codes.shape[0], -1)
            m = nibble % 8
            value = torch.where(m < 2, 0.5 * m.double(), (1.0 + 0.5 * (m % 2)) * torch.exp2((m // 2).double() - 1.0))
            value = torch.where(nibble >= 8, -value, value)
            value = value * torch.exp2(scales.double() - 127.0).repeat_interleave(BLOCK, dim=1)
            parts.append(hidden @ value[:, :width].t())
        return dict(logits=torch.cat(parts, dim=1))
    if kind == "sample":
        return exact_sample(s)
    loss, kls, grads = torch.zeros(1, dtype=torch.float64, device="cuda"), [], []
    for r in range(0, case["rows"], 1024):
        at = slice(r, r + 1024)
        logp = torch.log_softmax(s["logits"][at].double(), dim=1)
        logq = torch.log_softmax(s["teacher"][at].double(), dim=1)
        ids, w = s["ids"][at].long(), s["weight"][at].double()
        live = torch.ones_like(w) if s["valid"] is None else (s["valid"][at] != 0).double()
        kl = (logq.exp() * (logq - logp.gather(1, ids))).sum(dim=1) * live
        target = torch.zeros_like(logp).scatter_(1, ids, logq.exp())
        loss += (w * kl).sum()
        kls.append(kl)
        grads.append(((logp.exp() - target) * (w * live).unsqueeze(1)).to(torch.float64 if case["rows"] * case["vocab"] < 4e8
                                                                          else torch.float32))
    return dict(loss=loss, kl=torch.cat(kls), dlogits=torch.cat(grads))


def exact_sample(s):
    """Row by row: the kept tokens are the first of the ranked ones, as many as the tightest limit allows."""
    tokens, logps, fulls = [], [], []
    for r in range(s["case"]["rows"]):
        if s["valid"] is not None and not bool(s["valid"][r]):
            tokens.append(-1)
            logps.append(0.0)
            fulls.append(0.0)
            continue
        z = s["logits"][r].double()
        temperature = float(s["temperature"][r])
        ranked, order = torch.sort(z, descending=True, stable=True)
        if temperature == 0.0:
            tokens.append(int(order[0]))
            logps.append(0.0)
            fulls.append(0.0)
            continue
        logp = torch.log_softmax(ranked / temperature, dim=0)
        n = z.numel()
        k = 0 if s["top_k"] is None else int(s["top_k"][r])
        if k > 0:
            n = min(n, k)
        if s["top_p"] is not None and float(s["top_p"][r]) < 1.0:
            p = logp[:n].exp()
            before = torch.cumsum(p, dim=0) - p
            n = int((before < float(s["top_p"][r]) * p.sum()).sum())
        if s["min_p"] is not None:
            n = min(n, int((logp - logp[0] >= math.log(max(float(s["min_p"][r]), 1e-300))).sum()))
        score = logp[:n] - torch.log(s["noise"][r].double()[order[:n]])
        at = int(torch.argmax(score))
        tokens.append(int(order[at]))
        logps.append(float(logp[at] - torch.logsumexp(logp[:n], dim=0)))
        fulls.append(float(logp[at]))
    return dict(token=torch.tensor(tokens, dtype=torch.int32), logp=torch.tensor(logps, dtype=torch.float64),
                logp_full=torch.tensor(fulls, dtype=torch.float64))
