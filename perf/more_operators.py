"""The operators of a training step around the read-out: timed cases, a generator of more of the same kinds, and each operator
written in elementary operations.

A trainer normalises the last hidden states, reads out logits, forms a loss over whole responses, and steps the weights with the
gradient.  The losses over single tokens, the read-out and its gradient are timed elsewhere; these are the operators on either
side of them.

Kinds (the `kind` of a case):
  pairs      logits of preferred and other responses in turn -> loss over their log-ratios to a reference, rewards, dlogits
  scores     the same loss from log-probabilities of the tokens -> loss, rewards, coefficient of every row
  norm       rows -> normalised rows (layer norm, or root mean square), mean and reciprocal deviation
  norm_grad  gradient of the normalised rows -> gradient of the rows, of the weight and of the bias
  adamw      a step over many tensors at once, moments in 32 or in 8 bits; the moments' values are returned

`own` False computes them in plain torch operations, `own` True through `paper_2605_13907_amd.binding.AisContext`.
"""
import functools
import math

import torch

own = False

BLOCK = 32                    # elements of a tensor whose 8-bit moments share a scale
MASK = 0xFFFFFFFF
# odd constants of the rounding's random numbers: fractions of the golden ratio and of the square root of 2
PHI, ROOT2 = 0x9E3779B1, 0x6A09E667
LR, BETA1, BETA2, EPS, DECAY = 1e-4, 0.9, 0.999, 1e-8, 0.01


def listed():
    return [
        # Launch latency: the tiny workload of the benchmark, four pairs.
        dict(name="pairs-tiny-f32", kind="pairs", rows=512, vocab=1_024, pairs=4, dtype="f32", live=1.0, form="logistic"),
        # One step over 16 pairs of the flagship vocabulary, a fifth of the tokens prompt.
        dict(name="pairs-step-bf16", kind="pairs", rows=8_192, vocab=151_936, pairs=16, dtype="bf16", live=0.8, form="logistic"),
        # An odd vocabulary, padded responses, the squared form over means of the tokens.
        dict(name="pairs-odd-bf16", kind="pairs", rows=3_001, vocab=50_257, pairs=12, dtype="bf16", live=0.6, form="squared"),
        # Log-probabilities of a few responses from the read-out that keeps no logits: latency.
        dict(name="scores-few", kind="scores", rows=2_048, pairs=4, live=1.0, form="logistic"),
        # A whole set of preferences scored before training.
        dict(name="scores-set", kind="scores", rows=1_200_000, pairs=2_000, live=0.7, form="hinge"),
        # The hidden states of a decode batch of 64 sequences: the smallest call.
        dict(name="norm-decode-bf16", kind="norm", rows=64, width=4_096, dtype="bf16", centered=False),
        # All token rows of the flagship batch, layer norm.
        dict(name="norm-step-bf16", kind="norm", rows=41_643, width=4_096, dtype="bf16", centered=True),
        # Back from the read-out, whose gradient is fp32, to bf16 hidden states of the flagship batch.
        dict(name="norm-grad-step-bf16", kind="norm_grad", rows=41_643, width=4_096, dtype="bf16", dy="f32", centered=False),
        # An fp32 model of odd width with weight and bias.
        dict(name="norm-grad-odd-f32", kind="norm_grad", rows=5_001, width=1_100, dtype="f32", dy="f32", centered=True),
        # The small tensors of a model: norms, biases, adapters.
        dict(name="adamw-small-8", kind="adamw", tensors=150, least=1_000, most=30_000, bits=8, dtype="f32", grad="f32", copy=False),
        # The output embedding of the odd model, bf16 weights and gradients, moments in full.
        dict(name="adamw-odd-32", kind="adamw", tensors=3, least=5_000_000, most=55_282_700, bits=32, dtype="bf16", grad="bf16",
             copy=False),
        # The output embedding of the flagship workload: fp32 master weights, the read-out's fp32 gradient, a bf16 copy.
        dict(name="adamw-embedding-8", kind="adamw", tensors=1, least=622_329_856, most=622_329_856, bits=8, dtype="f32", grad="f32",
             copy=True),
    ]


def draw(rng):
    def log_int(lo, hi):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    kind = rng.choice(["pairs", "pairs", "scores", "norm", "norm", "norm_grad", "norm_grad", "adamw", "adamw"])
    form = rng.choice(["logistic", "logistic", "smooth", "hinge", "squared"])
    if kind == "pairs":
        v = log_int(1_000, 262_144)
        vocab = max(64, v // 64 * 64) if rng.random() < 0.6 else v
        rows = min(log_int(64, 8_000), 600_000_000 // vocab)
        return dict(kind=kind, rows=rows, vocab=vocab, pairs=max(1, min(log_int(1, 64), rows // 8)),
                    dtype=rng.choice(["bf16", "bf16", "f32"]), live=rng.choice([1.0, 0.8, 0.5]), form=form)
    if kind == "scores":
        rows = log_int(64, 1_200_000)
        return dict(kind=kind, rows=rows, pairs=max(1, min(log_int(1, 4_000), rows // 8)), live=rng.choice([1.0, 0.8, 0.5]), form=form)
    if kind in ("norm", "norm_grad"):
        width = 64 * log_int(2, 128) if rng.random() < 0.7 else log_int(100, 9_000)
        rows = min(log_int(1, 40_000), 150_000_000 // width)
        dtype = rng.choice(["bf16", "bf16", "f32"])
        case = dict(kind=kind, rows=rows, width=width, dtype=dtype, centered=rng.random() < 0.5)
        return dict(case, dy=rng.choice([dtype, "f32"])) if kind == "norm_grad" else case
    tensors = log_int(1, 200)
    most = log_int(64, 200_000_000 // tensors)
    dtype = rng.choice(["bf16", "f32", "f32"])
    return dict(kind=kind, tensors=tensors, least=max(1, most // 30), most=most, bits=rng.choice([8, 8, 32]), dtype=dtype,
                grad=rng.choice([dtype, "f32"]), copy=dtype == "f32" and rng.random() < 0.5)


# ---- inputs ----------------------------------------------------------------------------------------------------------

def type_of(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def form_of(case):
    """beta, kind of the loss, label smoothing, margin, means instead of sums."""
    return dict(logistic=(0.1, 0, 0.0, 0.0, False), smooth=(0.1, 0, 0.1, 0.0, False), hinge=(0.05, 1, 0.0, 0.2, False),
                squared=(0.5, 2, 0.0, 0.0, True))[case["form"]]


def cut(rows, parts, gen):
    """Offsets of `parts` responses of uneven lengths that share the rows."""
    share = torch.rand(parts, generator=gen, device="cuda", dtype=torch.float64) + 0.3
    at = (share.cumsum(0) / share.sum() * rows).round().long()
    at[-1] = rows
    return torch.cat((torch.zeros(1, dtype=torch.int64, device="cuda"), at))


def sizes_of(case):
    """Numbers of elements of the tensors, from `least` to `most`, in a geometric row that wanders."""
    n, lo, hi = case["tensors"], math.log(case["least"]), math.log(case["most"])
    return [int(round(math.exp(lo + (hi - lo) * ((i * 0.618033988749895) % 1.0 if i else 1.0)))) for i in range(n)]


def offsets_of(case):
    """Where each tensor begins in a buffer of all, at whole blocks, and the buffer's length."""
    at = [0]
    for n in sizes_of(case):
        at.append(at[-1] + -(-n // BLOCK) * BLOCK)
    return at


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    kind = case["kind"]

    def randn(*size):
        return torch.randn(*size, generator=gen, device="cuda")

    def uniform(*size):
        return torch.rand(*size, generator=gen, device="cuda")

    if kind in ("pairs", "scores"):
        rows, pairs = case["rows"], case["pairs"]
        state = dict(case=case, cu=cut(rows, 2 * pairs, gen), weight=(0.5 + uniform(pairs)) / pairs,
                     valid=None if case["live"] >= 1.0 else (uniform(rows) < case["live"]).to(torch.uint8))
        if kind == "scores":
            # confident and less confident tokens; the policy has moved a little from its reference
            logp = -torch.empty(rows, device="cuda").exponential_(generator=gen)
            return dict(state, logp=logp, ref=torch.clamp(logp + 0.15 * randn(rows) + 0.01, max=0.0))
        z = torch.empty(rows, case["vocab"], dtype=type_of(case["dtype"]), device="cuda")
        ids, logp = [], []
        for r in range(0, rows, 1024):
            at = z[r:r + 1024]
            # ranked probabilities that fall as a power of the rank
            part = torch.empty(at.shape, device="cuda").exponential_(generator=gen) * (1.2 + 1.8 * uniform(at.shape[0], 1))
            at.copy_(part)
            part = torch.log_softmax(at.float(), dim=1)
            ids.append((part - torch.empty(at.shape, device="cuda").exponential_(generator=gen).log_()).argmax(dim=1))
            logp.append(part.gather(1, ids[-1].unsqueeze(1)).squeeze(1))
        logp = torch.cat(logp)
        return dict(state, logits=z, ids=torch.cat(ids).to(torch.int32), ref=torch.clamp(logp + 0.15 * randn(rows) + 0.01, max=0.0))
    if kind in ("norm", "norm_grad"):
        rows, width, dtype = case["rows"], case["width"], type_of(case["dtype"])
        x = torch.randn(rows, width, generator=gen, device="cuda")
        # rows of different magnitudes, a few channels that stand out, as a residual stream has them
        x *= torch.exp(0.5 * randn(rows, 1))
        x[:, :: 97] *= 8.0
        state = dict(case=case, x=x.to(dtype), weight=(1.0 + 0.1 * randn(width)).to(dtype),
                     bias=(0.1 * randn(width)).to(dtype) if case["centered"] else None)
        if kind == "norm":
            return state
        wide = state["x"].float()
        mean = wide.mean(dim=1) if case["centered"] else None
        rest = wide - mean.unsqueeze(1) if case["centered"] else wide
        rstd = torch.rsqrt(rest.square().mean(dim=1) + 1e-5)
        dy = randn(rows, width).mul_(1e-3).to(type_of(case["dy"]))
        return dict(state, mean=mean, rstd=rstd, dy=dy)
    sizes, offsets = sizes_of(case), offsets_of(case)
    total, dtype, gtype = offsets[-1], type_of(case["dtype"]), type_of(case["grad"])
    p = torch.zeros(total, dtype=dtype, device="cuda")
    g = torch.zeros(total, dtype=gtype, device="cuda")
    state = dict(case=case, param=p, grad=g, params=[], grads=[], step=1_000, seed=17, copy=None, copies=None,
                 grad_scale=0.5 + 0.5 * uniform(1))
    if case["copy"]:
        state["copy"] = torch.zeros(total, dtype=torch.bfloat16, device="cuda")
        state["copies"] = [state["copy"][a:a + n] for a, n in zip(offsets, sizes)]
    if case["bits"] == 8:
        # moments as they stand after many steps: signed codes, and unsigned ones of squares, below the blocks' largest
        m = torch.zeros(total, dtype=torch.uint8, device="cuda")
        v = torch.zeros(total, dtype=torch.uint8, device="cuda")
        scales = torch.randint(102, 106, (2, total // BLOCK), generator=gen, device="cuda", dtype=torch.uint8)
        state.update(m=m, v=v, m_scale=scales[0], v_scale=scales[1] - 21)
    else:
        m = torch.zeros(total, device="cuda")
        v = torch.zeros(total, device="cuda")
        state.update(m=m, v=v, m_scale=None, v_scale=None)
    for a, n in zip(offsets, sizes):
        state["params"].append(p[a:a + n])
        state["grads"].append(g[a:a + n])
        for i in range(a, a + n, 1 << 27):
            at = slice(i, min(i + (1 << 27), a + n))
            size = at.stop - at.start
            p[at] = 0.02 * randn(size)
            g[at] = (1e-5 * randn(size)).to(gtype)
            if case["bits"] == 8:
                c = torch.randint(0, 256, (size,), generator=gen, device="cuda", dtype=torch.uint8)
                m[at] = torch.where(c % 128 > 117, c - 10, c)
                v[at] = torch.randint(180, 240, (size,), generator=gen, device="cuda", dtype=torch.uint8)
            else:
                m[at] = 3e-6 * randn(size)
                v[at] = 1e-10 * torch.empty(size, device="cuda").exponential_(generator=gen)
    return state


# ---- the plain forms -------------------------------------------------------------------------------------------------

def plain_scores(s, logp):
    """(loss, rewards, derivative of the loss by each row's log-probability) from the log-probabilities."""
    beta, kind, smooth, margin, mean = form_of(s["case"])
    rows, pairs = s["case"]["rows"], s["case"]["pairs"]
    here = torch.ones(rows, device=logp.device) if s["valid"] is None else (s["valid"] != 0).float()
    owner = torch.searchsorted(s["cu"][1:].contiguous(), torch.arange(rows, device=logp.device), right=True)
    # sums over long responses, whose terms cancel
    sums = torch.zeros(2 * pairs, dtype=torch.float64, device=logp.device)
    sums.index_add_(0, owner, ((logp.double() - s["ref"].double()) * here.double()))
    count = torch.zeros(2 * pairs, device=logp.device).index_add_(0, owner, here)
    each = torch.ones_like(count)
    if mean:
        each = torch.where(count > 0, 1.0 / torch.clamp(count, min=1.0), torch.zeros_like(count))
    d = (sums * each.double()).float()
    h = beta * (d[0::2] - d[1::2]) - margin
    if kind == 0:
        below, above = torch.log1p(torch.exp(-h.abs())) + torch.clamp(-h, min=0.0), torch.log1p(torch.exp(-h.abs())) + torch.clamp(h, min=0.0)
        loss, slope = (1.0 - smooth) * below + smooth * above, 1.0 / (1.0 + torch.exp(-h)) - (1.0 - smooth)
    elif kind == 1:
        loss, slope = torch.clamp(1.0 - h, min=0.0), -(h < 1.0).float()
    else:
        loss, slope = ((h - 0.5) / beta).square(), 2.0 * (h - 0.5) / beta / beta
    by = s["weight"] * slope * beta
    by = torch.stack((by, -by), dim=1).view(-1) * each
    return (s["weight"] * loss).sum().reshape(1), beta * d, by[owner] * here


def plain_pairs(s):
    z = s["logits"].float()
    ids = s["ids"].long().unsqueeze(1)
    top = z.amax(dim=1, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(dim=1, keepdim=True)
    # a log-probability is rounded once, to 32 bits: a response's log-ratios nearly cancel
    logp = ((z.gather(1, ids) - top).double() - torch.log(e.sum(dim=1, keepdim=True, dtype=torch.float64))).squeeze(1).float()
    loss, reward, by = plain_scores(s, logp)
    one = torch.ones_like(ids, dtype=torch.float32)
    grad = (e / total).scatter_add_(1, ids, -one) * -by.unsqueeze(1)
    return dict(loss=loss, reward=reward, dlogits=grad.to(s["logits"].dtype))


def plain_norm(s):
    x, width = s["x"].float(), s["case"]["width"]
    mean = x.sum(dim=1, keepdim=True) / width if s["case"]["centered"] else torch.zeros_like(x[:, :1])
    rest = x - mean
    rstd = 1.0 / torch.sqrt(rest.square().sum(dim=1, keepdim=True) / width + 1e-5)
    y = rest * rstd * s["weight"].float()
    if s["bias"] is not None:
        y = y + s["bias"].float()
    return dict(y=y.to(s["x"].dtype), mean=mean.squeeze(1) if s["case"]["centered"] else None, rstd=rstd.squeeze(1))


def plain_norm_grad(s):
    x, dy, rstd, width = s["x"].float(), s["dy"].float(), s["rstd"].unsqueeze(1), s["case"]["width"]
    unit = (x - s["mean"].unsqueeze(1)) * rstd if s["case"]["centered"] else x * rstd
    w = dy * s["weight"].float()
    back = w - unit * ((w * unit).sum(dim=1, keepdim=True) / width)
    if s["case"]["centered"]:
        back = back - w.sum(dim=1, keepdim=True) / width
    return dict(dx=(back * rstd).to(s["x"].dtype), dweight=(dy * unit).sum(dim=0), dbias=dy.sum(dim=0) if s["case"]["centered"] else None)


@functools.lru_cache(maxsize=None)
def grids():
    """What the 256 codes of each moment stand for under a scale of 1: sign, 4 exponent bits and 3 of fraction; 5 and 3."""
    def magnitude(c, bias):
        return (c % 8) / 8.0 * 2.0 ** (1 - bias) if c < 8 else (1.0 + c % 8 / 8.0) * 2.0 ** (c // 8 - bias)

    first = [(-1.0 if c > 127 else 1.0) * magnitude(c % 128, 7) for c in range(256)]
    return (torch.tensor(first, dtype=torch.float64, device="cuda"),
            torch.tensor([magnitude(c, 15) for c in range(256)], dtype=torch.float64, device="cuda"))


def power_of_two(e):
    """2^e in 64 bits, exactly, for whole e."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def moment_values(s):
    """Both moments in 64 bits, exactly."""
    if s["m_scale"] is None:
        return s["m"].double(), s["v"].double()
    out = []
    for codes, scale, grid in zip((s["m"], s["v"]), (s["m_scale"], s["v_scale"]), grids()):
        out.append((grid[codes.int()].view(-1, BLOCK) * power_of_two(scale.int() - 127).unsqueeze(1)).view(-1))
    return out


def mixed(x):
    x = ((x ^ (x >> 15)) * ROOT2) & MASK
    return x ^ (x >> 16)


def random_bits(case, step, seed):
    """32 random bits of every element, from the tensor's number and the element's place in it alone."""
    offsets = torch.tensor(offsets_of(case), device="cuda")
    i = torch.arange(int(offsets[-1]), device="cuda")
    if case["tensors"] == 1:
        return mixed((i * PHI & MASK) ^ mixed(mixed(seed ^ (step * PHI & MASK))))
    tensor = torch.searchsorted(offsets[1:].contiguous(), i, right=True)
    key = mixed(mixed(seed ^ (step * PHI & MASK)) ^ (tensor * PHI & MASK))
    return mixed(((i - offsets[tensor]) * PHI & MASK) ^ key)


def encoded(x, random, low, least_scale, top, never_zero):
    """(codes, scales) of non-negative x: under the block's scale the largest has the exponent `top` and the smallest whole
    exponent is `low`; of the two codes on either side of a value the random number takes one."""
    b = x.view(-1, BLOCK)
    largest = b.amax(dim=1)
    scale = torch.where(largest > 0, torch.frexp(largest).exponent - 1 - top + 127, torch.zeros_like(largest, dtype=torch.int32))
    scale = torch.clamp(scale, min=least_scale)
    t = b.double() * power_of_two(127 - scale).unsqueeze(1)
    e = torch.clamp(torch.where(t > 0, torch.frexp(t).exponent - 1, torch.full_like(t, low, dtype=torch.int32)), min=low)
    n = torch.floor(t * power_of_two(3 - e) + random.view(-1, BLOCK) / 65536.0).int() + 8 * (e - low)
    if never_zero:
        n = torch.where((t > 0) & (n < 1), torch.ones_like(n), n)
    return n.view(-1), scale.to(torch.uint8)


def plain_adamw(s):
    s["step"] += 1
    step, case = s["step"], s["case"]
    # the moments in 64 bits and then in 32, since a code next to a border goes by their last bits
    g = s["grad"].double() * s["grad_scale"].double()
    m, v = moment_values(s)
    m = (BETA1 * m + (1.0 - BETA1) * g).float()
    v = (BETA2 * v + (1.0 - BETA2) * (g * g)).float()
    del g
    p = s["param"].float()
    p = p - LR * (DECAY * p + m / (1.0 - BETA1 ** step) / (torch.sqrt(v / (1.0 - BETA2 ** step)) + EPS))
    s["param"].copy_(p)
    if s["copy"] is not None:
        s["copy"].copy_(p)
    del p
    if case["bits"] == 32:
        s["m"].copy_(m)
        s["v"].copy_(v)
    else:
        random = random_bits(case, step, s["seed"])
        codes, s["m_scale"] = encoded(m.abs(), random & 65535, -6, 7, 7, False)
        s["m"].copy_(torch.where(m < 0, codes + 128, codes))
        codes, s["v_scale"] = encoded(v, random >> 16, -14, 15, 15, True)
        s["v"].copy_(codes)
        m, v = (x.bfloat16() for x in moment_values(s))
    return dict(param=s["param"], copy=s["copy"], m=m, v=v)


# ---- one pass --------------------------------------------------------------------------------------------------------

@functools.lru_cache(maxsize=None)
def context():
    """The one context that a program keeps."""
    from paper_2605_13907_amd import binding
    return binding.AisContext()


def loss_params(case):
    from paper_2605_13907_amd import binding
    beta, kind, smooth, margin, mean = form_of(case)
    return binding.default_preference_params(beta=beta, kind=kind, label_smoothing=smooth, margin=margin, mean_logp=1 if mean else 0)


def optimizer(s):
    """The handle that a program keeps beside its weights."""
    if "optimizer" not in s:
        from paper_2605_13907_amd import binding
        s["optimizer"] = binding.AdamWState(s["params"], bits=s["case"]["bits"], copies=s["copies"], seed=s["seed"], step=s["step"],
                                            m=s["m"], v=s["v"], m_scale=s["m_scale"], v_scale=s["v_scale"])
    return s["optimizer"]


def run(state):
    case, s = state["case"], state
    kind = case["kind"]
    if not own:
        if kind == "scores":
            loss, reward, by = plain_scores(s, s["logp"])
            return dict(loss=loss, reward=reward, g=-by)
        return dict(pairs=plain_pairs, norm=plain_norm, norm_grad=plain_norm_grad, adamw=plain_adamw)[kind](s)
    ctx = context()
    if kind == "pairs":
        logp, lse = ctx.token_logprob(s["logits"], s["ids"], s["valid"])
        loss, reward, dlogits = ctx.preference_loss_grad(s["logits"], s["ids"], s["valid"], s["cu"], logp, lse, s["ref"],
                                                         loss_params(case), weight=s["weight"])
        return dict(loss=loss, reward=reward, dlogits=dlogits)
    if kind == "scores":
        loss, reward, g = ctx.preference_row_scale(s["logp"], s["ref"], s["valid"], s["cu"], loss_params(case), weight=s["weight"])
        return dict(loss=loss, reward=reward, g=g)
    if kind == "norm":
        y, mean, rstd = ctx.norm_rows(s["x"], s["weight"], s["bias"], eps=1e-5, centered=case["centered"])
        return dict(y=y, mean=mean, rstd=rstd)
    if kind == "norm_grad":
        dx, dweight, dbias = ctx.norm_rows_grad(s["dy"], s["x"], s["weight"], s["mean"], s["rstd"], want_bias=case["centered"])
        return dict(dx=dx, dweight=dweight, dbias=dbias)
    opt = optimizer(s)
    ctx.adamw_step(opt, s["grads"], lr=LR, beta1=BETA1, beta2=BETA2, eps=EPS, weight_decay=DECAY, grad_scale=s["grad_scale"])
    m, v = (opt.m, opt.v) if case["bits"] == 32 else ctx.adamw_values(opt, dtype=torch.bfloat16)
    return dict(param=s["param"], copy=s["copy"], m=m, v=v)


def work(case):
    kind = case["kind"]
    if kind == "adamw":
        n = sum(sizes_of(case))
        each = 2 * (2 if case["dtype"] == "bf16" else 4) + (2 if case["grad"] == "bf16" else 4) + (2 if case["copy"] else 0)
        # moments read and written, 8-bit ones with the values that are asked for
        each += 16 if case["bits"] == 32 else 4 + 4 / BLOCK + 4
        return dict(bytes=int(n * each), flops=15 * n)
    rows = case["rows"]
    if kind == "scores":
        return dict(bytes=int(rows * (8 * case["live"] + (1 if case["live"] < 1 else 0) + 4)) + 28 * case["pairs"], flops=4 * rows)
    e = 2 if case["dtype"] == "bf16" else 4
    if kind == "pairs":
        live = case["live"] * rows
        return dict(bytes=int(e * case["vocab"] * (live + rows)) + 9 * rows, flops=int(8 * live * case["vocab"]))
    width = case["width"]
    if kind == "norm":
        return dict(bytes=2 * e * rows * width + 8 * rows + 2 * e * width, flops=6 * rows * width)
    return dict(bytes=rows * width * (2 * e + (2 if case["dy"] == "bf16" else 4)) + 8 * rows + (8 + e) * width, flops=12 * rows * width)


# ---- the definitions in 64 bits --------------------------------------------------------------------------------------

def exact_scores(s, logp):
    """Response by response."""
    beta, kind, smooth, margin, mean = form_of(s["case"])
    cu = s["cu"].tolist()
    delta = logp.double() - s["ref"].double()
    live = torch.ones_like(delta) if s["valid"] is None else (s["valid"] != 0).double()
    rewards, loss, by = [], 0.0, torch.zeros_like(delta)
    # prefix sums would cancel: each response by itself
    sums = [float(x.sum()) for x in torch.split(delta * live, [b - a for a, b in zip(cu, cu[1:])])]
    counts = [float(x.sum()) for x in torch.split(live, [b - a for a, b in zip(cu, cu[1:])])]
    weight = s["weight"].double().tolist()
    for i, w in enumerate(weight):
        share = [(1.0 / counts[j] if counts[j] else 0.0) if mean else 1.0 for j in (2 * i, 2 * i + 1)]
        chosen, other = sums[2 * i] * share[0], sums[2 * i + 1] * share[1]
        rewards += [beta * chosen, beta * other]
        h = beta * (chosen - other) - margin
        if kind == 0:
            minus = -math.log1p(math.exp(-h)) if h > 0 else h - math.log1p(math.exp(h))       # log sigmoid(h)
            loss -= w * ((1.0 - smooth) * minus + smooth * (minus - h))
            slope = math.exp(minus) - (1.0 - smooth)
        elif kind == 1:
            loss += w * max(0.0, 1.0 - h)
            slope = -1.0 if h < 1.0 else 0.0
        else:
            loss += w * (chosen - other - margin / beta - 1.0 / (2.0 * beta)) ** 2
            slope = 2.0 * (chosen - other - margin / beta - 1.0 / (2.0 * beta)) / beta
        for j, sign in ((2 * i, 1.0), (2 * i + 1, -1.0)):
            by[cu[j]:cu[j + 1]] = sign * w * slope * beta * share[j - 2 * i]
    out = dict(loss=torch.tensor([loss], dtype=torch.float64), reward=torch.tensor(rewards, dtype=torch.float64))
    return out, by * live


def exact_pairs(s):
    z = s["logits"]
    logp = torch.cat([torch.log_softmax(x.double(), dim=1).gather(1, i.long().unsqueeze(1)).squeeze(1)
                      for x, i in zip(z.split(1024), s["ids"].split(1024))])
    out, by = exact_scores(s, logp)
    wide = torch.float64 if z.numel() < 4e8 else torch.float32
    grad = torch.empty(z.shape, dtype=wide, device=z.device)
    for r in range(0, z.shape[0], 1024):
        at = slice(r, r + 1024)
        hot = torch.nn.functional.one_hot(s["ids"][at].long(), z.shape[1])
        grad[at] = (by[at].unsqueeze(1) * (hot - torch.softmax(z[at].double(), dim=1))).to(wide)
    return dict(out, dlogits=grad)


def exact_norm(s):
    width, parts = s["case"]["width"], []
    for x in s["x"].split(4096):
        x = x.double()
        mean = x.mean(dim=1, keepdim=True) if s["case"]["centered"] else 0.0
        rstd = (((x - mean) ** 2).mean(dim=1, keepdim=True) + 1e-5) ** -0.5
        y = (x - mean) * rstd * s["weight"].double() + (0.0 if s["bias"] is None else s["bias"].double())
        parts.append((y, mean, rstd))
    return dict(y=torch.cat([p[0] for p in parts]), mean=torch.cat([p[1] for p in parts]).view(-1) if s["case"]["centered"] else None,
                rstd=torch.cat([p[2] for p in parts]).view(-1))


def exact_norm_grad(s):
    """The Jacobian of the normalised row, which takes out what lies along the ones and along the row itself."""
    centered, width = s["case"]["centered"], s["case"]["width"]
    dx, dweight, dbias = [], torch.zeros(width, dtype=torch.float64, device="cuda"), torch.zeros(width, dtype=torch.float64, device="cuda")
    for r in range(0, s["case"]["rows"], 4096):
        at = slice(r, r + 4096)
        x, dy, rstd = s["x"][at].double(), s["dy"][at].double(), s["rstd"][at].double()[:, None]
        n = (x - (s["mean"][at].double()[:, None] if centered else 0.0)) * rstd
        w = dy * s["weight"].double()
        along = torch.stack((n, torch.ones_like(n))) if centered else n[None]
        dx.append(rstd * (w - sum(a * (a * w).mean(dim=1, keepdim=True) for a in along)))
        dweight += torch.einsum("rd,rd->d", dy, n)
        dbias += dy.sum(dim=0)
    return dict(dx=torch.cat(dx), dweight=dweight, dbias=dbias if centered else None)


def product32(a, b):
    """The low 32 bits of a product, by halves."""
    low, high = a % 65536 * b, a // 65536 * b % 65536
    return (low + high * 65536) % 4294967296


def scrambled(a):
    a = product32(torch.bitwise_xor(a, a // 32768), ROOT2)
    return torch.bitwise_xor(a, a // 65536)


def exact_moment(value, random, bits, signed):
    """The value that `value` (32 bits wide) is rounded to: `bits` exponent bits above three of fraction, at a random side."""
    bias = 2 ** (bits - 1) - 1
    top, least = (7, 7) if signed else (15, 15)
    b = value.double().view(-1, BLOCK)
    a = b.abs()
    largest = a.max(dim=1, keepdim=True).values
    power = torch.where(largest > 0, torch.floor(torch.log2(largest)) - top, torch.full_like(largest, -1000.0)).clamp(min=least - 127.0)
    unit = torch.exp2(power)
    place = torch.floor(torch.log2(torch.clamp(a / unit, min=1e-300))).clamp(min=1.0 - bias)
    spacing = torch.exp2(place - 3.0) * unit
    below = torch.floor(a / spacing)
    up = (a / spacing - below) + random.double().view(-1, BLOCK) / 65536.0 >= 1.0
    out = (below + up.double()) * spacing
    if not signed:
        out = torch.where((a > 0) & (out == 0), spacing, out)
    return (torch.sign(b) * out).view(-1)


def exact_adamw(s):
    case, step = s["case"], s["step"] + 1
    scale, offsets = float(s["grad_scale"].double()), offsets_of(case)
    total = offsets[-1]
    param = torch.empty(total, dtype=torch.float64, device="cuda")
    # 8-bit moments are exact in bf16
    moments = [torch.empty(total, dtype=torch.float64 if case["bits"] == 32 else torch.bfloat16, device="cuda") for _ in range(2)]
    for t, (start, end) in enumerate(zip(offsets, offsets[1:])):
        for a in range(start, end, 1 << 25):
            at = slice(a, min(a + (1 << 25), end))
            g = s["grad"][at].double() * scale
            if case["bits"] == 32:
                old = s["m"][at].double(), s["v"][at].double()
            else:
                old = []
                blocks = slice(at.start // BLOCK, at.stop // BLOCK)
                for codes, powers, bias in ((s["m"][at] % 128, s["m_scale"], 7), (s["v"][at], s["v_scale"], 15)):
                    field, fraction = (codes // 8).double(), (codes % 8).double() / 8.0
                    x = torch.where(field > 0, (1.0 + fraction) * torch.exp2(field - bias), fraction * 2.0 ** (1 - bias))
                    old.append(x * torch.exp2(powers[blocks].double() - 127.0).repeat_interleave(BLOCK))
                old[0] = torch.where(s["m"][at] > 127, -old[0], old[0])
            m = BETA1 * old[0] + (1.0 - BETA1) * g
            v = BETA2 * old[1] + (1.0 - BETA2) * g ** 2
            p = s["param"][at].double()
            ahead = (m / (1.0 - BETA1 ** step)) / ((v / (1.0 - BETA2 ** step)) ** 0.5 + EPS)
            param[at] = p * (1.0 - LR * DECAY) - LR * ahead
            if case["bits"] == 8:
                key = torch.tensor(s["seed"], device="cuda") ^ product32(torch.tensor(step, device="cuda"), PHI)
                key = scrambled(scrambled(key) ^ product32(torch.tensor(t, device="cuda"), PHI))
                bits = scrambled(product32(torch.arange(at.start - start, at.stop - start, device="cuda"), PHI) ^ key)
                m, v = exact_moment(m.float(), bits % 65536, 4, True), exact_moment(v.float(), bits // 65536, 5, False)
            moments[0][at], moments[1][at] = m, v
    return dict(param=param, copy=param if case["copy"] else None, m=moments[0], v=moments[1])


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "scores":
        out, by = exact_scores(s, s["logp"])
        return dict(out, g=-by)
    return dict(pairs=exact_pairs, norm=exact_norm, norm_grad=exact_norm_grad, adamw=exact_adamw)[case["kind"]](s)
