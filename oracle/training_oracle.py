"""Plain 64-bit forms of the operators on either side of the read-out: the preference loss over pairs of responses, normalised rows
and their gradient, an AdamW step with moments of 32 or 8 bits.  numpy only."""
import math

import numpy as np

BLOCK = 32
M32 = 0xFFFFFFFF


# ---- preference loss -------------------------------------------------------------------------------------------------

def pair_loss(h, beta, kind, smoothing):
    """(loss, its derivative) at h."""
    if math.isnan(h):
        return h, h
    if kind == 0:
        log_up = -math.log1p(math.exp(-h)) if h >= 0 else h - math.log1p(math.exp(h))           # log sigmoid(h)
        log_down = -math.log1p(math.exp(h)) if h < 0 else -h - math.log1p(math.exp(-h))
        return -(1 - smoothing) * log_up - smoothing * log_down, -(1 - smoothing) * math.exp(log_down) + smoothing * math.exp(log_up)
    if kind == 1:
        return max(0.0, 1.0 - h), -1.0 if h < 1.0 else 0.0
    return ((h - 0.5) / beta) ** 2, 2.0 * (h - 0.5) / beta ** 2


def preference(logp, ref, valid, cu, weight=None, beta=0.1, kind=0, label_smoothing=0.0, margin=0.0, mean_logp=0, inv_temperature=1.0):
    """(loss, reward [B], g [R]); g is minus the derivative of the loss by each row's log-probability, times inv_temperature."""
    logp = np.asarray(logp, dtype=np.float64)
    ref = np.zeros_like(logp) if ref is None else np.asarray(ref, dtype=np.float64)
    live = np.ones(logp.shape, dtype=bool) if valid is None else np.asarray(valid) != 0
    n = len(cu) - 1
    weight = np.full(n // 2, 2.0 / n) if weight is None else np.asarray(weight, dtype=np.float64)
    d, share = np.zeros(n), np.ones(n)
    for i in range(n):
        rows = np.arange(cu[i], cu[i + 1])
        rows = rows[live[rows]]
        d[i] = math.fsum(logp[rows] - ref[rows]) if np.isfinite(logp[rows] - ref[rows]).all() else (logp[rows] - ref[rows]).sum()
        if mean_logp:
            share[i] = 1.0 / len(rows) if len(rows) else 0.0
        d[i] *= share[i]
    loss, g = 0.0, np.zeros_like(logp)
    with np.errstate(invalid="ignore"):
        for p in range(n // 2):
            h = beta * (d[2 * p] - d[2 * p + 1]) - margin
            value, slope = pair_loss(h, beta, kind, label_smoothing)
            loss += weight[p] * value
            for i, sign in ((2 * p, -1.0), (2 * p + 1, 1.0)):
                rows = np.arange(cu[i], cu[i + 1])
                g[rows] = np.where(live[rows], sign * weight[p] * slope * beta * share[i] * inv_temperature, 0.0)
    return loss, beta * d, g


# ---- normalised rows -------------------------------------------------------------------------------------------------

def norm(x, weight, bias, eps, centered, valid=None):
    """(y, mean or None, rstd)."""
    x = np.array(x, dtype=np.float64)
    live = np.ones(len(x), dtype=bool) if valid is None else np.asarray(valid) != 0
    x[~live] = 0.0
    mean = x.mean(axis=1) if centered else np.zeros(len(x))
    rest = x - mean[:, None]
    rstd = 1.0 / np.sqrt((rest ** 2).mean(axis=1) + eps)
    y = rest * rstd[:, None] * (1.0 if weight is None else weight) + (0.0 if bias is None else bias)
    y[~live], rstd[~live] = 0.0, 0.0
    return y, mean if centered else None, rstd


def norm_grad(dy, x, weight, mean, rstd, valid=None):
    """(dx, dweight, dbias)."""
    live = np.ones(len(x), dtype=bool) if valid is None else np.asarray(valid) != 0
    x, dy = np.where(live[:, None], x, 0.0).astype(np.float64), np.where(live[:, None], dy, 0.0).astype(np.float64)
    rstd = np.where(live, rstd, 0.0).astype(np.float64)[:, None]
    n = (x - (0.0 if mean is None else np.where(live, mean, 0.0)[:, None])) * rstd
    u = dy * (1.0 if weight is None else weight)
    dx = u - n * (u * n).mean(axis=1, keepdims=True)
    if mean is not None:
        dx = dx - u.mean(axis=1, keepdims=True)
    return dx * rstd, (dy * n).sum(axis=0), dy.sum(axis=0)


# ---- AdamW -----------------------------------------------------------------------------------------------------------

def mix(x):
    x = ((x ^ (x >> 15)) * 0x6A09E667) & M32
    return x ^ (x >> 16)


def random_bits(n, tensor, step, seed):
    """32 bits for every element of a tensor."""
    key = mix(mix(seed ^ (step * 0x9E3779B1 & M32)) ^ (tensor * 0x9E3779B1 & M32))
    i = np.arange(n, dtype=np.uint64)
    return mix((i * np.uint64(0x9E3779B1) & np.uint64(M32)) ^ np.uint64(key))


def grid(moment):
    """Values of the 256 codes under a scale of 1."""
    bits, bias = (7, 7) if moment == 1 else (8, 15)
    out = []
    for c in range(256):
        a = c & (1 << bits) - 1
        v = a % 8 / 8 * 2.0 ** (1 - bias) if a < 8 else (1 + a % 8 / 8) * 2.0 ** (a // 8 - bias)
        out.append(-v if c >> bits else v)
    return np.array(out)


def decode(codes, scales, moment):
    codes, n = np.asarray(codes), len(codes)
    scales = np.asarray(scales).astype(np.int64)
    power = np.where(scales == 255, np.nan, 2.0 ** (scales - 127.0))
    with np.errstate(invalid="ignore"):
        return grid(moment)[codes] * np.repeat(power, BLOCK)[:n]


def encode(x, random16, moment):
    """x fp32 [n] -> (codes, scales): each value goes to one of the two codes beside it."""
    n, top = len(x), 7 if moment == 1 else 15
    bias = top
    nb = -(-n // BLOCK)
    full = np.zeros(nb * BLOCK, dtype=np.float64)
    full[:n] = x
    rnd = np.zeros(nb * BLOCK)
    rnd[:n] = random16
    a = np.abs(full).reshape(nb, BLOCK)
    largest = a.max(axis=1)                                  # NaN if any is
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        e = np.where(largest > 0, np.frexp(largest)[1] - 1 + 127, 0)
        e = np.maximum(e, 0)                                 # subnormal fp32 numbers
        scale = np.where(np.isfinite(largest), np.maximum(e - top, top), 255)
        t = a / np.where(scale == 255, 1.0, 2.0 ** (scale - 127.0))[:, None]
        place = np.maximum(np.where(t > 0, np.frexp(t)[1] - 1, 1 - bias), 1 - bias)
        k = np.floor(t / 2.0 ** (place - 3.0) + rnd.reshape(nb, BLOCK) / 65536.0)
        code = k + 8 * (place - (1 - bias))
        if moment == 2:
            code = np.where((t > 0) & (code < 1), 1, code)
        code = np.where(scale[:, None] == 255, 0, code)
    code = code.astype(np.int64).reshape(-1)[:n]
    if moment == 1:
        code = code + np.where(np.signbit(full[:n]) & (np.repeat(scale, BLOCK)[:n] != 255), 128, 0)
    return code.astype(np.uint8), scale.astype(np.uint8)


def adamw(p, g, m, v, step, lr, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01, grad_scale=1.0):
    """(p, m, v): the moments as fp32 numbers, the parameters in 64 bits."""
    p, g = np.asarray(p, dtype=np.float64), np.asarray(g, dtype=np.float64) * grad_scale
    with np.errstate(invalid="ignore", over="ignore", divide="ignore"):
        m = (beta1 * np.asarray(m, dtype=np.float64) + (1 - beta1) * g).astype(np.float32)
        v = (beta2 * np.asarray(v, dtype=np.float64) + (1 - beta2) * g * g).astype(np.float32)
        ahead = m.astype(np.float64) / (1 - beta1 ** step) / (np.sqrt(v.astype(np.float64) / (1 - beta2 ** step)) + eps)
        return p - lr * (weight_decay * p + ahead), m, v
