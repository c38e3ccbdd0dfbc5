"""CPU fp64 oracle of the 4-bit rollout and of the distillation loss: MXFP4 rows and their product, the draw of a token under
temperature, top-k, top-p and min-p from given random numbers, and the divergence from a teacher's top logits with its
gradient.  Written from the definitions, one row at a time where that is the definition; shares no code with csrc/."""
from __future__ import annotations

import math

import numpy as np

BLOCK = 32
E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def nearest_e2m1(a):
    """Index of the E2M1 magnitude nearest to a >= 0 (ties to the even index), saturating at the largest."""
    a = np.asarray(a, dtype=np.float64)
    below = np.clip(np.searchsorted(E2M1, a, side="right") - 1, 0, 7)
    above = np.minimum(below + 1, 7)
    to_below, to_above = a - E2M1[below], E2M1[above] - a
    up = (to_above < to_below) | ((to_above == to_below) & (below % 2 == 1))
    return np.where((below < 7) & up, above, below)


def mxfp4_quantize(x):
    """x [R, D] -> (codes [R, 16 nb] uint8, scales [R, nb] uint8, values [R, D] float64)."""
    x = np.asarray(x, dtype=np.float64)
    rows, width = x.shape
    blocks = -(-width // BLOCK)
    full = np.zeros((rows, blocks * BLOCK))
    full[:, :width] = x
    full = full.reshape(rows, blocks, BLOCK)
    index = np.zeros(full.shape, dtype=np.uint8)
    scales = np.zeros((rows, blocks), dtype=np.uint8)
    values = np.zeros(full.shape)
    for r in range(rows):
        for b in range(blocks):
            block = full[r, b]
            if not np.isfinite(block).all():
                scales[r, b] = 255
                values[r, b] = np.nan
                continue
            largest = np.abs(block).max()
            e = max(math.frexp(largest)[1] - 1 - 2, -127) if largest > 0 else -127
            mag = nearest_e2m1(np.abs(block) / 2.0 ** e)
            index[r, b] = mag + 8 * np.signbit(block)
            scales[r, b] = e + 127
            values[r, b] = np.copysign(E2M1[mag], block) * 2.0 ** e
    index = index.reshape(rows, blocks * 16, 2)
    return index[..., 0] | index[..., 1] << 4, scales, values.reshape(rows, -1)[:, :width]


def mxfp4_values(codes, scales):
    """What codes [R, 16 nb] and scales [R, nb] stand for, [R, 32 nb] float64 (NaN where the scale is 255)."""
    codes = np.asarray(codes)
    index = np.stack((codes & 15, codes >> 4), axis=2).reshape(codes.shape[0], -1)
    v = np.where(index >= 8, -1.0, 1.0) * E2M1[index & 7]
    scale = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127.0))
    return v * np.repeat(scale, BLOCK, axis=1)


def mxfp4_logits(hidden, weight):
    """Both operands as (codes, scales) -> logits [R, V]."""
    return mxfp4_values(*hidden) @ mxfp4_values(*weight).T


def kept_tokens(z, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(kept tokens in ranked order, their t - max t, log of the row's sum of exp(t - max t)), or None for a row without a
    distribution."""
    z = np.asarray(z, dtype=np.float64)
    if np.isnan(z).any() or np.isposinf(z).any() or np.isneginf(z).all() or not temperature >= 0 or math.isinf(temperature) \
            or math.isnan(top_p) or math.isnan(min_p):
        return None
    finite = np.flatnonzero(np.isfinite(z))
    order = finite[np.argsort(-z[finite], kind="stable")]
    t = (z[order] - z[order[0]]) / (temperature if temperature > 0 else 1.0)
    mass = np.exp(t)
    log_total = math.log(mass.sum())
    if temperature == 0 or top_p <= 0 or min_p > 1:
        return order[:1], t[:1], log_total
    n = len(order)
    if top_k > 0:
        n = min(n, top_k)
    if top_p < 1:
        before = np.concatenate(([0.0], np.cumsum(mass[:n])))[:n]
        target = top_p * mass[:n].sum()
        n = int((before < target).sum())
    if min_p > 0:
        n = min(n, int((t >= math.log(min_p)).sum()))
    return order[:n], t[:n], log_total


def sample(z, noise, **limits):
    """(token, logp, logp_full, lead of the winner's score over the next one's) of one row."""
    kept = kept_tokens(z, **limits)
    if kept is None:
        return -1, 0.0, 0.0, math.inf
    order, t, log_total = kept
    if limits.get("temperature", 1.0) == 0:
        return int(order[0]), 0.0, 0.0, math.inf
    e = np.asarray(noise, dtype=np.float64)[order]
    e = np.where(np.isnan(e), 3.0e38, np.clip(e, float(np.float32(1.17549435e-38)), 3.0e38))
    score = t - np.log(e)
    best = np.lexsort((order, -score))
    lead = score[best[0]] - score[best[1]] if len(best) > 1 else math.inf
    at = best[0]
    return int(order[at]), t[at] - math.log(np.exp(t).sum()), t[at] - log_total, lead


def distill(z, ids, teacher, weight, inv_temperature=1.0, valid=None):
    """(loss, kl [R], dlogits [R, V]): divergence from the teacher's listed tokens and the gradient of sum weight kl."""
    z = np.asarray(z, dtype=np.float64)
    rows, vocab = z.shape
    kl, grad = np.zeros(rows), np.zeros((rows, vocab))
    for r in range(rows):
        listed = (ids[r] >= 0) & (ids[r] < vocab)
        t = np.asarray(teacher[r], dtype=np.float64)[listed] * inv_temperature
        if (valid is not None and not valid[r]) or not listed.any() or np.isneginf(t).all():
            continue
        with np.errstate(invalid="ignore", divide="ignore"):
            q = np.exp(t - t.max())
            q /= q.sum()
            s = z[r] * inv_temperature
            logp = s - s.max() - math.log(np.exp(s - s.max()).sum())
            some = ~(q == 0)
            kl[r] = (q[some] * (np.log(q[some]) - logp[ids[r][listed][some]])).sum()
            grad[r] = np.exp(logp)
            np.add.at(grad[r], ids[r][listed], -q)
            grad[r] *= weight[r] * inv_temperature
    live = np.ones(rows, dtype=bool) if valid is None else np.asarray(valid) != 0
    return float((np.asarray(weight, dtype=np.float64) * kl)[live].sum()), kl, grad
