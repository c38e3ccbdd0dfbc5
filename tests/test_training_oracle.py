"""Pins of the 64-bit forms of the preference loss, the normalised rows and the AdamW step: gradients against differences, a step
by hand, the 8-bit grids, and roundings that keep the mean."""
import math

import numpy as np
import pytest

import oracle.training_oracle as O

FORMS = [dict(), dict(label_smoothing=0.2), dict(kind=1, margin=0.3), dict(kind=2, beta=0.5), dict(kind=2, mean_logp=1, beta=0.7, margin=0.1),
         dict(mean_logp=1, beta=2.0, inv_temperature=0.8)]


def batch(seed=0, rows=40):
    r = np.random.default_rng(seed)
    logp = -r.exponential(size=rows)
    cu = np.array([0, 7, 7, 18, 25, 39, 40])
    return logp, logp + 0.3 * r.standard_normal(rows), (r.random(rows) < 0.8).astype(np.uint8), cu, r.random(3)


@pytest.mark.parametrize("form", FORMS)
def test_preference_gradient_is_the_difference_of_losses(form):
    logp, ref, valid, cu, weight = batch()
    _, _, g = O.preference(logp, ref, valid, cu, weight, **form)
    for t in range(len(logp)):
        at = [logp.copy(), logp.copy()]
        at[0][t] -= 1e-6
        at[1][t] += 1e-6
        lo, hi = (O.preference(z, ref, valid, cu, weight, **form)[0] for z in at)
        assert -g[t] / form.get("inv_temperature", 1.0) == pytest.approx((hi - lo) / 2e-6, rel=1e-5, abs=1e-8)


def test_preference_by_hand():
    loss, reward, g = O.preference([-1.0, -2.0, -0.5], None, None, [0, 2, 3], None, beta=0.5)
    h = 0.5 * (-3.0 + 0.5)
    assert loss == pytest.approx(math.log(1 + math.exp(-h))) and list(reward) == [-1.5, -0.25]
    assert g == pytest.approx([0.5 / (1 + math.exp(h))] * 2 + [-0.5 / (1 + math.exp(h))])
    assert O.pair_loss(1.0, 1.0, 1, 0) == (0.0, 0.0) and O.pair_loss(0.25, 1.0, 1, 0) == (0.75, -1.0)
    for h in (-900.0, 900.0):
        assert O.pair_loss(h, 1.0, 0, 0.0) == (max(-h, 0.0), -1.0 if h < 0 else -math.exp(-900.0))


@pytest.mark.parametrize("centered", [True, False])
def test_norm_gradient_is_the_difference_of_losses(centered):
    r = np.random.default_rng(1)
    x, w, b, dy = r.standard_normal((5, 9)), r.standard_normal(9), r.standard_normal(9), r.standard_normal((5, 9))
    valid = np.array([1, 1, 0, 1, 1])
    y, mean, rstd = O.norm(x, w, b, 1e-3, centered, valid)
    dx, dw, db = O.norm_grad(dy, x, w, mean, rstd, valid)
    f = lambda x, w, b: (dy * O.norm(x, w, b, 1e-3, centered, valid)[0]).sum()
    for i in range(9):
        e = np.eye(9)[i] * 1e-6
        assert dw[i] == pytest.approx((f(x, w + e, b) - f(x, w - e, b)) / 2e-6, abs=1e-7)
        assert db[i] == pytest.approx((dy * valid[:, None]).sum(axis=0)[i])
        for row in range(5):
            d = np.zeros_like(x)
            d[row, i] = 1e-6
            assert dx[row, i] == pytest.approx((f(x + d, w, b) - f(x - d, w, b)) / 2e-6, abs=1e-7)


def test_a_step_by_hand():
    p, m, v = O.adamw([1.0], [2.0], [0.0], [0.0], 1, 0.1, weight_decay=0.5)
    # a first step has the gradient's sign for its direction
    assert p[0] == pytest.approx(1.0 - 0.1 * (0.5 + 1.0), rel=1e-7) and m[0] == np.float32(0.2) and v[0] == pytest.approx(0.004)


def test_grids():
    first, second = O.grid(1), O.grid(2)
    assert first[1] == 2.0 ** -9 and first[8] == 2.0 ** -6 and first[0x78] == 256.0 and first[128 + 9] == -first[9]
    assert second[1] == 2.0 ** -17 and second[8] == 2.0 ** -14 and second[255] == 1.875 * 2.0 ** 16
    assert (np.diff(second) > 0).all() and (np.diff(first[:128]) > 0).all()


@pytest.mark.parametrize("moment", [1, 2])
def test_codes_stay_codes(moment):
    """A value that a code stands for keeps it whatever the random number, under the scale that its block then has."""
    r = np.random.default_rng(2)
    codes = r.integers(0, 0x78 if moment == 1 else 247, 320).astype(np.uint8)
    codes[::32] = 0x77 if moment == 1 else 246
    x = O.decode(codes, np.full(10, 100), moment)
    got, scales = O.encode(x.astype(np.float32), np.full(320, 65535), moment)
    assert (O.decode(got, scales, moment) == x).all()


@pytest.mark.parametrize("moment", [1, 2])
def test_the_mean_is_kept(moment):
    """Of 4,096 roundings of one value with the steps' random numbers the mean is the value, within five deviations of its own: a
    rounding is off by one of two amounts that sum to a step, half a step being the most that they deviate."""
    r = np.random.default_rng(3)
    x = (r.standard_normal(256) if moment == 1 else r.standard_normal(256) ** 2 + 1e-4).astype(np.float32)
    total = np.zeros(256)
    for step in range(1, 4097):
        bits = O.random_bits(256, 0, step, 11)
        codes, scales = O.encode(x, bits & np.uint64(65535) if moment == 1 else bits >> np.uint64(16), moment)
        total += O.decode(codes, scales, moment)
    step = np.maximum(2.0 ** (np.floor(np.log2(np.abs(x))) - 3), np.repeat(np.abs(x).reshape(-1, 32).max(axis=1), 32) * 2.0 ** -15)
    assert (np.abs(total / 4096 - x) <= 5 * 0.5 * step / 64 + step * 2.0 ** -16).all()


def test_slow_averages_move():
    """What nearest rounding would hold in place: an average whose steps are a hundredth of a code's spacing reaches its end."""
    v = np.full(32, 1.0, dtype=np.float32)
    codes, scales = O.encode(v, np.zeros(32), 2)
    for step in range(1, 3001):
        new = (0.999 * O.decode(codes, scales, 2) + 0.001 * 4.0).astype(np.float32)
        codes, scales = O.encode(new, O.random_bits(32, 0, step, 5) >> np.uint64(16), 2)
    want = 4.0 - 3.0 * 0.999 ** 3000
    # a code's spacing there is 1/8 to 1/4: the deviation of an average over 1 / (2 * 0.001) steps of roundings is below 0.25 / 2 / 0.04^(1/2)
    assert abs(O.decode(codes, scales, 2).mean() - want) <= 0.5
