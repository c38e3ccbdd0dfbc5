"""The oracle of the 4-bit rollout and the distillation loss against independent statements of the same definitions."""
import math

import numpy as np
import pytest
import torch

import oracle.rollout_oracle as O


def test_rounding_to_the_grid_by_hand():
    want = {0.0: 0, 0.25: 0, 0.2500001: 1, 0.5: 1, 0.75: 2, 1.0: 2, 1.25: 2, 1.26: 3, 1.5: 3, 1.75: 4, 2.5: 4, 2.51: 5, 3.5: 6,
            3.49: 5, 4.0: 6, 5.0: 6, 5.01: 7, 6.0: 7, 7.9: 7, 100.0: 7}
    for a, i in want.items():
        assert O.nearest_e2m1(a) == i, a


def test_block_scales_by_hand():
    x = np.zeros((1, 96))
    x[0, 0], x[0, 1] = 1.0, -0.3            # exponent of 1.0 is 0: scale 2^-2, 1.0 -> 4, -0.3 -> -1.2 -> -1
    x[0, 40] = 7.99                          # scale 1, saturates at 6
    codes, scales, values = O.mxfp4_quantize(x)
    assert scales.tolist() == [[125, 127, 0]]
    assert values[0, 0] == 1.0 and values[0, 1] == -0.25 and values[0, 40] == 6.0
    assert codes[0, 0] == 6 | (8 + 2) << 4 and codes[0, 20] == 7
    assert (O.mxfp4_values(codes, scales)[:, :96] == values).all()


def test_error_of_a_block_is_bounded():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((16, 128)) * np.exp(rng.standard_normal((16, 1)) * 4)
    _, scales, values = O.mxfp4_quantize(x)
    unit = np.repeat(2.0 ** (scales.astype(float) - 127), 32, axis=1)
    # half of the widest spacing, or what saturation at 6 leaves of numbers below 8
    assert (np.abs(values - x) <= unit * np.where(np.abs(x) > 6 * unit, 2.0, 1.0)).all()


@pytest.mark.parametrize("limits", [dict(), dict(top_k=3), dict(top_p=0.7), dict(min_p=0.2), dict(top_k=4, top_p=0.8),
                                    dict(top_p=0.9, min_p=0.1, temperature=0.5), dict(top_k=1), dict(temperature=0.0)])
def test_kept_tokens_by_brute_force(limits):
    rng = np.random.default_rng(2)
    for _ in range(50):
        z = rng.integers(-3, 4, 9) * 0.5
        kept, _, _ = O.kept_tokens(z, **limits)
        temperature = limits.get("temperature", 1.0)
        ranked = sorted(range(9), key=lambda v: (-z[v], v))
        p = torch.softmax(torch.tensor(z) / (temperature or 1.0), 0)
        want, within = [], ranked[:limits.get("top_k", 0) or 9]
        mass = sum(float(p[v]) for v in within)
        before = 0.0
        for v in within:
            if before < limits.get("top_p", 1.0) * mass and float(p[v]) >= limits.get("min_p", 0.0) * float(p.max()) - 1e-15:
                want.append(v)
            before += float(p[v])
        if temperature == 0.0:
            want = ranked[:1]
        assert kept.tolist() == want


def test_draws_follow_the_distribution():
    rng = np.random.default_rng(3)
    z = np.array([0.0, 1.0, -1.0, 2.0, 0.5])
    counts = np.zeros(5)
    n = 20_000
    for _ in range(n):
        counts[O.sample(z, rng.exponential(size=5), top_k=4)[0]] += 1
    p = np.exp(z) * (z > -1.0)
    p /= p.sum()
    assert (np.abs(counts / n - p) <= 5 * np.sqrt(p * (1 - p) / n)).all()


def test_rows_without_a_distribution():
    e = np.ones(3)
    for z in ([math.nan, 0, 0], [math.inf, 0, 0], [-math.inf] * 3):
        assert O.sample(np.array(z), e)[0] == -1
    assert O.sample(np.array([0.0, 1.0, 2.0]), e, temperature=-1.0)[0] == -1
    assert O.sample(np.array([-math.inf, 1.0, -math.inf]), e)[:2] == (1, 0.0)


def distill_loss(z, ids, teacher, weight, inv_t):
    """Torch float64, by its own log-softmax."""
    logp = torch.log_softmax(z * inv_t, dim=1)
    loss = z.new_zeros(())
    for r in range(z.shape[0]):
        on = ids[r] >= 0
        logq = torch.log_softmax(teacher[r][on] * inv_t, dim=0)
        loss = loss + weight[r] * (logq.exp() * (logq - logp[r][ids[r][on]])).sum()
    return loss


@pytest.mark.parametrize("inv_t", [1.0, 0.5, 2.0])
def test_distillation_gradient(inv_t):
    gen = torch.Generator().manual_seed(4)
    z = torch.randn(5, 17, generator=gen, dtype=torch.float64, requires_grad=True)
    ids = torch.stack([torch.randperm(17, generator=gen)[:6] for _ in range(5)])
    ids[1, 3:] = -1
    ids[2, 1] = ids[2, 0]                    # listed twice
    teacher = torch.randn(5, 6, generator=gen, dtype=torch.float64)
    weight = torch.rand(5, generator=gen, dtype=torch.float64)
    want = distill_loss(z, ids, teacher, weight, inv_t)
    want.backward()
    loss, kl, grad = O.distill(z.detach().numpy(), ids.numpy(), teacher.numpy(), weight.numpy(), inv_t)
    assert loss == pytest.approx(float(want.detach()), rel=1e-12)
    assert np.abs(grad - z.grad.numpy()).max() < 1e-13
    # ... and against differences
    h, zn = 1e-6, z.detach().numpy()
    for r, v in ((0, 0), (1, 5), (2, int(ids[2, 0])), (4, 16)):
        step = np.zeros_like(zn)
        step[r, v] = h
        up = O.distill(zn + step, ids.numpy(), teacher.numpy(), weight.numpy(), inv_t)[0]
        down = O.distill(zn - step, ids.numpy(), teacher.numpy(), weight.numpy(), inv_t)[0]
        assert (up - down) / (2 * h) == pytest.approx(grad[r, v], abs=1e-8)


def test_distillation_of_rows_without_a_teacher():
    z, ids = np.zeros((3, 4)), np.array([[-1, -1], [0, 1], [2, 3]])
    teacher = np.array([[0.0, 0.0], [-math.inf, -math.inf], [0.0, 1.0]])
    loss, kl, grad = O.distill(z, ids, teacher, np.ones(3), valid=np.array([1, 1, 0]))
    assert loss == 0 and not kl.any() and not grad.any()
