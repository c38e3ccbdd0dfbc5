"""Token sampling on the GPU against the fp64 oracle.

The drawn token has to be the oracle's, except where fp32 cannot tell: the winner's score leads the next one's by less than
2e-5 (scores are of the size of t = (z - max z) / T, |t| < 90 for any token with a chance, so two roundings of 2^-24 |t| and the
logarithm's stay below 2e-5).  Top-p and min-p decide by masses that are 2^-23 off each: what the oracle draws with top_p and
min_p 1e-6 lower or higher is right as well, and log-probs lie between the oracle's, give or take 2e-5 + 3e-7 |t| (for
temperatures that make t large)."""
import math

import numpy as np
import pytest
import torch

import oracle.rollout_oracle as O
from paper_2605_13907_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = B.AisContext()
    yield c
    c.close()


def limits_of(limits, r):
    out = {}
    for name, v in limits.items():
        if v is not None:
            x = v[r].item() if isinstance(v, torch.Tensor) else v
            out[name] = int(x) if name == "top_k" else float(x)
    if out.get("top_k", 1) < 0:
        out["top_k"] = 0
    return out


def check(ctx, z, noise, valid=None, **limits):
    """Compares every row; returns the tokens."""
    ctx.status()
    token, logp, full = ctx.sample_tokens(z, noise, valid, **limits)
    assert token.dtype == torch.int32 and logp.dtype == torch.float32 and full.dtype == torch.float32
    got, lp, lf = token.cpu().numpy(), logp.double().cpu().numpy(), full.double().cpu().numpy()
    zs, es = z.double().cpu().numpy(), noise.double().cpu().numpy()
    unclear, bad = 0, False
    for r in range(z.shape[0]):
        if valid is not None and not valid[r]:
            assert (got[r], lp[r], lf[r]) == (-1, 0.0, 0.0)
            continue
        lim = limits_of(limits, r)
        wants = [O.sample(zs[r], es[r], **{**lim, **{n: lim[n] * (1 + d) for n in ("top_p", "min_p") if 0 < lim.get(n, 0) < 1}})
                 for d in (0.0, 1e-6, -1e-6)]
        if wants[0][0] < 0:
            assert (got[r], lp[r], lf[r]) == (-1, 0.0, 0.0), r
            bad = True
            continue
        if wants[0][3] < 2e-5:
            unclear += 1
            continue
        mine = [w for w in wants if w[0] == got[r]]
        assert mine, (r, lim, got[r], wants)
        t = (zs[r][got[r]] - zs[r][np.isfinite(zs[r])].max()) / (lim.get("temperature", 1.0) or 1.0)
        tol = 2e-5 + 3e-7 * abs(t)
        for have, k in ((lp[r], 1), (lf[r], 2)):
            assert min(w[k] for w in mine) - tol <= have <= max(w[k] for w in mine) + tol, (r, lim, have, mine)
    assert bool(ctx.status() & B.STATUS_BAD_ROW) == bad
    assert unclear <= 0.02 * z.shape[0] + 1
    return got


def logits(rows, vocab, dtype, seed, scale=3.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    z = torch.randn(rows, vocab, generator=gen, device="cuda") * scale
    e = torch.empty(rows, vocab, device="cuda").exponential_(generator=gen)
    return z.to(dtype), e


LIMITS = [dict(), dict(temperature=0.7), dict(top_k=1), dict(top_k=20), dict(top_p=0.9), dict(min_p=0.05), dict(temperature=0.0),
          dict(top_k=50, top_p=0.8), dict(top_k=40, top_p=0.95, min_p=0.02, temperature=1.3), dict(top_p=0.99, min_p=0.001),
          dict(top_k=100_000_000), dict(top_p=1.0, min_p=0.0, top_k=0), dict(top_p=0.0), dict(min_p=1.0), dict(min_p=2.0),
          dict(top_p=-1.0, top_k=-5)]


@pytest.mark.parametrize("limits", LIMITS)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("vocab", [1, 2, 9, 64, 1000, 5003, 33_000])
def test_limits(ctx, dtype, vocab, limits):
    check(ctx, *logits(6, vocab, dtype, vocab), **limits)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("limits", [dict(top_k=20, top_p=0.9), dict(top_p=0.95), dict(top_k=3000), dict()])
def test_wide_vocabulary(ctx, dtype, limits):
    check(ctx, *logits(2, 262_144, dtype, 7), **limits)


@pytest.mark.parametrize("limits", [dict(top_k=700), dict(top_k=3000), dict(top_k=9000, top_p=0.6), dict(top_p=0.5),
                                    dict(top_p=0.999), dict(top_k=2049), dict(min_p=0.5), dict(top_k=5000, min_p=0.9),
                                    dict(top_k=4000, top_p=0.7, min_p=0.4, temperature=2.0)])
@pytest.mark.parametrize("kind", ["equal", "two", "steps", "flat"])
def test_many_tokens_kept(ctx, kind, limits):
    """More tokens than are sorted at once, and equal ones on both sides of a cut: the lower indices are kept."""
    vocab = 20_000
    z, e = logits(4, vocab, torch.float32, 11)
    if kind == "equal":
        z = torch.full_like(z, 1.5)
    elif kind == "two":
        z = torch.where(z > 0, torch.full_like(z, 0.25), torch.full_like(z, -0.25))
    elif kind == "steps":
        z = torch.round(z)
    else:
        z = z * 0.01
    check(ctx, z.to(torch.bfloat16 if kind != "flat" else torch.float32), e, **limits)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("vocab", [1, 4, 9, 70, 5000, 30_000])
@pytest.mark.parametrize("value", [0.0, 1e-45, -1e-45, 1.0, -1.0])
def test_rows_of_one_value(ctx, dtype, vocab, value):
    """The cut lies behind the last token of a value; a zero of either sign is a zero."""
    z, e = logits(4, vocab, dtype, 83)
    z = torch.full_like(z, value) * torch.where(z > 0, 1.0, -1.0 if value == 0.0 else 1.0).to(dtype)
    for limits in (dict(top_p=0.99), dict(top_p=0.9999, min_p=1.0), dict(top_p=0.3), dict(top_k=vocab - 1, top_p=0.9999),
                   dict(top_k=max(vocab // 2, 1)), dict(min_p=1.0)):
        check(ctx, z, e, **limits)


@pytest.mark.parametrize("limits", [dict(top_p=0.97), dict(top_k=6000), dict(top_k=9000, top_p=0.9), dict(min_p=0.5),
                                    dict(top_p=0.97, min_p=0.6), dict(top_k=7000, min_p=0.6), dict(top_p=0.3)])
@pytest.mark.parametrize("centre", [0.0, 1e-12, -5.0, 100.0, -3e4, 4e9, -4e9])
def test_flat_rows_of_few_values(ctx, centre, limits):
    """bf16 rows whose every token is about as likely, at both ends of the values that are told apart and beyond them."""
    z, e = logits(3, 30_001, torch.float32, 31, scale=1.0)
    spread = max(0.02 * abs(centre), 1e-14)
    z = (centre + spread * z).to(torch.bfloat16)
    z[1, 5::7] = -math.inf
    z[2, :20_000] = z[2, 0]
    check(ctx, z, e, temperature=2.5 * spread, **limits)


def test_the_cut_between_equal_logits(ctx):
    """2,500 equal logits, the random numbers favour the last of those kept."""
    for k in (1, 2, 63, 64, 65, 1000, 1024, 1025, 2048, 2049, 2499, 2500):
        z = torch.zeros(1, 2500, device="cuda")
        e = torch.ones(1, 2500, device="cuda")
        e[0, k - 1], e[0, k:] = 0.5, 0.25
        token, logp, full = ctx.sample_tokens(z, e, top_k=k)
        assert token.item() == k - 1
        assert logp.item() == pytest.approx(-math.log(k), abs=1e-5) and full.item() == pytest.approx(-math.log(2500), abs=1e-5)
    for n in (1, 10, 999, 2100):
        z = torch.zeros(1, 2500, device="cuda")
        e = torch.ones(1, 2500, device="cuda")
        e[0, n - 1], e[0, n:] = 0.5, 0.25
        assert ctx.sample_tokens(z, e, top_p=(n - 0.5) / 2500)[0].item() == n - 1


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_limits_of_each_row(ctx, dtype):
    z, e = logits(40, 4001, dtype, 13)
    gen = torch.Generator(device="cuda").manual_seed(5)

    def pick(values, kind):
        return torch.tensor(values, dtype=kind, device="cuda")[torch.randint(0, len(values), (40,), generator=gen, device="cuda")]

    valid = (torch.arange(40, device="cuda") % 5 != 3).to(torch.uint8)
    check(ctx, z, e, valid, temperature=pick([0.0, 0.5, 1.0, 1.7], torch.float32), top_k=pick([0, -1, 1, 7, 400, 3000], torch.int32),
          top_p=pick([0.3, 0.9, 1.0, 1.5], torch.float32), min_p=pick([0.0, 0.01, 0.3], torch.float32))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("limits", [dict(), dict(top_k=5), dict(top_p=0.9), dict(min_p=0.1), dict(temperature=0.0), dict(top_k=900)])
def test_masks(ctx, dtype, limits):
    z, e = logits(12, 777, dtype, 17)
    lowest = torch.finfo(dtype).min
    z[0] = -math.inf                          # nothing is left
    z[1] = -math.inf
    z[1, 400] = -3.0                          # one is
    z[2, 100:] = -math.inf
    z[3, :700] = -math.inf
    z[4, 5] = math.nan
    z[5, 5] = math.inf
    z[6, 5:9] = math.inf
    z[7, 300:] = lowest
    z[8, 1:] = lowest
    z[9] = -math.inf
    z[9, ::100] = 2.0
    z[10] = math.nan
    got = check(ctx, z, e, **limits)
    assert got[1] == 400 and got[8] == 0 and got[2] < 100 and got[3] >= 700 and got[7] < 300 and got[9] % 100 == 0
    assert (got[[0, 4, 5, 6, 10]] == -1).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("limits", [dict(), dict(top_k=5), dict(top_p=0.9), dict(min_p=0.1), dict(temperature=0.0), dict(top_k=900),
                                    dict(temperature=5.0, top_p=0.5), dict(top_p=0.7, min_p=0.2)])
@pytest.mark.parametrize("vocab", [9, 777, 40_001])
def test_logits_as_large_as_the_type_holds(ctx, dtype, vocab, limits):
    z, e = logits(7, vocab, dtype, 61)
    lowest, most = torch.finfo(dtype).min, torch.finfo(dtype).max
    z[0] = lowest                              # nothing but masked tokens, all alike
    z[1] = lowest
    z[1, ::3] = -math.inf
    z[2] = most
    z[3, :] = lowest
    z[3, 5] = most
    z[4] = z[4] * 1e30                         # one token takes everything, its products with 1 / T fit
    z[5] = 1e10
    z[6] = lowest
    z[6, vocab - 1] = math.nan
    got = check(ctx, z, e, **limits)
    assert got[3] == 5 and got[1] % 3 != 0 and got[6] == -1


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("limits", [dict(), dict(top_k=5), dict(top_p=0.9), dict(min_p=0.1), dict(top_k=900)])
@pytest.mark.parametrize("temperature", [0.3, 1.6, 1.7, 5.0, 1000.0])
def test_lowest_masks_at_any_temperature(ctx, dtype, limits, temperature):
    z, e = logits(6, 30_000, dtype, 73)
    lowest = torch.finfo(dtype).min
    for r, left in enumerate((1, 2, 40, 1000, 20_000)):
        z[r, left:] = lowest
    z[5, 100:] = lowest
    z[5, 20_000:] = -math.inf
    check(ctx, z, e, temperature=temperature, **limits)


def test_temperatures_as_small_as_there_are(ctx):
    z, e = logits(4, 3000, torch.float32, 67)
    temperature = torch.tensor([1e-9, 1e-30, 1e-38, 1e-44], device="cuda")
    for limits in (dict(), dict(top_k=5), dict(top_p=0.9)):
        token, logp, full = ctx.sample_tokens(z, e, temperature=temperature, **limits)
        assert torch.equal(token.long(), z.argmax(dim=1)) and not logp.any() and not full.any()
    assert ctx.status() == 0


def test_limits_without_a_meaning(ctx):
    z, e = logits(8, 100, torch.float32, 19)
    nan, inf = math.nan, math.inf
    f = lambda *v: torch.tensor(v, device="cuda")  # noqa: E731
    token, logp, full = ctx.sample_tokens(z, e, temperature=f(1.0, -1.0, nan, inf, 1.0, 1.0, 1.0, 0.0),
                                          top_p=f(1.0, 1.0, 1.0, 1.0, nan, 1.0, 0.5, 0.5),
                                          min_p=f(0.0, 0.0, 0.0, 0.0, 0.0, nan, 0.0, 0.0))
    assert (token.cpu().numpy() == -1).tolist() == [False, True, True, True, True, True, False, False]
    assert not logp[1:6].any() and not full[1:6].any()
    assert ctx.status() == B.STATUS_BAD_ROW


def test_random_numbers_outside_their_range(ctx):
    z = torch.zeros(5, 300, device="cuda")
    e = torch.ones(5, 300, device="cuda")
    e[0, 7] = 0.0                              # as the smallest number
    e[1] = math.inf
    e[1, 9] = 2.0
    e[2] = math.nan
    e[2, 11] = 5.0
    e[3, 13] = -1.0
    e[4] = math.nan                            # all as the largest: equal scores, the lowest index
    for limits in (dict(), dict(top_k=200)):
        assert ctx.sample_tokens(z, e, **limits)[0].tolist() == [7, 9, 11, 13, 0]


def test_small_temperatures(ctx):
    z, e = logits(20, 3000, torch.float32, 23)
    check(ctx, z, e, temperature=0.05)
    check(ctx, z, e, temperature=0.05, top_p=0.9)
    check(ctx, z, e, temperature=1e-3, top_k=30)
    check(ctx, z * 1e-3, e, temperature=1e-3, top_k=30)
    check(ctx, z + 1000.0, e, top_p=0.9)
    check(ctx, z, e, temperature=50.0, top_p=0.5)


@pytest.mark.parametrize("vocab", [700, 40_000])
def test_scores_that_a_large_offset_would_round_to_one(ctx, vocab):
    """x / T is up to 1e6, where floats lie 1/16 apart: many tokens of a row, of one thread too, come that near its best."""
    z, e = logits(12, vocab, torch.float32, 59)
    check(ctx, 1000.0 + z * 1e-3, e, temperature=1e-3)
    check(ctx, z * 1e-3 - 1000.0, e, temperature=1e-3)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("offset", [0, 1, 3, 7, 33])
def test_rows_that_begin_anywhere(ctx, dtype, offset):
    z, e = logits(5, 2100, dtype, 29)
    z = z[:, offset:offset + 1999]
    e = e[:, offset:offset + 1999]
    check(ctx, z, e)
    check(ctx, z, e, top_k=30, top_p=0.9)
    check(ctx, z, e, top_p=0.95)
    check(ctx, z[:, :5], e[:, :5], top_p=0.95)


def test_same_answer_every_time(ctx):
    z, e = logits(64, 40_000, torch.bfloat16, 31)
    for limits in (dict(), dict(top_p=0.999), dict(top_k=5000, top_p=0.9), dict(top_k=64)):
        first = ctx.sample_tokens(z, e, **limits)
        for _ in range(3):
            assert all(torch.equal(a, b) for a, b in zip(first, ctx.sample_tokens(z, e, **limits)))


def test_draws_follow_the_distribution(ctx):
    """20,000 draws of one row: counts within five standard deviations of what top-k leaves."""
    n, vocab = 20_000, 50
    gen = torch.Generator(device="cuda").manual_seed(1)
    row = torch.randn(1, vocab, generator=gen, device="cuda")
    e = torch.empty(n, vocab, device="cuda").exponential_(generator=gen)
    token, logp, _ = ctx.sample_tokens(row.expand(n, vocab).contiguous(), e, temperature=0.8, top_k=12)
    p = torch.softmax(row[0].double() / 0.8, 0)
    kept = torch.topk(p, 12).indices
    q = torch.zeros_like(p)
    q[kept] = p[kept] / p[kept].sum()
    share = torch.bincount(token.long(), minlength=vocab).double() / n
    assert ((share - q).abs() <= 5 * torch.sqrt(q * (1 - q) / n)).all()
    assert (logp.double() - torch.log(q)[token.long()]).abs().max() < 2e-5


def test_no_rows_streams_and_graphs(ctx):
    z, e = logits(0, 10, torch.float32, 1)
    assert [t.shape for t in ctx.sample_tokens(z, e)] == [(0,)] * 3
    z, e = logits(9, 5000, torch.bfloat16, 37)
    p = torch.full((9,), 0.9, device="cuda")
    want = ctx.sample_tokens(z, e, top_p=p)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = ctx.sample_tokens(z, e, top_p=p)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = ctx.sample_tokens(z, e, top_p=p)
    for seed in range(4):
        new = logits(9, 5000, torch.bfloat16, 40 + seed)
        z.copy_(new[0])
        e.copy_(new[1])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, ctx.sample_tokens(z, e, top_p=p)))


def test_refusals(ctx):
    z, e = logits(4, 100, torch.float32, 1)
    one = torch.ones(4, device="cuda")
    for bad in (dict(temperature=one.double()), dict(top_k=one), dict(top_p=one.half())):
        with pytest.raises(TypeError):
            ctx.sample_tokens(z, e, **bad)
    for bad in (dict(temperature=one[:3]), dict(min_p=one.cpu()), dict(valid=torch.ones(5, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(ValueError):
            ctx.sample_tokens(z, e, **bad)
    with pytest.raises(TypeError):
        ctx.sample_tokens(z, e.double())
    with pytest.raises(TypeError):
        ctx.sample_tokens(z.half(), e)
    for noise in (e[:3], e[:, :99], e.cpu(), e.t()):
        with pytest.raises(ValueError):
            ctx.sample_tokens(z, noise)
