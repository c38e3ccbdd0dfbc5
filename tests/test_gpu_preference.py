"""The preference loss on the GPU against its 64-bit form: tiles that responses begin and end in, empty responses, masks, every form,
rows that must not be read, faulty offsets, and the gradient through logits.

Tolerances.  Sums and pairs are formed in fp64 from the same fp32 numbers; a reward and a loss are rounded once (2^-24) and a
coefficient up to three times (itself, times the temperature, and that product's operand), each allowed twice over for the fp64
sums' own order: 2^-23 and 2^-22.  Sums that cancel add their terms' absolute sum times 2^-50."""
import numpy as np
import pytest
import torch

import oracle.training_oracle as O
from paper_2605_13907_amd import binding as B

pytestmark = pytest.mark.gpu

TILE = 2048
FORMS = [dict(), dict(label_smoothing=0.2, margin=0.1), dict(kind=1, margin=0.3, beta=0.5), dict(kind=2, beta=0.5),
         dict(kind=2, mean_logp=1, beta=0.7, margin=0.1), dict(mean_logp=1, beta=2.0, inv_temperature=0.8)]


@pytest.fixture(scope="module")
def ctx():
    c = B.AisContext()
    yield c
    c.close()


def cuda(a, dtype=None):
    return None if a is None else torch.tensor(a, dtype=dtype, device="cuda")


def compare(ctx, logp, ref, valid, cu, weight, **form):
    p = B.default_preference_params(**form)
    loss, reward, g = ctx.preference_row_scale(cuda(logp), cuda(ref), cuda(valid), cuda(cu, torch.int64), p, weight=cuda(weight))
    exact = dict(form)
    for k in ("beta", "label_smoothing", "margin", "inv_temperature"):
        exact[k] = float(getattr(p, k))                          # as the fp32 fields hold them
    want, want_reward, want_g = O.preference(logp, ref, valid, cu, weight, **exact)
    live = np.ones(len(logp), bool) if valid is None else valid != 0
    size = np.abs(np.where(live, logp, 0.0)).sum() + (0 if ref is None else np.abs(np.where(live, ref, 0.0)).sum())
    beta = exact.get("beta", 0.1)
    noise = beta * size * 2.0 ** -50
    reward, g = reward.cpu().numpy(), g.cpu().numpy()
    assert np.abs(reward - want_reward).max(initial=0.0) <= np.abs(want_reward).max(initial=0.0) * 2.0 ** -23 + noise
    assert np.allclose(reward, want_reward, rtol=2.0 ** -23, atol=noise)
    assert np.allclose(g, want_g, rtol=2.0 ** -22, atol=beta * 40 * noise)
    assert (g[~live] == 0).all()
    assert loss.item() == pytest.approx(want, rel=2.0 ** -22, abs=40 * noise + 1e-300)
    assert ctx.status() == 0


def batch(lengths, seed=0, live=0.8, with_ref=True):
    r = np.random.default_rng(seed)
    cu = np.concatenate(([0], np.cumsum(lengths))).astype(np.int64)
    n = int(cu[-1])
    logp = (-r.exponential(size=n)).astype(np.float32)
    ref = (logp + 0.2 * r.standard_normal(n)).astype(np.float32) if with_ref else None
    valid = None if live >= 1 else (r.random(n) < live).astype(np.uint8)
    return logp, ref, valid, cu, r.random(len(lengths) // 2).astype(np.float32)


LENGTHS = {
    "one row": [1, 0], "two rows": [1, 1], "nothing": [0, 0], "empty ones between": [0, 3, 0, 0, 5, 0, 0, 0, 7, 2],
    "a tile": [TILE, 0], "a tile and one": [TILE, 1], "borders": [TILE - 1, 1, 1, TILE - 1, TILE, TILE],
    "inside tiles": [700, 900, 1_100, 3_000, 5, 6_001], "long": [50_001, 3], "many short": [1, 2, 0, 3] * 1_500,
    "mixed": [9_000, 1, 1, 1, 0, 4_096, 2, 2], "one workgroup's": [4_000, 4_192], "one more": [4_000, 4_193], "one workgroup's many": [1, 2, 0] * 2_700 + [1, 1], "ragged": [int(v) for v in np.random.default_rng(5).integers(0, 400, 600)],
}


@pytest.mark.parametrize("name", LENGTHS)
def test_lengths(ctx, name):
    lengths = LENGTHS[name]
    compare(ctx, *batch(lengths), **FORMS[0])
    compare(ctx, *batch(lengths, seed=1, live=1.0, with_ref=False), **FORMS[4])


@pytest.mark.parametrize("form", FORMS)
def test_forms(ctx, form):
    logp, ref, valid, cu, weight = batch([300, 200, 1, 900, 0, 12, 2_500, 2_100], seed=2)
    compare(ctx, logp, ref, valid, cu, weight, **form)
    compare(ctx, logp, ref, None, cu, None, **form)


def test_a_response_without_a_valid_token(ctx):
    logp, ref, _, cu, weight = batch([10, 20, 30, 40], live=1.0)
    valid = np.ones(100, np.uint8)
    valid[10:30] = 0
    for form in FORMS:
        compare(ctx, logp, ref, valid, cu, weight, **form)
    compare(ctx, logp, ref, np.zeros(100, np.uint8), cu, weight)


def test_masked_rows_are_not_looked_at(ctx):
    logp, ref, valid, cu, weight = batch([40, 60, 30, 70], seed=3, live=0.5)
    p = B.default_preference_params()
    run = lambda a, b: ctx.preference_row_scale(cuda(a), cuda(b), cuda(valid), cuda(cu), p, weight=cuda(weight))
    want = run(logp, ref)
    a, b = logp.copy(), ref.copy()
    a[valid == 0], b[valid == 0] = np.nan, np.inf
    for x, y in zip(want, run(a, b)):
        assert torch.equal(x, y)


@pytest.mark.parametrize("value", [np.nan, -np.inf])
def test_what_is_not_finite_stays_in_its_pair(ctx, value):
    logp, ref, _, cu, weight = batch([1_500, 900, 700, 300, 2_000, 100], live=1.0)
    run = lambda a: ctx.preference_row_scale(cuda(a), cuda(ref), None, cuda(cu), B.default_preference_params(), weight=cuda(weight))
    _, reward, g = run(logp)
    bad = logp.copy()
    bad[2_600] = value                                           # the third response
    loss, bad_reward, bad_g = run(bad)
    keep = [0, 1, 4, 5]
    assert torch.equal(bad_reward[keep], reward[keep])
    rows = np.r_[0:2_400, 3_400:5_500]
    assert torch.equal(bad_g[rows], g[rows])
    assert not torch.isfinite(bad_reward[2]) and not torch.isfinite(loss)
    assert bool(torch.isnan(bad_g[2_400:3_400]).all()) == bool(np.isnan(value))


@pytest.mark.parametrize("h", [-2_000.0, -40.0, -1e-3, 0.0, 1e-3, 40.0, 700.0])
def test_far_margins(ctx, h):
    logp = np.array([h, 0.0], np.float32)
    for form in (dict(beta=1.0), dict(beta=1.0, label_smoothing=0.25), dict(beta=1.0, kind=1), dict(beta=1.0, kind=2)):
        compare(ctx, logp, None, None, np.array([0, 1, 2]), None, **form)


@pytest.mark.parametrize("cu", [[1, 4, 8, 9, 10], [0, 4, 3, 9, 10], [0, 4, 8, 9, 9], [0, 4, 8, 30, 10], [-5, 4, 8, 9, 10],
                                [0, 2 ** 40, 8, 9, 10]])
def test_faulty_offsets_are_reported(ctx, cu):
    logp = cuda(np.full(10, -1.0, np.float32))
    _, _, g = ctx.preference_row_scale(logp, None, None, cuda(cu, torch.int64))
    assert g.shape == (10,)
    assert ctx.status() == B.STATUS_BAD_CU and ctx.status() == 0
    z, ids = torch.randn(10, 64, device="cuda"), torch.zeros(10, dtype=torch.int32, device="cuda")
    dz = ctx.preference_loss_grad(z, ids, None, cuda(cu, torch.int64), None)[3]
    assert dz.shape == z.shape
    assert ctx.status() == B.STATUS_BAD_CU and ctx.status() == 0


def test_no_rows(ctx):
    none = torch.empty(0, device="cuda")
    loss, reward, g = ctx.preference_row_scale(none, None, None, cuda([0, 0, 0], torch.int64), B.default_preference_params(margin=1.0))
    assert loss.item() == pytest.approx(np.log1p(np.exp(1.0)), rel=2.0 ** -22) and reward.tolist() == [0.0, 0.0] and g.numel() == 0


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab,pitch", [(1, 1), (70, 70), (1_000, 1_003), (4_096, 4_096), (33_001, 33_001), (140_000, 140_000)])
def test_through_logits(ctx, dtype, vocab, pitch):
    """Log-probs: each term is off by 2^-22 (an exponential's 2^-23, its exponent's rounding of at most 2^-24 times 40 of a term that is
    then below e^-20), a batch's sum of 16 by 16 of 2^-25; 2^-20 of min(1, the other tokens' share) covers them, and 2^-24 its own rounding.
    dlogits are the coefficients times softmax less the token's one: half a step of the type, and in fp32 the exponential and the shift by
    an lse of up to 20: 2^-19."""
    through_logits(ctx, dtype, vocab, pitch, [5, 11, 0, 40, 17, 3])


def through_logits(ctx, dtype, vocab, pitch, lengths):
    gen = torch.Generator(device="cuda").manual_seed(7)
    logp0, _, valid, cu, weight = batch(lengths, seed=4)
    rows = len(logp0)
    z = (3 * torch.randn(rows, pitch, generator=gen, device="cuda")).to(dtype)[:, :vocab]
    ids = torch.randint(0, vocab, (rows,), generator=gen, device="cuda", dtype=torch.int32)
    valid, cu, weight = cuda(valid), cuda(cu), cuda(weight)
    p = B.default_preference_params(beta=0.3, inv_temperature=0.9)
    temperature = float(np.float32(0.9))
    exact = torch.log_softmax(z.double() * temperature, dim=1).gather(1, ids.long()[:, None])[:, 0]
    live = valid != 0
    ref = (exact + 0.1 * torch.randn(rows, generator=gen, device="cuda")).float()
    loss, reward, logp, dz = ctx.preference_loss_grad(z, ids, valid, cu, ref, p, weight=weight)
    others = -torch.expm1(exact)
    slack = 2.0 ** -20 * others + 1e-300
    assert (torch.where(live, (logp.double() - exact).abs() <= slack + 2.0 ** -24 * exact.abs(), logp == 0)).all()
    form = dict(beta=float(p.beta), inv_temperature=temperature)
    want_loss, want_reward, g = O.preference(exact.cpu().numpy(), ref.cpu().numpy(), valid.cpu().numpy(), cu.cpu().numpy(),
                                             weight.cpu().numpy(), **form)
    each = float(p.beta) * float(slack.sum())
    assert np.allclose(reward.cpu().numpy(), want_reward, rtol=2.0 ** -23, atol=each)
    assert loss.item() == pytest.approx(want_loss, rel=2.0 ** -22, abs=2 * each * float(weight.sum()))
    g = torch.tensor(g, device="cuda")
    soft = torch.softmax(z.double() * temperature, dim=1)
    soft[torch.arange(rows), ids.long()] = torch.expm1(exact)
    want = g[:, None] * soft
    # a slope changes by at most a quarter of what its argument does
    off = 2.0 ** -19 + each
    tol = want.abs() * (off + (2.0 ** -8 if dtype == torch.bfloat16 else 0.0)) * 1.01 + g.abs()[:, None] * (slack[:, None] + 2.0 ** -24) \
        + float(p.beta) * each * weight.max().double() * soft.abs()
    assert ((dz.double() - want).abs() <= tol).all()
    alone = ctx.preference_loss_grad(z, ids, valid, cu, ref, p, weight=weight, want_grad=False)
    assert alone[3] is None and all(torch.equal(a, b) for a, b in zip(alone[:3], (loss, reward, logp)))
    inplace = ctx.preference_loss_grad(z, ids, valid, cu, ref, p, weight=weight, dlogits=z)[3]
    assert inplace.data_ptr() == z.data_ptr() and torch.equal(inplace, dz)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("lengths", [[1_000, 24], [1_024, 1], [0, 1_024], [16] * 64, [15] * 66, [0] * 62 + [3, 2], [700, 1, 300, 0], [1_500, 1_000],
                                     [300] * 10])
def test_through_logits_of_more_rows(ctx, lengths, dtype):
    """Batches whose coefficients the gradient's own workgroups form (up to 1,024 rows in 64 responses), and the next larger ones."""
    through_logits(ctx, dtype, 136, 136, lengths)
    through_logits(ctx, dtype, 1_501, 1_501, lengths)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("rows", [90, 1_500])
def test_forms_through_logits(ctx, form, rows):
    """Either way to the coefficients gives what the log-probs of the same logits give by themselves, up to those log-probs' own
    rounding: 2^-24 of each, under beta."""
    logp0, ref, valid, cu, weight = batch([rows // 3, rows // 3, rows // 6, rows // 6], seed=8)
    gen = torch.Generator(device="cuda").manual_seed(2)
    n, vocab = len(logp0), 200
    z = torch.randn(n, vocab, generator=gen, device="cuda")
    ids = torch.randint(0, vocab, (n,), generator=gen, device="cuda", dtype=torch.int32)
    valid, cu, weight = cuda(valid), cuda(cu), cuda(weight)
    p = B.default_preference_params(**form)
    exact = torch.log_softmax(z.double() * p.inv_temperature, dim=1).gather(1, ids.long()[:, None])[:, 0]
    ref = (exact + 0.05 * torch.randn(n, generator=gen, device="cuda")).float()
    loss, reward, logp, dz = ctx.preference_loss_grad(z, ids, valid, cu, ref, p, weight=weight)
    want_loss, want_reward, g = ctx.preference_row_scale(logp, ref, valid, cu, p, weight=weight)
    off = float(p.beta) * (float(logp.abs().sum()) * 2.0 ** -24 if not p.mean_logp else 8 * 2.0 ** -24) + 2.0 ** -22 * float(want_reward.abs().max())
    assert torch.allclose(reward, want_reward, rtol=2.0 ** -22, atol=off)
    scale = 1.0 if p.kind < 2 else 2.0 / p.beta ** 2 * max(1.0, float(want_reward.abs().max()))
    assert abs(loss.item() - want_loss.item()) <= 2.0 ** -22 * abs(want_loss.item()) + 2 * off * scale * float(weight.sum())
    want = g.double()[:, None] * torch.softmax(z.double() * p.inv_temperature, dim=1)
    want[torch.arange(n), ids.long()] = g.double() * torch.expm1(exact)
    slope = float(p.beta) * float(weight.max()) * (2 * off * scale if p.kind != 1 else 0.0)
    assert ((dz.double() - want).abs() <= 2.0 ** -19 * want.abs() + slope + 1e-30).all()


def test_small_terms_of_long_responses_add_up(ctx):
    """A response's log-ratios, each of which a sum in 32 bits leaves 3e-7 too large, are the sum of exact ones: rows of a large and 60,000
    small terms, all alike, whose error does not average out.  A term is off by 2^-23 + 2^-24 at most, the same one for all small ones."""
    rows, vocab = 512, 60_001
    z = torch.full((rows, vocab), -15.0, device="cuda")
    z[:, 0] = 0.0
    ids = torch.ones(rows, dtype=torch.int32, device="cuda")
    exact = torch.log_softmax(z[:1].double(), dim=1)[0, 1].item()
    cu = cuda([0, rows, rows], torch.int64)
    ref = torch.full((rows,), float(np.float32(exact)), device="cuda")
    _, reward, _, _ = ctx.preference_loss_grad(z, ids, None, cu, ref, B.default_preference_params(beta=1.0), want_grad=False)
    want = rows * (exact - float(np.float32(exact)))
    share = 60_000 * np.exp(-15.0) / (1 + 60_000 * np.exp(-15.0))
    # 15 log2(e) in fp32 is off by 2^-25 times 22, as the terms' common exponent: e^-15's relative error 22 * 2^-25 + 2^-23
    assert abs(reward[0].item() - want) <= rows * (share * (22 * 2.0 ** -25 + 2.0 ** -23 + 16 * 2.0 ** -25) + 15 * 2.0 ** -50)


@pytest.mark.parametrize("shift", [-8_000.0, 8_000.0])
def test_tokens_far_from_the_rest(ctx, shift):
    """A sampled token thousands below the row's largest, or above all others."""
    z = torch.randn(6, 300, device="cuda")
    z[:, 7] += shift
    ids = torch.full((6,), 7, dtype=torch.int32, device="cuda")
    exact = torch.log_softmax(z.double(), dim=1)[:, 7]
    logp = ctx.preference_loss_grad(z, ids, None, cuda([0, 3, 6], torch.int64), None)[2]
    assert torch.allclose(logp.double(), exact, rtol=2.0 ** -22, atol=1e-300)


def test_faulty_tokens_are_reported(ctx):
    z = torch.randn(4, 300, device="cuda")
    ids = cuda(np.array([3, 300, -1, 299], np.int32))
    _, _, logp, dz = ctx.preference_loss_grad(z, ids, None, cuda([0, 2, 4], torch.int64), None)
    assert logp[1] == 0 and logp[2] == 0 and logp[0] < 0 and torch.isfinite(dz).all()
    assert ctx.status() == B.STATUS_BAD_TOKEN and ctx.status() == 0


def test_more_rows_than_a_launch_of_tiles_fills(ctx):
    compare(ctx, *batch([int(v) for v in np.random.default_rng(9).integers(0, 3_000, 400)], seed=9))


@pytest.mark.parametrize("lengths", [[30, 70], [5_000, 4_000, 300, 0]])
def test_arrays_that_begin_anywhere(ctx, lengths):
    logp, ref, valid, cu, weight = batch(lengths, seed=11)
    n = len(logp)
    p = B.default_preference_params()
    want = ctx.preference_row_scale(cuda(logp), cuda(ref), cuda(valid), cuda(cu), p, weight=cuda(weight))
    for shift in (1, 2, 3, 5):
        moved = []
        for a in (logp, ref, valid):
            t = torch.zeros(n + 8, dtype=torch.from_numpy(a).dtype, device="cuda")
            t[shift:shift + n] = cuda(a)
            moved.append(t[shift:shift + n])
        for a, b in zip(want, ctx.preference_row_scale(*moved, cuda(cu), p, weight=cuda(weight))):
            assert torch.equal(a, b)


def test_a_million_responses(ctx):
    """More responses than rows in most places, and one of half the batch among them."""
    r = np.random.default_rng(12)
    lengths = r.integers(0, 2, 1 << 20)
    lengths[123_457] = 500_000
    logp, ref, valid, cu, weight = batch([int(v) for v in lengths], seed=12)
    loss, reward, g = ctx.preference_row_scale(cuda(logp), cuda(ref), cuda(valid), cuda(cu), weight=cuda(weight))
    delta = np.where(valid != 0, logp.astype(np.float64) - ref, 0.0)
    d = np.add.reduceat(np.concatenate((delta, [0.0])), cu[:-1]) * (lengths > 0)
    beta = float(B.default_preference_params().beta)
    h = beta * (d[0::2] - d[1::2])
    want = (weight.astype(np.float64) * np.logaddexp(0.0, -h)).sum()
    c = weight * beta / (1.0 + np.exp(h))
    rows = np.repeat(np.arange(1 << 20), lengths)
    want_g = np.where(rows % 2 == 0, 1.0, -1.0) * c[rows // 2] * (valid != 0)
    noise = beta * np.abs(delta).sum() * 2.0 ** -50
    assert np.allclose(reward.cpu().numpy(), beta * d, rtol=2.0 ** -23, atol=noise)
    assert np.allclose(g.cpu().numpy(), want_g, rtol=2.0 ** -22, atol=noise)
    assert loss.item() == pytest.approx(want, rel=2.0 ** -22)
    assert ctx.status() == 0


def test_runs_alike(ctx):
    logp, ref, valid, cu, weight = (cuda(a) for a in batch([5_000, 7_000, 3, 9_000], seed=6))
    first = ctx.preference_row_scale(logp, ref, valid, cu, weight=weight)
    for _ in range(5):
        for a, b in zip(first, ctx.preference_row_scale(logp, ref, valid, cu, weight=weight)):
            assert torch.equal(a, b)
