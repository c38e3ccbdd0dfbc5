"""The distillation loss and its gradient on the GPU against the fp64 oracle.

kl and loss: 2e-6 of the sum of |terms| (q, log q and log p are fp32 numbers of a few roundings each, |log p| <= 60) and the
same relative; the gradient element by element: 1e-5 of weight inv_temperature (p + q) for the fp32 soft-max, and half a unit in
the last place of the result's type."""
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


def case(rows, vocab, top, dtype, seed, scale=3.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    z = (torch.randn(rows, vocab, generator=gen, device="cuda") * scale).to(dtype)
    noisy = z.float() + 0.5 * torch.randn(rows, vocab, generator=gen, device="cuda")
    t = torch.topk(noisy, top, dim=1)
    return z, t.indices.to(torch.int32), t.values.contiguous(), torch.rand(rows, generator=gen, device="cuda")


def check(ctx, z, ids, teacher, weight=None, valid=None, inv_t=1.0, **kw):
    before = z.clone()
    loss, kl, grad = ctx.distill_topk(z, ids, teacher, weight, valid, inv_t, **kw)
    w = np.full(z.shape[0], 1.0 / z.shape[0]) if weight is None else weight.double().cpu().numpy()
    zs, idn, tn = before.double().cpu().numpy(), ids.cpu().numpy(), teacher.double().cpu().numpy()
    live = None if valid is None else valid.cpu().numpy()
    want_loss, want_kl, want = O.distill(zs, idn, tn, w, inv_t, live)
    size = 60.0 + np.abs(want_kl)
    got_kl = kl.double().cpu().numpy()
    fine = np.isfinite(want_kl)
    assert (np.abs(got_kl - want_kl) <= 2e-6 * size)[fine].all(), np.abs(got_kl - want_kl)[fine].max()
    np.testing.assert_array_equal(got_kl[~fine], want_kl[~fine])
    if fine.all():
        assert abs(loss.item() - want_loss) <= 2e-6 * (w * size).sum()
    if grad is not None:
        assert grad.dtype == z.dtype and grad.shape == z.shape
        got = grad.double().cpu().numpy()
        ulp = 2.0 ** -8 if z.dtype == torch.bfloat16 else 2.0 ** -23
        listed = np.zeros_like(want)
        for r in range(z.shape[0]):
            on = (idn[r] >= 0) & (idn[r] < z.shape[1])
            if on.any() and np.isfinite(tn[r][on]).all():
                q = np.exp((tn[r][on] - tn[r][on].max()) * inv_t)
                np.add.at(listed[r], idn[r][on], 2 * q / q.sum() * w[r] * inv_t)
        bound = 1e-5 * (np.abs(want) + listed) + ulp * np.abs(want) + 2.0 ** -126
        assert (np.abs(got - want) <= bound)[np.isfinite(want)].all()
        assert (np.isnan(got) == np.isnan(want)).all()
    return loss, kl, grad


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,vocab,top", [(1, 1, 1), (3, 2, 2), (5, 7, 3), (2, 64, 64), (40, 1000, 8), (9, 1024, 200), (4, 2050, 1024),
                                            (6, 4099, 33), (3, 8192, 64), (2, 17_000, 50), (2, 50_257, 128), (1, 151_936, 64),
                                            (1, 200_003, 20), (1, 262_144, 7), (1, 300_000, 5)])
def test_sizes(ctx, dtype, rows, vocab, top):
    z, ids, teacher, weight = case(rows, vocab, top, dtype, rows + vocab)
    check(ctx, z, ids, teacher, weight)
    loss, kl, none = check(ctx, z, ids, teacher, weight, want_grad=False)
    assert none is None


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("inv_t", [0.25, 1.0, 1.7])
def test_temperature_mask_and_mean(ctx, dtype, inv_t):
    z, ids, teacher, weight = case(37, 3001, 20, dtype, 3)
    valid = (torch.arange(37, device="cuda") % 3 != 1).to(torch.uint8)
    _, kl, grad = check(ctx, z, ids, teacher, weight, valid, inv_t)
    assert not kl[1::3].any() and not grad[1::3].any()
    check(ctx, z, ids, teacher, None, valid, inv_t)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_of_fewer_entries(ctx, dtype):
    z, ids, teacher, weight = case(12, 500, 16, dtype, 5)
    ids[0] = -1                               # none at all
    ids[1, 3:] = -1
    ids[2, ::2] = -1
    teacher[3, 4:] = -math.inf
    teacher[4] = -math.inf                    # nothing that counts
    ids[5, 1] = ids[5, 0]                     # listed twice, three times, always the same
    ids[6, 4] = ids[6, 9] = ids[6, 2]
    ids[7] = 77
    teacher[8] = 1.25                         # all alike
    teacher[9, 0] = 500.0                     # one token
    ids[11, 15] = -1
    teacher[11, 15] = math.nan                # of an entry that is none
    ctx.status()
    _, kl, grad = check(ctx, z, ids, teacher, weight)
    assert kl[0] == 0 and kl[4] == 0 and not grad[0].any() and not grad[4].any()
    assert ctx.status() == 0


def test_ids_outside_the_vocabulary(ctx):
    z, ids, teacher, weight = case(6, 300, 8, torch.float32, 7)
    ids[1, 2], ids[3, 0], ids[4, 5] = 300, 2 ** 31 - 1, -7
    ctx.status()
    check(ctx, z, ids, teacher, weight)
    assert ctx.status() == B.STATUS_BAD_TOKEN


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_masked_logits(ctx, dtype):
    """Tokens that the policy cannot take: without a teacher's entry they cost nothing, with one the divergence is infinite."""
    z, ids, teacher, weight = case(4, 600, 5, dtype, 9)
    z[0, 300:] = -math.inf
    ids[0] = torch.arange(5, device="cuda")
    z[1, int(ids[1, 0])] = -math.inf
    z[2, 50:] = torch.finfo(dtype).min
    ids[2] = torch.arange(5, device="cuda")
    _, kl, grad = check(ctx, z, ids, teacher, weight)
    assert math.isinf(kl[1].item()) and torch.isfinite(grad).all()


def test_numbers_that_are_none(ctx):
    z, ids, teacher, weight = case(4, 600, 5, torch.float32, 9)
    z[0, 10] = math.nan
    teacher[1, 2] = math.nan
    teacher[2, 2] = math.inf
    _, kl, grad = ctx.distill_topk(z, ids, teacher, weight)
    assert torch.isnan(kl[:3]).all() and torch.isfinite(kl[3])
    assert torch.isnan(grad[0]).all() and torch.isfinite(grad[3]).all()
    assert torch.isnan(grad[1][ids[1].long()]).all() and torch.isnan(grad[2][ids[2].long()]).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("vocab", [600, 152_000])
def test_rows_without_a_distribution(ctx, dtype, vocab):
    z, ids, teacher, weight = case(4, vocab, 5, dtype, 10)
    z[0] = -math.inf
    z[1, 17] = math.inf
    z[2, vocab - 1] = math.nan
    _, kl, grad = ctx.distill_topk(z, ids, teacher, weight)
    assert torch.isnan(kl[:3]).all() and torch.isnan(grad[:3]).all()
    assert torch.isfinite(kl[3]) and torch.isfinite(grad[3]).all()
    alone = ctx.distill_topk(z, ids, teacher, weight, want_grad=False)[1]
    assert torch.isnan(alone[:3]).all() and torch.isfinite(alone[3])


def test_policy_that_is_its_teacher(ctx):
    """The whole vocabulary listed with the policy's own logits: divergence and gradient vanish."""
    z, _, _, weight = case(8, 500, 1, torch.float32, 11)
    order = torch.argsort(torch.rand(8, 500, device="cuda"), dim=1)
    _, kl, grad = ctx.distill_topk(z, order.to(torch.int32), z.gather(1, order), weight)
    assert kl.abs().max() < 2e-6 and grad.abs().max() < 2e-7


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("offset", [0, 1, 5, 8, 64])
@pytest.mark.parametrize("vocab", [900, 9001])
def test_strides_and_in_place(ctx, dtype, offset, vocab):
    z, ids, teacher, weight = case(6, vocab, 12, dtype, 13)
    wide = torch.zeros(6, vocab + 100, dtype=dtype, device="cuda")
    view = wide[:, offset:offset + vocab]
    view.copy_(z)
    loss, kl, grad = check(ctx, view, ids, teacher, weight)
    keep = wide.clone()
    loss2, kl2, same = ctx.distill_topk(view, ids, teacher, weight, dlogits=view)
    assert same.data_ptr() == view.data_ptr() and torch.equal(same, grad) and torch.equal(kl, kl2) and torch.equal(loss, loss2)
    keep[:, offset:offset + vocab] = grad
    assert torch.equal(keep, wide)


def test_gradient_in_another_place(ctx):
    """Logits and gradient that lie differently relative to 128-byte lines, through the C interface."""
    z, ids, teacher, weight = case(5, 3000, 9, torch.bfloat16, 15)
    want = ctx.distill_topk(z, ids, teacher, weight)
    out = torch.zeros(5, 3100, dtype=torch.bfloat16, device="cuda")
    kl, loss = torch.empty(5, device="cuda"), torch.empty(1, device="cuda")
    for offset in (0, 1, 8, 33):
        out.zero_()
        ctx._sync_stream()
        rc = B._lib().ais_distill_topk(ctx._h, z.data_ptr(), B.AIS_BF16, 5, 3000, 3000, ids.data_ptr(), teacher.data_ptr(), 9, None,
                                       weight.data_ptr(), 1.0, kl.data_ptr(), loss.data_ptr(), out[:, offset:].data_ptr(), 3100)
        assert rc == 0
        torch.testing.assert_close(out[:, offset:offset + 3000].float(), want[2].float(), rtol=2.0 ** -7, atol=1e-9)
        assert not out[:, :offset].any() and not out[:, offset + 3000:].any()


def test_gradient_against_differences(ctx):
    """The loss moves as the gradient says: along a random direction, fp32, symmetric differences of 1e-2."""
    z, ids, teacher, weight = case(64, 200, 10, torch.float32, 17, scale=1.0)
    _, _, grad = ctx.distill_topk(z, ids, teacher, weight)
    gen = torch.Generator(device="cuda").manual_seed(1)
    for _ in range(4):
        d = torch.randn(z.shape, generator=gen, device="cuda")
        up, down = (ctx.distill_topk(z + s * 1e-2 * d, ids, teacher, weight, want_grad=False)[0].item() for s in (1, -1))
        # the third derivative of a log-sum-exp is at most of order one along d, times 1e-4 / 6 a row; the loss is 2e-6 x 60 off
        assert (up - down) / 2e-2 == pytest.approx((grad * d).sum().item(), abs=64 * 1e-4 + 64 * 60 * 2e-6 / 1e-2 * 0.1)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("vocab", [9, 1000, 50_257, 152_000, 270_000])
def test_logits_as_large_as_the_type_holds(ctx, dtype, vocab):
    """Rows whose products with 1 / T do not fit: of equal values, every token is as likely."""
    z, ids, teacher, weight = case(5, vocab, 7, dtype, 71)
    lowest, most = torch.finfo(dtype).min, torch.finfo(dtype).max
    z[0] = lowest
    z[1] = lowest
    z[1, ::2] = -math.inf
    z[1, ids[1].long()] = lowest
    z[2] = most
    z[3] = 1e10
    for want_grad in (True, False):
        check(ctx, z, ids, teacher, weight, want_grad=want_grad)
    shifted = torch.zeros(5, vocab + 3, dtype=dtype, device="cuda")[:, 1:vocab + 1]
    shifted.copy_(z)
    check(ctx, shifted, ids, teacher, weight)
    loss, kl, grad = ctx.distill_topk(z, ids, teacher, weight)
    again = ctx.distill_topk(z, ids, teacher, weight, dlogits=z)
    assert torch.equal(grad, again[2]) and torch.equal(kl, again[1])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("inv_t", [0.001, 0.2, 0.6, 1.0, 3.0])
@pytest.mark.parametrize("vocab", [300, 20_000, 152_000])
def test_lowest_masks_at_any_temperature(ctx, dtype, inv_t, vocab):
    z, ids, teacher, weight = case(4, vocab, 6, dtype, 79)
    lowest = torch.finfo(dtype).min
    keep = z.gather(1, ids.long())
    z[0] = lowest
    z[1, 10:] = lowest
    z[2, vocab // 2:] = lowest
    z[3, 100:] = -math.inf
    z.scatter_(1, ids.long(), keep)
    check(ctx, z, ids, teacher, weight, inv_t=inv_t)
    check(ctx, z, ids, teacher, weight, inv_t=inv_t, want_grad=False)


def test_no_rows_streams_and_graphs(ctx):
    z, ids, teacher, weight = case(3, 50, 4, torch.float32, 1)
    loss, kl, grad = ctx.distill_topk(z[:0], ids[:0], teacher[:0])
    assert loss.item() == 0 and kl.shape == (0,) and grad.shape == (0, 50)
    z, ids, teacher, weight = case(30, 5000, 16, torch.bfloat16, 19)
    want = ctx.distill_topk(z, ids, teacher, weight)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = ctx.distill_topk(z, ids, teacher, weight)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = ctx.distill_topk(z, ids, teacher, weight)
    for seed in range(4):
        for old, new in zip((z, ids, teacher, weight), case(30, 5000, 16, torch.bfloat16, 50 + seed)):
            old.copy_(new)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, ctx.distill_topk(z, ids, teacher, weight)))


def test_refusals(ctx):
    z, ids, teacher, weight = case(4, 50, 4, torch.float32, 1)
    for bad in ((z.half(), ids, teacher), (z, ids.long(), teacher), (z, ids, teacher.double())):
        with pytest.raises(TypeError):
            ctx.distill_topk(*bad)
    for bad in ((z, ids[:3], teacher[:3]), (z, ids, teacher[:, :3]), (z, ids.cpu(), teacher), (z, ids.t(), teacher.t())):
        with pytest.raises(ValueError):
            ctx.distill_topk(*bad)
    with pytest.raises(ValueError):
        ctx.distill_topk(z, ids, teacher, weight[:2])
    with pytest.raises(ValueError):
        ctx.distill_topk(z, ids, teacher, weight, dlogits=z.bfloat16())
    with pytest.raises(B.AisError) as e:
        ctx.distill_topk(z, ids, teacher, weight, inv_temperature=0.0)
    assert e.value.code == -5
    wide = torch.zeros(4, 1025, device="cuda")
    with pytest.raises(B.AisError) as e:
        ctx.distill_topk(z, wide.int(), wide)
    assert e.value.code == -2
