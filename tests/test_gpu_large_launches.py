"""Calls with more elements or rows than one launch has threads for (no launch has 2^32): what lies behind the first launch's share, or what a
workgroup comes to after its first share, is what it is in a call by itself."""
import numpy as np
import pytest
import torch

import oracle.training_oracle as O
from paper_2605_13907_amd import binding as B
from tests.test_gpu_adamw import HALF, RULE, U, numbers, tensor

pytestmark = pytest.mark.gpu

GIB = 1 << 30


@pytest.fixture(scope="module")
def ctx():
    c = B.AisContext()
    yield c
    c.close()
    torch.cuda.empty_cache()


def room(gib):
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < gib * GIB:
        pytest.skip(f"needs {gib} GiB")


def test_a_step_of_many_billions(ctx):
    """Six tensors of 2.9 billion elements, 16,992,192 workgroups of 256 threads in all: each one's end is stepped as by itself."""
    room(80)
    n, count, tail = 2_900_000_011, 6, 200
    g = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    g[-tail:] = tensor(tail, torch.bfloat16, 2, 1e-3)
    params = [torch.zeros(n, dtype=torch.bfloat16, device="cuda") for _ in range(count)]
    for i, p in enumerate(params):
        p[-tail:] = tensor(tail, torch.bfloat16, 10 + i)
    before, grad = [numbers(p[-tail:]) for p in params], numbers(g[-tail:])
    state = B.AdamWState(params, bits=8, seed=5)
    ctx.adamw_step(state, [g] * count, **RULE)
    assert state.step == 1
    first = (n - tail) // 32 * 32                                # the block that the tail begins in
    at = np.arange(first, n, dtype=np.uint64)
    for i, p in enumerate(params):
        want, m, v = O.adamw(before[i], grad, np.zeros(tail), np.zeros(tail), 1, **RULE)
        assert (np.abs(numbers(p[-tail:]) - want) <= HALF[torch.bfloat16] * np.abs(want) + 20 * U * (np.abs(want) + RULE["lr"])).all(), i
        assert not p[:-tail].any()
        key = O.mix(O.mix(5 ^ 0x9E3779B1) ^ (i * 0x9E3779B1 & O.M32))
        bits = O.mix((at * np.uint64(0x9E3779B1) & np.uint64(O.M32)) ^ np.uint64(key))
        for which, x, flat, rnd in ((1, m, state.m, bits & np.uint64(65535)), (2, v, state.v, bits >> np.uint64(16))):
            codes, _ = O.encode(np.concatenate((np.zeros(n - tail - first, np.float32), x)), rnd, which)
            assert (flat[state.offsets[i] + first:state.offsets[i] + n].cpu().numpy() == codes).all(), (i, which)


@pytest.mark.parametrize("moment", [0, 1])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_values_of_billions(ctx, dtype, moment):
    """2^31 elements are a workgroup's eight by 256 of the most that a launch has."""
    room(16)
    n, part = (1 << 31) + 2_077, 1 << 20
    gen = torch.Generator(device="cuda").manual_seed(1)
    codes = torch.randint(0, 256, (n,), generator=gen, device="cuda", dtype=torch.uint8)
    scales = torch.randint(90, 160, (-(-n // 32),), generator=gen, device="cuda", dtype=torch.uint8)

    def values(at, count):
        out = torch.full((count + 8,), 7.0, dtype=dtype, device="cuda")
        arrays = [codes.data_ptr() + at, scales.data_ptr() + at // 32]
        arrays = [*arrays, None, None, count, out.data_ptr(), None] if moment == 0 else [None, None, *arrays, count, None, out.data_ptr()]
        assert ctx._lib.ais_adamw_values(ctx._h, *arrays, B.AIS_BF16 if dtype == torch.bfloat16 else B.AIS_F32) == 0
        assert (out[count:] == 7.0).all()
        return out[:count]

    got = values(0, n)
    for at in (0, (1 << 30) + 32, (1 << 31) - part, n // 32 * 32 - part):
        assert torch.equal(got[at:at + part], values(at, part))
    end = n // 32 * 32
    assert torch.equal(got[end:], values(end, n - end))


def same_rows(got, want, at, live):
    """Rows from `at` on of a call's outputs against those rows' own, zero where they are masked."""
    for a, b in zip(got, want):
        if a is None:
            assert b is None
            continue
        part = a[at:at + len(b)]
        assert torch.equal(part, b if live is None else torch.where(live.view(-1, *[1] * (b.dim() - 1)), b, torch.zeros_like(b)))


@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("centered", [True, False])
@pytest.mark.parametrize("width,n,gib", [(64, (1 << 21) + 70_001, 4), (2_568, (1 << 21) + 3_001, 40), (16_392, (1 << 16) + 301, 12)])
def test_rows_of_large_batches(ctx, width, n, gib, centered, masked):
    """A million workgroups have more than two rows each; of rows that are not held, 65,536 workgroups more than one."""
    room(gib)
    gen = torch.Generator(device="cuda").manual_seed(4)
    x = torch.empty(n, width, dtype=torch.bfloat16, device="cuda")
    for part in x.split(1 << 18):
        part.copy_(torch.randn(part.shape, generator=gen, device="cuda"))
    weight, bias = (torch.randn(width, generator=gen, device="cuda") for _ in range(2))
    # live, masked, live at the distance that a workgroup's rows have
    valid = ((torch.arange(n, device="cuda") // (1 << 16)) % 16 % 3 != 1).to(torch.uint8) if masked else None
    got = ctx.norm_rows(x, weight, bias, centered=centered, valid=valid)
    for at in range(0, n, 4_000 if width == 64 else 300_000 if width < 10_000 else 2_000):
        some = x[at:at + 2_000]
        same_rows(got, ctx.norm_rows(some, weight, bias, centered=centered), at, None if valid is None else valid[at:at + 2_000] != 0)
    at = n - 2_000
    same_rows(got, ctx.norm_rows(x[at:], weight, bias, centered=centered), at, None if valid is None else valid[at:] != 0)


@pytest.mark.parametrize("masked", [False, True])
def test_gradient_of_many_wide_rows(ctx, masked):
    room(12)
    n, width = (1 << 16) + 301, 8_200
    gen = torch.Generator(device="cuda").manual_seed(6)
    x, dy = (torch.empty(n, width, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for t in (x, dy):
        for part in t.split(1 << 15):
            part.copy_(torch.randn(part.shape, generator=gen, device="cuda"))
    weight, mean, rstd = torch.randn(width, generator=gen, device="cuda"), torch.randn(n, generator=gen, device="cuda"), torch.ones(n, device="cuda")
    valid = (torch.arange(n, device="cuda") % 3 != 1).to(torch.uint8) if masked else None
    dx = ctx.norm_rows_grad(dy, x, weight, mean, rstd, valid=valid)[0]
    for at in (*range(0, n, 8_000), n - 2_000):
        here = slice(at, at + 2_000)
        want = ctx.norm_rows_grad(dy[here], x[here], weight, mean[here], rstd[here])[0]
        same_rows([dx], [want], at, None if valid is None else valid[here] != 0)


def test_sums_of_very_wide_rows(ctx):
    """More than 2^26 columns, of one row: each one's sum is its one term."""
    room(8)
    width = (1 << 26) + 1_003
    gen = torch.Generator(device="cuda").manual_seed(8)
    x, dy = (torch.randn(1, width, generator=gen, device="cuda") for _ in range(2))
    rstd = torch.full((1,), 0.75, device="cuda")
    _, dw, db = ctx.norm_rows_grad(dy, x, torch.ones(width, device="cuda"), None, rstd)
    assert torch.equal(dw, dy[0] * (x[0] * 0.75)) and torch.equal(db, dy[0])


@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("masked", [False, True])
def test_sweeps_over_many_rows(ctx, masked, offset):
    """More rows than 2^32 threads of 256 to a row.  The hinge's slope is -1 behind a margin that no response reaches, so that a row's
    gradient is its own."""
    room(24)
    n, vocab, part = (1 << 24) + 1_003, 64, 4_096
    gen = torch.Generator(device="cuda").manual_seed(9)
    flat = torch.empty(n * vocab + offset, dtype=torch.bfloat16, device="cuda")
    z = flat[offset:].view(n, vocab)
    for some in z.split(1 << 22):
        some.copy_(torch.randn(some.shape, generator=gen, device="cuda"))
    ids = torch.randint(0, vocab, (n,), generator=gen, device="cuda", dtype=torch.int32)
    valid = (torch.rand(n, generator=gen, device="cuda") < 0.7).to(torch.uint8) if masked else None
    p = B.default_preference_params(kind=1, margin=1e6, beta=1e-3)
    cu = lambda rows: torch.tensor([0, rows, rows], device="cuda")

    def calls(at, rows):
        rows = min(rows, n - at)
        some = slice(at, at + rows)
        mask = None if valid is None else valid[some]
        logp, lse = ctx.token_logprob(z[some], ids[some], mask)
        loss = ctx.preference_loss_grad(z[some], ids[some], mask, cu(rows), None, p, weight=torch.ones(1, device="cuda"))
        return logp, lse, loss[2], loss[3], *ctx.token_logprob_softmax_grad(z[some], ids[some], mask)

    got = calls(0, n)
    for at in (0, (1 << 21) - 2_000, 3 << 21, (1 << 22) - 1, (1 << 24) - 2_000, n - part):
        for a, b in zip(got, calls(at, part)):
            assert torch.equal(a[at:at + part], b)
    assert ctx.status() == 0
