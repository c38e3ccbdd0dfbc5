"""The AdamW step against its 64-bit form: lists of tensors of every size and type, tensors that begin anywhere, moments in 32 and in 8
bits, whose codes have to be equal.

Tolerances, in units of u = 2^-24.  The moments are formed in fp64 and rounded once: half a step, u, and a subnormal's 2^-150.  Where their two
terms cancel, fp64's own roundings show: each of the two products and their sum is off by 2^-53 of itself at most, in the kernel and in the form it is
compared with, so by 2^-51 of the terms' sizes together (a gradient of -3.8e-3 against 9 times its average left 7.5e-20 for 5.4e-20).  The step
is lr (wd p + m c1 / (sqrt(v c2) + eps)) in fp32: c1, c2, lr, wd and eps are rounded (5), products, root, sum, quotient and sum again (7),
m and v before (2), some of them under the root: 14 u of its parts' sizes; the last subtraction u of the result; a parameter's type half its step."""
import numpy as np
import pytest
import torch

import oracle.training_oracle as O
from paper_2605_13907_amd import binding as B

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
RULE = dict(lr=1e-2, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.1)


@pytest.fixture(scope="module")
def ctx():
    c = B.AisContext()
    yield c
    c.close()


def numbers(t):
    return t.detach().double().cpu().numpy().reshape(-1)


class Twin:
    """A state on the GPU and what it has to hold."""

    def __init__(self, params, bits, copies=None, seed=3, step=0):
        self.state = B.AdamWState(params, bits=bits, copies=copies, seed=seed, step=step)
        self.bits, self.seed, self.step = bits, seed, step
        self.m = [np.zeros(p.numel(), np.float64) for p in params]
        self.v = [np.zeros(p.numel(), np.float64) for p in params]

    def check_step(self, ctx, grads, scale=None, **rule):
        rule = dict(RULE, **rule)
        before = [numbers(p) for p in self.state.params]
        ctx.adamw_step(self.state, grads, grad_scale=scale, **rule)
        self.step += 1
        values = ctx.adamw_values(self.state) if self.bits == 8 else (self.state.m, self.state.v)
        for i, (p, copy) in enumerate(zip(self.state.params, self.state.copies)):
            got, n = numbers(p), p.numel()
            if grads[i] is None:
                assert (got == before[i]).all()
                continue
            want, m, v = O.adamw(before[i], numbers(grads[i]), self.m[i], self.v[i], self.step, grad_scale=1.0 if scale is None else float(scale),
                                 **rule)
            ahead = np.abs(want - before[i] * (1 - rule["lr"] * rule["weight_decay"]))
            tol = 14 * U * rule["lr"] * (rule["weight_decay"] * np.abs(before[i])) + 14 * U * ahead + U * np.abs(want) + 2.0 ** -149
            tol = tol * (1 + HALF[p.dtype]) + HALF[p.dtype] * np.abs(want)
            assert (np.abs(got - want) <= tol).all(), i
            if copy is not None:
                assert torch.equal(copy, p.bfloat16())
            at = slice(self.state.offsets[i], self.state.offsets[i] + n)
            if self.bits == 32:
                g = np.abs(numbers(grads[i])) * (1.0 if scale is None else float(scale))
                terms = rule["beta1"] * np.abs(self.m[i]) + (1 - rule["beta1"]) * g, np.zeros(n)
                for flat, x, size in ((self.state.m, m, terms[0]), (self.state.v, v, terms[1])):
                    x = x.astype(np.float64)
                    assert (np.abs(numbers(flat[at]) - x) <= 2.01 * U * np.abs(x) + 2.0 ** -149 + 2.0 ** -51 * size).all()
                self.m[i], self.v[i] = numbers(self.state.m[at]), numbers(self.state.v[at])
                continue
            bits = O.random_bits(n, i, self.step, self.seed)
            blocks = slice(at.start // 32, at.start // 32 + -(-n // 32))
            for which, x, rnd, flat, scales, out in ((1, m, bits & np.uint64(65535), self.state.m, self.state.m_scale, values[0]),
                                                     (2, v, bits >> np.uint64(16), self.state.v, self.state.v_scale, values[1])):
                codes, sc = O.encode(x, rnd, which)
                assert (scales[blocks].cpu().numpy() == sc).all()
                assert (flat[at].cpu().numpy() == codes).all()
                held = O.decode(codes, sc, which)
                np.testing.assert_array_equal(numbers(out[at]), held.astype(np.float32))
                if which == 1:
                    self.m[i] = held
                else:
                    self.v[i] = held


def tensor(n, dtype, seed, size=1.0, offset=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    flat = torch.full((offset + n + 8,), float("nan"), dtype=dtype, device="cuda")
    t = flat[offset:offset + n]
    t.copy_(size * torch.randn(n, generator=gen, device="cuda"))
    return t


def grads_of(sizes, dtypes, seed, size=1e-3, offset=0):
    # gradients of many magnitudes, some of them zero (formed in fp32: torch's mixed products leave the device less memory)
    out = []
    for i, n in enumerate(sizes):
        g = tensor(n, dtypes[i % len(dtypes)], seed + i, size, offset)
        gen = torch.Generator(device="cuda").manual_seed(seed + 1_000 + i)
        wide = g.float() * torch.exp(3 * torch.randn(n, generator=gen, device="cuda"))
        wide[torch.rand(n, generator=gen, device="cuda") < 0.05] = 0.0
        g.copy_(wide)
        out.append(g)
    return out


BOTH = (torch.float32, torch.bfloat16)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("param", BOTH)
@pytest.mark.parametrize("grad", BOTH)
def test_sizes_and_types(ctx, bits, param, grad):
    sizes = [1, 7, 8, 9, 31, 32, 33, 63, 64, 65, 100, 2_047, 2_048, 2_049, 5_000, 70_001]
    twin = Twin([tensor(n, param, n) for n in sizes], bits)
    for step in range(3):
        twin.check_step(ctx, grads_of(sizes, [grad], 10 * step))


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("count", [1, 63, 64, 65, 319, 320, 321, 700])
def test_many_tensors_of_mixed_types(ctx, bits, count):
    sizes = [(37 * i) % 301 for i in range(count)]               # the first has no element at all
    params = [tensor(n, BOTH[i % 3 == 1], i) for i, n in enumerate(sizes)]
    copies = [torch.zeros(n, dtype=torch.bfloat16, device="cuda") if i % 2 else None for i, n in enumerate(sizes)]
    twin = Twin(params, bits, copies)
    for step in range(2):
        twin.check_step(ctx, grads_of(sizes, BOTH, step), scale=torch.full((1,), 0.37, device="cuda"))


@pytest.mark.parametrize("bits", [32, 8])
def test_tensors_that_begin_anywhere(ctx, bits):
    sizes = [5, 100, 2_049, 4_001]
    for offset in (1, 2, 3, 7):
        for param in BOTH:
            twin = Twin([tensor(n, param, n, offset=offset) for n in sizes], bits,
                        [tensor(n, torch.bfloat16, n, offset=offset) for n in sizes])
            twin.check_step(ctx, grads_of(sizes, BOTH, offset, offset=offset))


@pytest.mark.parametrize("bits", [32, 8])
def test_more_than_32_bits_of_bytes(ctx, bits):
    """A tensor of 2^31 and some elements: its end is stepped as by itself, in an element's place that the random numbers know."""
    n, tail = (1 << 31) + 77, 200
    p = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    g = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    p[-tail:], g[-tail:] = tensor(tail, torch.bfloat16, 1), tensor(tail, torch.bfloat16, 2, 1e-3)
    before, grad = numbers(p[-tail:]), numbers(g[-tail:])
    state = B.AdamWState([p], bits=bits, seed=5)
    ctx.adamw_step(state, [g], **RULE)
    want, m, v = O.adamw(before, grad, np.zeros(tail), np.zeros(tail), 1, **RULE)
    assert (np.abs(numbers(p[-tail:]) - want) <= HALF[torch.bfloat16] * np.abs(want) + 20 * U * (np.abs(want) + RULE["lr"])).all()
    assert not p[:-tail].any()
    if bits == 32:
        assert np.allclose(numbers(state.m[n - tail:n]), m.astype(np.float64), rtol=2.01 * U) and not state.m[:n - tail].any()
        return
    first = (n - tail) // 32 * 32                                # the block that the tail begins in
    pad = n - tail - first
    key = O.mix(O.mix(5 ^ 0x9E3779B1) ^ 0)
    at = np.arange(first, n, dtype=np.uint64)
    bits_of = O.mix((at * np.uint64(0x9E3779B1) & np.uint64(O.M32)) ^ np.uint64(key))
    for which, x, flat, rnd in ((1, m, state.m, bits_of & np.uint64(65535)), (2, v, state.v, bits_of >> np.uint64(16))):
        codes, _ = O.encode(np.concatenate((np.zeros(pad, np.float32), x)), rnd, which)
        assert (flat[first:n].cpu().numpy() == codes).all()


def test_a_tensor_without_a_gradient_stays(ctx):
    for bits in (32, 8):
        params = [tensor(n, torch.float32, n) for n in (100, 200, 300)]
        twin = Twin(params, bits)
        g = grads_of((100, 200, 300), BOTH, 1)
        twin.check_step(ctx, g)
        twin.check_step(ctx, [g[0], None, g[2]])
        m = twin.state.of(twin.state.m, 1).clone()
        twin.check_step(ctx, [None, None, None])
        assert torch.equal(m, twin.state.of(twin.state.m, 1))


@pytest.mark.parametrize("size", [1e-30, 1e-12, 1.0, 1e12])
def test_magnitudes(ctx, size):
    sizes = [64, 1_000]
    for bits in (32, 8):
        twin = Twin([tensor(n, torch.float32, n) for n in sizes], bits)
        for step in range(4):
            twin.check_step(ctx, grads_of(sizes, [torch.float32], step, size))


@pytest.mark.parametrize("bits", [32, 8])
def test_subnormal_second_moments(ctx, bits):
    """Squares below fp32's normal numbers are as good as others beside an eps that is smaller still; they are held to 2^-149, which a
    root takes half of."""
    twin = Twin([tensor(256, torch.float32, 1)], bits)
    twin.check_step(ctx, [torch.full((256,), 3e-19, device="cuda")], eps=1e-30)
    twin.check_step(ctx, [torch.full((256,), -2e-19, device="cuda")], eps=1e-30)


def test_blocks_of_zeros_and_of_one_number(ctx):
    g = torch.zeros(160, device="cuda")
    g[40] = 3.0
    g[64:96] = 2.0 ** -20
    g[96:128] = -1.5
    g[159] = 1e-38
    twin = Twin([tensor(160, torch.float32, 1)], 8)
    for _ in range(4):
        twin.check_step(ctx, [g])


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_what_is_not_finite_stays_in_its_block(ctx, bad):
    params = [tensor(200, torch.float32, 1), tensor(50, torch.float32, 2)]
    clean = [p.clone() for p in params]
    g = grads_of((200, 50), [torch.float32], 1)
    one, other = B.AdamWState(params, bits=8), B.AdamWState(clean, bits=8)
    hurt = [g[0].clone(), g[1]]
    hurt[0][70] = bad
    ctx.adamw_step(one, hurt)
    ctx.adamw_step(other, g)
    keep = torch.arange(200, device="cuda") != 70
    assert torch.equal(params[0][keep], clean[0][keep]) and torch.isnan(params[0][70]) and torch.equal(params[1], clean[1])
    for a, b in zip(ctx.adamw_values(one), ctx.adamw_values(other)):
        block = torch.arange(a.numel(), device="cuda") // 32 == 2
        assert torch.isnan(a[block]).all() and torch.equal(a[~block], b[~block])
    assert one.m_scale[2] == 255 and one.v_scale[2] == 255 and (one.m_scale[:2] != 255).all()


def test_step_and_rate_on_the_gpu(ctx):
    """The same steps with their number and rate in device memory."""
    sizes = [100, 3_000]
    for bits in (32, 8):
        params = [tensor(n, torch.float32, n) for n in sizes]
        again = [p.clone() for p in params]
        here = B.AdamWState(params, bits=bits, step=4)
        there = B.AdamWState(again, bits=bits, step=torch.full((1,), 4, dtype=torch.int64, device="cuda"))
        rate = torch.full((1,), 0.125, device="cuda")
        for step in range(3):
            g = grads_of(sizes, BOTH, step)
            ctx.adamw_step(here, g, lr=0.125)
            ctx.adamw_step(there, g, lr=rate)
            for a, b in zip(params + [here.m, here.v], again + [there.m, there.v]):
                assert torch.equal(a, b)
        assert here.step == 7 and there.step.item() == 7


def test_large_steps_count_and_seeds_differ(ctx):
    p = [tensor(4_096, torch.float32, 1)]
    g = grads_of([4_096], [torch.float32], 1)
    twin = Twin([p[0].clone()], 8, seed=0xFFFFFFFF, step=(1 << 33) + 5)
    twin.check_step(ctx, g)
    a, b = B.AdamWState([p[0].clone()], bits=8, seed=1), B.AdamWState([p[0].clone()], bits=8, seed=2)
    ctx.adamw_step(a, g)
    ctx.adamw_step(b, g)
    assert not torch.equal(a.m, b.m) and torch.equal(a.m_scale, b.m_scale) and torch.equal(a.params[0], b.params[0])


def test_values_of_every_code(ctx):
    codes = torch.arange(256, dtype=torch.uint8, device="cuda").repeat(6)
    for scale in (7, 15, 100, 127, 200, 247, 255):
        scales = torch.full((48,), scale, dtype=torch.uint8, device="cuda")
        for moment in (1, 2):
            want = torch.tensor(O.decode(codes.cpu().numpy(), scales.cpu().numpy(), moment), device="cuda")
            for dtype in BOTH:
                out = torch.empty(codes.numel(), dtype=dtype, device="cuda")
                arrays = [codes.data_ptr(), scales.data_ptr()]
                arrays = [*arrays, None, None, codes.numel(), out.data_ptr(), None] if moment == 1 else \
                    [None, None, *arrays, codes.numel(), None, out.data_ptr()]
                assert ctx._lib.ais_adamw_values(ctx._h, *arrays, B.AIS_BF16 if dtype == torch.bfloat16 else B.AIS_F32) == 0
                assert torch.equal(torch.nan_to_num(out, nan=7.0), torch.nan_to_num(want.to(dtype), nan=7.0)), (scale, moment, dtype)


def test_refusals(ctx):
    p = [tensor(64, torch.float32, 1), tensor(32, torch.bfloat16, 2)]
    g = grads_of((64, 32), [torch.float32], 1)
    with pytest.raises(ValueError):
        B.AdamWState([])
    with pytest.raises(ValueError):
        B.AdamWState(p, bits=16)
    with pytest.raises(ValueError):
        B.AdamWState([p[0], p[0]])
    with pytest.raises(ValueError):
        B.AdamWState([p[0], p[0][32:]])
    with pytest.raises(ValueError):
        B.AdamWState([p[0][::2]])
    with pytest.raises(ValueError):
        B.AdamWState([p[0].cpu()])
    with pytest.raises(TypeError):
        B.AdamWState([p[0].half()])
    with pytest.raises(TypeError):
        B.AdamWState([p[0]], copies=[torch.zeros(64, device="cuda")])
    with pytest.raises(ValueError):
        B.AdamWState([p[0]], copies=[p[1]])
    with pytest.raises(ValueError):
        B.AdamWState([p[1]], copies=[p[1]])
    with pytest.raises(ValueError):
        B.AdamWState(p, bits=32, m_scale=torch.zeros(3, dtype=torch.uint8, device="cuda"))
    with pytest.raises(TypeError):
        B.AdamWState(p, bits=8, m=torch.zeros(96, device="cuda"))
    with pytest.raises(ValueError):
        B.AdamWState(p, bits=8, m=torch.zeros(97, dtype=torch.uint8, device="cuda")[1:])
    state = B.AdamWState(p, bits=8)
    for bad, error in (([g[0]], ValueError), ([g[0], g[0]], ValueError), ([g[0], g[1].half()], TypeError), ([g[0], g[1].cpu()], ValueError),
                       ([g[0], 3], TypeError), ([torch.zeros(128, device="cuda")[::2], g[1]], ValueError)):
        with pytest.raises(error):
            ctx.adamw_step(state, bad)
    for rule in (dict(lr=-1.0), dict(beta1=1.0), dict(eps=0.0), dict(weight_decay=float("nan"))):
        with pytest.raises(B.AisError):
            ctx.adamw_step(state, g, **rule)
    with pytest.raises(TypeError):
        ctx.adamw_step(state, g, grad_scale=torch.ones(1, dtype=torch.float64, device="cuda"))
    assert state.step == 0
    p[0].data = p[0].clone()
    with pytest.raises(ValueError):
        ctx.adamw_step(state, g)
    assert state.step == 0
    with pytest.raises(TypeError):
        ctx.adamw_values(state, dtype=torch.float16)
    with pytest.raises(ValueError):
        ctx.adamw_values(B.AdamWState([tensor(64, torch.float32, 1)]))
