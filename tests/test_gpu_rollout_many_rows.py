"""More rows than one launch has threads for: 2^21 and some, of which every thousand are the same."""
import pytest
import torch

from paper_2605_13907_amd import binding as B

pytestmark = pytest.mark.gpu

ROWS, SAME = (1 << 21) + 1003, 1000


@pytest.fixture(scope="module")
def ctx():
    c = B.AisContext()
    yield c
    c.close()


def repeated(t):
    return t.repeat(ROWS // SAME + 1, *[1] * (t.dim() - 1))[:ROWS].contiguous()


def rows(width, seed, dtype=torch.bfloat16):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(SAME, width, generator=gen, device="cuda").to(dtype)


def test_sample(ctx):
    z = rows(5, 1)
    e = torch.empty(SAME, 5, device="cuda").exponential_(generator=torch.Generator(device="cuda").manual_seed(2))
    limits = dict(valid=(torch.arange(SAME, device="cuda") % 7 != 0).to(torch.uint8),
                  temperature=torch.linspace(0.2, 2.0, SAME, device="cuda"),
                  top_k=(torch.arange(SAME, device="cuda") % 4).int())
    few = ctx.sample_tokens(z, e, **limits)
    many = ctx.sample_tokens(repeated(z), repeated(e), **{n: repeated(v) for n, v in limits.items()})
    for a, b in zip(few, many):
        assert torch.equal(repeated(a), b)


@pytest.mark.parametrize("want_grad", [False, True])
def test_distill(ctx, want_grad):
    z = rows(6, 3)
    ids = torch.arange(2, dtype=torch.int32, device="cuda").repeat(SAME, 1)
    teacher = rows(2, 4, torch.float32)
    valid = (torch.arange(SAME, device="cuda") % 7 != 0).to(torch.uint8)
    weight = torch.full((SAME,), 0.25, device="cuda")
    few = ctx.distill_topk(z, ids, teacher, weight, valid, want_grad=want_grad)
    many = ctx.distill_topk(repeated(z), repeated(ids), repeated(teacher), repeated(weight), repeated(valid), want_grad=want_grad)
    assert torch.equal(repeated(few[1]), many[1])
    want = 0.25 * many[1].double().sum().item()
    assert abs(many[0].item() - want) <= 2.0 ** -24 * abs(want) * 1.01         # summed in fp64, rounded once
    if want_grad:
        assert torch.equal(repeated(few[2]), many[2])


def test_quantize(ctx):
    x = rows(9, 5)
    few, many = ctx.mxfp4_quantize_rows(x, want_values=True), ctx.mxfp4_quantize_rows(repeated(x), want_values=True)
    for a, b in zip(few, many):
        assert torch.equal(repeated(a), b)
