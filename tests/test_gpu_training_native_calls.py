"""The native calls of the preference loss, the normalised rows and the AdamW step against the methods' own way: same results to the bit,
same refusals."""
import pytest
import torch

from paper_2605_13907_amd import binding as B
from tests.test_gpu_native_calls import bad_forms, both, same  # noqa: F401 (both: a fixture)

pytestmark = pytest.mark.gpu


def arguments():
    n, v, d = 8, 70, 100
    gen = torch.Generator(device="cuda").manual_seed(3)
    randn = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    z, x, dy = randn(n, v), randn(n, d), randn(n, d)
    logp = -torch.rand(n, generator=gen, device="cuda")
    valid = torch.tensor([1, 1, 0, 1, 1, 1, 0, 1], device="cuda", dtype=torch.uint8)
    cu = torch.tensor([0, 3, 5, 6, 8], device="cuda")
    pair = dict(logp_train=logp, logp_ref=logp - 0.1, valid=valid, cu_rows=cu, weight=torch.rand(2, generator=gen, device="cuda"))
    through = {k: t for k, t in pair.items() if k != "logp_train"}
    return {
        "preference_row_scale": pair,
        "preference_loss_grad": dict(through, logits=z, token_ids=torch.arange(n, device="cuda", dtype=torch.int32)),
        "norm_rows": dict(x=x, weight=randn(d), bias=randn(d), valid=valid),
        "norm_rows_grad": dict(dy=dy, x=x, weight=randn(d), mean=0.1 * randn(n), rstd=1.0 + logp.abs(), valid=valid),
    }


def test_same_results(both):  # noqa: F811
    for name, args in arguments().items():
        variants = [args, dict(args, valid=None)]
        if name.startswith("preference"):
            variants += [dict(args, logp_ref=None, weight=None), dict(args, params=B.default_preference_params(kind=2, mean_logp=1))]
        if name == "preference_loss_grad":
            variants += [dict(args, logits=args["logits"].bfloat16()), dict(args, logits=args["logits"][:, 1:]),
                         dict(args, dlogits=torch.zeros_like(args["logits"])), dict(args, want_grad=False)]
        if name == "norm_rows":
            x = args["x"]
            variants += [dict(x=x), dict(args, centered=False, bias=None), dict(args, x=x.bfloat16()), dict(args, weight=None),
                         dict(x=x[:, 3:40], eps=0.1), dict(x=x[:1]), dict(x=x[:0]), dict(args, weight=args["weight"].bfloat16(),
                                                                                          bias=args["bias"].bfloat16())]
        if name == "norm_rows_grad":
            variants += [dict(args, mean=None), dict(args, weight=None, want_bias=False), dict(args, dy=args["dy"].bfloat16()),
                         dict(args, x=args["x"].bfloat16(), weight=args["weight"].bfloat16()), dict(args, want_bias=False),
                         {k: t[:0] if k != "weight" else t for k, t in args.items()}]
        for v in variants:
            assert both[0]._native is not None
            same(getattr(both[0], name)(**v), getattr(both[1], name)(**v))


def test_one_wrong_argument_at_a_time(both):  # noqa: F811
    """Every array of every call: refused by both ways, before anything is launched, with the same error."""
    # of an array that gives the call its sizes a shorter one is the others' fault, or none's
    alone = {("preference_row_scale", "cu_rows"), ("preference_loss_grad", "cu_rows")}
    for name, args in arguments().items():
        for arg, t in args.items():
            for k, wrong in enumerate(bad_forms(t)):
                if k == 2 and (name, arg) in alone:
                    continue
                errors = []
                for ctx in both:
                    with pytest.raises((TypeError, ValueError)) as e:
                        getattr(ctx, name)(**{**args, arg: wrong})
                    errors.append((type(e.value), str(e.value)))
                assert errors[0] == errors[1], (name, arg, k, errors)
    a = arguments()
    for ctx in both:
        for cu in (a["preference_row_scale"]["cu_rows"][:4], torch.zeros(1, dtype=torch.int64, device="cuda")):
            with pytest.raises((B.AisError, ValueError)):
                ctx.preference_row_scale(**dict(a["preference_row_scale"], cu_rows=cu, weight=None))
        with pytest.raises(B.AisError):
            ctx.preference_row_scale(**a["preference_row_scale"], params=B.default_preference_params(beta=-1.0))
        with pytest.raises(B.AisError):
            ctx.norm_rows(**a["norm_rows"], eps=0.0)
        with pytest.raises(TypeError):
            ctx.norm_rows(**dict(a["norm_rows"], bias=a["norm_rows"]["bias"].bfloat16()))
        with pytest.raises(ValueError):
            ctx.norm_rows_grad(**dict(a["norm_rows_grad"], dy=a["norm_rows_grad"]["dy"][:, 1:]))
        with pytest.raises(ValueError):
            ctx.preference_loss_grad(**a["preference_loss_grad"], dlogits=torch.zeros(8, 80, device="cuda")[:, :70])


@pytest.mark.parametrize("bits", [32, 8])
def test_the_step(both, bits):  # noqa: F811
    gen = torch.Generator(device="cuda").manual_seed(1)
    sizes, types = [100, 0, 2_049, 31], [torch.float32, torch.bfloat16]
    states = []
    params = [torch.randn(n, generator=gen, device="cuda").to(types[i % 2]) for i, n in enumerate(sizes)]
    for _ in both:
        mine = [torch.nn.Parameter(p.clone()) for p in params]
        states.append(B.AdamWState(mine, bits=bits, copies=[torch.zeros(n, dtype=torch.bfloat16, device="cuda") for n in sizes], seed=9))
    scale, rate = torch.full((1,), 0.5, device="cuda"), torch.full((1,), 0.01, device="cuda")
    for step in range(4):
        grads = [torch.randn(n, generator=gen, device="cuda").to(types[(i + step) % 2]) for i, n in enumerate(sizes)]
        if step == 2:
            grads[2] = None
        for ctx, s in zip(both, states):
            ctx.adamw_step(s, tuple(grads) if step == 1 else grads, lr=rate if step % 2 else 0.02, grad_scale=scale if step else None)
        torch.cuda.synchronize()
        for a, b in zip((*states[0].params, *states[0].copies, states[0].m, states[0].v), (*states[1].params, *states[1].copies, states[1].m,
                                                                                     states[1].v)):
            assert torch.equal(a, b), step
        assert states[0].step == states[1].step == step + 1
    if bits == 8:
        same(both[0].adamw_values(states[0]), both[1].adamw_values(states[1]))
        same(both[0].adamw_values(states[0], torch.bfloat16), both[1].adamw_values(states[1], torch.bfloat16))


def test_moved_arrays_are_refused(both):  # noqa: F811
    for ctx in both:
        for name in ("m", "v", "m_scale", "v_scale"):
            s = B.AdamWState([torch.ones(64, device="cuda")], bits=8, copies=[torch.zeros(64, dtype=torch.bfloat16, device="cuda")])
            setattr(s, name, getattr(s, name).clone())
            with pytest.raises(ValueError, match=f"{name} is not where it was"):
                ctx.adamw_step(s, [torch.ones(64, device="cuda")])
        s.copies[0].data = s.copies[0].clone()
        s = B.AdamWState([torch.ones(64, device="cuda")], copies=[torch.zeros(64, dtype=torch.bfloat16, device="cuda")])
        s.copies[0].data = s.copies[0].clone()
        with pytest.raises(ValueError, match="is not where it was"):
            ctx.adamw_step(s, [torch.ones(64, device="cuda")])


def test_storage_that_refuses_its_address(both):  # noqa: F811
    """A C++ exception in the middle of a native call: the method's own way raises it, and the interpreter goes on."""
    a = arguments()
    for t in (a["preference_row_scale"]["logp_train"], a["preference_loss_grad"]["logits"], a["norm_rows"]["x"], a["norm_rows_grad"]["dy"]):
        torch._C._set_throw_on_mutable_data_ptr(t)
    for name, args in a.items():
        for ctx in both:
            with pytest.raises(RuntimeError, match="Cannot access data pointer"):
                getattr(ctx, name)(**args)
    g = torch.ones(64, device="cuda")
    state = B.AdamWState([torch.ones(64, device="cuda")])
    torch._C._set_throw_on_mutable_data_ptr(g)
    for ctx in both:
        with pytest.raises(RuntimeError, match="Cannot access data pointer"):
            ctx.adamw_step(state, [g])
    assert state.step == 0
    torch.cuda.synchronize()
