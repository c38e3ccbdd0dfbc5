"""The native calls of the 4-bit rollout and the distillation loss against the methods' own way: same results to the bit, same
refusals."""
import pytest
import torch

from paper_2605_13907_amd import binding as B
from tests.test_gpu_native_calls import bad_forms, both, same  # noqa: F401 (both: a fixture)

pytestmark = pytest.mark.gpu


def arguments():
    n, v, d = 8, 70, 100
    gen = torch.Generator(device="cuda").manual_seed(3)
    z = torch.randn(n, v, generator=gen, device="cuda")
    h, w = torch.randn(n, d, generator=gen, device="cuda"), torch.randn(v, d, generator=gen, device="cuda").bfloat16()
    f = torch.rand(n, generator=gen, device="cuda")
    ids = torch.topk(z, 5, dim=1)
    ctx = B.AisContext()
    hc, hs = ctx.mxfp4_quantize_rows(h)
    wc, ws = ctx.mxfp4_quantize_rows(w)
    torch.cuda.synchronize()
    ctx.close()
    valid = torch.tensor([1, 1, 0, 1, 1, 1, 0, 1], device="cuda", dtype=torch.uint8)
    return {
        "mxfp4_quantize_rows": dict(x=h),
        "mxfp4_logits": dict(hidden_codes=hc, hidden_scales=hs, weight_codes=wc, weight_scales=ws),
        "sample_tokens": dict(logits=z, noise=torch.empty_like(z).exponential_(generator=gen), valid=valid, temperature=f + 0.5,
                              top_k=torch.arange(n, device="cuda", dtype=torch.int32), top_p=f, min_p=f * 0.1),
        "distill_topk": dict(logits=z, teacher_ids=ids.indices.int(), teacher_logits=ids.values, weight=f, valid=valid),
    }


def test_same_results(both):  # noqa: F811
    for name, args in arguments().items():
        variants = [args]
        if name == "mxfp4_quantize_rows":
            variants += [dict(args, want_values=True), dict(x=args["x"].bfloat16()), dict(x=args["x"][:, 3:40], want_values=True),
                         dict(x=args["x"][:1]), dict(x=args["x"][:0])]
        if name == "mxfp4_logits":
            variants += [dict(args, dtype=torch.float32), dict(args, hidden_codes=args["hidden_codes"][::2], hidden_scales=args["hidden_scales"][::2])]
        if name == "sample_tokens":
            variants += [{k: args[k] for k in ("logits", "noise")}, dict(args, logits=args["logits"].bfloat16()),
                         dict(args, logits=args["logits"][:, 1:], noise=args["noise"][:, 1:])]
        if name == "distill_topk":
            variants += [dict(args, want_grad=False), dict(args, weight=None, valid=None, inv_temperature=0.5),
                         dict(args, logits=args["logits"][:, 1:], teacher_ids=args["teacher_ids"] - 1),
                         dict(args, dlogits=torch.zeros_like(args["logits"]))]
        for v in variants:
            assert both[0]._native is not None
            same(getattr(both[0], name)(**v), getattr(both[1], name)(**v))


def test_numbers_for_all_rows(both):  # noqa: F811
    a = arguments()["sample_tokens"]
    n = a["logits"].shape[0]
    full = [torch.full((n,), x, device="cuda", dtype=t) for x, t in ((0.7, torch.float32), (9, torch.int32), (0.8, torch.float32), (0.01, torch.float32))]
    want = both[0].sample_tokens(a["logits"], a["noise"], None, *full)
    for ctx in both:
        same(ctx.sample_tokens(a["logits"], a["noise"], None, 0.7, 9, 0.8, 0.01), want)


def test_one_wrong_argument_at_a_time(both):  # noqa: F811
    """Every array of every call: refused by both ways, before anything is launched, with the same error."""
    sized_by_others = {("mxfp4_quantize_rows", "x")}
    for name, args in arguments().items():
        for arg, t in args.items():
            for k, wrong in enumerate(bad_forms(t)):
                if k == 2 and (name, arg) in sized_by_others:
                    continue
                errors = []
                for ctx in both:
                    with pytest.raises((TypeError, ValueError)) as e:
                        getattr(ctx, name)(**{**args, arg: wrong})
                    errors.append((type(e.value), str(e.value)))
                assert errors[0] == errors[1], (name, arg, k, errors)
    z = arguments()["distill_topk"]
    for ctx in both:
        for out in (z["logits"].bfloat16(), z["logits"][:4], torch.zeros(8, 80, device="cuda")[:, :70]):
            with pytest.raises(ValueError):
                ctx.distill_topk(**z, dlogits=out)
        with pytest.raises(B.AisError):
            ctx.distill_topk(**z, inv_temperature=-1.0)
        with pytest.raises(TypeError):
            ctx.mxfp4_logits(**arguments()["mxfp4_logits"], dtype=torch.float16)


def test_storage_that_refuses_its_address(both):  # noqa: F811
    """A C++ exception in the middle of a native call: the method's own way raises it, and the interpreter goes on."""
    a = arguments()
    for t in (a["mxfp4_quantize_rows"]["x"], a["mxfp4_logits"]["hidden_codes"], a["sample_tokens"]["logits"], a["distill_topk"]["logits"]):
        torch._C._set_throw_on_mutable_data_ptr(t)
    for name, args in a.items():
        for ctx in both:
            with pytest.raises(RuntimeError, match="Cannot access data pointer"):
                getattr(ctx, name)(**args)
    torch.cuda.synchronize()
