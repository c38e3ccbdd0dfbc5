"""Argument checks of the 4-bit rollout's and the distillation's entry points: on the host, before any launch, so that no GPU is
needed (every pointer below is one that is never looked at)."""
import ctypes as C

from paper_2605_13907_amd import binding as B

P, Q = C.c_void_p(0x1000), C.c_void_p(0x20000)


def caller(name, order, defaults):
    fn = getattr(B._lib(), name)

    def call(**kw):
        assert set(kw) <= set(defaults), kw
        a = {**defaults, **kw}
        return fn(*[a[k] for k in order])

    return call


def test_quantize_rows():
    order = ("ctx x dtype n_rows width stride codes codes_stride scales scales_stride values values_stride").split()
    call = caller("ais_mxfp4_quantize_rows", order, dict(ctx=None, x=P, dtype=B.AIS_BF16, n_rows=3, width=100, stride=100, codes=Q,
                                                         codes_stride=64, scales=Q, scales_stride=4, values=P, values_stride=100))
    assert call() == -1                                          # everything fine except the NULL context
    assert call(values=None, values_stride=0) == -1
    for missing in ("x", "codes", "scales"):
        assert call(**{missing: None}) == -1
    assert call(n_rows=-1) == -2 and call(width=0) == -2 and call(width=2 ** 31 - 60, stride=2 ** 31) == -2
    assert call(stride=99) == -3 and call(codes_stride=48) == -3 and call(scales_stride=0) == -3 and call(values_stride=99) == -3
    assert call(dtype=2) == -7
    assert call(codes_stride=72) == -4 and call(scales_stride=6) == -4
    assert call(codes=C.c_void_p(0x1008)) == -4 and call(scales=C.c_void_p(0x1002)) == -4
    assert call(x=C.c_void_p(0x1001)) == -4 and call(values=C.c_void_p(0x1001)) == -4
    assert call(dtype=B.AIS_F32, values=C.c_void_p(0x1002)) == -4
    assert call(n_rows=0, x=None, codes=None, scales=None, values=None) == -1


def test_logits():
    order = "ctx h hs hsc hscs n_rows w ws wsc wscs vocab width out dtype out_stride".split()
    call = caller("ais_mxfp4_logits", order, dict(ctx=None, h=P, hs=64, hsc=P, hscs=4, n_rows=5, w=Q, ws=64, wsc=Q, wscs=4, vocab=50,
                                                  width=128, out=P, dtype=B.AIS_F32, out_stride=50))
    assert call() == -1
    for missing in ("h", "hsc", "w", "wsc", "out"):
        assert call(**{missing: None}) == -1
    assert call(n_rows=-2) == -2 and call(vocab=0) == -2 and call(width=0) == -2 and call(width=2 ** 31) == -2
    assert call(hs=48) == -3 and call(ws=48) == -3 and call(hscs=3) == -3 and call(wscs=0) == -3 and call(out_stride=49) == -3
    assert call(hs=72) == -4 and call(ws=88) == -4 and call(hscs=5) == -4 and call(wscs=7) == -4
    for odd in ("h", "w"):
        assert call(**{odd: C.c_void_p(0x1004)}) == -4
    for odd in ("hsc", "wsc", "out"):
        assert call(**{odd: C.c_void_p(0x1002)}) == -4
    assert call(dtype=5) == -7
    assert call(n_rows=0, h=None, hsc=None, w=None, wsc=None, out=None) == -1


def test_sample_tokens():
    order = "ctx z dtype n_rows vocab stride noise noise_stride valid temperature top_k top_p min_p token logp full".split()
    call = caller("ais_sample_tokens", order, dict(ctx=None, z=P, dtype=B.AIS_BF16, n_rows=4, vocab=64, stride=64, noise=P,
                                                   noise_stride=64, valid=None, temperature=None, top_k=None, top_p=None, min_p=None,
                                                   token=Q, logp=Q, full=None))
    assert call() == -1
    for missing in ("z", "noise", "token", "logp"):
        assert call(**{missing: None}) == -1
    assert call(n_rows=-1) == -2 and call(vocab=0) == -2 and call(vocab=2 ** 31) == -2
    assert call(stride=63) == -3 and call(noise_stride=63) == -3
    assert call(z=C.c_void_p(0x1001)) == -4 and call(noise=C.c_void_p(0x1002)) == -4
    assert call(dtype=9) == -7
    assert call(n_rows=0, z=None, noise=None, token=None, logp=None) == -1


def test_distill_topk():
    order = "ctx z dtype n_rows vocab stride ids teacher top valid weight inv_t kl loss dz dz_stride".split()
    call = caller("ais_distill_topk", order, dict(ctx=None, z=P, dtype=B.AIS_F32, n_rows=4, vocab=64, stride=70, ids=P, teacher=P, top=8,
                                                  valid=None, weight=None, inv_t=1.0, kl=Q, loss=Q, dz=Q, dz_stride=64))
    assert call() == -1
    assert call(dz=None, dz_stride=0) == -1
    for missing in ("z", "ids", "teacher", "kl", "loss"):
        assert call(**{missing: None}) == -1
    assert call(n_rows=-1) == -2 and call(vocab=0) == -2 and call(top=0) == -2 and call(top=1025) == -2
    assert call(stride=63) == -3 and call(dz_stride=63) == -3
    assert call(z=C.c_void_p(0x1002)) == -4 and call(dz=C.c_void_p(0x1002)) == -4
    assert call(inv_t=0.0) == -5 and call(inv_t=float("inf")) == -5 and call(inv_t=float("nan")) == -5
    assert call(dtype=-1) == -7
    assert call(n_rows=0, z=None, ids=None, teacher=None, kl=None, dz=None) == -1


def test_logits_whose_indices_reach_beyond_32_bits():
    """A tile's indices go on behind the last row: the sizes that leave no room for that are refused."""
    order = "ctx h hs hsc hscs n_rows w ws wsc wscs vocab width out dtype out_stride".split()
    call = caller("ais_mxfp4_logits", order, dict(ctx=None, h=P, hs=64, hsc=P, hscs=4, n_rows=5, w=Q, ws=64, wsc=Q, wscs=4, vocab=50,
                                                  width=128, out=P, dtype=B.AIS_F32, out_stride=2 ** 31))
    most = 2 ** 31 - 1025
    assert call(vocab=most) == -1 and call(vocab=most + 1) == -2
    assert call(n_rows=most) == -1 and call(n_rows=most + 1) == -2
