"""Argument checks of the preference loss's, the normalised rows' and the AdamW step's entry points: on the host, before any launch,
so that no GPU is needed (every pointer below is one that is never looked at)."""
import ctypes as C

import pytest

from paper_2605_13907_amd import binding as B
from tests.test_rollout_abi import P, Q, caller

NAN, INF = float("nan"), float("inf")


def preference(**kw):
    return C.byref(B.default_preference_params(**kw))


BAD_PREFERENCE = [dict(beta=0.0), dict(beta=-1.0), dict(beta=NAN), dict(beta=INF), dict(kind=-1), dict(kind=3), dict(label_smoothing=-0.1),
                  dict(label_smoothing=0.6), dict(label_smoothing=NAN), dict(kind=1, label_smoothing=0.1), dict(kind=2, label_smoothing=0.1),
                  dict(margin=NAN), dict(margin=INF), dict(mean_logp=2), dict(mean_logp=-1), dict(inv_temperature=0.0),
                  dict(inv_temperature=NAN)]


def test_preference_defaults():
    p = B.default_preference_params()
    assert (p.kind, p.mean_logp, p.margin, p.label_smoothing, p.inv_temperature) == (0, 0, 0.0, 0.0, 1.0)
    assert p.beta == pytest.approx(0.1)
    B._lib().ais_preference_params_default(None)
    B._lib().ais_adamw_params_default(None)
    with pytest.raises(AttributeError):
        B.default_preference_params(gamma=1.0)


def test_preference_row_scale():
    order = "ctx logp ref valid n_rows cu n_resp weight params reward loss g".split()
    call = caller("ais_preference_row_scale", order, dict(ctx=None, logp=P, ref=None, valid=None, n_rows=10, cu=P, n_resp=4, weight=None,
                                                          params=preference(), reward=Q, loss=Q, g=Q))
    assert call() == -1                                          # everything fine except the NULL context
    for missing in ("logp", "cu", "params", "reward", "loss", "g"):
        assert call(**{missing: None}) == -1
    assert call(n_rows=-1) == -2 and call(n_rows=2 ** 31) == -2 and call(n_resp=0) == -2 and call(n_resp=2 ** 24 + 2) == -2
    assert call(n_resp=3) == -6
    for bad in BAD_PREFERENCE:
        assert call(params=preference(**bad)) == -5, bad
    assert call(n_rows=0, logp=None, g=None) == -1


def test_preference_loss_grad():
    order = "ctx z dtype n_rows vocab stride ids valid cu n_resp ref weight params reward loss logp dz".split()
    call = caller("ais_preference_loss_grad", order,
                  dict(ctx=None, z=P, dtype=B.AIS_BF16, n_rows=10, vocab=64, stride=64, ids=P, valid=None, cu=P, n_resp=2, ref=None,
                       weight=None, params=preference(), reward=Q, loss=Q, logp=Q, dz=Q))
    assert call() == -1 and call(dz=None) == -1
    for missing in ("z", "ids", "cu", "logp", "params", "reward", "loss"):
        assert call(**{missing: None}) == -1
    assert call(vocab=0) == -2 and call(n_rows=-1) == -2 and call(stride=63) == -3 and call(dtype=2) == -7 and call(n_resp=5) == -6
    assert call(z=C.c_void_p(0x1001)) == -4 and call(dz=C.c_void_p(0x1001)) == -4
    for bad in BAD_PREFERENCE:
        assert call(params=preference(**bad)) == -5, bad
    assert call(n_rows=0, z=None, ids=None, logp=None, dz=None) == -1


def test_norm_rows():
    order = "ctx x dtype n_rows width stride valid weight bias param_dtype eps centered y y_stride mean rstd".split()
    call = caller("ais_norm_rows", order, dict(ctx=None, x=P, dtype=B.AIS_BF16, n_rows=3, width=100, stride=100, valid=None, weight=P, bias=P,
                                               param_dtype=B.AIS_F32, eps=1e-5, centered=1, y=Q, y_stride=100, mean=Q, rstd=Q))
    assert call() == -1 and call(weight=None, bias=None) == -1 and call(centered=0, mean=None) == -1
    for missing in ("x", "y", "mean", "rstd"):
        assert call(**{missing: None}) == -1
    assert call(n_rows=-1) == -2 and call(width=0) == -2 and call(width=2 ** 31 - 4, stride=2 ** 31, y_stride=2 ** 31) == -2
    assert call(stride=99) == -3 and call(y_stride=99) == -3
    assert call(dtype=2) == -7 and call(param_dtype=2) == -7
    for bad in (0.0, -1.0, NAN, INF):
        assert call(eps=bad) == -5
    assert call(centered=2) == -5
    assert call(x=C.c_void_p(0x1001)) == -4 and call(y=C.c_void_p(0x1001)) == -4
    assert call(weight=C.c_void_p(0x1002)) == -4 and call(bias=C.c_void_p(0x1002)) == -4
    assert call(param_dtype=B.AIS_BF16, weight=C.c_void_p(0x1002)) == -1
    assert call(n_rows=0, x=None, y=None, mean=None, rstd=None) == -1


def test_norm_rows_grad():
    order = ("ctx dy dy_dtype dy_stride x dtype n_rows width stride valid weight param_dtype mean rstd dx dx_stride dweight dbias").split()
    call = caller("ais_norm_rows_grad", order,
                  dict(ctx=None, dy=P, dy_dtype=B.AIS_F32, dy_stride=100, x=P, dtype=B.AIS_BF16, n_rows=3, width=100, stride=100, valid=None,
                       weight=P, param_dtype=B.AIS_F32, mean=None, rstd=P, dx=Q, dx_stride=100, dweight=Q, dbias=Q))
    assert call() == -1 and call(weight=None, dweight=None, dbias=None) == -1
    for missing in ("dy", "x", "rstd", "dx"):
        assert call(**{missing: None}) == -1
    assert call(n_rows=-1) == -2 and call(width=0) == -2
    assert call(stride=99) == -3 and call(dy_stride=99) == -3 and call(dx_stride=99) == -3
    assert call(dtype=2) == -7 and call(dy_dtype=3) == -7 and call(param_dtype=-1) == -7
    assert call(x=C.c_void_p(0x1001)) == -4 and call(dy=C.c_void_p(0x1002)) == -4 and call(dx=C.c_void_p(0x1001)) == -4
    assert call(weight=C.c_void_p(0x1002)) == -4
    assert call(n_rows=0, dy=None, x=None, rstd=None, dx=None) == -1


def adamw(tensors=None, n=1, ctx=None, table=P, scale=None, step_dev=None, lr_dev=None, **rule):
    p = B.AisAdamWParams()
    B._lib().ais_adamw_params_default(C.byref(p))
    for k, v in rule.items():
        setattr(p, k, v)
    t = dict(param=0x1000, grad=0x2000, copy=None, m=0x3000, v=0x4000, m_scale=0x5000, v_scale=0x5000, n=100, param_dtype=1, grad_dtype=1)
    t.update(tensors or {})
    return B._lib().ais_adamw_step(ctx, (B.AisAdamWTensor * 2)(B.AisAdamWTensor(**t), B.AisAdamWTensor(**t)), table, n, C.byref(p), scale, step_dev,
                                   lr_dev)


def test_adamw_step():
    assert adamw() == -1 and adamw(state_bits=8) == -1 and adamw(n=2) == -1 and adamw(n=0) == -1
    assert adamw(n=-1) == -2
    for missing in ("param", "m", "v"):
        assert adamw({missing: None}) == -1
    assert adamw(table=None) == -1 and adamw(table=C.c_void_p(0x1004)) == -4
    assert adamw(dict(grad=None, param=None, m=0x3001)) == -1    # not stepped, so nothing else about it counts
    assert adamw(dict(m_scale=None), state_bits=8) == -1 and adamw(dict(m_scale=None)) == -1
    assert adamw(dict(n=-1)) == -2 and adamw(dict(n=2 ** 32 - 4096)) == -2
    assert adamw(dict(n=0, param=None, grad=None, m=None, v=None)) == -1
    assert adamw(dict(param_dtype=2)) == -7 and adamw(dict(grad_dtype=-1)) == -7
    for odd in (dict(param=0x1002), dict(grad=0x2002), dict(copy=0x2001), dict(m=0x3008), dict(v=0x4004)):
        assert adamw(odd) == -4, odd
    for bad in (dict(lr=-1.0), dict(lr=NAN), dict(beta1=-0.1), dict(beta1=1.0), dict(beta2=1.0), dict(beta2=NAN), dict(eps=0.0), dict(eps=INF),
                dict(eps=1e-31), dict(weight_decay=-1.0), dict(weight_decay=INF), dict(state_bits=16), dict(step=0), dict(step=-5)):
        assert adamw(**bad) == -5, bad
    lib = B._lib()
    assert lib.ais_adamw_step(None, None, P, 1, C.byref(B.AisAdamWParams()), None, None, None) == -1
    assert lib.ais_adamw_step(None, (B.AisAdamWTensor * 1)(), P, 1, None, None, None, None) == -1


def test_adamw_values():
    order = "ctx m m_scale v v_scale n m_out v_out dtype".split()
    call = caller("ais_adamw_values", order, dict(ctx=None, m=P, m_scale=P, v=P, v_scale=P, n=100, m_out=Q, v_out=Q, dtype=B.AIS_F32))
    assert call() == -1 and call(dtype=B.AIS_BF16) == -1 and call(m=None, m_scale=None, m_out=None) == -1
    for missing in ("m", "m_scale", "v", "v_scale"):
        assert call(**{missing: None}) == -1
    assert call(m_out=None, v_out=None) == -1 and call(n=-1) == -2 and call(n=2 ** 40 + 1) == -2
    assert call(m=C.c_void_p(0x1008)) == -4 and call(v=C.c_void_p(0x1008)) == -4 and call(m_out=C.c_void_p(0x1002)) == -4
    assert call(v_out=C.c_void_p(0x1002)) == -4 and call(dtype=7) == -7


def test_descriptors_are_laid_out_as_in_the_header():
    assert C.sizeof(B.AisAdamWTensor) == 72 and C.sizeof(B.AisAdamWParams) == 56 and C.sizeof(B.AisPreferenceParams) == 24
