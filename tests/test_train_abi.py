"""The training-side calls validate their arguments on the host before anything is launched (no GPU needed)."""
import ctypes

import pytest
import torch

import paper_2303_08999_b200 as sr
from paper_2303_08999_b200 import api, build

FAKE = 0x1000        # never dereferenced: every call below fails validation before any launch
BIG = 1 << 40


@pytest.fixture(scope="module")
def lib():
    build.build()
    return sr.load_library()


def _dims(**kw):
    base = dict(n=1, c=3, h=4, w=4, scale=2, k=5, D=8)
    base.update(kw)
    return api.sr_dims(*(base[f] for f in ("n", "c", "h", "w", "scale", "k", "D")))


def test_dense_gradient_refusals(lib):
    def call(d=None, lr=FAKE, coef=FAKE, dt=api.SR_F16, dict_=FAKE, gout=FAKE, gcoef=FAKE, gdict=FAKE, flags=0, scratch=FAKE, nbytes=BIG):
        return lib.sr_dict_regress_dense_grad(lr, coef, dt, dict_, gout, gcoef, gdict, ctypes.byref(d or _dims()), flags, scratch, nbytes, None)
    for name in ("lr", "dict_", "gout", "coef", "scratch"):
        assert call(**{name: None}) == api.SR_ERR_NULL, name
    assert call(gcoef=None, gdict=None) == api.SR_ERR_NULL
    assert lib.sr_dict_regress_dense_grad(FAKE, FAKE, 1, FAKE, FAKE, FAKE, FAKE, None, 0, FAKE, BIG, None) == api.SR_ERR_NULL
    for d, want in ((_dims(k=4), api.SR_ERR_UNSUPPORTED), (_dims(k=11), api.SR_ERR_UNSUPPORTED), (_dims(scale=9), api.SR_ERR_UNSUPPORTED),
                    (_dims(D=257), api.SR_ERR_UNSUPPORTED), (_dims(D=0), api.SR_ERR_SHAPE), (_dims(n=0), api.SR_ERR_SHAPE),
                    (_dims(h=70000, w=70000), api.SR_ERR_SHAPE)):
        assert call(d) == want
        assert lib.sr_dict_regress_grad_scratch_bytes(ctypes.byref(d)) == 0
    assert lib.sr_dict_regress_grad_scratch_bytes(None) == 0
    assert call(dt=2) == api.SR_ERR_UNSUPPORTED                       # bfloat16 exists for the optimiser only
    for flag in (api.SR_CLAMP01, api.SR_IDX_GLOBAL, api.SR_COEF_COMPACT, api.SR_OUT_F16, api.SR_OUT_U8, api.SR_LUMA_ONLY, api.SR_GRAD_ADD, 512):
        assert call(flags=flag) == api.SR_ERR_UNSUPPORTED
    for name in ("lr", "dict_", "gout", "gdict"):
        assert call(**{name: FAKE + 2}) == api.SR_ERR_ALIGN, name
    assert call(coef=FAKE + 1) == api.SR_ERR_ALIGN and call(gcoef=FAKE + 1) == api.SR_ERR_ALIGN
    assert call(gcoef=FAKE + 2, dt=api.SR_F32) == api.SR_ERR_ALIGN and call(scratch=FAKE + 8) == api.SR_ERR_ALIGN
    need = lib.sr_dict_regress_grad_scratch_bytes(ctypes.byref(_dims()))
    assert need > 0 and call(nbytes=need - 1) == api.SR_ERR_SHAPE


def test_selected_gradient_refusals(lib):
    def call(d=None, s=4, idx=FAKE, gamma=None, ggamma=None, flags=0, gcoef=FAKE, gdict=FAKE, coef=FAKE, scratch=FAKE, nbytes=BIG):
        return lib.sr_dict_regress_selected_grad(FAKE, coef, api.SR_F16, idx, gamma, FAKE, FAKE, gcoef, gdict, ggamma, ctypes.byref(d or _dims()), s,
                                                 flags, scratch, nbytes, None)
    assert call(idx=None) == api.SR_ERR_NULL and call(idx=None, flags=api.SR_IDX_GLOBAL) == api.SR_ERR_NULL
    assert call(gcoef=None, gdict=None) == api.SR_ERR_NULL
    assert call(s=0) == api.SR_ERR_SHAPE and call(s=9) == api.SR_ERR_SHAPE
    assert call(gamma=FAKE) == api.SR_ERR_UNSUPPORTED and call(ggamma=FAKE) == api.SR_ERR_UNSUPPORTED       # the subset's alone
    assert call(flags=api.SR_CLAMP01) == api.SR_ERR_UNSUPPORTED
    assert call(gamma=FAKE + 2, flags=api.SR_IDX_GLOBAL) == api.SR_ERR_ALIGN
    assert call(ggamma=FAKE + 2, flags=api.SR_IDX_GLOBAL) == api.SR_ERR_ALIGN
    assert call(gcoef=None, gdict=None, ggamma=FAKE, flags=api.SR_IDX_GLOBAL, scratch=None) == api.SR_ERR_NULL
    assert call(coef=None) == api.SR_ERR_NULL and call(nbytes=16) == api.SR_ERR_SHAPE


def test_balance_refusals(lib):
    def call(d=None, s=4, coef=FAKE, idx=FAKE, dt=api.SR_F16, loss=FAKE, counts=FAKE, share=FAKE, slope=FAKE, flags=0, scratch=FAKE, nbytes=BIG):
        return lib.sr_select_balance(coef, dt, idx, None, loss, counts, share, slope, ctypes.byref(d or _dims()), s, flags, scratch, nbytes, None)
    for name in ("coef", "idx", "loss", "counts", "share", "slope", "scratch"):
        assert call(**{name: None}) == api.SR_ERR_NULL, name
    assert call(s=0) == api.SR_ERR_SHAPE and call(s=9) == api.SR_ERR_SHAPE and call(dt=5) == api.SR_ERR_UNSUPPORTED
    assert call(flags=api.SR_GRAD_ADD) == api.SR_ERR_UNSUPPORTED and call(_dims(D=300)) == api.SR_ERR_UNSUPPORTED
    for name in ("loss", "counts", "share", "slope", "scratch"):
        assert call(**{name: FAKE + 2}) == api.SR_ERR_ALIGN, name
    assert call(coef=FAKE + 1) == api.SR_ERR_ALIGN
    need = lib.sr_select_balance_scratch_bytes(ctypes.byref(_dims()))
    assert need > 0 and call(nbytes=need - 1) == api.SR_ERR_SHAPE and lib.sr_select_balance_scratch_bytes(None) == 0

    def grad(coef=FAKE, slope=FAKE, out=FAKE, dt=api.SR_F16, flags=0, gl=None, d=None):
        return lib.sr_select_balance_grad(coef, dt, None, slope, gl, 1.0, out, ctypes.byref(d or _dims()), flags, None)
    assert grad(coef=None) == api.SR_ERR_NULL and grad(slope=None) == api.SR_ERR_NULL and grad(out=None) == api.SR_ERR_NULL
    assert grad(flags=api.SR_BALANCE_PER_FRAME) == api.SR_ERR_UNSUPPORTED and grad(dt=2) == api.SR_ERR_UNSUPPORTED
    assert grad(out=FAKE + 1) == api.SR_ERR_ALIGN and grad(slope=FAKE + 2) == api.SR_ERR_ALIGN and grad(gl=FAKE + 2) == api.SR_ERR_ALIGN
    assert grad(d=_dims(w=0)) == api.SR_ERR_SHAPE


def test_adamw_refusals(lib):
    def call(count=1, pd=0, gd=0, bits=32, tensor=None, **opts):
        o = api.sr_adamw_opts(1e-3, 0.9, 0.999, 1e-8, 0.01, 1.0, 1, None, None, None)
        for name, value in opts.items():
            setattr(o, name, value)
        t = dict(param=FAKE, grad=FAKE, m=FAKE, v=FAKE, m_scale=FAKE, v_scale=FAKE, n=5)
        t.update(tensor or {})
        return lib.sr_adamw_step((api.sr_adamw_tensor * 1)(api.sr_adamw_tensor(**t)), count, pd, gd, bits, ctypes.byref(o), None)
    o = api.sr_adamw_opts(1e-3, 0.9, 0.999, 1e-8, 0.01, 1.0, 1, None, None, None)
    assert lib.sr_adamw_step(None, 1, 0, 0, 32, ctypes.byref(o), None) == api.SR_ERR_NULL
    assert lib.sr_adamw_step((api.sr_adamw_tensor * 1)(), 1, 0, 0, 32, None, None) == api.SR_ERR_NULL
    assert lib.sr_adamw_step(None, 0, 0, 0, 32, ctypes.byref(o), None) == api.SR_OK          # nothing to do, nothing launched
    assert call(tensor=dict(n=0, param=None, grad=None, m=None, v=None)) == api.SR_OK
    assert call(count=-1) == api.SR_ERR_SHAPE
    for pd, gd, bits in ((3, 0, 32), (0, 3, 32), (-1, 0, 32), (0, 0, 16), (0, 0, 4)):
        assert call(pd=pd, gd=gd, bits=bits) == api.SR_ERR_UNSUPPORTED
    nan, inf = float("nan"), float("inf")
    for bad in (dict(beta1=1.0), dict(beta2=-0.1), dict(beta1=nan), dict(eps=-1.0), dict(eps=inf), dict(lr=nan), dict(weight_decay=inf),
                dict(grad_scale=nan), dict(step=0)):
        assert call(**bad) == api.SR_ERR_SHAPE, bad
    for name in ("param", "grad", "m", "v"):
        assert call(tensor={name: None}) == api.SR_ERR_NULL and call(tensor={name: FAKE + 2}) == api.SR_ERR_ALIGN, name
    assert call(pd=1, bits=8, tensor=dict(param=FAKE + 1)) == api.SR_ERR_ALIGN and call(gd=2, bits=8, tensor=dict(grad=FAKE + 1)) == api.SR_ERR_ALIGN
    assert call(bits=8, tensor=dict(m_scale=None)) == api.SR_ERR_NULL and call(bits=8, tensor=dict(v_scale=FAKE + 1)) == api.SR_ERR_ALIGN
    assert call(tensor=dict(n=-1)) == api.SR_ERR_SHAPE
    assert call(lr_dev=FAKE + 2) == api.SR_ERR_ALIGN and call(step_dev=FAKE + 4) == api.SR_ERR_ALIGN and call(skip_dev=FAKE + 1) == api.SR_ERR_ALIGN


def test_binding_refuses_cpu_tensors_and_bad_lists():
    z = torch.zeros
    with pytest.raises(TypeError):
        sr.sr_dict_regress_dense_grad(z(1, 3, 4, 4), z(1, 8, 8, 8), z(8, 25), z(1, 3, 8, 8), 2, 5)
    with pytest.raises(TypeError):
        sr.sr_select_balance(z(1, 8, 4, 4), z(1, 2, 4, 4, dtype=torch.uint8))
    with pytest.raises(TypeError):
        sr.sr_select_balance_grad(z(1, 8, 4, 4), z(1, 8))
    with pytest.raises(TypeError):
        sr.sr_adamw_plan([z(4)], [z(4)], [z(4)])
    with pytest.raises(ValueError):
        sr.sr_adamw_plan([z(4)], [], [z(4)])
    with pytest.raises(ValueError):
        sr.sr_adamw_plan([], [], [])
