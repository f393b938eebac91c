"""What hag_rms_norm, hag_rms_norm_fp8, hag_rms_norm_grad, hag_fp8_product and hag_adamw refuse, by the status they return before anything is launched (no GPU)."""
import ctypes
import math

import pytest

from paper_1906_03707_amd import binding as B

P = 1 << 20                                                # an address that nothing reads
BIG = 1 << 31


def refused(rc):
    assert rc == B.HAG_EINVAL and B.lib().hag_last_error()


@pytest.mark.parametrize("n,d,dtype,param,x_stride,r_stride,eps", [(-1, 4, 0, 0, 4, 4, 1e-5), (BIG, 4, 0, 0, 4, 4, 1e-5), (2, 0, 0, 0, 4, 4, 1e-5), (2, (1 << 20) + 1, 0, 0, 4, 4, 1e-5),
                                                                   (2, 4, 1, 0, 4, 4, 1e-5), (2, 4, 2, 3, 4, 4, 1e-5), (2, 4, 0, 2, 4, 4, 1e-5), (2, 4, 0, 0, -4, 4, 1e-5), (2, 4, 0, 0, 4, -4, 1e-5),
                                                                   (2, 4, 0, 0, 4, 4, -1e-5), (2, 4, 0, 0, 4, 4, math.nan), (2, 4, 0, 0, 4, 4, math.inf)])
def test_rms_norm_refusals(n, d, dtype, param, x_stride, r_stride, eps):
    L = B.lib()
    refused(L.hag_rms_norm(n, d, dtype, P, x_stride, P, r_stride, param, P, eps, P, P, P, None))
    refused(L.hag_rms_norm_fp8(n, d, dtype, P, x_stride, P, r_stride, param, P, eps, P, P, 1 << 21, P, 1 << 20, None))
    if eps == 1e-5:
        refused(L.hag_rms_norm_grad(n, d, dtype, P, x_stride, P, r_stride, P, 4, param, P, P, P, P, P, None))
        refused(L.hag_rms_norm_grad(n, d, dtype, P, 4, P, r_stride, P, x_stride, param, P, P, P, P, P, None))


def test_rms_norm_refuses_null_pointers():
    L = B.lib()
    refused(L.hag_rms_norm(2, 4, 0, None, 4, None, 0, 0, P, 1e-5, None, P, P, None))
    refused(L.hag_rms_norm(2, 4, 0, P, 4, P, 4, 0, P, 1e-5, None, P, P, None))                          # a residual and nowhere to put the sum
    refused(L.hag_rms_norm(2, 4, 0, P, 4, None, 0, 0, P, 1e-5, None, None, P, None))
    refused(L.hag_rms_norm_fp8(2, 4, 0, P, 4, None, 0, 0, P, 1e-5, None, None, 4, P, 1, None))
    refused(L.hag_rms_norm_fp8(2, 4, 0, P, 4, None, 0, 0, P, 1e-5, None, P, 4, None, 1, None))
    refused(L.hag_rms_norm_fp8(2, 40, 0, P, 40, None, 0, 0, P, 1e-5, None, P, 39, P, 2, None))          # rows that overlap
    refused(L.hag_rms_norm_fp8(2, 40, 0, P, 40, None, 0, 0, P, 1e-5, None, P, 40, P, 1, None))
    for gy, h, rstd, gx, ws in ((None, P, P, P, P), (P, None, P, P, P), (P, P, None, P, P), (P, P, P, None, P), (P, P, P, P, None), (P, P, P, P, P + 4)):
        refused(L.hag_rms_norm_grad(2, 4, 0, gy, 4, None, 0, h, 4, 0, P, rstd, gx, P, ws, None))
    assert L.hag_rms_norm(0, 4, 0, None, 4, None, 0, 0, None, 1e-5, None, None, None, None) == B.HAG_OK
    assert L.hag_rms_norm_fp8(0, 4, 0, None, 4, None, 0, 0, None, 1e-5, None, None, 4, None, 1, None) == B.HAG_OK
    assert L.hag_rms_norm_grad(0, 4, 0, None, 4, None, 0, None, 4, 0, None, None, None, None, None, None) == B.HAG_OK
    assert L.hag_rms_norm_grad_workspace_bytes(5, 0) == 0 and L.hag_rms_norm_grad_workspace_bytes(5, 7) > 0


def test_product_refusals():
    L = B.lib()

    def call(n=2, d=40, k=3, x=P, xs=40, sx=P, ssx=2, w=P, ws=40, sw=P, ssw=2, dtype=0, y=P):
        return L.hag_fp8_product(n, d, k, x, xs, sx, ssx, w, ws, sw, ssw, dtype, y, None)

    for bad in (dict(n=-1), dict(n=BIG), dict(k=-1), dict(k=(1 << 20) + 1), dict(d=0), dict(d=(1 << 20) + 1), dict(xs=-40), dict(ssx=-1), dict(ws=-1), dict(ssw=-2), dict(dtype=1), dict(dtype=4),
                dict(x=None), dict(sx=None), dict(w=None), dict(sw=None), dict(y=None)):
        refused(call(**bad))
    assert call(n=0, x=None, sx=None, y=None) == B.HAG_OK and call(k=0, w=None, sw=None, y=None) == B.HAG_OK


def test_adamw_refusals():
    L = B.lib()

    def entry(param=P, grad=P, m=P, v=P, copy=0, m_scales=P, v_scales=P, count=5, types=0, copy_type=0):
        return (ctypes.c_int64 * 10)(param, grad, m, v, copy, m_scales, v_scales, count, types, copy_type)

    def options(**how):
        o = B.hag_adamw_options_t(1e-3, 0.9, 0.999, 1e-8, 0.01, 1.0, 1, None, None, None, 0, 32)
        for k, v in how.items():
            setattr(o, k, v)
        return ctypes.byref(o)

    good = entry()
    for how in (dict(bits=16), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0), dict(beta2=math.nan), dict(eps=0.0), dict(eps=-1.0), dict(eps=math.inf), dict(lr=math.nan), dict(lr=math.inf),
                dict(weight_decay=math.nan), dict(step=0), dict(norm=P, max_norm=0.0), dict(norm=P, max_norm=math.nan)):
        refused(L.hag_adamw(1, good, options(**how), None))
    refused(L.hag_adamw(-1, good, options(), None))
    refused(L.hag_adamw((1 << 24) + 1, good, options(), None))
    refused(L.hag_adamw(1, None, options(), None))
    refused(L.hag_adamw(1, good, None, None))
    f32, bf16, f16 = B.HAG_F32, B.HAG_BF16, B.HAG_F16
    for how in (dict(param=0), dict(grad=0), dict(m=0), dict(v=0), dict(count=-1), dict(count=1 << 50), dict(types=1), dict(types=f32 | B.HAG_I64 << 32), dict(types=bf16 | f32 << 32), dict(types=f16 | bf16 << 32),
                dict(copy=P, copy_type=1)):
        refused(L.hag_adamw(1, entry(**how), options(), None))
    for how in (dict(m_scales=0), dict(v_scales=0)):
        refused(L.hag_adamw(1, entry(**how), options(bits=8), None))
    assert L.hag_adamw(0, None, options(), None) == B.HAG_OK
    assert L.hag_adamw(1, entry(param=0, grad=0, m=0, v=0, count=0), options(), None) == B.HAG_OK


def test_structures_are_those_of_the_header():
    assert ctypes.sizeof(B.hag_adamw_options_t) == 88
    assert B.hag_adamw_options_t.step.offset == 48 and B.hag_adamw_options_t.seed.offset == 80
