"""What the operators at the ends of a stage refuse, through the C ABI, before anything is enqueued: none of these calls needs a GPU
(on a machine without one a call that is in order ends with HXT_EHIP)."""
import ctypes as C

import pytest
import torch

from paper_2602_18007_amd import hxt

BF16, F32, E4M3 = torch.bfloat16, torch.float32, torch.float8_e4m3fn
BASE = 1 << 32                      # addresses that are never accessed


def at(i):
    return BASE + i * (1 << 28)


def status(name, block, *more):
    return getattr(hxt.lib(), name)(*more, C.byref(block), None)


def norm_block(**kw):
    b = hxt._Norm(rows=8, cols=64, dtype=hxt.HXT_BF16, eps=1e-5, x=at(0), x_stride=64, h=at(1), h_stride=64, q=at(2), q_stride=64, scale=at(3),
                  weight=at(4))
    for k, v in kw.items():
        setattr(b, k, v)
    return b


@pytest.mark.parametrize("change,want", [
    (dict(rows=-1), hxt.HXT_EINVAL), (dict(cols=0), hxt.HXT_EINVAL), (dict(dtype=hxt.HXT_F16), hxt.HXT_EINVAL), (dict(eps=0.0), hxt.HXT_EINVAL),
    (dict(eps=float("nan")), hxt.HXT_EINVAL), (dict(eps=float("inf")), hxt.HXT_EINVAL), (dict(x=None), hxt.HXT_EINVAL),
    (dict(h=None, q=None), hxt.HXT_EINVAL), (dict(scale=None), hxt.HXT_EINVAL), (dict(cols=32769, x_stride=40000, h_stride=40000, q_stride=40000), hxt.HXT_EUNSUPPORTED),
    (dict(rows=1 << 31), hxt.HXT_EUNSUPPORTED), (dict(x=at(0) + 1), hxt.HXT_EALIGN), (dict(weight=at(4) + 1), hxt.HXT_EALIGN),
    (dict(scale=at(3) + 2), hxt.HXT_EALIGN), (dict(x_stride=-64), hxt.HXT_EINVAL), (dict(h_stride=63), hxt.HXT_EINVAL), (dict(q_stride=63), hxt.HXT_EINVAL),
    (dict(x_stride=1 << 41), hxt.HXT_EUNSUPPORTED),
    (dict(h=at(0) + 2), hxt.HXT_EOVERLAP), (dict(h=at(0), h_stride=65, rows=9), hxt.HXT_EOVERLAP), (dict(q=at(0)), hxt.HXT_EOVERLAP),
    (dict(y=at(0), y_stride=64), hxt.HXT_EOVERLAP), (dict(y=at(1), y_stride=64), hxt.HXT_EOVERLAP), (dict(scale=at(1) + 4), hxt.HXT_EOVERLAP),
    (dict(h=at(4)), hxt.HXT_EOVERLAP), (dict(residual=at(0), residual_stride=0, h=at(0), x=at(5)), hxt.HXT_EOVERLAP),
])
def test_norm_refuses(change, want):
    assert status("hxt_norm", norm_block(**change)) == want


NO_GPU = pytest.mark.skipif(torch.cuda.is_available(), reason="the addresses stand for nothing")


@NO_GPU
@pytest.mark.parametrize("change", [
    {}, dict(rows=1, x_stride=0), dict(x_stride=0), dict(h=at(0)), dict(h=None, y=at(0), y_stride=64),
    dict(x_stride=128, h=at(0) + 128, h_stride=128),                       # columns 64.. of the buffer whose columns 0.. are x
    dict(residual=at(5), residual_stride=64, h=at(5)), dict(weight=None, h=None),
])
def test_norm_takes(change):
    assert status("hxt_norm", norm_block(**change)) == hxt.HXT_EHIP


def test_norm_without_rows_is_nothing():
    assert status("hxt_norm", norm_block(rows=0)) == hxt.HXT_OK
    assert status("hxt_norm", norm_block(rows=0, x=None)) == hxt.HXT_OK


def grad_block(**kw):
    b = hxt._NormGrad(rows=8, cols=64, dtype=hxt.HXT_F32, eps=1e-5, h=at(0), h_stride=64, dy=at(1), dy_stride=64, dx=at(2), dx_stride=64, weight=at(3),
                      dweight=at(4), work=at(5), work_bytes=hxt.hxt_norm_grad_work_bytes(8, 64))
    for k, v in kw.items():
        setattr(b, k, v)
    return b


@pytest.mark.parametrize("change,want", [
    (dict(h=None), hxt.HXT_EINVAL), (dict(dy=None), hxt.HXT_EINVAL), (dict(dx=None), hxt.HXT_EINVAL), (dict(work=None), hxt.HXT_EINVAL),
    (dict(work_bytes=hxt.hxt_norm_grad_work_bytes(8, 64) - 1), hxt.HXT_EINVAL), (dict(work=at(5) + 8), hxt.HXT_EALIGN), (dict(dtype=hxt.HXT_E4M3), hxt.HXT_EINVAL),
    (dict(dh=at(6) + 2, dh_stride=64), hxt.HXT_EALIGN), (dict(dx=at(0) + 4), hxt.HXT_EOVERLAP), (dict(dweight=at(1)), hxt.HXT_EOVERLAP),
    (dict(work=at(0)), hxt.HXT_EOVERLAP), (dict(dweight=at(3)), hxt.HXT_EOVERLAP), (dict(dweight_add=at(4) + 4), hxt.HXT_EOVERLAP), (dict(dx=at(5)), hxt.HXT_EOVERLAP),
])
def test_norm_grad_refuses(change, want):
    assert status("hxt_norm_grad", grad_block(**change)) == want


@NO_GPU
@pytest.mark.parametrize("change", [{}, dict(dx=at(0)), dict(dx=at(1)), dict(dh=at(2), dh_stride=64), dict(dweight_add=at(4)), dict(dweight=None, work=None),
                                    dict(rows=0), dict(dy_stride=0)])
def test_norm_grad_takes(change):
    assert status("hxt_norm_grad", grad_block(**change)) == hxt.HXT_EHIP


def product_block(**kw):
    b = hxt._Product(m=16, n=32, k=64, dtype=hxt.HXT_BF16, out_dtype=hxt.HXT_BF16, act=1, a=at(0), a_stride=64, b=at(1), b_stride=64, bias=at(2),
                     residual=at(3), residual_stride=32, pre=at(4), pre_stride=32, c=at(5), c_stride=32)
    for k, v in kw.items():
        setattr(b, k, v)
    return b


@pytest.mark.parametrize("change,want", [
    (dict(m=-1), hxt.HXT_EINVAL), (dict(dtype=hxt.HXT_F32), hxt.HXT_EINVAL), (dict(out_dtype=hxt.HXT_E4M3), hxt.HXT_EINVAL), (dict(act=4), hxt.HXT_EINVAL),
    (dict(act=-1), hxt.HXT_EINVAL), (dict(a=None), hxt.HXT_EINVAL), (dict(b=None), hxt.HXT_EINVAL), (dict(c=None), hxt.HXT_EINVAL),
    (dict(a_scale=at(6)), hxt.HXT_EINVAL), (dict(dtype=hxt.HXT_E4M3, out_dtype=hxt.HXT_F32), hxt.HXT_EUNSUPPORTED), (dict(k=(1 << 24) + 1, a_stride=1 << 25, b_stride=1 << 25), hxt.HXT_EUNSUPPORTED), (dict(m=1 << 31), hxt.HXT_EUNSUPPORTED),
    (dict(a_stride=(1 << 22) + 1), hxt.HXT_EUNSUPPORTED), (dict(c_stride=31), hxt.HXT_EINVAL), (dict(pre_stride=31), hxt.HXT_EINVAL), (dict(b_stride=-1), hxt.HXT_EINVAL),
    (dict(a=at(0) + 1), hxt.HXT_EALIGN), (dict(bias=at(2) + 1), hxt.HXT_EALIGN), (dict(c=at(5) + 2, out_dtype=hxt.HXT_F32), hxt.HXT_EALIGN),
    (dict(c=at(0)), hxt.HXT_EOVERLAP), (dict(c=at(1) + 64), hxt.HXT_EOVERLAP), (dict(c=at(2)), hxt.HXT_EOVERLAP), (dict(c=at(3) + 2), hxt.HXT_EOVERLAP),
    (dict(c=at(4)), hxt.HXT_EOVERLAP), (dict(pre=at(3)), hxt.HXT_EOVERLAP), (dict(dtype=hxt.HXT_E4M3, a_scale=at(5) + 4), hxt.HXT_EOVERLAP),
])
def test_product_refuses(change, want):
    assert status("hxt_product", product_block(**change)) == want


def test_product_wants_its_workspace():
    m, n, k = 1, 128, 14336
    need = hxt.hxt_product_work_bytes(m, n, k)
    if need:
        kw = dict(m=m, n=n, k=k, a_stride=k, b_stride=k, residual_stride=n, pre_stride=n, c_stride=n)
        assert status("hxt_product", product_block(**kw)) == hxt.HXT_EINVAL
        assert status("hxt_product", product_block(work=at(7), work_bytes=need - 1, **kw)) == hxt.HXT_EINVAL
        assert status("hxt_product", product_block(work=at(7) + 4, work_bytes=need, **kw)) == hxt.HXT_EALIGN
        assert status("hxt_product", product_block(work=at(1), work_bytes=need, **kw)) == hxt.HXT_EOVERLAP
    # more than is needed may be used: none of it may be another argument's
    assert status("hxt_product", product_block(work=at(1) - 4096, work_bytes=8192)) == hxt.HXT_EOVERLAP
    assert status("hxt_product", product_block(work=at(7) + 8, work_bytes=8192)) == hxt.HXT_EALIGN


@NO_GPU
@pytest.mark.parametrize("change", [{}, dict(residual=at(5)), dict(k=0, a=None, b=None), dict(a_stride=0), dict(m=1, a_stride=0),
                                    dict(dtype=hxt.HXT_E4M3, a_scale=at(6), b_scale=at(7), a=at(0) + 1)])
def test_product_takes(change):
    assert status("hxt_product", product_block(**change)) == hxt.HXT_EHIP


def test_product_of_nothing():
    assert status("hxt_product", product_block(m=0)) == hxt.HXT_OK
    assert status("hxt_product", product_block(n=0, bias=None, residual=None, pre=None, c=None)) == hxt.HXT_OK


def product_grad_block(**kw):
    b = hxt._ProductGrad(m=16, n=32, k=64, db_dtype=hxt.HXT_F32, act=2, dc=at(0), dc_stride=32, pre=at(1), pre_stride=32, a=at(2), a_stride=64, b=at(3),
                         b_stride=64, dz=at(4), dz_stride=32, da=at(5), da_stride=64, db=at(6), db_stride=64, dbias=at(7), work=at(8),
                         work_bytes=hxt.hxt_product_grad_work_bytes(16, 32, 64))
    for k, v in kw.items():
        setattr(b, k, v)
    return b


@pytest.mark.parametrize("change,want", [
    (dict(dc=None), hxt.HXT_EINVAL), (dict(pre=None), hxt.HXT_EINVAL), (dict(dz=None), hxt.HXT_EINVAL), (dict(a=None), hxt.HXT_EINVAL), (dict(b=None), hxt.HXT_EINVAL),
    (dict(db_dtype=hxt.HXT_F16), hxt.HXT_EINVAL), (dict(act=9), hxt.HXT_EINVAL), (dict(work=None), hxt.HXT_EINVAL), (dict(work_bytes=0), hxt.HXT_EINVAL),
    (dict(work=at(8) + 4), hxt.HXT_EALIGN), (dict(da_stride=63), hxt.HXT_EINVAL), (dict(db=at(6) + 2), hxt.HXT_EALIGN), (dict(k=1 << 31), hxt.HXT_EUNSUPPORTED),
    (dict(n=(1 << 24) + 1, dc_stride=1 << 22), hxt.HXT_EUNSUPPORTED),
    (dict(da=at(3)), hxt.HXT_EOVERLAP), (dict(da=at(0)), hxt.HXT_EOVERLAP), (dict(dz=at(0) + 2), hxt.HXT_EOVERLAP), (dict(db=at(5)), hxt.HXT_EOVERLAP),
    (dict(db_add=at(6) + 4, db_add_stride=64), hxt.HXT_EOVERLAP), (dict(dbias=at(8)), hxt.HXT_EOVERLAP), (dict(dbias_add=at(7) + 4), hxt.HXT_EOVERLAP),
])
def test_product_grad_refuses(change, want):
    assert status("hxt_product_grad", product_grad_block(**change)) == want


@NO_GPU
@pytest.mark.parametrize("change", [{}, dict(dz=at(0)), dict(dz=at(1)), dict(db_add=at(6), db_add_stride=64), dict(dbias_add=at(7)), dict(act=0, pre=None, dz=None),
                                    dict(da=None, b=None), dict(db=None, a=None)])
def test_product_grad_takes(change):
    assert status("hxt_product_grad", product_grad_block(**change)) == hxt.HXT_EHIP


# ---- the message forms -----------------------------------------------------------------------------

def plan_of(*shapes, dtype=BF16):
    return hxt.hxt_plan_multi([(s, None, dtype) for s in shapes], 2, 256)


def unpack_norm(plan, packed=at(8), sums=None, **kw):
    b = norm_block(**dict(dict(x=None), **kw))
    return hxt.lib().hxt_unpack_norm(plan.handle, packed, C.byref(b), sums, None)


def test_unpack_norm_refuses():
    one, two = plan_of((8, 64)), plan_of((8, 64), (8, 64))
    assert unpack_norm(one, x=at(0)) == hxt.HXT_EINVAL
    assert unpack_norm(two, residual=at(5), residual_stride=64) == hxt.HXT_EINVAL
    assert unpack_norm(plan_of((8, 63))) == hxt.HXT_EUNSUPPORTED
    assert unpack_norm(plan_of((8, 64), (8, 63))) == hxt.HXT_EUNSUPPORTED
    assert unpack_norm(plan_of((8, 64), (8, 64), (8, 64))) == hxt.HXT_EUNSUPPORTED
    assert unpack_norm(plan_of((8, 64), dtype=F32)) == hxt.HXT_EUNSUPPORTED
    strided = hxt.hxt_plan((8, 64), (128, 1), BF16, 2, 256)
    assert unpack_norm(strided) == hxt.HXT_EUNSUPPORTED
    assert unpack_norm(one, packed=None) == hxt.HXT_EINVAL
    assert unpack_norm(one, packed=at(8) + 16) == hxt.HXT_EALIGN
    b = norm_block(x=None)
    assert hxt.lib().hxt_unpack_norm(None, at(8), C.byref(b), None, None) == hxt.HXT_EINVAL
    with pytest.raises(ValueError):
        hxt.hxt_unpack_norm(hxt.hxt_plan((8, 64), None, 2, 2, 256), None, None)


@NO_GPU
def test_message_forms_take_what_is_in_order_and_no_overlap():
    plan = plan_of((8, 64))
    assert unpack_norm(plan) == hxt.HXT_EHIP
    g = grad_block(dx=None, dtype=hxt.HXT_BF16, weight=None, dweight=None)
    assert hxt.lib().hxt_pack_norm_grad(plan.handle, C.byref(g), at(9), None, None) == hxt.HXT_EHIP
    p = product_block(c=None)
    assert hxt.lib().hxt_pack_product(plan_of((16, 32)).handle, C.byref(p), at(9), None, None) == hxt.HXT_EHIP


def test_pack_forms_refuse():
    plan = plan_of((8, 64))
    for change, want in ((dict(), hxt.HXT_EINVAL), (dict(dx=None), hxt.HXT_EUNSUPPORTED), (dict(dx=None, dtype=hxt.HXT_BF16, rows=7), hxt.HXT_EUNSUPPORTED)):
        g = grad_block(**change)
        assert hxt.lib().hxt_pack_norm_grad(plan.handle, C.byref(g), at(9), None, None) == want
    for change, want in ((dict(), hxt.HXT_EINVAL), (dict(c=None, out_dtype=hxt.HXT_F32, residual=None), hxt.HXT_EUNSUPPORTED), (dict(c=None, m=15), hxt.HXT_EUNSUPPORTED)):
        p = product_block(**change)
        assert hxt.lib().hxt_pack_product(plan_of((16, 32)).handle, C.byref(p), at(9), None, None) == want


def test_the_binding_checks_what_pointers_do_not_show():
    x, w = torch.zeros(4, 64, dtype=BF16), torch.zeros(64, dtype=BF16)
    hxt.Norm(w, x=x, h=torch.zeros_like(x))
    hxt.Norm(w, x=torch.zeros(2, 2, 64, dtype=BF16), y=x)                       # [seq, batch, hidden]
    for bad in (dict(x=x, h=x.float()), dict(x=x, h=torch.zeros(4, 63, dtype=BF16)), dict(x=x.t(), h=x.t()), dict(x=x, q=x, scale=w),
                dict(x=x, q=torch.zeros(4, 64, dtype=E4M3), scale=torch.zeros(3)), dict(x=x.half(), h=x.half())):
        with pytest.raises((ValueError, TypeError)):
            hxt.Norm(w if bad["x"].dtype == BF16 else None, **bad)
    with pytest.raises(ValueError):
        hxt.Product(x, torch.zeros(8, 63, dtype=BF16), c=torch.zeros(4, 8, dtype=BF16))
    with pytest.raises(ValueError):
        hxt.Product(x, torch.zeros(8, 64, dtype=BF16), act="tanh", c=torch.zeros(4, 8, dtype=BF16))
    with pytest.raises(ValueError):
        hxt.ProductGrad(torch.zeros(4, 8, dtype=F32), a=x)
