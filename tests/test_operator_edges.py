"""What the operators at the ends of a stage take and refuse at an edge, through the C ABI and the binding, on the CPU."""
import ctypes as C
import os
import re

import pytest
import torch

from paper_2602_18007_amd import hxt
from tests.test_operator_refusals import BF16, E4M3, F32, NO_GPU, at, product_block, status


@pytest.mark.parametrize("m,n,k,dtype", [(40, 1000, 4160, hxt.HXT_BF16), (60, 2000, 4224, hxt.HXT_E4M3), (130, 520, 8201, hxt.HXT_BF16)])
def test_product_refuses_a_workspace_that_is_missing_small_or_misplaced(m, n, k, dtype):
    need = hxt.lib().hxt_product_work_bytes(m, n, k, dtype)
    assert need > 4096
    kw = dict(m=m, n=n, k=k, dtype=dtype, a_stride=k, b_stride=k, residual_stride=n, pre_stride=n, c_stride=n)
    assert status("hxt_product", product_block(**kw)) == hxt.HXT_EINVAL
    assert status("hxt_product", product_block(work=at(7), work_bytes=need - 1, **kw)) == hxt.HXT_EINVAL
    assert status("hxt_product", product_block(work=None, work_bytes=need, **kw)) == hxt.HXT_EINVAL
    assert status("hxt_product", product_block(work=at(7) + 4, work_bytes=need, **kw)) == hxt.HXT_EALIGN
    for other in (0, 1, 2, 3, 4, 5):                     # a, b, bias, residual, pre, c
        assert status("hxt_product", product_block(work=at(other), work_bytes=need, **kw)) == hxt.HXT_EOVERLAP
    plan = hxt.hxt_plan((m, n), None, BF16, 2, 4096)
    kw.pop("c_stride")
    for work, size in ((None, 0), (at(7), need - 1)):
        block = product_block(c=None, work=work, work_bytes=size, **kw)
        assert hxt.lib().hxt_pack_product(plan.handle, C.byref(block), at(9), None, None) == hxt.HXT_EINVAL


def test_norms_of_no_rows_through_the_binding():
    """A tensor without elements has no address: that its rows are none is no missing output."""
    dev = "cuda:0" if torch.cuda.is_available() else "cpu"
    for dt in (BF16, F32):
        e, q, s = torch.empty(0, 64, dtype=dt, device=dev), torch.empty(0, 64, dtype=E4M3, device=dev), torch.empty(0, device=dev)
        w = torch.ones(64, dtype=dt, device=dev)
        hxt.hxt_norm(hxt.Norm(w, x=e, y=e))
        hxt.hxt_norm(hxt.Norm(w, x=e, residual=e, h=e, y=e, q=q, scale=s))
        hxt.hxt_norm(hxt.Norm(w, x=e, q=q, scale=s))
    b = hxt._Norm(rows=0, cols=64, dtype=hxt.HXT_BF16, eps=1e-5)
    assert status("hxt_norm", b) == hxt.HXT_OK
    b.rows, b.x, b.x_stride = 1, at(0), 64
    assert status("hxt_norm", b) == hxt.HXT_EINVAL       # (with rows an output is needed)


def test_message_norm_of_no_rows():
    plan = hxt.hxt_plan((0, 64), None, BF16, 2, 256)
    assert plan.num_chunks == 0
    b = hxt._Norm(rows=0, cols=64, dtype=hxt.HXT_BF16, eps=1e-5)
    assert hxt.lib().hxt_unpack_norm(plan.handle, None, C.byref(b), None, None) == hxt.HXT_OK


@NO_GPU
@pytest.mark.parametrize("change", [
    dict(m=1, n=(1 << 22) + 8, k=64, a_stride=64, b_stride=64, residual_stride=(1 << 22) + 8, pre_stride=(1 << 22) + 8, c_stride=(1 << 22) + 8, bias=None),
    dict(m=1, a_stride=1 << 40, residual_stride=1 << 62, pre_stride=0, c_stride=1 << 40),
    dict(n=1, k=64, b_stride=1 << 40, residual_stride=1, pre_stride=1, c_stride=1),
    dict(m=1, n=1, k=(1 << 22) + 64, a=at(0), a_stride=(1 << 22) + 64, b_stride=(1 << 22) + 64, work=at(7), work_bytes=1 << 20),
])
def test_one_row_has_no_stride_to_speak_of(change):
    """A [1, n] tensor's row stride is n or anything else: it is no distance between rows.  (Addresses here are 2^28 apart.)"""
    assert status("hxt_product", product_block(**change)) == hxt.HXT_EHIP


@NO_GPU
def test_one_row_of_a_gradient_has_no_stride_to_speak_of():
    n = (1 << 22) + 8
    b = hxt._ProductGrad(m=1, n=n, k=8, db_dtype=hxt.HXT_BF16, act=2, dc=at(0), dc_stride=n, pre=at(1), pre_stride=1 << 50, a=at(2), a_stride=1 << 41, b=at(3),
                         b_stride=8, dz=at(4), dz_stride=n, da=at(5), da_stride=1 << 60, db=at(6), db_stride=8, work=at(8), work_bytes=1 << 27)
    assert status("hxt_product_grad", b) == hxt.HXT_EHIP
    b.m = 2
    assert status("hxt_product_grad", b) == hxt.HXT_EUNSUPPORTED
    b.m, b.dc_stride = 1, -1
    assert status("hxt_product_grad", b) == hxt.HXT_EINVAL


def test_the_binding_takes_rows_of_no_elements():
    """An empty contraction of [batch, seq, 0] factors, and no rows of [0, seq, n]."""
    a, b = torch.empty(2, 3, 0, dtype=BF16), torch.empty(5, 0, dtype=BF16)
    p = hxt.Product(a, b, c=torch.empty(2, 3, 5, dtype=BF16))
    assert (p.c.m, p.c.n, p.c.k) == (6, 5, 0)
    p = hxt.Product(torch.empty(0, 3, 8, dtype=BF16), torch.empty(5, 8, dtype=BF16), c=torch.empty(0, 3, 5, dtype=BF16))
    assert (p.c.m, p.c.n, p.c.k) == (0, 5, 8)
    g = hxt.ProductGrad(torch.empty(2, 3, 0, dtype=BF16), b=torch.empty(0, 8, dtype=BF16), da=torch.empty(2, 3, 8, dtype=BF16))
    assert (g.c.m, g.c.n, g.c.k) == (6, 0, 8)
    with pytest.raises(ValueError):
        hxt.Product(a, b, c=torch.empty(5, 5, dtype=BF16))


def test_assembly_says_that_it_writes_m0():
    """The compiler may set m0 for itself and rely on it later: a statement that writes it names it among what it changes."""
    csrc = os.path.join(os.path.dirname(hxt.LIB_PATH), "csrc")
    writes = 0
    for name in sorted(os.listdir(csrc)):
        text = open(os.path.join(csrc, name)).read()
        for statement in re.findall(r"asm volatile\((.*?)\);", text, flags=re.S):
            if re.search(r"s_mov_b32 m0\b", statement):
                writes += 1
                assert re.search(r':[^:]*"m0"', statement), "%s: %s" % (name, statement)
    assert writes > 0
