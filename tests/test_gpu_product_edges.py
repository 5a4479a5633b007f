"""hxt_product, hxt_pack_product and hxt_product_grad where sizes and values are at an edge: infinities in front of an activation, empty
contractions of large results, more columns than one launch has threads for, scales whose product leaves binary32."""
import pytest
import torch

from paper_2602_18007_amd import hxt
from tests.operator_cases import BF16, DEV, E4M3, F32, HALF, f64, generator, normal, within

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")

# few rows, tens of rows, tens of rows in parts, tiles in parts, tiles; whole rows of 8 results and odd ones
WAYS = [(3, 40, 72), (3, 33, 72), (40, 264, 520), (40, 1000, 4160), (130, 267, 2056), (300, 520, 64), (257, 261, 72)]


def whole(shape, g, most=4):
    return torch.randint(-most, most + 1, shape, generator=g, device=DEV).to(F32)


def workspace(m, n, k, dtype=BF16):
    return torch.empty(hxt.hxt_product_work_bytes(m, n, k, dtype), dtype=torch.uint8, device=DEV)


@pytest.mark.parametrize("m,n,k", WAYS)
def test_relu_of_infinities(m, n, k):
    """0 for whatever is not above 0, minus infinity among it (a bias that masks a column), without a sign; NaN stays NaN."""
    g = generator(m + n + k)
    a, b = whole((m, k), g).to(BF16), whole((n, k), g).to(BF16)
    a[1, 2] = -INF                                       # a row of infinities of either sign, and of NaN where b has 0
    bias = whole((n,), g).to(BF16)
    bias[0], bias[n // 2], bias[n - 1], bias[n - 2] = -INF, -INF, INF, NAN
    z = (a.float().cpu().double() @ b.float().cpu().double().t().contiguous() + bias.float().cpu().double()).to(DEV)
    want = torch.where(torch.isnan(z), z, torch.where(z > 0, z, torch.zeros_like(z)))
    for out in (BF16, F32):
        c = torch.empty(m, n, dtype=out, device=DEV)
        hxt.hxt_product(hxt.Product(a, b, bias=bias, act="relu", c=c, out_dtype=out, work=workspace(m, n, k)))
        within(c, want, torch.nan_to_num(want, 0.0, 0.0, 0.0).abs() * HALF[out], "c")
        assert not bool((torch.signbit(c) & (c == 0)).any())
    assert bool((c[0, [0, n // 2]] == 0).all()) and c[0, n - 1].item() == INF and bool(torch.isnan(c[:, n - 2]).all())


def test_relu_gradient_at_infinities():
    m, n = 70, 90
    g = generator(4)
    dc, pre = whole((m, n), g).to(BF16), whole((m, n), g).to(BF16)
    pre[:, 3], pre[5] = -INF, INF
    dz = torch.empty_like(dc)
    hxt.hxt_product_grad(hxt.ProductGrad(dc, pre=pre, act="relu", dz=dz, work=torch.empty(hxt.hxt_product_grad_work_bytes(m, n, 0), dtype=torch.uint8, device=DEV)))
    assert torch.equal(dz.float(), torch.where(pre > 0, dc.float(), torch.zeros(m, n, device=DEV)))
