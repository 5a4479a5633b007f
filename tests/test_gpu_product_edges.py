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


@pytest.mark.parametrize("m,n", [(4096, 4096), (3000, 3001), (1024, 14336), (4, 9000), (9, 20000), (64, 14336), (20, 30)])
@pytest.mark.parametrize("dtype", [BF16, E4M3])
def test_empty_sums_of_any_size(m, n, dtype):
    """Rows of no elements have a stride of 1 in a tensor and count neither as whole vectors nor as anything to copy."""
    g = generator(m + n)
    a, b = torch.empty(m, 0, dtype=dtype, device=DEV), torch.empty(n, 0, dtype=dtype, device=DEV)
    bias, r = whole((n,), g).to(BF16), whole((m, n), g).to(BF16)
    want = bias.float() + r.float()
    assert hxt.hxt_product_work_bytes(m, n, 0, dtype) == 0
    for work in (None, torch.empty(1 << 20, dtype=torch.uint8, device=DEV)):
        c = torch.full((m, n), 7.0, dtype=BF16, device=DEV)
        hxt.hxt_product(hxt.Product(a, b, bias=bias, residual=r, c=c, work=work))
        assert torch.equal(c.float(), want)
        plan = hxt.hxt_plan((m, n), None, BF16, 4, 1 << 16)
        packed, again = (torch.full((plan.packed_bytes,), 0xA5, dtype=torch.uint8, device=DEV) for _ in range(2))
        sums, want_sums = (torch.empty(plan.num_chunks, dtype=torch.int64, device=DEV) for _ in range(2))
        hxt.hxt_pack_product(plan, hxt.Product(a, b, bias=bias, residual=r, work=work), packed, sums)
        hxt.hxt_pack(plan, [c], again, want_sums)
        assert torch.equal(packed, again) and torch.equal(sums, want_sums)


@pytest.mark.parametrize("out", [BF16, F32])
@pytest.mark.parametrize("n,k", [(4097, 4097), (4096, 4100), (3001, 3000), (4096, 4096), (14336, 1024)])
def test_gradients_of_an_empty_micro_batch(n, k, out):
    """m = 0: the gradients are what was added, of any size."""
    g = generator(n + k)
    add, badd = whole((n, k), g).to(out), whole((n,), g)
    db, dbias = torch.full((n, k), 7.0, dtype=out, device=DEV), torch.full((n,), 7.0, device=DEV)
    hxt.hxt_product_grad(hxt.ProductGrad(torch.empty(0, n, dtype=BF16, device=DEV), torch.empty(0, k, dtype=BF16, device=DEV), db=db, db_add=add,
                                         dbias=dbias, dbias_add=badd))
    assert torch.equal(db, add) and torch.equal(dbias, badd)
    hxt.hxt_product_grad(hxt.ProductGrad(torch.empty(0, n, dtype=BF16, device=DEV), torch.empty(0, k, dtype=BF16, device=DEV), db=db, dbias=dbias))
    assert bool((db == 0).all()) and bool((dbias == 0).all())


@pytest.mark.parametrize("m,k", [(4097, 4097), (4099, 4104), (4096, 4096), (3, 14336)])
def test_gradient_through_no_columns(m, k):
    """n = 0: da is 0, of any size."""
    da = torch.full((m, k), 7.0, dtype=BF16, device=DEV)
    hxt.hxt_product_grad(hxt.ProductGrad(torch.empty(m, 0, dtype=BF16, device=DEV), b=torch.empty(0, k, dtype=BF16, device=DEV), da=da))
    assert bool((da == 0).all())


@pytest.mark.parametrize("m", [1, 3])
def test_more_columns_than_a_launch_has_threads_for(m):
    """The kernel for few rows has 32 threads a column: of 2^27 columns and more one launch cannot hold them."""
    n, k = (1 << 27) + 24, 8
    g = generator(m)
    a, b = whole((m, k), g).to(BF16), whole((n, k), g).to(BF16)
    plan = hxt.hxt_plan((m * n,), None, BF16, 4, 64 << 20)
    packed = torch.full((plan.packed_bytes,), 0xA5, dtype=torch.uint8, device=DEV)
    sums, got_sums = (torch.empty(plan.num_chunks, dtype=torch.int64, device=DEV) for _ in range(2))
    hxt.hxt_pack_product(plan, hxt.Product(a, b, work=workspace(m, n, k)), packed, sums)
    got = torch.empty(m, n, dtype=BF16, device=DEV)
    hxt.hxt_unpack(plan, packed, [got], got_sums)
    assert torch.equal(sums, got_sums)
    for i in range(m):
        assert torch.equal(got[i], (b.float() * a[i].float()).sum(1).to(BF16))


def test_more_copied_vectors_than_a_launch_has_threads_for():
    """Rows at an odd address are copied to whole vectors first, 16 bytes a thread; here one row stands for 2^23 of 513 vectors."""
    m, n, k = 1 << 23, 1024, 4104
    g = generator(9)
    one, b = whole((k + 1,), g, 1).to(BF16)[1:], whole((n, k), g, 1).to(BF16)
    room = m * k * 2 + n * k * 2 + (1 << 20)
    c, work = torch.empty(m, n, dtype=BF16, device=DEV), torch.empty(room, dtype=torch.uint8, device=DEV)
    hxt.hxt_product(hxt.Product(one.expand(m, k), b, c=c, work=work))
    want = (b.float() * one.float()).sum(1).to(BF16)
    for part in c.view(64, -1, n):
        assert bool((part == want).all())


@pytest.mark.parametrize("m,n,k", WAYS)
def test_scales_whose_product_leaves_binary32(m, n, k):
    """A row's scale may be 2^-126 (hxt_norm's least): times a column's 2^-19 it would be subnormal, with a few bits left, though sums are
    2^22 and more here; two large ones would be infinite, and a sum of 0 NaN.  Every step in front of the rounding to bf16 is off by
    2^-24 of its value at most, the results by 2^-8 and 3 of those."""
    g = generator(m * n + k)
    a, b = ((torch.randint(8, 15, (r, k), generator=g, device=DEV) * 32).float().to(E4M3) for r in (m, n))      # 256 .. 448
    a.view(torch.uint8)[2], b.view(torch.uint8)[1] = 0, 0
    sa = (torch.rand(m, generator=g, device=DEV) + 1) * 2.0 ** -126
    sb = (torch.rand(n, generator=g, device=DEV) + 1) * 2.0 ** -19
    sa[1], sa[2], sb[1] = 2.0 ** 100, 2.0 ** 100, 2.0 ** 40
    c = torch.empty(m, n, dtype=BF16, device=DEV)
    hxt.hxt_product(hxt.Product(a, b, a_scale=sa, b_scale=sb, c=c, work=workspace(m, n, k, E4M3)))
    sums = f64(a) @ f64(b).t().contiguous()
    want = sums * f64(sa)[:, None] * f64(sb)
    # the matrix instruction for 8 bits adds 128 products with 20 bits below the largest; results below 2^-126 have steps of 2^-133
    within(c, want, want.abs() * (HALF[BF16] + 2.0 ** -13 + (k + 4) * 2.0 ** -24 + 3 * 2.0 ** -24) + 2.0 ** -134, "c")
    assert bool((c[2] == 0).all()) and bool((c[:, 1] == 0).all())


def test_long_single_rows():
    """One row of a result, of a gradient or of a factor may be longer than the distance that rows may have."""
    n, k = (1 << 22) + 24, 40
    g = generator(11)
    a, b, bias = whole((1, k), g).to(BF16), whole((n, k), g).to(BF16), whole((n,), g).to(BF16)
    pre, c, r = torch.empty(1, n, dtype=BF16, device=DEV), torch.empty(1, n, dtype=BF16, device=DEV), whole((1, n), g).to(BF16)
    hxt.hxt_product(hxt.Product(a, b, bias=bias, act="relu", pre=pre, residual=r, c=c, work=workspace(1, n, k)))
    z = (b.float() * a.float()).sum(1) + bias.float()
    assert torch.equal(pre[0], z.to(BF16)) and torch.equal(c[0], (torch.relu(z) + r[0].float()).to(BF16))
    dc = whole((1, n), g).to(BF16)
    dz, da, db, dbias = torch.empty_like(dc), torch.empty_like(a), torch.empty_like(b), torch.empty(n, device=DEV)
    work = torch.empty(hxt.hxt_product_grad_work_bytes(1, n, k), dtype=torch.uint8, device=DEV)
    hxt.hxt_product_grad(hxt.ProductGrad(dc, a, b, pre=pre, act="relu", dz=dz, da=da, db=db, dbias=dbias, work=work))
    d = torch.where(pre > 0, dc.float(), torch.zeros_like(dc, dtype=F32))
    assert torch.equal(dz.float(), d) and torch.equal(dbias, d[0]) and torch.equal(db, (d[0][:, None] * a.float()).to(BF16))
    assert torch.equal(da[0], (f64(d[0])[:, None] * f64(b)).sum(0).to(F32).to(BF16))
    long = (1 << 22) + 72
    x, y = whole((1, long), g, 1).to(BF16), whole((1, long), g, 1).to(BF16)
    one = torch.empty(1, 1, device=DEV)
    hxt.hxt_product(hxt.Product(x, y, c=one, out_dtype=F32, work=workspace(1, 1, long)))
    assert one.item() == (f64(x) * f64(y)).sum().item()
    spread = torch.zeros(1, 3, (1 << 23) + 8, dtype=BF16, device=DEV)[:, 1:2, :k]      # (a stride of 2^23 + 8)
    spread.copy_(a)
    out = torch.empty(1, 1, n, dtype=BF16, device=DEV)
    hxt.hxt_product(hxt.Product(spread, b, bias=bias, c=out, work=workspace(1, n, k)))
    assert torch.equal(out.view(-1), z.to(BF16))
