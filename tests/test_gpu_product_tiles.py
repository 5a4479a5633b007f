"""Products in large tiles: whole numbers, whose sums are exact in binary32 in whatever order, against 64 bits, to the last bit.  The sizes are
those that the launch code's rule sends to each kind of tile (tests/product_tiles.py)."""
import pytest
import torch

from paper_2602_18007_amd import hxt
from tests.operator_cases import BF16, DEV, E4M3, F32, Guarded, f64, generator
from tests.product_tiles import LARGE, SMALLER, pad_to_vectors

pytestmark = pytest.mark.gpu


def whole(shape, g, most=3):
    return torch.randint(-most, most + 1, shape, generator=g, device=DEV).to(F32)


def factor(rows, cols, dtype, g):
    """Rows of whole vectors at 16-byte multiples, whatever their length."""
    return Guarded(rows, cols, dtype, pad_to_vectors(cols, dtype)).set(whole((rows, cols), g)).m


def same(got, want, what):
    differ = int((got != want).sum())
    assert differ == 0, "%s: %d of %d differ" % (what, differ, want.numel())


FORWARD = [c for c in LARGE + SMALLER if c[0] == "forward"]


@pytest.mark.parametrize("kind,dtype,m,n,k,tile,half", FORWARD)
def test_products(kind, dtype, m, n, k, tile, half):
    print("product", m, n, k, dtype, tile, half, flush=True)
    g = generator(m + n + k)
    a, b = factor(m, k, dtype, g), factor(n, k, dtype, g)
    z = f64(a) @ f64(b).t().contiguous()
    work = torch.empty(hxt.hxt_product_work_bytes(m, n, k, dtype), dtype=torch.uint8, device=DEV)
    for out, pad in ((BF16, 0), (BF16, 5), (F32, 3)) if dtype == BF16 else ((BF16, 0), (BF16, 5)):
        c = Guarded(m, n, out, pad)
        hxt.hxt_product(hxt.Product(a, b, c=c.m, out_dtype=out, work=work))
        same(c.m, z.to(F32).to(out), "c")
        assert c.untouched()
    # the whole epilogue: scales that are powers of two, bias, pre, an activation that whole numbers stay whole in, residual
    sa, sb = ((2.0 ** torch.randint(-3, 4, (r,), generator=g, device=DEV).float() for r in (m, n)) if dtype == E4M3 else (None, None))
    bias, r = whole((n,), g).to(BF16), Guarded(m, n, BF16, 1).set(whole((m, n), g))
    pre, c = Guarded(m, n, BF16, 2), Guarded(m, n, BF16, 7)
    hxt.hxt_product(hxt.Product(a, b, a_scale=sa, b_scale=sb, bias=bias, act="relu", residual=r.m, pre=pre.m, c=c.m, work=work))
    if sa is not None:
        z = z * f64(sa)[:, None] * f64(sb)
    z = z + f64(bias)
    same(pre.m, z.to(F32).to(BF16), "pre")
    same(c.m, (z.clamp_min(0) + f64(r.m)).to(F32).to(BF16), "c of the epilogue")
    assert pre.untouched() and c.untouched()


@pytest.mark.parametrize("lanes,chunk", [(3, 8192), (2, 768), (4, 1 << 20)])
@pytest.mark.parametrize("kind,dtype,m,n,k,tile,half", [c for c in FORWARD if c[2] > 4000 and c[3] % 2 or c[6] == 2])
def test_products_into_messages(kind, dtype, m, n, k, tile, half, lanes, chunk):
    """Chunk borders in every row, so in the columns of the half tiles too; gaps and padding are zeros, bytes outside stay."""
    print("pack product", m, n, k, dtype, tile, half, lanes, chunk, flush=True)
    g = generator(m + n + k)
    a, b = factor(m, k, dtype, g), factor(n, k, dtype, g)
    z = f64(a) @ f64(b).t().contiguous()
    work = torch.empty(hxt.hxt_product_work_bytes(m, n, k, dtype), dtype=torch.uint8, device=DEV)
    for out in (BF16, F32) if dtype == BF16 else (BF16,):
        plan = hxt.hxt_plan((m, n), None, out, lanes, chunk)
        packed, want = (torch.full((plan.packed_bytes,), 0xA5, dtype=torch.uint8, device=DEV) for _ in range(2))
        sums, want_sums = (torch.empty(plan.num_chunks, dtype=torch.int64, device=DEV) for _ in range(2))
        hxt.hxt_pack(plan, [z.to(F32).to(out)], want, want_sums)
        hxt.hxt_pack_product(plan, hxt.Product(a, b, out_dtype=out, work=work), packed, sums)
        same(packed, want, "message")
        assert torch.equal(sums, want_sums)


@pytest.mark.parametrize("kind,dtype,m,n,k,tile,half", [c for c in LARGE + SMALLER if c[0] != "forward"])
def test_gradients(kind, dtype, m, n, k, tile, half):
    """da [m, n] contracts the k columns of dc and rows of b; db [m, n] the k rows of dc and of a."""
    print(kind, m, n, k, tile, half, flush=True)
    g = generator(m + n + k)
    if kind == "da":
        dc, b = factor(m, k, BF16, g), factor(k, n, BF16, g)
        work = torch.empty(hxt.hxt_product_grad_work_bytes(m, k, n), dtype=torch.uint8, device=DEV)
        da = Guarded(m, n, BF16, 3)
        hxt.hxt_product_grad(hxt.ProductGrad(dc, b=b, da=da.m, work=work))
        same(da.m, (f64(dc) @ f64(b)).to(F32).to(BF16), "da")
        assert da.untouched()
        return
    dc, a = factor(k, m, BF16, g), factor(k, n, BF16, g)
    work = torch.empty(hxt.hxt_product_grad_work_bytes(k, m, n), dtype=torch.uint8, device=DEV)
    want = f64(dc).t().contiguous() @ f64(a)
    for out in (F32, BF16):
        db, add = Guarded(m, n, out, 3), whole((m, n), g).to(out)
        hxt.hxt_product_grad(hxt.ProductGrad(dc, a, db=db.m, work=work))
        same(db.m, want.to(F32).to(out), "db")
        hxt.hxt_product_grad(hxt.ProductGrad(dc, a, db=db.m, db_add=add, work=work))
        same(db.m, (want + f64(add)).to(F32).to(out), "db added")
        assert db.untouched()
