"""hxt_norm, hxt_unpack_norm, hxt_norm_grad and hxt_pack_norm_grad against their formulas in 64 bits.

Bounds: a result that is one expression of its inputs is rounded once (half a step, HALF) from a binary32 value whose relative
error is EPS32 = 2^-17 at most: a row's sum of squares adds at most 64 squares a thread and 10 levels of partial sums (74 roundings
of 2^-24, all terms positive), the root halves that, and scaling adds a few roundings more."""
import pytest
import torch

from paper_2602_18007_amd import hxt
from tests.operator_cases import BF16, DEV, E4M3, F32, HALF, Guarded, f64, generator, norm_exact, norm_grad_exact, normal, within

pytestmark = pytest.mark.gpu
EPS, EPS32 = 1e-5, 2.0 ** -17
SMALLEST = {BF16: 2.0 ** -134, F32: 2.0 ** -150}         # half of the smallest number


def check_norm(h, y, q, scale, want, dtype):
    H, Y, S = want
    if h is not None:
        within(h, H, H.abs() * (HALF[dtype] + 2.0 ** -24) + SMALLEST[dtype], "h")
    if y is not None:
        within(y, Y, Y.abs() * (HALF[dtype] + EPS32) + SMALLEST[dtype], "y")
    if q is not None:
        within(scale, S, S * EPS32, "scale")
        # e4m3 below 2^-6 has steps of 2^-9; q * scale stands for y
        within(f64(q) * f64(scale)[:, None], Y, Y.abs() * (HALF[E4M3] + 2 * EPS32) + (S * 2.0 ** -10)[:, None], "q")
        assert not bool((f64(q).abs() > 448).any())


SHAPES = [(1, 1), (3, 5), (1, 64), (7, 65), (5, 511), (4, 512), (6, 520), (3, 1003), (2, 2048), (3, 2056), (1, 4096), (37, 4096), (2, 4104), (3, 8191),
          (2, 8192), (2, 8200), (2, 16384), (1, 16391), (2, 32768)]


MANY_ROWS = [(1030, 600), (1025, 1500), (1027, 4000), (1024, 4096), (1025, 6001), (1026, 12000), (1024, 20008)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,cols", SHAPES + MANY_ROWS)
def test_norm_of_tensors(rows, cols, dtype):
    print("norm", rows, cols, dtype, flush=True)
    g = generator(rows * 70001 + cols)
    for pad, offset, residual, weight in ((0, 0, True, True), (3, 1, True, True), (8, 0, False, True), (0, 0, False, False)):
        x = Guarded(rows, cols, dtype, pad, offset).set(normal((rows, cols), g, 2.0))
        r = Guarded(rows, cols, dtype, pad + 2, offset).set(normal((rows, cols), g, 3.0)) if residual else None
        w = (1 + 0.2 * normal((cols,), g)).to(dtype) if weight else None
        h, y = Guarded(rows, cols, dtype, pad, offset), Guarded(rows, cols, dtype, pad + 1, offset)
        q = Guarded(rows, cols, E4M3, pad, offset)
        scale = torch.full((rows,), -1.0, device=DEV)
        hxt.hxt_norm(hxt.Norm(w, EPS, x=x.m, residual=r.m if r else None, h=h.m, y=y.m, q=q.m, scale=scale))
        check_norm(h.m, y.m, q.m, scale, norm_exact(x.m, r.m if r else None, w, EPS), dtype)
        assert h.untouched() and y.untouched() and q.untouched()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_norm_outputs_alone_in_place_and_broadcast(dtype):
    g = generator(3)
    rows, cols = 9, 1000
    x, r, w = normal((rows, cols), g, 1.0, dtype), normal((rows, cols), g, 1.0, dtype), (1 + 0.2 * normal((cols,), g)).to(dtype)
    want = norm_exact(x, r, w, EPS)
    y = torch.empty_like(x)
    hxt.hxt_norm(hxt.Norm(w, EPS, x=x, residual=r, y=y))
    check_norm(None, y, None, None, want, dtype)
    q, scale = torch.empty(rows, cols, dtype=E4M3, device=DEV), torch.empty(rows, device=DEV)
    hxt.hxt_norm(hxt.Norm(w, EPS, x=x, residual=r, q=q, scale=scale))
    check_norm(None, None, q, scale, want, dtype)
    for into in ("x", "r"):                              # the sum goes where an input was
        x2, r2 = x.clone(), r.clone()
        t = x2 if into == "x" else r2
        hxt.hxt_norm(hxt.Norm(w, EPS, x=x2, residual=r2, h=t, y=y))
        check_norm(t, y, None, None, want, dtype)
    x2 = x.clone()
    hxt.hxt_norm(hxt.Norm(w, EPS, x=x2, residual=r, y=x2))
    check_norm(None, x2, None, None, want, dtype)
    one = r[:1].expand(rows, cols)                       # one row for all
    hxt.hxt_norm(hxt.Norm(w, EPS, x=x, residual=one, y=y))
    check_norm(None, y, None, None, norm_exact(x, one, w, EPS), dtype)
    both = torch.full((rows, 2 * cols), 7.0, dtype=dtype, device=DEV)          # input and output side by side in one buffer
    both[:, :cols] = x
    hxt.hxt_norm(hxt.Norm(w, EPS, x=both[:, :cols], residual=r, y=both[:, cols:]))
    check_norm(None, both[:, cols:], None, None, want, dtype)
    assert torch.equal(both[:, :cols], x)


@pytest.mark.parametrize("rows,cols", [(9, 64), (9, 1000), (9, 4096), (1031, 520), (1025, 1100), (1027, 3000), (1025, 5000)])
def test_norm_of_rows_with_unusual_values(rows, cols):
    """Rows of zeros, of the type's largest and smallest values, with NaN and with infinities; each row apart from the others."""
    for dtype in (BF16, F32):
        big, tiny = torch.finfo(dtype).max, torch.finfo(dtype).tiny
        x = normal((rows, cols), generator(5), 1.0, dtype)
        x[0] = 0
        x[1] = big / 4
        x[2] = tiny
        x[3, 1] = float("nan")
        x[4, cols - 1] = float("inf")
        x[5, 0] = -float("inf")
        x[6] *= 1e25
        x[7, : cols // 2] = 0
        y, h = torch.empty_like(x), torch.empty_like(x)
        q, scale = torch.empty(rows, cols, dtype=E4M3, device=DEV), torch.empty(rows, device=DEV)
        hxt.hxt_norm(hxt.Norm(None, EPS, x=x, h=h, y=y, q=q, scale=scale))
        H, Y, S = norm_exact(x, None, None, EPS)
        S = torch.where(torch.isnan(Y).any(1), torch.full_like(S, float("nan")), S)
        check_norm(h, y, None, None, (H, Y, S), dtype)
        within(scale, S, torch.nan_to_num(S) * EPS32, "scale")
        good = torch.isfinite(S)
        check_norm(None, None, q[good], scale[good], (H[good], Y[good], S[good]), dtype)
        assert bool((f64(q[0]) == 0).all()) and scale[0].item() == 2.0 ** -126
        assert bool(torch.isnan(f64(q[3])).all())


def packed_of(plan, tensors):
    packed = torch.full((plan.packed_bytes,), 0xA5, dtype=torch.uint8, device=DEV)
    hxt.hxt_pack(plan, tensors, packed)
    return packed


MESSAGES = [(1, 4096, 2, 16384), (37, 512, 3, 4096), (64, 1000, 4, 65536), (33, 1001, 2, 768), (5, 4096, 2, 256), (129, 4096, 4, 1 << 20), (4, 8, 2, 256),
            (19, 3584, 8, 32768), (3, 16384, 2, 1 << 16),
            (1030, 3584, 4, 1 << 18), (1025, 2048, 2, 4096), (1027, 264, 3, 768), (1026, 5000, 2, 1 << 20)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("residual", ["message", "local", "none"])
@pytest.mark.parametrize("rows,cols,lanes,chunk", MESSAGES)
def test_norm_of_a_message(rows, cols, lanes, chunk, residual, dtype):
    """Rows across chunks of any size, checksums as hxt_unpack's, twice in a row (the accumulators are clean again)."""
    print("unpack norm", rows, cols, lanes, chunk, residual, dtype, flush=True)
    g = generator(rows + cols)
    x, r = normal((rows, cols), g, 1.0, dtype), normal((rows, cols), g, 2.0, dtype)
    w = (1 + 0.2 * normal((cols,), g)).to(dtype)
    tensors = [x, r] if residual == "message" else [x]
    plan = hxt.hxt_plan_multi([((rows, 1, cols), None, dtype)] * len(tensors), lanes, chunk)
    packed = packed_of(plan, tensors)
    before = packed.clone()
    want_sums = torch.empty(plan.num_chunks, dtype=torch.int64, device=DEV)
    hxt.hxt_checksum(plan, packed, want_sums)
    want = norm_exact(x, None if residual == "none" else r, w, EPS)
    for sums in (torch.full_like(want_sums, -1), None, torch.full_like(want_sums, -2)):
        h, y, q = Guarded(rows, cols, dtype, 3), Guarded(rows, cols, dtype), Guarded(rows, cols, E4M3, 1)
        scale = torch.full((rows,), -1.0, device=DEV)
        a = hxt.Norm(w, EPS, residual=r if residual == "local" else None, h=h.m, y=y.m, q=q.m, scale=scale)
        hxt.hxt_unpack_norm(plan, packed, a, sums)
        check_norm(h.m, y.m, q.m, scale, want, dtype)
        assert h.untouched() and y.untouched() and q.untouched()
        assert sums is None or torch.equal(sums, want_sums)
    assert torch.equal(packed, before)


def test_norm_of_a_message_shares_its_sums_with_unpack():
    """The accumulators are hxt_unpack's: calls of both, on two streams, with a damaged byte in between."""
    rows, cols = 300, 2048
    x = normal((rows, cols), generator(1), 1.0, BF16)
    plan = hxt.hxt_plan(x.shape, None, BF16, 4, 1 << 16)
    packed = packed_of(plan, [x])
    y, dst, want = torch.empty_like(x), torch.empty_like(x), torch.empty(plan.num_chunks, dtype=torch.int64, device=DEV)
    hxt.hxt_checksum(plan, packed, want)
    a = hxt.Norm(None, EPS, y=y)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    sums = [torch.empty_like(want) for _ in range(6)]
    for i, s in enumerate(sums):
        st = streams[i % 2]
        if i % 3 == 1:
            hxt.hxt_unpack(plan, packed, [dst], s, st)
        else:
            hxt.hxt_unpack_norm(plan, packed, a, s, st)
    torch.cuda.synchronize()
    assert all(torch.equal(s, want) for s in sums)
    packed[70000] += 1
    hxt.hxt_unpack_norm(plan, packed, a, sums[0])
    assert int((sums[0] != want).sum()) == 1


def check_grad(dx, dweight, h, dy, dh, w, dtype, add=None):
    DX, size, DW, dw_size = norm_grad_exact(h, dy, dh, w, EPS)
    within(dx, DX, DX.abs() * (HALF[dtype] + 2.0 ** -24) + size * 4 * EPS32 + SMALLEST[dtype], "dx")
    if dweight is not None:
        # rows are added one after another by at most a few hundred threads, then 16 slices of those, then the slices: for
        # these sizes fewer than 200 roundings, and the terms' own (2 EPS32)
        DW = DW if add is None else DW + f64(add)
        within(dweight, DW, dw_size * (200 * 2.0 ** -24 + 2 * EPS32) + DW.abs() * 2.0 ** -23, "dweight")


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,cols", SHAPES + [(1537, 512), (2000, 64), (1600, 1000)])
def test_norm_grad_of_tensors(rows, cols, dtype):
    print("norm grad", rows, cols, dtype, flush=True)
    g = generator(rows * 3 + cols)
    for pad, offset, with_dh, with_w in ((0, 0, True, True), (5, 1, False, True), (0, 0, False, False)):
        h = Guarded(rows, cols, dtype, pad, offset).set(normal((rows, cols), g, 2.0))
        dy = Guarded(rows, cols, dtype, pad + 1, offset).set(normal((rows, cols), g, 0.1))
        dh = Guarded(rows, cols, dtype, pad, offset).set(normal((rows, cols), g, 0.1)) if with_dh else None
        w = (1 + 0.2 * normal((cols,), g)).to(dtype) if with_w else None
        dx = Guarded(rows, cols, dtype, pad, offset)
        dweight, add = Guarded(1, cols, F32), normal((cols,), g)
        need = hxt.hxt_norm_grad_work_bytes(rows, cols)
        work = Guarded(1, need, torch.uint8)
        hxt.hxt_norm_grad(hxt.NormGrad(w, EPS, h=h.m, dy=dy.m, dh=dh.m if dh else None, dx=dx.m, dweight=dweight.m.view(-1),
                                       dweight_add=add if with_dh else None, work=work.m.view(-1)))
        check_grad(dx.m, dweight.m.view(-1), h.m, dy.m, dh.m if dh else None, w, dtype, add if with_dh else None)
        assert dx.untouched() and dweight.untouched() and work.untouched()


def test_norm_grad_alone_in_place_and_with_unusual_rows():
    g = generator(8)
    rows, cols = 11, 776
    for dtype in (BF16, F32):
        h, dy, dh = (normal((rows, cols), g, s, dtype) for s in (1.0, 0.1, 0.1))
        h[0] = 0
        h[1] *= 1e25
        w = (1 + 0.2 * normal((cols,), g)).to(dtype)
        for into in range(3):
            ts = [h.clone(), dy.clone(), dh.clone()]
            hxt.hxt_norm_grad(hxt.NormGrad(w, EPS, h=ts[0], dy=ts[1], dh=ts[2], dx=ts[into]))
            check_grad(ts[into], None, h, dy, dh, w, dtype)
        bad = h.clone()
        bad[4, 3] = float("nan")
        dx = torch.empty_like(h)
        hxt.hxt_norm_grad(hxt.NormGrad(w, EPS, h=bad, dy=dy, dh=dh, dx=dx))
        assert bool(torch.isnan(dx[4]).all())
        keep = [i for i in range(rows) if i != 4]
        check_grad(dx[keep], None, h[keep], dy[keep], dh[keep], w, dtype)
        one = dy[:1].expand(rows, cols)                  # one gradient row for all
        hxt.hxt_norm_grad(hxt.NormGrad(w, EPS, h=h, dy=one, dx=dx))
        check_grad(dx, None, h, one, None, w, dtype)


def test_norm_grad_of_no_rows_gives_what_was_added():
    add = normal((64,), generator(2))
    dweight = torch.full((64,), 9.0, device=DEV)
    e = torch.empty(0, 64, device=DEV)
    hxt.hxt_norm_grad(hxt.NormGrad(None, EPS, h=e, dy=e, dx=e, dweight=dweight, dweight_add=add))
    assert torch.equal(dweight, add)
    hxt.hxt_norm_grad(hxt.NormGrad(None, EPS, h=e, dy=e, dx=e, dweight=dweight))
    assert bool((dweight == 0).all())


def test_norm_grad_against_differences():
    """Central differences of the 64-bit norm: the step's own error is below 1e-7 of the gradient's size here."""
    g = generator(4)
    rows, cols = 3, 24
    x, w, c = normal((rows, cols), g), 1 + 0.2 * normal((cols,), g), normal((rows, cols), g)
    dx, dweight = torch.empty_like(x), torch.empty(cols, device=DEV)
    work = torch.empty(hxt.hxt_norm_grad_work_bytes(rows, cols), dtype=torch.uint8, device=DEV)
    hxt.hxt_norm_grad(hxt.NormGrad(w, EPS, h=x, dy=c, dx=dx, dweight=dweight, work=work))
    loss = lambda x_, w_: (norm_exact(x_, None, w_, EPS)[1] * f64(c)).sum()              # noqa: E731
    x64, w64, step = f64(x), f64(w), 1e-5
    for t, got in ((x64, dx), (w64, dweight)):
        flat = t.view(-1)
        for i in range(0, flat.numel(), 7):
            keep = flat[i].item()
            flat[i] = keep + step
            up = loss(x64, w64).item()
            flat[i] = keep - step
            down = loss(x64, w64).item()
            flat[i] = keep
            assert abs((up - down) / (2 * step) - got.view(-1)[i].item()) < 1e-4
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,cols,lanes,chunk", MESSAGES)
def test_norm_grad_into_a_message(rows, cols, lanes, chunk, dtype):
    print("pack norm grad", rows, cols, lanes, chunk, dtype, flush=True)
    g = generator(rows + cols)
    h, dy, dh = (normal((rows, cols), g, s, dtype) for s in (1.0, 0.1, 0.1))
    w = (1 + 0.2 * normal((cols,), g)).to(dtype)
    plan = hxt.hxt_plan((rows, cols), None, dtype, lanes, chunk)
    dweight = torch.empty(cols, device=DEV)
    work = torch.empty(hxt.hxt_norm_grad_work_bytes(rows, cols), dtype=torch.uint8, device=DEV)
    a = hxt.NormGrad(w, EPS, h=h, dy=dy, dh=dh, dweight=dweight, work=work)
    for sums in (None, torch.empty(plan.num_chunks, dtype=torch.int64, device=DEV)):
        packed = torch.full((plan.packed_bytes,), 0xA5, dtype=torch.uint8, device=DEV)
        hxt.hxt_pack_norm_grad(plan, a, packed, sums)
        dx, got = torch.empty_like(h), torch.empty(plan.num_chunks, dtype=torch.int64, device=DEV)
        hxt.hxt_unpack(plan, packed, [dx], got)
        check_grad(dx, dweight, h, dy, dh, w, dtype)
        again = torch.full_like(packed, 0xA5)            # pads are zero, bytes outside the chunks as they were
        hxt.hxt_pack(plan, [dx], again)
        assert torch.equal(packed, again)
        assert sums is None or torch.equal(sums, got)


def test_norm_calls_captured_and_replayed():
    """Forward and backward in one graph, on inputs that change between the replays, with eager work on the same plan beside them."""
    rows, cols = 257, 4096
    g = generator(11)
    x, r, dy = (normal((rows, cols), g, 1.0, BF16) for _ in range(3))
    w = (1 + 0.2 * normal((cols,), g)).to(BF16)
    plan, back = hxt.hxt_plan_multi([((rows, cols), None, BF16)] * 2, 4, 1 << 17), hxt.hxt_plan((rows, cols), None, BF16, 4, 1 << 17)
    packed, sent = packed_of(plan, [x, r]), torch.empty(back.packed_bytes, dtype=torch.uint8, device=DEV)
    h, q, scale = torch.empty_like(x), torch.empty(rows, cols, dtype=E4M3, device=DEV), torch.empty(rows, device=DEV)
    sums, sent_sums = torch.empty(plan.num_chunks, dtype=torch.int64, device=DEV), torch.empty(back.num_chunks, dtype=torch.int64, device=DEV)
    dweight, work = torch.empty(cols, device=DEV), torch.empty(hxt.hxt_norm_grad_work_bytes(rows, cols), dtype=torch.uint8, device=DEV)
    fwd, bwd = hxt.Norm(w, EPS, h=h, q=q, scale=scale), hxt.NormGrad(w, EPS, h=h, dy=dy, dweight=dweight, work=work)
    side = torch.cuda.Stream()

    def both(st):
        hxt.hxt_unpack_norm(plan, packed, fwd, sums, st)
        hxt.hxt_pack_norm_grad(back, bwd, sent, sent_sums, st)

    side.wait_stream(torch.cuda.current_stream())
    both(side)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        both(side)
    for i in range(3):
        x, r = normal((rows, cols), g, 1.0, BF16), normal((rows, cols), g, 1.0, BF16)
        hxt.hxt_pack(plan, [x, r], packed)
        dy.copy_(normal((rows, cols), g, 1.0, BF16))
        for t in (h, q, scale, dweight, sent, sums, sent_sums):
            t.view(torch.uint8).fill_(0x77)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        check_norm(h, None, q, scale, norm_exact(x, r, w, EPS), BF16)
        dx, got, want = torch.empty_like(x), torch.empty_like(sent_sums), torch.empty_like(sums)
        hxt.hxt_unpack(back, sent, [dx], got)
        hxt.hxt_checksum(plan, packed, want)
        check_grad(dx, dweight, h, dy, None, w, BF16)
        assert torch.equal(got, sent_sums) and torch.equal(want, sums)


def test_norm_repeats_bit_for_bit():
    rows, cols = 1500, 2048
    g = generator(12)
    h, dy = normal((rows, cols), g, 1.0, BF16), normal((rows, cols), g, 1.0, BF16)
    work = torch.empty(hxt.hxt_norm_grad_work_bytes(rows, cols), dtype=torch.uint8, device=DEV)
    got = []
    for _ in range(3):
        dx, dweight = torch.empty_like(h), torch.empty(cols, device=DEV)
        hxt.hxt_norm_grad(hxt.NormGrad(None, EPS, h=h, dy=dy, dx=dx, dweight=dweight, work=work))
        got.append((dx, dweight))
    assert all(torch.equal(a, got[0][0]) and torch.equal(b, got[0][1]) for a, b in got)


def test_rows_past_four_gigabytes():
    """Offsets beyond 32 bits, of tensors and in a message: the rows repeat every 1000, so that all of them are known."""
    rows, cols, every = 140000, 16384, 1000
    g = generator(13)
    base, w = normal((every, cols), g, 1.0, BF16), (1 + 0.2 * normal((cols,), g)).to(BF16)
    x = base.repeat(rows // every, 1)
    y = torch.empty_like(x)
    want = norm_exact(base, None, w, EPS)
    hxt.hxt_norm(hxt.Norm(w, EPS, x=x, y=y))
    check_norm(None, y[:every], None, None, want, BF16)
    assert bool((y.view(-1, every, cols) == y[:every]).all())
    plan = hxt.hxt_plan((rows, cols), None, BF16, 8, 25 << 20)
    packed = torch.empty(plan.packed_bytes, dtype=torch.uint8, device=DEV)
    hxt.hxt_pack(plan, [x], packed)
    first = y[:every].clone()
    y.zero_()
    got, sums = torch.empty(plan.num_chunks, dtype=torch.int64, device=DEV), torch.empty(plan.num_chunks, dtype=torch.int64, device=DEV)
    hxt.hxt_checksum(plan, packed, got)
    hxt.hxt_unpack_norm(plan, packed, hxt.Norm(w, EPS, y=y), sums)
    within(y[:every], want[1], want[1].abs() * (HALF[BF16] + EPS32) + SMALLEST[BF16], "y")
    assert bool((y.view(-1, every, cols) == y[:every]).all()) and torch.equal(sums, got)
    del packed, first
    dx, dweight = torch.empty_like(x), torch.empty(cols, device=DEV)
    work = torch.empty(hxt.hxt_norm_grad_work_bytes(rows, cols), dtype=torch.uint8, device=DEV)
    hxt.hxt_norm_grad(hxt.NormGrad(w, EPS, h=x, dy=x, dx=dx, dweight=dweight, work=work))
    check_grad(dx[:every], None, base, base, None, w, BF16)
    assert bool((dx.view(-1, every, cols) == dx[:every]).all())
    _, _, DW, size = norm_grad_exact(base, base, None, w, EPS)
    # 140000 rows over 512 workgroups: 274 additions each, then 64 and 8
    within(dweight, DW * (rows // every), size * (rows // every) * (400 * 2.0 ** -24 + 2 * EPS32), "dweight")


def test_the_binding_refuses_tensors_of_the_host():
    x = torch.zeros(4, 64)
    with pytest.raises(ValueError):
        hxt.hxt_norm(hxt.Norm(x=x, y=torch.empty_like(x)))
    with pytest.raises(ValueError):
        hxt.Norm(x=x, y=torch.empty(4, 64, device=DEV))
