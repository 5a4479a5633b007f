"""hxt_norm, hxt_unpack_norm and hxt_norm_grad at an edge: more rows than one launch has threads for, values half way between two steps
of 8 bits, scales of infinity, sums of products that leave binary32."""
import pytest
import torch

from paper_2602_18007_amd import hxt
from tests.operator_cases import BF16, DEV, E4M3, F32, HALF, f64, generator, norm_grad_exact, normal, within

pytestmark = pytest.mark.gpu
EPS, EPS32 = 1e-5, 2.0 ** -17                            # the latter: relative error of a binary32 value before its rounding
SMALLEST = {BF16: 2.0 ** -134, F32: 2.0 ** -150}         # half of the smallest number


def test_more_rows_than_a_launch_has_threads_for():
    """Norms of short rows have 64 threads a row: 2^26 rows are 2^32 threads."""
    rows = (1 << 26) + 5
    g = generator(1)
    x = normal((rows, 1), g, 2.0, BF16)
    y, scale = torch.empty_like(x), torch.full((rows,), -1.0, device=DEV)
    q = torch.empty(rows, 1, dtype=E4M3, device=DEV)
    hxt.hxt_norm(hxt.Norm(None, EPS, x=x, y=y, q=q, scale=scale))
    for part in range(0, rows, 1 << 24):
        at = slice(part, part + (1 << 24))
        X = f64(x[at])
        Y = X / torch.sqrt(X * X + EPS)
        within(y[at], Y, Y.abs() * (HALF[BF16] + EPS32) + SMALLEST[BF16], "y")
        S = (Y.abs().view(-1) / 448).clamp_min(2.0 ** -126)
        within(scale[at], S, S * EPS32, "scale")
        # one value a row: 448, or 0 where the value is 0
        assert bool((q[at].float() == torch.where(X == 0, X, 448 * X.sign()).float()).all())


def test_more_rows_of_a_message_than_a_launch_has_threads_for():
    rows, cols = (1 << 26) + 5, 8
    x = normal((rows, cols), generator(2), 2.0, BF16)
    plan = hxt.hxt_plan((rows, cols), None, BF16, 4, 1 << 20)
    packed = torch.empty(plan.packed_bytes, dtype=torch.uint8, device=DEV)
    sums, want_sums = (torch.empty(plan.num_chunks, dtype=torch.int64, device=DEV) for _ in range(2))
    hxt.hxt_pack(plan, [x], packed, want_sums)
    y = torch.empty_like(x)
    hxt.hxt_unpack_norm(plan, packed, hxt.Norm(None, EPS, y=y), sums)
    assert torch.equal(sums, want_sums)
    for part in range(0, rows, 1 << 24):
        at = slice(part, part + (1 << 24))
        X = f64(x[at])
        Y = X / torch.sqrt((X * X).mean(1, keepdim=True) + EPS)
        within(y[at], Y, Y.abs() * (HALF[BF16] + EPS32) + SMALLEST[BF16], "y")
