"""hxt_norm, hxt_unpack_norm and hxt_norm_grad at an edge: more rows than one launch has threads for, values half way between two steps
of 8 bits, scales of infinity, sums of products that leave binary32."""
import pytest
import torch

from paper_2602_18007_amd import hxt
from tests.operator_cases import BF16, DEV, E4M3, F32, HALF, f64, generator, norm_grad_exact, normal, within

pytestmark = pytest.mark.gpu
EPS, EPS32 = 1e-5, 2.0 ** -17                            # the latter: relative error of a binary32 value before its rounding
SMALLEST = {BF16: 2.0 ** -134, F32: 2.0 ** -150}         # half of the smallest number
