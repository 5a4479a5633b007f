"""Which kernel serves a product, by the launch code's own rule, on the CPU: the sizes of the GPU tests go where those mean them to, and what
is chosen fits the workspace that is asked for."""
import ctypes as C
import os
import random
import subprocess

import pytest

from paper_2602_18007_amd import hxt
from tests.product_tiles import E4M3, LARGE, SMALLER
from tests.test_gpu_product import GRADS, SIZES

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("rules") / "libproduct_rules.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-Wall", "-Wextra", "-Werror", "-fsanitize=undefined", "-fno-sanitize-recover=all",
                    "-I", os.path.join(ROOT, "paper_2602_18007_amd", "csrc"), "-o", out, os.path.join(ROOT, "tests", "host", "product_rules.cpp")], check=True)
    lib = C.CDLL(out)
    lib.product_work.restype = C.c_uint64
    return lib


class Way:
    def __init__(self, lib, m, n, k, es, across=(False, False), direct=(True, True), work=1 << 60):
        out = (C.c_uint64 * 8)()
        lib.product_way(*map(C.c_int64, (m, n, k, es)), *map(int, across + direct), C.c_uint64(work), out)
        self.tile, self.parts, self.steps, self.half, self.direct, self.copy_p, self.copy_q, self.used = out


ACROSS = {"forward": (False, False), "da": (False, True), "db": (True, True)}


@pytest.mark.parametrize("kind,dtype,m,n,k,tile,half", LARGE + SMALLER)
def test_sizes_go_to_the_tiles_they_are_meant_for(rules, kind, dtype, m, n, k, tile, half):
    es = 1 if dtype == E4M3 else 2
    w = Way(rules, m, n, k, es, ACROSS[kind])
    assert (w.tile, w.half, w.direct) == (tile, half, 1)
    whole = k // (128 // es)
    if tile == 256:
        assert w.parts == 1 and whole >= 9 and whole // 8 > 0
    else:
        assert min(w.steps, whole) >= 5


def test_the_remainder_and_both_ways_of_a_workspace_are_among_them(rules):
    assert {(kind, dtype) for kind, dtype, *_, half in LARGE if half} == {(kind, dtype) for kind, dtype, *_ in LARGE}
    parts = {(kind, dtype, Way(rules, m, n, k, 1 if dtype == E4M3 else 2, ACROSS[kind]).parts > 1) for kind, dtype, m, n, k, *_ in SMALLER}
    assert parts >= {("forward", hxt_dtype, False) for hxt_dtype in {d for k, d, *_ in SMALLER if k == "forward"}}
    assert {kind for kind, _, several in parts if several} == {"forward", "da", "db"}


@pytest.mark.parametrize("m,n", [(1, 1), (4, 9000), (20, 30), (64, 14336), (3000, 3001), (4096, 4096), (1024, 14336), (40000, 40000)])
@pytest.mark.parametrize("across", list(ACROSS.values()))
def test_of_an_empty_contraction_nothing_is_copied(rules, m, n, across):
    for direct in ((True, True), (False, False), (True, False)):
        w = Way(rules, m, n, 0, 2, across, direct)
        assert w.direct and not w.copy_p and not w.copy_q and w.used == 0 and w.parts == 1


def test_what_is_chosen_fits_the_workspace(rules):
    """Any sizes, operands in whole vectors by their length or by neither length nor base: with the workspace that the query gives, all that
    the chosen way keeps there fits."""
    rng = random.Random(5)
    sizes = [(m, n, k) for m, n, k in SIZES + GRADS] + [tuple(int(2 ** rng.uniform(0, 14)) for _ in range(3)) for _ in range(600)]
    for m, n, k in sizes:
        for kind, across in ACROSS.items():
            for es in (2, 1) if kind == "forward" else (2,):
                need = rules.product_work(*map(C.c_int64, (m, n, k, es)), *map(int, across))
                if kind == "forward":
                    assert need == hxt.lib().hxt_product_work_bytes(m, n, k, hxt.HXT_E4M3 if es == 1 else hxt.HXT_BF16)
                whole = tuple((outer if a else k) * es % 16 == 0 for a, outer in zip(across, (m, n)))
                for direct in {whole, (False, whole[1]), (whole[0], False), (False, False)}:
                    w = Way(rules, m, n, k, es, across, direct, need)
                    assert w.used <= need, (m, n, k, kind, es, direct)
                    assert w.direct or w.tile in (16, 128)
                    if across != (False, False):
                        assert w.tile in (128, 256)
