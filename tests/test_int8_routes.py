"""Which kernels the sizes of the GPU tests reach, asked of the library's own rules (host code, compiled here)."""

import ctypes
import os
import subprocess

import pytest

from paper_2608_10010_amd import build as B
from tests import test_gpu_int8_kernels as K
from tests.test_gpu_int8_moe_range import SIZES

KERNELS = ["DOT", "FEW4", "FEW8", "FEW32", "T64", "T64_128", "T128", "T256_128", "T256"]
STAGES = {"T64": 4, "T64_128": 3, "T128": 3, "T256_128": 3, "T256": 2}
SOURCE = """
#include "int8_routes.hpp"
using namespace cfint8;
extern "C" int product(int64_t M, int64_t N, int64_t K, int trans) {
    const bool t = trans && turned(M, N, K);
    return (t ? 100 : 0) + route_direct(M, N, K, trans && !t).kernel;
}
extern "C" int slots(int digits, int64_t T, int64_t E, int64_t k, int64_t H, int64_t I) {
    return digits == 3 ? by_slots<3>(T, E, k, H, I) : by_slots<4>(T, E, k, H, I);
}
static_assert(T256 == 8 && DOT == 0, "the order of names in the test");
"""


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    d = tmp_path_factory.mktemp("routes")
    src, lib = os.path.join(d, "routes.cpp"), os.path.join(d, "routes.so")
    with open(src, "w") as f:
        f.write(SOURCE)
    subprocess.run([B.cxx(), "-O1", "-std=c++17", "-Wall", "-shared", "-fPIC", f"-I{B.CSRC}", src, "-o", lib], check=True)
    L = ctypes.CDLL(lib)
    i64 = ctypes.c_int64
    L.product.argtypes, L.slots.argtypes = [i64, i64, i64, ctypes.c_int], [ctypes.c_int, i64, i64, i64, i64, i64]
    return L


def kernel(rules, M, N, k, trans):
    v = rules.product(M, N, k, trans)
    return ("turned " if v >= 100 else "") + KERNELS[v % 100]


def test_products_reach_their_kernels(rules):
    for name, M, N, k, trans in K.PRODUCT_CASES:
        assert kernel(rules, M, N, k, trans) == name, (M, N, k, trans)
    for name, M, N, trans in K.LONG:
        assert kernel(rules, M, N, 131056, trans) == name, (M, N, trans)


def test_products_cover_every_kernel_and_stage():
    seen = {}
    for name, _, _, k, trans in K.PRODUCT_CASES:
        seen.setdefault((name, trans), set()).add(-(-k // 128) % STAGES.get(name, 1))
    for name, n in STAGES.items():
        for trans in (0, 1):
            assert seen[name, trans] == set(range(n)), (name, trans)
    assert {n for n, _ in seen} >= set(KERNELS)


@pytest.mark.parametrize("digits", [3, 4])
def test_layers_go_their_way(rules, digits):
    for T, E, topk, H, I, way in K.LAYERS:
        assert bool(rules.slots(digits, T, E, topk, H, I)) == (way == "slots"), (T, E, topk, H, I)
    ways = [bool(rules.slots(digits, *s)) for s in SIZES]
    assert ways == [True, True, False, False]
