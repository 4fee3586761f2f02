"""Every kernel of the 8-bit product and both ways through the mixture-of-experts layer, at sizes chosen by the kernel
that they reach (tests/test_int8_routes.py asks the library's own rules whether they do): each stage that a tile
kernel can start on, tiles, blocks and pieces that end inside, the longest K, rings that go round several times."""

import numpy as np
import pytest
import torch

from paper_2608_10010_amd import cfint8 as i8
from tests import int8_ref as R
from tests.gpu_util import say
from tests.test_gpu_int8_moe import dev, make, reference

pytestmark = pytest.mark.gpu

# kernel, M, N, K's, second operands ([N][K]: 0, [K][N]: 1).  K in blocks of 128: a tile kernel of S stages starts on
# another one for each remainder by S (T64: 4, T64_128, T128 and T256_128: 3, T256: 2)
PRODUCTS = [
    ("DOT", 1, 9001, (1100, 2049), (0,)), ("DOT", 2, 16400, (333, 4113), (0,)), ("FEW4", 16, 4090, (1000, 130), (0,)),
    ("FEW8", 9, 4000, (2049, 2300), (0,)), ("FEW32", 20, 9001, (257, 1000), (0,)), ("FEW32", 333, 700, (641, 1027), (0,)),
    ("T64", 250, 4090, (100, 515, 641, 805, 1001), (0, 1)), ("T64_128", 700, 1500, (515, 641, 805), (0, 1)),
    ("T128", 1000, 4090, (100, 515, 641, 805), (0, 1)), ("T128", 500, 4100, (515, 641, 1003), (0, 1)),
    ("T256_128", 2040, 4090, (100, 515, 641, 805, 1037), (0, 1)), ("T256", 4090, 4093, (100, 300, 900, 1037), (0, 1)),
    ("turned FEW8", 16, 1030, (4100,), (1,)), ("turned FEW32", 20, 1030, (9000,), (1,)),
]
PRODUCT_CASES = [(k, M, N, K, t) for k, M, N, Ks, ts in PRODUCTS for K in Ks for t in ts]
LONG = [("T64", 1000, 1000, 0), ("turned T64", 1000, 1000, 1)] + [
    (k, M, N, t) for k, M, N in (("T64_128", 500, 3500), ("T128", 500, 4100), ("T256_128", 2040, 4090), ("T256", 4090, 4093))
    for t in (0, 1)]


@pytest.mark.parametrize("kernel,M,N,K,trans", PRODUCT_CASES)
def test_product(kernel, M, N, K, trans):
    say(f"[int8 kernels] {kernel} {M} {N} {K} trans={trans}")
    rng = np.random.default_rng(M + 3 * N + 7 * K)
    a, b = R.random_codes(rng, M, K), R.random_codes(rng, N, K)
    bias = (rng.standard_normal(N) * 1e3).astype(np.float32)
    ta = R.codes_tensor(a, fill=101, ld=R.ceil16(K) + 16)
    tb = R.codes_tensor(b.T if trans else b, fill=-93, ld=R.ceil16(N if trans else K) + 48)
    up = lambda v: torch.from_numpy(v).to(R.DEV)  # noqa: E731
    for dtype, spread in ((torch.float32, 1.0), (torch.bfloat16, 30.0)):      # scales that are moderate, and not
        sa, sb = (np.exp(rng.standard_normal(n) * spread).astype(np.float32) for n in (M, N))
        wide = torch.full((M + 1, N + 3), -3.0, dtype=dtype, device=R.DEV)
        i8.cfint8_gemm(ta, up(sa), tb, up(sb), M, N, K, trans_b=trans, bias=up(bias), c=wide[:M, :N])
        torch.cuda.synchronize()
        R.same_bits(wide[:M, :N], R.gemm(a, b, sa, sb, bias, dtype), f"{kernel} {dtype}")
        assert bool((wide[:M, N:] == -3).all()) and bool((wide[M] == -3).all()), "written outside C"


@pytest.mark.parametrize("kernel,M,N,trans", LONG)
def test_longest_sums(kernel, M, N, trans):
    """K = 131056 with codes at their ends, where sums come within 2^18 of 2^31, and with random ones."""
    K = 131056
    say(f"[int8 kernels] longest K, {kernel} {M} {N} trans={trans}")
    rng = np.random.default_rng(M)
    for p, q in ((np.full(K, -128), np.full(K, -128)), (rng.integers(-127, 128, K), rng.integers(-127, 128, K))):
        signs = [rng.choice([-1, 1], n) if p[0] != -128 else np.ones(n, np.int64) for n in (M, N)]
        P, Q, s, t = (torch.from_numpy(v.astype(np.int8)).to(R.DEV) for v in (p, q, *signs))
        a = s[:, None] * P
        b = Q[:, None] * t if trans else t[:, None] * Q
        if trans and N % 16:
            wide = torch.zeros((K, R.ceil16(N)), dtype=torch.int8, device=R.DEV)
            wide[:, :N] = b
            b = wide[:, :N]
        total = int((p.astype(np.int64) * q).sum())
        assert abs(total) < 2 ** 31
        c = i8.cfint8_gemm(a, None, b, None, M, N, K, trans_b=trans)
        torch.cuda.synchronize()
        want = torch.from_numpy((np.outer(*signs) * total).astype(np.float32))
        R.same_bits(c, want, f"{kernel} longest K")


# (T, E, topk, H, I, way): several blocks of 128 for every wave, odd ends; the widest and the most of everything
LAYERS = [
    (40, 4, 2, 2064, 1040, "experts"), (33, 5, 2, 1040, 592, "experts"), (24, 3, 1, 2064, 1040, "experts"),
    (20, 260, 2, 1040, 144, "experts"), (64, 4, 1, 16384, 48, "experts"), (48, 4, 2, 64, 16384, "experts"),
    (1, 8, 2, 16384, 80, "slots"), (3, 6, 2, 4112, 144, "slots"), (1, 8, 8, 640, 16384, "slots"),
    (1, 32, 32, 512, 4096, "slots"), (2, 4, 2, 2064, 1040, "slots")]


def layer(T, E, topk, H, I, dtype, rows=None, seed=0):
    say(f"[int8 kernels] moe T={T} E={E} topk={topk} H={H} I={I} {dtype}")
    x, r, gu, gus, dn, dns = make(T, E, H, I, dtype, seed)
    rows = list(range(T)) if rows is None else rows
    y, ids, w = i8.cfint8_moe(*dev(x, r, gu, gus, dn, dns), topk)
    torch.cuda.synchronize()
    Y, bound, wi, wp, dp = reference(x[rows], r, gu, gus, dn, dns, topk, True, None, dtype)
    assert np.array_equal(ids[rows].cpu().numpy(), wi), "ids"
    assert (np.abs(w[rows].cpu().double().numpy() - wp) <= dp).all(), "weights"
    err = np.abs(y[rows].cpu().double().numpy() - Y)
    assert (err <= bound).all(), f"{(err > bound).sum()} beyond the bound, worst {np.max(err / bound):.3g} of it"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,E,topk,H,I,way", LAYERS)
def test_layer(T, E, topk, H, I, way, dtype):
    # rows are independent of each other: every expert's first tiles of sixteen and its last rows
    layer(T, E, topk, H, I, dtype, rows=sorted({*range(0, T, 3), T - 1}))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,E,topk,H,I", [(256, 32, 32, 16, 16384), (256, 1024, 32, 48, 16)])
def test_most_slots(T, E, topk, H, I, dtype):
    """8192 slots: h's digits lie up to 2^29 bytes from the first."""
    layer(T, E, topk, H, I, dtype, rows=[0, 1, 128, 254, 255])
