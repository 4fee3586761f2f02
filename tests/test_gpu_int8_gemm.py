"""The product of 8-bit codes with scales for each token and channel.  The sum is exact, so every result
is compared bit for bit with the same few fp32 operations on the exact sum."""

import numpy as np
import pytest
import torch

from paper_2608_10010_amd import cfint8 as i8
from tests import int8_ref as R
from tests.gpu_util import say

pytestmark = pytest.mark.gpu


def case(M, N, K, trans=0, dtype=torch.float32, scales="ab", bias=True, ldc=None, seed=0, spread=1.0, codes=None):
    rng = np.random.default_rng(seed + 7 * M + 13 * N + 31 * K)
    a, b = R.random_codes(rng, M, K), R.random_codes(rng, N, K)
    if codes is not None:
        a[:], b[:] = codes
    sa = np.exp(rng.standard_normal(M) * spread).astype(np.float32) if "a" in scales else None
    sb = np.exp(rng.standard_normal(N) * spread).astype(np.float32) if "b" in scales else None
    bs = (rng.standard_normal(N) * 1e3).astype(np.float32) if bias else None
    return a, b, sa, sb, bs


def dev(v):
    return None if v is None else torch.from_numpy(v).to(R.DEV)


def run(M, N, K, trans=0, dtype=torch.float32, ld_extra=0, c_pad=0, **kw):
    say(f"[int8 gemm] M={M} N={N} K={K} trans={trans} {dtype} {kw}")
    a, b, sa, sb, bs = case(M, N, K, **kw)
    ta = R.codes_tensor(a, fill=101, ld=R.ceil16(K) + ld_extra)
    tb = R.codes_tensor(b.T if trans else b, fill=-93, ld=R.ceil16(N if trans else K) + ld_extra)
    wide = torch.full((M + 1, N + c_pad), -3.0, dtype=dtype, device=R.DEV)
    i8.cfint8_gemm(ta, dev(sa), tb, dev(sb), M, N, K, trans_b=trans, bias=dev(bs), c=wide[:M, :N])
    torch.cuda.synchronize()
    R.same_bits(wide[:M, :N], R.gemm(a, b, sa, sb, bs, dtype), f"{M}x{N}x{K}")
    assert bool((wide[:M, N:] == -3).all()) and bool((wide[M] == -3).all()), "written outside C"


# sizes on both sides of tiles, of pieces of 16 codes and of the split of K
@pytest.mark.parametrize("trans", [0, 1])
@pytest.mark.parametrize("M,N,K", [
    (1, 1, 1), (1, 5, 16), (2, 17, 15), (3, 16, 17), (1, 4096, 4096), (4, 1000, 4099), (16, 33, 64), (17, 64, 129),
    (31, 130, 100), (33, 257, 63), (64, 256, 128), (65, 63, 257), (100, 511, 1000), (128, 128, 128), (129, 127, 500),
    (255, 300, 255), (256, 256, 2048), (257, 513, 130), (333, 700, 1027), (513, 1025, 400), (1024, 2048, 256)])
def test_sizes(M, N, K, trans):
    run(M, N, K, trans)
    run(M, N, K, trans, dtype=torch.bfloat16, ld_extra=48, c_pad=5)


@pytest.mark.parametrize("trans", [0, 1])
@pytest.mark.parametrize("scales,bias", [("", False), ("a", True), ("b", False), ("ab", True)])
def test_optional_vectors(scales, bias, trans):
    for M, N, K in ((5, 70, 200), (300, 260, 300)):
        run(M, N, K, trans, scales=scales, bias=bias)


@pytest.mark.parametrize("M,N", [(1, 64), (40, 48), (300, 520)])
def test_largest_sums(M, N):
    """Every product of the longest K at the codes' ends: the sum stays exact in 32 bits."""
    K = 131056
    for codes in ((-128, -128), (127, -128), (127, 127)):
        run(M, N, K, codes=codes, scales="", bias=False)


def test_scales_far_apart():
    """Scales whose products leave fp32's range although no result does, results that do, zeros, NaN."""
    M, N, K = 70, 300, 160
    a, b, _, _, _ = case(M, N, K)
    sa, sb = np.full(M, 1e-37, np.float32), np.full(N, 1e-20, np.float32)
    sb[1::4], sb[2::4], sb[3::4] = 1e30, 0.0, 1e-42
    sa[1::3], sa[2::3] = 2e36, 1e-45
    sa[5], sb[7] = np.nan, np.nan
    for dtype in (torch.float32, torch.bfloat16):
        say(f"[int8 gemm] scales far apart {dtype}")
        c = i8.cfint8_gemm(R.codes_tensor(a), dev(sa), R.codes_tensor(b), dev(sb), M, N, K, dtype=dtype)
        torch.cuda.synchronize()
        R.same_bits(c, R.gemm(a, b, sa, sb, None, dtype), "scales far apart")
        assert bool(torch.isnan(c[5]).all()) and bool(torch.isnan(c[:, 7]).all())


@pytest.mark.parametrize("trans", [0, 1])
def test_leading_dimensions_past_32_bits(trans):
    """A's and B's last rows lie past 2^31 bytes from the first."""
    M, N, K = 600, 520, 48
    ld = 4194304
    rng = np.random.default_rng(3)
    a, b = R.random_codes(rng, M, K), R.random_codes(rng, N, K)
    wide = torch.zeros((M, ld), dtype=torch.int8, device=R.DEV)
    wide[:, :K] = torch.from_numpy(a).to(R.DEV)
    say(f"[int8 gemm] lda = 2^22, trans={trans}")
    c = i8.cfint8_gemm(wide, None, R.codes_tensor(b.T if trans else b), None, M, N, K, trans_b=trans)
    torch.cuda.synchronize()
    R.same_bits(c, R.gemm(a, b, None, None, None, torch.float32), "lda")
    if not trans:
        c = i8.cfint8_gemm(R.codes_tensor(b), None, wide, None, N, M, K)
    else:                                           # K x N codes with K = 600 rows of 2^22
        wide[:, :48] = torch.from_numpy(a).to(R.DEV)
        q = R.random_codes(rng, 70, M)
        c = i8.cfint8_gemm(R.codes_tensor(q), None, wide, None, 70, 48, M, trans_b=1)
        b, a = q, np.ascontiguousarray(a.T)
    torch.cuda.synchronize()
    R.same_bits(c, R.gemm(b, a, None, None, None, torch.float32), "ldb")


def test_outputs_past_32_bits():
    """Outputs past 2^31 elements from C's first."""
    M, N, K = 40000, 60000, 32
    rng = np.random.default_rng(4)
    a, b = R.random_codes(rng, M, K), R.random_codes(rng, N, K)
    say("[int8 gemm] 40000 x 60000")
    c = i8.cfint8_gemm(R.codes_tensor(a), None, R.codes_tensor(b), None, M, N, K, dtype=torch.bfloat16)
    torch.cuda.synchronize()
    rows = [0, 1, 20000, 35791, 39999]
    R.same_bits(c[rows], R.gemm(a[rows], b, None, None, None, torch.bfloat16), "rows")


# large enough for each tile shape: 64 x 64, 64 x 128, 128 x 128, 256 x 128, 256 x 256, with ends inside tiles, blocks of
# 128 codes (one, two and three of them over) and pieces of 16; one and two rows against many columns, up to 16
# rows against few
@pytest.mark.parametrize("M,N,K", [
    (1, 9001, 1100), (2, 8193, 333), (2, 16400, 4113), (16, 4090, 1000), (9, 4000, 2049), (16, 100, 5000),
    (200, 4000, 1000), (250, 4090, 1001), (500, 4100, 1003), (1000, 4090, 900), (2040, 4090, 515), (2040, 4090, 641),
    (4090, 4093, 129), (4090, 4093, 1037), (4096, 4096, 256)])
def test_routes(M, N, K):
    run(M, N, K, ld_extra=16)
    run(M, N, K, dtype=torch.bfloat16, spread=30.0)        # scales that are not moderate


def test_results_do_not_depend_on_the_route():
    """The same rows and columns in products that take different kernels."""
    K = 1537
    rng = np.random.default_rng(8)
    a, b = R.random_codes(rng, 4090, K), R.random_codes(rng, 4100, K)
    sa, sb = np.exp(rng.standard_normal(4090)).astype(np.float32), np.exp(rng.standard_normal(4100)).astype(np.float32)
    ta, tb, ga, gb = R.codes_tensor(a), R.codes_tensor(b), dev(sa), dev(sb)
    whole = i8.cfint8_gemm(ta, ga, tb, gb, 4090, 4100, K)
    for M, N in ((1, 4100), (2, 4100), (14, 3000), (40, 4100), (250, 4100), (512, 4100), (1024, 2100), (2048, 4100)):
        say(f"[int8 gemm] route {M} x {N} x {K}")
        c = i8.cfint8_gemm(ta, ga, tb, gb, M, N, K)
        torch.cuda.synchronize()
        R.same_bits(c, whole[:M, :N], f"{M} x {N}")


@pytest.mark.parametrize("M,N,K", [(600, 4096, 300), (1500, 2300, 4097), (2100, 4100, 1001), (4097, 4200, 259),
                                   (16, 1030, 4100), (40, 200, 9000), (2, 9000, 530)])
def test_transposed_operands_of_every_tile(M, N, K):
    """The same product from [N][K] and from [K][N] codes, bit for bit."""
    say(f"[int8 gemm] transposed {M} {N} {K}")
    a, b, sa, sb, bs = case(M, N, K)
    ta, tb, tt = R.codes_tensor(a, fill=5), R.codes_tensor(b, fill=9), R.codes_tensor(b.T, fill=-7)
    for dtype in (torch.float32, torch.bfloat16):
        want = i8.cfint8_gemm(ta, dev(sa), tb, dev(sb), M, N, K, bias=dev(bs), dtype=dtype)
        got = i8.cfint8_gemm(ta, dev(sa), tt, dev(sb), M, N, K, trans_b=1, bias=dev(bs), dtype=dtype)
        torch.cuda.synchronize()
        R.same_bits(got, want.cpu(), f"{M}x{N}x{K}")


@pytest.mark.parametrize("M,N,K", [(1, 17, 2048), (2, 4099, 2050), (1, 5, 4095), (2, 3, 6000), (1, 70001, 1929), (2, 33000, 4100),
                                   (1, 8195, 1), (3, 9000, 100), (32, 9001, 257)])
def test_one_or_two_rows(M, N, K):
    run(M, N, K)
    run(M, N, K, dtype=torch.bfloat16, ld_extra=32, c_pad=5)


@pytest.mark.parametrize("M,N,trans", [((1 << 21) + 70, 3, 0), ((1 << 21) + 70, 20, 1), (1, (1 << 21) + 33, 0),
                                       (3, (1 << 21) + 33, 0), (70, (1 << 21) + 65, 1)])
def test_more_lines_than_a_launch_takes(M, N, trans):
    run(M, N, 19, trans=trans)
