// Product of 8-bit integer codes with a scale for each token and channel on the gfx950 matrix cores.
//
// C[m][n] = (sum_k qa[m][k] qb[n][k]) sa[m] sb[n] + bias[n]: v_mfma_i32_32x32x32_i8 sums exactly, so the
// result depends neither on the tiling nor on the order of K.
#include "int8_internal.hpp"

namespace cfint8 {

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));

// the 16 codes at position k of a line of n, zeros past its end
__device__ __forceinline__ i32x4 load16(const int8_t* p, int64_t k, int64_t n) {
    i32x4 v = {0, 0, 0, 0};
    if (k >= n) return v;
    v = *reinterpret_cast<const i32x4*>(p + k);
    if (k + 16 > n) {
        const int left = (int)(n - k);
#pragma unroll
        for (int w = 0; w < 4; w++) {
            const int b = left - 4 * w;   // codes of this word
            v[w] = b >= 4 ? v[w] : b <= 0 ? 0 : (int)((uint32_t)v[w] & ((1u << (8 * b)) - 1));
        }
    }
    return v;
}

__device__ __forceinline__ uint32_t to_bf16(float f) {   // nearest even; NaN stays one
    uint32_t u = __float_as_uint(f);
    if ((u & 0x7FFFFFFFu) > 0x7F800000u) return 0x7FC0u;
    u += 0x7FFFu + ((u >> 16) & 1u);
    return u >> 16;
}

// sum * sa * sb + bias.  The scales' significands multiply the sum and their exponents are applied in one
// step, so nothing leaves fp32's range in between
__device__ __forceinline__ float scaled(int sum, float sa, float sb, float bias) {
    const float m = (float)sum * (__builtin_amdgcn_frexp_mantf(sa) * __builtin_amdgcn_frexp_mantf(sb));
    return __builtin_amdgcn_ldexpf(m, __builtin_amdgcn_frexp_expf(sa) + __builtin_amdgcn_frexp_expf(sb)) + bias;
}

constexpr int BM = 64, BN = 64, BK = 64, PITCH = BK + 16;

__global__ __launch_bounds__(256) void simple_kernel(GemmArgs g, int64_t tiles_n) {
    __shared__ __attribute__((aligned(16))) int8_t sa[BM * PITCH], sb[BN * PITCH];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t m0 = (blockIdx.x / tiles_n) * BM, n0 = (blockIdx.x % tiles_n) * BN;
    i32x16 acc = {};
    const int row = tid >> 2, chunk = tid & 3;
    for (int64_t k0 = 0; k0 < g.K; k0 += BK) {
        const i32x4 zero = {0, 0, 0, 0};
        const i32x4 a = m0 + row < g.M ? load16(g.a + (m0 + row) * g.lda, k0 + 16 * chunk, g.K) : zero;
        i32x4 b;
        if (g.trans) b = k0 + row < g.K ? load16(g.b + (k0 + row) * g.ldb, n0 + 16 * chunk, g.N) : zero;
        else b = n0 + row < g.N ? load16(g.b + (n0 + row) * g.ldb, k0 + 16 * chunk, g.K) : zero;
        __syncthreads();
        *reinterpret_cast<i32x4*>(sa + row * PITCH + 16 * chunk) = a;
        if (g.trans) {
#pragma unroll
            for (int i = 0; i < 16; i++) sb[(16 * chunk + i) * PITCH + row] = (int8_t)(b[i >> 2] >> (8 * (i & 3)));
        } else {
            *reinterpret_cast<i32x4*>(sb + row * PITCH + 16 * chunk) = b;
        }
        __syncthreads();
        const int8_t* pa = sa + ((wave >> 1) * 32 + (lane & 31)) * PITCH + 16 * (lane >> 5);
        const int8_t* pb = sb + ((wave & 1) * 32 + (lane & 31)) * PITCH + 16 * (lane >> 5);
#pragma unroll
        for (int k = 0; k < BK; k += 32)
            acc = __builtin_amdgcn_mfma_i32_32x32x32_i8(*reinterpret_cast<const i32x4*>(pa + k),
                                                        *reinterpret_cast<const i32x4*>(pb + k), acc, 0, 0, 0);
    }
    const int64_t n = n0 + (wave & 1) * 32 + (lane & 31);
    if (n >= g.N) return;
    const float sb_n = g.bs ? g.bs[n] : 1.f, bias = g.bias ? g.bias[n] : 0.f;
#pragma unroll
    for (int v = 0; v < 16; v++) {
        const int64_t m = m0 + (wave >> 1) * 32 + 8 * (v >> 2) + 4 * (lane >> 5) + (v & 3);
        if (m >= g.M) continue;
        const float y = scaled(acc[v], g.as ? g.as[m] : 1.f, sb_n, bias);
        if (g.c_bf16) static_cast<uint16_t*>(g.c)[m * g.ldc + n] = (uint16_t)to_bf16(y);
        else static_cast<float*>(g.c)[m * g.ldc + n] = y;
    }
}

}  // namespace

int64_t gemm_workspace_bytes(int64_t, int64_t, int64_t, int) { return 0; }

hipError_t launch_gemm(const GemmArgs& g, hipStream_t s) {
    const int64_t tn = (g.N + BN - 1) / BN, tm = (g.M + BM - 1) / BM;
    simple_kernel<<<(unsigned)(tm * tn), 256, 0, s>>>(g, tn);
    return hipGetLastError();
}

}  // namespace cfint8
