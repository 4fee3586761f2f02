// C ABI of the 8-bit integer operators: argument validation and dispatch.  Every argument error is
// found before any HIP call.

#include "../../include/cfint8.h"
#include "int8_internal.hpp"

using namespace cfint8;

namespace {

constexpr int64_t kMaxExtent = (int64_t)1 << 31;

bool aligned(const void* p, uintptr_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
bool dtype_ok(int d) { return d == CURVEFP_F32 || d == CURVEFP_BF16; }
int64_t esize(int d) { return d == CURVEFP_F32 ? 4 : 2; }
bool extent_ok(int64_t n) { return n >= 1 && n < kMaxExtent; }
// leading dimension of a matrix of codes with n in each row: its size, then its alignment
bool ld_ok(int64_t ld, int64_t n) { return ld >= n && ld <= CFINT8_MAX_LD; }

int hip_status(hipError_t e) { return e == hipSuccess ? CURVEFP_OK : CURVEFP_ERR_HIP; }

bool gemm_sizes_ok(int64_t M, int64_t N, int64_t K) {
    return extent_ok(M) && extent_ok(N) && K >= 1 && K <= CFINT8_MAX_K;
}

bool moe_sizes_ok(int64_t T, int64_t E, int64_t topk, int64_t H, int64_t I) {
    return T >= 1 && T <= CFINT8_MOE_MAX_TOKENS && E >= 1 && E <= CFINT8_MOE_MAX_EXPERTS && topk >= 1 && topk <= E &&
           topk <= CFINT8_MOE_MAX_TOPK && H >= 16 && H % 16 == 0 && H <= CFINT8_MOE_MAX_WIDTH && I >= 16 &&
           I % 16 == 0 && I <= CFINT8_MOE_MAX_WIDTH;
}

}  // namespace

#pragma GCC visibility push(default)
extern "C" {

int64_t cfint8_quantize_workspace_bytes(int64_t rows, int64_t cols, int block_axis) {
    if (block_axis != 0 && block_axis != 1) return CURVEFP_ERR_BLOCK;
    if (!extent_ok(rows) || !extent_ok(cols)) return CURVEFP_ERR_SHAPE;
    return quantize_workspace_bytes(rows, cols, block_axis);
}

int cfint8_quantize(const void* src, int dtype, int64_t rows, int64_t cols, int64_t ld_src, int block_axis,
                    const float* mul, int8_t* codes, int64_t ld_codes, float* scales, void* workspace,
                    int64_t workspace_bytes, void* stream) {
    if (!src || !codes || !scales) return CURVEFP_ERR_NULL;
    if (!dtype_ok(dtype)) return CURVEFP_ERR_FORMAT;
    if (block_axis != 0 && block_axis != 1) return CURVEFP_ERR_BLOCK;
    if (!extent_ok(rows) || !extent_ok(cols) || ld_src < cols || ld_src > ((int64_t)1 << 30)) return CURVEFP_ERR_SHAPE;
    if (!ld_ok(ld_codes, block_axis == 1 ? cols : rows)) return CURVEFP_ERR_SHAPE;
    const int64_t need = quantize_workspace_bytes(rows, cols, block_axis);
    if (need > 0 && !workspace) return CURVEFP_ERR_NULL;
    if (workspace_bytes < need) return CURVEFP_ERR_SHAPE;
    if (!aligned(codes, 16) || ld_codes % 16 || !aligned(scales, 4) || !aligned(mul, 16)) return CURVEFP_ERR_ALIGN;
    if (need > 0 && !aligned(workspace, 16)) return CURVEFP_ERR_ALIGN;
    if (block_axis == 1 ? !aligned(src, 16) || (ld_src * esize(dtype)) % 16 : !aligned(src, (uintptr_t)esize(dtype)))
        return CURVEFP_ERR_ALIGN;
    return hip_status(launch_quantize(src, dtype, rows, cols, ld_src, block_axis, mul, codes, ld_codes, scales, workspace,
                                      reinterpret_cast<hipStream_t>(stream)));
}

int cfint8_dequantize(const int8_t* codes, int64_t ld_codes, const float* scales, int64_t outer, int64_t k, void* dst,
                      int dtype, int64_t ld_dst, void* stream) {
    if (!codes || !scales || !dst) return CURVEFP_ERR_NULL;
    if (!dtype_ok(dtype)) return CURVEFP_ERR_FORMAT;
    if (!extent_ok(outer) || !extent_ok(k) || !ld_ok(ld_codes, k) || ld_dst < k || ld_dst > ((int64_t)1 << 30))
        return CURVEFP_ERR_SHAPE;
    if (!aligned(codes, 16) || ld_codes % 16 || !aligned(scales, 4) || !aligned(dst, 16) || (ld_dst * esize(dtype)) % 16)
        return CURVEFP_ERR_ALIGN;
    return hip_status(launch_dequantize(codes, ld_codes, scales, outer, k, dst, dtype, ld_dst,
                                        reinterpret_cast<hipStream_t>(stream)));
}

int64_t cfint8_gemm_workspace_bytes(int64_t M, int64_t N, int64_t K, int trans_b) {
    if (trans_b != 0 && trans_b != 1) return CURVEFP_ERR_BLOCK;
    if (!gemm_sizes_ok(M, N, K)) return CURVEFP_ERR_SHAPE;
    return gemm_workspace_bytes(M, N, K, trans_b);
}

int cfint8_gemm(const int8_t* a, int64_t lda, const float* a_scales, const int8_t* b, int64_t ldb, int trans_b,
                const float* b_scales, const float* bias, int64_t M, int64_t N, int64_t K, void* c, int c_dtype,
                int64_t ldc, void* workspace, int64_t workspace_bytes, void* stream) {
    if (!a || !b || !c) return CURVEFP_ERR_NULL;
    if (!dtype_ok(c_dtype)) return CURVEFP_ERR_FORMAT;
    if (trans_b != 0 && trans_b != 1) return CURVEFP_ERR_BLOCK;
    if (!gemm_sizes_ok(M, N, K)) return CURVEFP_ERR_SHAPE;
    if (!ld_ok(lda, K) || !ld_ok(ldb, trans_b ? N : K) || ldc < N || ldc >= kMaxExtent) return CURVEFP_ERR_SHAPE;
    const int64_t need = gemm_workspace_bytes(M, N, K, trans_b);
    if (need > 0 && !workspace) return CURVEFP_ERR_NULL;
    if (workspace_bytes < need) return CURVEFP_ERR_SHAPE;
    if (!aligned(a, 16) || lda % 16 || !aligned(b, 16) || ldb % 16 || !aligned(c, 16)) return CURVEFP_ERR_ALIGN;
    if (!aligned(a_scales, 4) || !aligned(b_scales, 4) || !aligned(bias, 4)) return CURVEFP_ERR_ALIGN;
    if (need > 0 && !aligned(workspace, 256)) return CURVEFP_ERR_ALIGN;
    GemmArgs g;
    g.a = a;
    g.lda = lda;
    g.as = a_scales;
    g.b = b;
    g.ldb = ldb;
    g.trans = trans_b;
    g.bs = b_scales;
    g.bias = bias;
    g.M = M;
    g.N = N;
    g.K = K;
    g.c = c;
    g.c_bf16 = c_dtype == CURVEFP_BF16;
    g.ldc = ldc;
    g.ws = workspace;
    return hip_status(launch_gemm(g, reinterpret_cast<hipStream_t>(stream)));
}

int64_t cfint8_moe_workspace_bytes(int64_t T, int64_t E, int64_t topk, int64_t H, int64_t I) {
    if (!moe_sizes_ok(T, E, topk, H, I)) return CURVEFP_ERR_SHAPE;
    return moe_workspace_bytes(T, E, topk, H, I);
}

int cfint8_moe(const void* x, int dtype, int64_t T, int64_t H, int64_t ld_x, const void* router, int64_t E,
               const int8_t* gate_up, const float* gate_up_scales, const int8_t* down, const float* down_scales,
               int64_t I, int64_t topk, int renormalize, const uint8_t* active, void* y, int64_t ld_y, int32_t* ids,
               float* weights, void* workspace, int64_t workspace_bytes, void* stream) {
    if (!x || !router || !gate_up || !gate_up_scales || !down || !down_scales || !y || !ids || !weights || !workspace)
        return CURVEFP_ERR_NULL;
    if (!dtype_ok(dtype)) return CURVEFP_ERR_FORMAT;
    if (!moe_sizes_ok(T, E, topk, H, I) || (renormalize != 0 && renormalize != 1)) return CURVEFP_ERR_SHAPE;
    if (ld_x < H || ld_x > ((int64_t)1 << 30) || ld_y < H || ld_y > ((int64_t)1 << 30)) return CURVEFP_ERR_SHAPE;
    if (workspace_bytes < moe_workspace_bytes(T, E, topk, H, I)) return CURVEFP_ERR_SHAPE;
    const int64_t es = esize(dtype);
    if (!aligned(x, 16) || (ld_x * es) % 16 || !aligned(y, 16) || (ld_y * es) % 16 || !aligned(router, 16) ||
        !aligned(gate_up, 16) || !aligned(down, 16) || !aligned(gate_up_scales, 4) || !aligned(down_scales, 4) ||
        !aligned(ids, 4) || !aligned(weights, 4) || !aligned(workspace, 256))
        return CURVEFP_ERR_ALIGN;
    MoeArgs m;
    m.x = x;
    m.bf16 = dtype == CURVEFP_BF16;
    m.T = T;
    m.H = H;
    m.ldx = ld_x;
    m.router = router;
    m.E = E;
    m.gu = gate_up;
    m.gus = gate_up_scales;
    m.dn = down;
    m.dns = down_scales;
    m.I = I;
    m.topk = topk;
    m.renorm = renormalize;
    m.active = active;
    m.y = y;
    m.ldy = ld_y;
    m.ids = ids;
    m.weights = weights;
    m.ws = workspace;
    return hip_status(launch_moe(m, reinterpret_cast<hipStream_t>(stream)));
}

}  // extern "C"
#pragma GCC visibility pop
