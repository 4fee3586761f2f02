// Internal declarations of the 8-bit integer operators (not part of the C ABI).
#pragma once

#include <cstdint>
#include <hip/hip_runtime.h>

namespace cfint8 {

// A launch has fewer than 2^32 threads: operands of more lines go in parts of so many
constexpr int64_t PART = (int64_t)1 << 21;

int64_t quantize_workspace_bytes(int64_t rows, int64_t cols, int axis);
hipError_t launch_quantize(const void* src, int dtype, int64_t rows, int64_t cols, int64_t ld, int axis,
                           const float* mul, int8_t* codes, int64_t ldq, float* scales, void* ws, hipStream_t s);
hipError_t launch_dequantize(const int8_t* codes, int64_t ldq, const float* scales, int64_t outer, int64_t k, void* dst,
                             int dtype, int64_t ld, hipStream_t s);

struct GemmArgs {
    const int8_t* a;
    int64_t lda;
    const float* as;      // null: 1
    const int8_t* b;
    int64_t ldb;
    int trans;
    const float* bs;      // null: 1
    const float* bias;    // null: none
    int64_t M, N, K;
    void* c;
    int c_bf16;
    int64_t ldc;
    void* ws;
};
int64_t gemm_workspace_bytes(int64_t M, int64_t N, int64_t K, int trans);
hipError_t launch_gemm(const GemmArgs& g, hipStream_t s);

struct MoeArgs {
    const void* x;
    int bf16;
    int64_t T, H, ldx;
    const void* router;
    int64_t E;
    const int8_t* gu;
    const float* gus;
    const int8_t* dn;
    const float* dns;
    int64_t I, topk;
    int renorm;
    const uint8_t* active;
    void* y;
    int64_t ldy;
    int32_t* ids;
    float* weights;
    void* ws;
};
int64_t moe_workspace_bytes(int64_t T, int64_t E, int64_t topk, int64_t H, int64_t I);
hipError_t launch_moe(const MoeArgs& m, hipStream_t s);

}  // namespace cfint8
