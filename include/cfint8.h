/*
 * cfint8.h -- C ABI of the 8-bit integer operators of libcurvefp on AMD Instinct MI355X (gfx950):
 * quantization with one real scale for each token or channel, reconstruction, the matrix product of
 * such codes, and a mixture-of-experts layer for a few tokens with such weights.
 *
 * INT8 with real scales is the format that the paper measures CurveFP against (arXiv 2608.10010,
 * Sec. 4.2).  The calls follow curvefp.h: its dtypes and status codes; device pointers that the caller
 * owns; asynchronous on `stream` (a hipStream_t, NULL = the legacy default stream), nothing allocated,
 * kept or synchronized, so every call may be captured into a HIP graph; argument errors returned as a
 * negative curvefp_status before any HIP call.
 *
 * A line is what shares a scale s >= 0: a row of the source (block_axis = 1) or a column (block_axis = 0).
 * Codes q are int8 in [-127, 127] and stand for q s.  Matrices of codes are row-major with a leading
 * dimension `ld` in bytes that is a multiple of 16 and at most CFINT8_MAX_LD, 16-byte aligned; each of
 * their rows, the last one too, must be readable up to the next multiple of 16 bytes.  What these bytes
 * behind the last code hold does not matter, and no call writes them.
 */
#ifndef CFINT8_H
#define CFINT8_H

#include "curvefp.h"

#ifdef __cplusplus
extern "C" {
#endif

#define CFINT8_MAX_LD ((int64_t)4194304)
/* largest K of a product: 131056 products of codes stay below 2^31 whatever the codes */
#define CFINT8_MAX_K ((int64_t)131056)

/*
 * Quantization.  For each line with elements x_k
 *   v_k = x_k, or x_k * mul[k] rounded to fp32 where mul is not null (fp32 [k], k along the line:
 *         for a gradient whose product contracts over the axis that another operand's scales lie on);
 *   s   = max |v_k| / 127, rounded to fp32;
 *   q_k = v_k / s (the exact quotient) rounded to the nearest integer, ties to even.
 * A line whose s is 0 (of zeros, or of values so small that s rounds to 0) has zero codes.  A line that holds a NaN or an infinity (in v) has s = NaN
 * and zero codes.  Where s is subnormal (max |v| below about 1.5e-36) codes are clamped to +-127.
 *   src     [rows][ld_src] of `dtype` (fp32 or bf16).  block_axis = 1: 16-byte aligned rows, each readable
 *           up to the next multiple of 16 bytes; block_axis = 0: element alignment suffices.
 *   mul     null, or fp32, one for each position of a line, 16-byte aligned.
 *   codes   block_axis = 1: [rows][ld_codes], codes in the first cols of each row;
 *           block_axis = 0: [cols][ld_codes], codes in the first rows of each (quantize-transpose).
 *   scales  fp32, one for each line.
 *   workspace  at least cfint8_quantize_workspace_bytes bytes, 16-byte aligned (may be null when that
 *           is 0, as for block_axis = 1); scratch, so calls that share it must be ordered.
 * Any rows and cols >= 1 below 2^31; ld_src <= 2^30.  Errors: CURVEFP_ERR_NULL, _FORMAT (dtype), _BLOCK
 * (block_axis), _SHAPE (sizes, leading dimensions, workspace too small), _ALIGN, _HIP.
 */
int64_t cfint8_quantize_workspace_bytes(int64_t rows, int64_t cols, int block_axis);
int cfint8_quantize(const void* src, int dtype, int64_t rows, int64_t cols, int64_t ld_src, int block_axis,
                    const float* mul, int8_t* codes, int64_t ld_codes, float* scales, void* workspace,
                    int64_t workspace_bytes, void* stream);

/*
 * Reconstruction: dst[o][i] = codes[o][i] * scales[o], rounded once to `dtype` (fp32, or bf16: the
 * product in fp32, then to bf16, ties to even).  codes [outer][ld_codes], scales [outer], dst
 * [outer][ld_dst] with 16-byte aligned rows.  A line with s = NaN gives NaN.
 */
int cfint8_dequantize(const int8_t* codes, int64_t ld_codes, const float* scales, int64_t outer, int64_t k,
                      void* dst, int dtype, int64_t ld_dst, void* stream);

/*
 * Product with scales for each token and channel:
 *   C[m][n] = (sum_k qa[m][k] qb[n][k]) a_scales[m] b_scales[n] + bias[n]
 * The sum is exact (int32); it is converted to fp32, multiplied by the two scales and added to the bias
 * in fp32 (scales that would leave fp32's range in between do not, only results do), and rounded to bf16
 * where c_dtype is bf16.
 *   a        codes [M][lda].
 *   b        trans_b = 0: codes [N][ldb]; trans_b = 1: codes [K][ldb], i.e. the operand of another product
 *            read transposed (the backward products below).
 *   a_scales [M], b_scales [N], bias [N]: fp32; each may be null (scales of 1, no bias).
 *   c        [M][ldc] of c_dtype (fp32 or bf16), overwritten; 16-byte aligned, any ldc >= N.
 *   workspace  at least cfint8_gemm_workspace_bytes(M, N, K, trans_b) bytes, 256-byte aligned (may be null
 *            when that is 0); scratch, so calls that share it must be ordered.
 * Any M, N >= 1 below 2^31 and 1 <= K <= CFINT8_MAX_K.  A scale that is NaN gives NaN in its whole row or
 * column.  The result does not depend on the route the sizes take.
 * Gradients of Y = X W^T from the forward pass's codes (qx, sx of X along its rows, qw, sw of W along its
 * rows), each with the forward scales folded into the quantized gradient:
 *   dX = Q(dY * sw along the rows) Qw   : quantize(dY, block_axis 1, mul = sw), gemm(.., b = qw, trans_b = 1, b_scales = null)
 *   dW = Q(dY * sx along the columns) Qx: quantize(dY, block_axis 0, mul = sx), gemm(.., b = qx, trans_b = 1, b_scales = null)
 * Errors: CURVEFP_ERR_NULL, _FORMAT (c_dtype), _BLOCK (trans_b not 0 or 1), _SHAPE, _ALIGN, _HIP.
 */
int64_t cfint8_gemm_workspace_bytes(int64_t M, int64_t N, int64_t K, int trans_b);
int cfint8_gemm(const int8_t* a, int64_t lda, const float* a_scales, const int8_t* b, int64_t ldb, int trans_b,
                const float* b_scales, const float* bias, int64_t M, int64_t N, int64_t K, void* c, int c_dtype,
                int64_t ldc, void* workspace, int64_t workspace_bytes, void* stream);

/*
 * Mixture-of-experts layer for a few tokens, weights in 8 bits (codes and scales of cfint8_quantize along
 * the rows), activations as they are:
 *   l[t][e] = x[t] . router[e], summed in 64 bits and held in fp32;
 *   slot j of token t takes the expert with the j-th largest l[t] (ties: the lowest e; NaN below all else);
 *   p[t][j] = exp(l_j - l_0) / sum over the topk slots (renormalize = 1) or over all experts (0);
 *   g = (x[t] . gate_up[e][i]) s, u = (x[t] . gate_up[e][I + i]) s, h[i] = g / (1 + exp(-g)) u;
 *   y[t] = sum_j p[t][j] (h . down[e_j]) s, rounded once to x's dtype.
 * Codes enter the products exactly.  x and h enter them in fixed point, 22 bits (dtype bf16) or 30 bits (fp32)
 * below a power of two above the largest of a row of x or of up to 64 neighbours of h; the sums of up to 64 such
 * products (all of a row's for x) are exact, their order in fp32 depends on the sizes alone.
 *   x        [T][ld_x] of `dtype` (fp32 or bf16), 16-byte aligned rows; T in [1, CFINT8_MOE_MAX_TOKENS].
 *   router   [E][H] of `dtype`, 16-byte aligned; E in [1, CFINT8_MOE_MAX_EXPERTS].
 *   gate_up  codes [E][2 I][H] (I gate rows, then I up rows), scales [E][2 I];
 *   down     codes [E][H][I], scales [E][H]; H and I multiples of 16, at most CFINT8_MOE_MAX_WIDTH.
 *   topk     in [1, min(E, CFINT8_MOE_MAX_TOPK)].
 *   active   null, or [T] bytes: a token whose byte is 0 (a padded one) takes no expert, reads no weight and
 *            gets a zero row, ids of -1 and weights of 0, whatever its x holds.
 *   y        [T][ld_y] of `dtype`, 16-byte aligned rows; ids int32 and weights fp32 [T][topk].
 *   workspace  at least cfint8_moe_workspace_bytes bytes, 256-byte aligned; scratch, so calls that share it must be
 *            ordered.
 * Values leave fp32's range where g, u, h, a slot's (h . down) s or y do, not where a sum of codes does that its scale
 * brings back.
 * A NaN or an infinity in x gives NaN in that token's y (in no other's).
 * Errors: CURVEFP_ERR_NULL, _FORMAT (dtype), _SHAPE, _ALIGN, _HIP.
 */
#define CFINT8_MOE_MAX_TOKENS ((int64_t)256)
#define CFINT8_MOE_MAX_EXPERTS ((int64_t)1024)
#define CFINT8_MOE_MAX_TOPK ((int64_t)32)
#define CFINT8_MOE_MAX_WIDTH ((int64_t)16384)
int64_t cfint8_moe_workspace_bytes(int64_t T, int64_t E, int64_t topk, int64_t H, int64_t I);
int cfint8_moe(const void* x, int dtype, int64_t T, int64_t H, int64_t ld_x, const void* router, int64_t E,
               const int8_t* gate_up, const float* gate_up_scales, const int8_t* down, const float* down_scales,
               int64_t I, int64_t topk, int renormalize, const uint8_t* active, void* y, int64_t ld_y, int32_t* ids,
               float* weights, void* workspace, int64_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* CFINT8_H */
