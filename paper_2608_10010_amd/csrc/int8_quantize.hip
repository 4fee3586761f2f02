// 8-bit integer quantization with one fp32 scale for each line (a row, or a column through the
// transpose), and its reconstruction.
//
//   s = fl32(max |v| / 127),  q = v / s rounded to nearest even, the quotient exact.
//
// The exact quotient matters: max / 2 lies within 2^-25 of 63.5 s in every line that holds it, on the side
// that the rounding of s decides.  q0 = rint(v * fl32(1/s)) is within one of q, and v - q0 s is exact in one
// fma (a multiple of half an ulp of s below s), so comparing it with s/2 settles q; that comparison
// finds something to mend only next to a tie, and eight elements share it.
//
// Rows: held in registers by a wave (up to 1024) or a workgroup (up to 32768), the source
// read once; longer ones read twice.  Columns: partial maxima of row chunks into the workspace (maxima, so no order
// to depend on), then 128 x 128 tiles turned in LDS; up to 256 rows all at once.  Bound by memory: 8192 x 14336 bf16 rows
// in 57 to 64 us (5.5 to 6.2 TB/s of source and codes; vector instructions take 93% of a busy unit's issue slots, so not much
// more would fit), 4096 x 11008 columns, whose source is read twice, in 42.
#include <type_traits>

#include "device_util.hpp"
#include "int8_internal.hpp"

namespace cfint8 {

using curvefp::Div32;
using curvefp::div32;
using curvefp::ld16;
using curvefp::make_div32;
using curvefp::st16;
using curvefp::st8;

namespace {

constexpr uint32_t INF_BITS = 0x7F800000u;

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {   // nearest even, low half first
    const f32x2 v = {lo, hi};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}

// what a line's elements are quantized with; pre = 2^64 for lines so small that 1 / s would overflow
struct Line {
    float s, inv, half, pre;
    bool zero;   // zero codes: a line of zeros, or one that holds a NaN or an infinity
    float out;   // the scale as stored
};

__device__ __forceinline__ Line make_line(uint32_t amax) {
    Line l;
    const float m = __uint_as_float(amax);
    l.out = amax >= INF_BITS ? __uint_as_float(0x7FC00000u) : m / 127.0f;
    l.zero = amax >= INF_BITS || l.out == 0.f;
    l.pre = l.out < 0x1p-60f ? 0x1p64f : 1.f;
    l.s = l.zero ? 1.f : l.out * l.pre;
    l.inv = 1.f / l.s;
    l.half = 0.5f * l.s;
    return l;
}

// codes of 8 elements as two little-endian words; TINY: some line's pre is not 1 (and its codes may need the clamp)
template <bool TINY>
__device__ __forceinline__ uint2 quant8(const float* v, const Line& l) {
    float q[8], r[8], far = 0.f;
#pragma unroll
    for (int i = 0; i < 8; i++) {
        const float x = TINY ? v[i] * l.pre : v[i];
        q[i] = __builtin_rintf(x * l.inv);
        r[i] = __builtin_fmaf(-q[i], l.s, x);
        far = fmaxf(far, fabsf(r[i]));
    }
    if (far >= l.half) {
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const float a = fabsf(r[i]);
            const bool up = a > l.half || (a == l.half && ((int)q[i] & 1) != 0);
            q[i] += up ? __builtin_copysignf(1.f, r[i]) : 0.f;
        }
    }
    uint32_t w[2];
#pragma unroll
    for (int h = 0; h < 2; h++) {
        uint32_t b[4];
#pragma unroll
        for (int i = 0; i < 4; i++)
            b[i] = (uint32_t)(int)(TINY ? __builtin_amdgcn_fmed3f(q[4 * h + i], -127.f, 127.f) : q[4 * h + i]);
        // byte 0 of each word, two at a time
        const uint32_t lo = __builtin_amdgcn_perm(b[1], b[0], 0x0C0C0400u);
        const uint32_t hi = __builtin_amdgcn_perm(b[3], b[2], 0x04000C0Cu);
        w[h] = lo | hi;
    }
    if (l.zero) w[0] = w[1] = 0;
    return make_uint2(w[0], w[1]);
}

__device__ __forceinline__ void unpack_bf16(const uint4& u, float* v) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; i++) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
}

// Eight source elements as loaded.  Loads have no branches around them, so that many are out at once: what lies past
// an edge is loaded from the edge and masked, or not stored, afterwards
template <bool BF16>
struct Raw {
    uint4 a, b;   // b: fp32 only

    __device__ __forceinline__ void unpack(float* v) const {
        if (BF16) {
            unpack_bf16(a, v);
        } else {
            const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
            for (int i = 0; i < 8; i++) v[i] = __uint_as_float(w[i]);
        }
    }
};

// elements c .. c + 7 of a row of n with 16-byte aligned pieces, the last of which may reach behind the row's end.
// LAST: not read again, by streaming loads (8192 x 4096 fp32 rows 60 -> 32 us)
template <bool BF16, bool LAST, class I>
__device__ __forceinline__ Raw<BF16> load_pieces(const char* p, I c, I n) {
    constexpr int PER = BF16 ? 8 : 4;   // elements of a piece
    const I last = (n - 1) / PER * PER;
    Raw<BF16> r;
    r.a = ld16<LAST>(reinterpret_cast<const uint4*>(p + (int64_t)min(c, last) * (BF16 ? 2 : 4)));
    if (!BF16) r.b = ld16<LAST>(reinterpret_cast<const uint4*>(p + (int64_t)min((I)(c + 4), last) * 4));
    return r;
}

template <class I>
__device__ __forceinline__ void mask8(float* v, I c, I n) {
    if (c + 8 > n) {
#pragma unroll
        for (int i = 0; i < 8; i++) v[i] = c + i < n ? v[i] : 0.f;
    }
}

// Eight elements of a row for the column kernels, by pieces (past the last whole eight these again) or, where the row's
// pieces are not aligned or end among the eight, element by element (past the last it again)
template <bool BF16, bool PIECES, bool LAST>
__device__ __forceinline__ Raw<BF16> load_columns(const char* p, int64_t c, int64_t n) {
    Raw<BF16> r;
    if (PIECES) {
        const uint4* q = reinterpret_cast<const uint4*>(p + min(c, n / 8 * 8 - 8) * (BF16 ? 2 : 4));
        r.a = ld16<LAST>(q);
        if (!BF16) r.b = ld16<LAST>(q + 1);
        return r;
    }
    uint32_t e[8];
#pragma unroll
    for (int i = 0; i < 8; i++) {
        const int64_t at = min(c + i, n - 1);
        e[i] = BF16 ? (uint32_t)reinterpret_cast<const uint16_t*>(p)[at] : reinterpret_cast<const uint32_t*>(p)[at];
    }
    if (BF16) {
        r.a = make_uint4(e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16);
    } else {
        r.a = make_uint4(e[0], e[1], e[2], e[3]);
        r.b = make_uint4(e[4], e[5], e[6], e[7]);
    }
    return r;
}

// times mul[c .. c + 7] (16-byte aligned), elements past the end left alone
template <class I>
__device__ __forceinline__ void mul8(const float* __restrict__ mul, I c, I n, float* v) {
    if (c + 8 <= n) {
        const float4 a = *reinterpret_cast<const float4*>(mul + c), b = *reinterpret_cast<const float4*>(mul + c + 4);
        v[0] *= a.x, v[1] *= a.y, v[2] *= a.z, v[3] *= a.w;
        v[4] *= b.x, v[5] *= b.y, v[6] *= b.z, v[7] *= b.w;
    } else {
#pragma unroll
        for (int i = 0; i < 7; i++)
            if (c + i < n) v[i] *= mul[c + i];
    }
}

__device__ __forceinline__ uint32_t max8(uint32_t m, const float* v) {
#pragma unroll
    for (int i = 0; i < 8; i++) m = max(m, __float_as_uint(v[i]) & 0x7FFFFFFFu);
    return m;
}

__device__ __forceinline__ uint32_t wave_max(uint32_t m) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o));
    return m;
}

// codes c .. c + 7 of a row of n (c a multiple of 8); nothing behind the row's last
template <class I>
__device__ __forceinline__ void store8(int8_t* q, I c, I n, uint2 w) {
    if (c + 8 <= n) {
        *reinterpret_cast<uint2*>(q + c) = w;
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; i++)
        if (c + i < n) q[c + i] = (int8_t)((i < 4 ? w.x : w.y) >> (8 * (i & 3)));
}

// ---------------------------------------------------------------- rows

// TPR threads hold a row of up to 8 TPR NU elements
template <bool BF16, bool MUL, int TPR, int NU>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void rows_kernel(
    const char* __restrict__ src, int64_t rows, int cols, int64_t ld, const float* __restrict__ mul,
    int8_t* __restrict__ codes, int64_t ldq, float* __restrict__ scales) {
    constexpr int THREADS = TPR < 256 ? 256 : TPR, WAVES = TPR / 64;
    __shared__ uint32_t red[WAVES > 1 ? WAVES : 1];
    const int t = threadIdx.x % TPR;
    const int64_t row = (int64_t)blockIdx.x * (THREADS / TPR) + threadIdx.x / TPR;
    if (row >= rows) return;   // TPR = 64: whole waves, no barrier below
    const char* p = src + row * ld * (BF16 ? 2 : 4);
    Raw<BF16> raw[NU];
    float v[NU][8];
    uint32_t m = 0;
#pragma unroll
    for (int u = 0; u < NU; u++) raw[u] = load_pieces<BF16, true>(p, (u * TPR + t) * 8, cols);
#pragma unroll
    for (int u = 0; u < NU; u++) {
        raw[u].unpack(v[u]);
        mask8(v[u], (u * TPR + t) * 8, cols);
        if (MUL) mul8(mul, (u * TPR + t) * 8, cols, v[u]);
        m = max8(m, v[u]);
    }
    m = wave_max(m);
    if (WAVES > 1) {
        if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = m;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < WAVES; w++) m = max(m, red[w]);
    }
    const Line l = make_line(m);
    int8_t* q = codes + row * ldq;
    auto store = [&](auto tiny) {
#pragma unroll
        for (int u = 0; u < NU; u++) {
            const int c = (u * TPR + t) * 8;
            if (c < cols) store8(q, c, cols, quant8<decltype(tiny)::value>(v[u], l));
        }
    };
    if (l.pre != 1.f) store(std::true_type{});
    else store(std::false_type{});
    if (t == 0) scales[row] = l.out;
}

// rows past the register kernels' reach: the source is read twice
template <bool BF16, bool MUL>
__global__ __launch_bounds__(1024) void long_rows_kernel(const char* __restrict__ src, int64_t cols, int64_t ld,
                                                         const float* __restrict__ mul, int8_t* __restrict__ codes,
                                                         int64_t ldq, float* __restrict__ scales) {
    __shared__ uint32_t red[16];
    const int64_t row = blockIdx.x;
    const char* p = src + row * ld * (BF16 ? 2 : 4);
    float v[8];
    uint32_t m = 0;
    for (int64_t c = (int64_t)threadIdx.x * 8; c < cols; c += 8192) {
        load_pieces<BF16, false>(p, c, cols).unpack(v);
        mask8(v, c, cols);
        if (MUL) mul8(mul, c, cols, v);
        m = max8(m, v);
    }
    m = wave_max(m);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = m;
    __syncthreads();
    for (int w = 0; w < 16; w++) m = max(m, red[w]);
    const Line l = make_line(m);
    for (int64_t c = (int64_t)threadIdx.x * 8; c < cols; c += 8192) {
        load_pieces<BF16, true>(p, c, cols).unpack(v);
        mask8(v, c, cols);
        if (MUL) mul8(mul, c, cols, v);
        store8(codes + row * ldq, c, cols, quant8<true>(v, l));
    }
    if (threadIdx.x == 0) scales[row] = l.out;
}

template <bool BF16, bool MUL>
hipError_t launch_rows(const void* src, int64_t rows, int64_t cols, int64_t ld, const float* mul, int8_t* codes,
                       int64_t ldq, float* scales, hipStream_t s) {
    const char* p = static_cast<const char*>(src);
    const dim3 wave_grid((unsigned)((rows + 3) / 4)), row_grid((unsigned)rows);
#define CFINT8_ROWS(TPR, NU)                                                                                       \
    rows_kernel<BF16, MUL, TPR, NU><<<TPR < 256 ? wave_grid : row_grid, TPR < 256 ? 256 : TPR, 0, s>>>(            \
        p, rows, (int)cols, ld, mul, codes, ldq, scales)
    // units a thread by thirds where a half of them would stay empty (8192 x 5120 bf16 28.4 -> 27.0 us with three of four)
    if (cols <= 512) CFINT8_ROWS(64, 1);
    else if (cols <= 1024) CFINT8_ROWS(64, 2);
    else if (cols <= 2048) CFINT8_ROWS(256, 1);
    else if (cols <= 4096) CFINT8_ROWS(256, 2);
    else if (cols <= 6144) CFINT8_ROWS(256, 3);
    else if (cols <= 8192) CFINT8_ROWS(256, 4);
    else if (cols <= 12288) CFINT8_ROWS(512, 3);
    else if (cols <= 16384) CFINT8_ROWS(512, 4);
    else if (cols <= 32768) CFINT8_ROWS(1024, 4);
    else long_rows_kernel<BF16, MUL><<<row_grid, 1024, 0, s>>>(p, cols, ld, mul, codes, ldq, scales);
#undef CFINT8_ROWS
    return hipGetLastError();
}

// ---------------------------------------------------------------- columns

constexpr int TILE = 128;         // columns and rows of a tile
constexpr int MAX_CHUNKS = 32;    // row chunks with a partial maximum of their own

// As many as give col_max 1024 workgroups, of at least 64 rows: every tile reads all of its columns' partial maxima
// (2048 x 14336 bf16: 10 chunks 28.8 us, 32 chunks 30.7 us; 4096 x 11008: 12 and 32 alike)
int64_t col_chunks(int64_t rows, int64_t cols) {
    const int64_t tiles = (cols + TILE - 1) / TILE, want = (1024 + tiles - 1) / tiles, most = (rows + 63) / 64;
    const int64_t n = want < most ? want : most;
    return n < MAX_CHUNKS ? n : MAX_CHUNKS;
}

// partial[chunk][col] = largest |v| of the chunk's rows (fp32 bits)
template <bool BF16, bool MUL, bool ALIGNED>
__global__ __launch_bounds__(256) void col_max_kernel(const char* __restrict__ src, int64_t rows, int64_t cols,
                                                      int64_t ld, const float* __restrict__ mul, int64_t chunk_rows,
                                                      uint32_t* __restrict__ partial) {
    __shared__ uint32_t red[16][TILE];
    constexpr int BATCH = 8;   // rows requested at once; past the chunk's last the last again
    const int cl = threadIdx.x & 15, rl = threadIdx.x >> 4;
    const int64_t c0 = (int64_t)blockIdx.x * TILE, c = c0 + cl * 8;
    const int64_t r0 = (int64_t)blockIdx.y * chunk_rows, r1 = min(rows, r0 + chunk_rows);
    uint32_t m[8];
#pragma unroll
    for (int i = 0; i < 8; i++) m[i] = 0;
    const bool ends = c < cols && c + 8 > cols;   // the row ends among this thread's columns
    auto scan = [&](auto pieces) {
        for (int64_t r = r0 + rl; r < r1; r += 16 * BATCH) {
            Raw<BF16> raw[BATCH];
            float f[BATCH];
#pragma unroll
            for (int u = 0; u < BATCH; u++) {
                const int64_t at = min(r + 16 * u, r1 - 1);
                raw[u] = load_columns<BF16, decltype(pieces)::value, false>(src + at * ld * (BF16 ? 2 : 4), c, cols);
                f[u] = MUL ? mul[at] : 1.f;
            }
            if (decltype(pieces)::value && ends)
#pragma unroll
                for (int u = 0; u < BATCH; u++)
                    raw[u] = load_columns<BF16, false, false>(src + min(r + 16 * u, r1 - 1) * ld * (BF16 ? 2 : 4), c, cols);
#pragma unroll
            for (int u = 0; u < BATCH; u++) {
                float v[8];
                raw[u].unpack(v);
#pragma unroll
                for (int i = 0; i < 8; i++) m[i] = max(m[i], __float_as_uint(MUL ? v[i] * f[u] : v[i]) & 0x7FFFFFFFu);
            }
        }
    };
    if (ALIGNED && cols >= 8) scan(std::true_type{});
    else scan(std::false_type{});
#pragma unroll
    for (int i = 0; i < 8; i++) red[rl][cl * 8 + i] = m[i];
    __syncthreads();
    const int64_t col = c0 + threadIdx.x;
    if (threadIdx.x < TILE && col < cols) {
        uint32_t x = 0;
#pragma unroll
        for (int k = 0; k < 16; k++) x = max(x, red[k][threadIdx.x]);
        partial[(int64_t)blockIdx.y * cols + col] = x;
    }
}

// A tile of 128 rows x 128 columns: a thread quantizes 4 rows x 8 columns twice from its registers, words of 4 codes of
// one column go to LDS (16-byte pieces of a column's 128 bytes XOR-swizzled by the column's group of 8, so that the
// 16 lanes of a row segment spread over the banks), and leave as 16-byte pieces of code rows.  (Turning the values in
// LDS before they are quantized takes 53 KB, so three workgroups a unit: 37 us on 4096 x 11008 bf16, this form 29 then
// and 24 now.)
// ONCE > 0: up to 128 ONCE rows in one launch, 256 threads for each 128 of them, which find the columns' maxima in LDS.
template <bool BF16, bool MUL, bool ALIGNED, int ONCE>
__global__ __launch_bounds__(ONCE > 0 ? 256 * ONCE : 256) void cols_kernel(const char* __restrict__ src, int64_t rows, int64_t cols, int64_t ld,
                                                   const float* __restrict__ mul, const uint32_t* __restrict__ partial,
                                                   int chunks, int8_t* __restrict__ codes, int64_t ldq,
                                                   float* __restrict__ scales) {
    constexpr int TILES = ONCE > 0 ? ONCE : 1;
    __shared__ uint32_t top[ONCE > 0 ? 4 * ONCE : 2][TILE];
    __shared__ __attribute__((aligned(16))) float4 line[TILE];   // s, 1 / s, pre, zero
    __shared__ __attribute__((aligned(16))) uint32_t tiles[TILES][TILE * TILE / 4];
    const int tid = threadIdx.x & 255, block = ONCE > 0 ? threadIdx.x >> 8 : (int)blockIdx.y;
    uint32_t* tile = tiles[ONCE > 0 ? block : 0];
    const int64_t c0 = (int64_t)blockIdx.x * TILE, r0 = (int64_t)block * TILE;
    uint32_t part[MAX_CHUNKS / 2];   // every other chunk; past the last one it again
    if (ONCE == 0) {
        const int64_t col = min(c0 + (tid & 127), cols - 1);
#pragma unroll
        for (int k = 0; k < MAX_CHUNKS / 2; k++)
            if (2 * k < chunks) part[k] = partial[(int64_t)min(2 * k + (tid >> 7), chunks - 1) * cols + col];
    }
    const int cl = tid & 15, rl = tid >> 4;
    const int64_t c = c0 + cl * 8;
    Raw<BF16> raw[8];
    float f[8];
    auto load = [&](auto pieces) {
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const int64_t r = min(r0 + (i >> 2) * 64 + rl * 4 + (i & 3), rows - 1);
            raw[i] = load_columns<BF16, decltype(pieces)::value, true>(src + r * ld * (BF16 ? 2 : 4), c, cols);
            f[i] = MUL ? mul[r] : 1.f;
        }
    };
    if (!ALIGNED || cols < 8) load(std::false_type{});
    else load(std::true_type{});
    if (ALIGNED && cols >= 8 && c < cols && c + 8 > cols) load(std::false_type{});   // the row ends among these eight
    if (ONCE > 0) {   // rows past the last one repeat it
        uint32_t m[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < 8; i++) {
            float x[8];
            raw[i].unpack(x);
#pragma unroll
            for (int j = 0; j < 8; j++) m[j] = max(m[j], __float_as_uint(MUL ? x[j] * f[i] : x[j]) & 0x7FFFFFFFu);
        }
#pragma unroll
        for (int j = 0; j < 8; j++) {   // over the wave's four row groups
            m[j] = max(m[j], (uint32_t)__shfl_xor((int)m[j], 16));
            m[j] = max(m[j], (uint32_t)__shfl_xor((int)m[j], 32));
            if ((tid & 63) < 16) top[threadIdx.x >> 6][cl * 8 + j] = m[j];
        }
    } else {
        uint32_t m = 0;
#pragma unroll
        for (int k = 0; k < MAX_CHUNKS / 2; k++)
            if (2 * k < chunks) m = max(m, part[k]);
        top[tid >> 7][tid & 127] = m;
    }
    __syncthreads();
    if (threadIdx.x < TILE) {
        uint32_t m = top[0][tid];
#pragma unroll
        for (int k = 1; k < (ONCE > 0 ? 4 * ONCE : 2); k++) m = max(m, top[k][tid]);
        const Line l = make_line(m);
        line[tid] = make_float4(l.s, l.inv, l.pre, l.zero ? 1.f : 0.f);
        if (r0 == 0 && c0 + tid < cols) scales[c0 + tid] = l.out;
    }
    float v[2][4][8];
#pragma unroll
    for (int i = 0; i < 8; i++) {
        raw[i].unpack(v[i >> 2][i & 3]);
        if (MUL)
#pragma unroll
            for (int j = 0; j < 8; j++) v[i >> 2][i & 3][j] *= f[i];
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 8; j++) {
        const float4 q = line[cl * 8 + j];
        Line l;
        l.s = q.x, l.inv = q.y, l.pre = q.z, l.zero = q.w != 0.f, l.half = 0.5f * q.x;
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; i++) x[i] = v[i >> 2][i & 3][j];
        const uint2 w = __any(l.pre != 1.f) ? quant8<true>(x, l) : quant8<false>(x, l);
        // word of rows 4 rl .. (first half: piece rl / 4; second: 4 + rl / 4)
        uint32_t* t = tile + (cl * 8 + j) * 32;
        t[(((rl >> 2) ^ (cl & 7)) << 2) + (rl & 3)] = w.x;
        t[(((4 + (rl >> 2)) ^ (cl & 7)) << 2) + (rl & 3)] = w.y;
    }
    __syncthreads();
    // 128 columns x 8 pieces of 16 codes
#pragma unroll
    for (int k = 0; k < 4; k++) {
        const int e = tid + k * 256, col = e >> 3, piece = e & 7;
        const int64_t r = r0 + piece * 16;
        if (c0 + col >= cols || r >= rows) continue;
        const uint4 w = *reinterpret_cast<const uint4*>(tile + col * 32 + ((piece ^ ((col >> 3) & 7)) << 2));
        int8_t* q = codes + (c0 + col) * ldq + r;
        if (r + 16 <= rows) {
            *reinterpret_cast<uint4*>(q) = w;
        } else {
            const uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int i = 0; i < 16; i++)
                if (r + i < rows) q[i] = (int8_t)(x[i >> 2] >> (8 * (i & 3)));
        }
    }
}

template <bool BF16, bool MUL, bool ALIGNED>
hipError_t launch_cols(const void* src, int64_t rows, int64_t cols, int64_t ld, const float* mul, int8_t* codes,
                       int64_t ldq, float* scales, void* ws, hipStream_t s) {
    const char* p = static_cast<const char*>(src);
    uint32_t* partial = static_cast<uint32_t*>(ws);
    const int64_t chunks = col_chunks(rows, cols), chunk_rows = (rows + chunks - 1) / chunks;
    const unsigned ct = (unsigned)((cols + TILE - 1) / TILE);
    // few rows: one launch, the source read once (64 x 4096 bf16 9.0 -> 6.6 us, 200 x 14336 fp32 10.2 -> 8.3; with 512 rows
    // in a workgroup 512 x 14336 fp32 takes 14.4 instead of 11.8)
    if (rows <= 2 * TILE) {
        if (rows <= TILE)
            cols_kernel<BF16, MUL, ALIGNED, 1><<<ct, 256, 0, s>>>(p, rows, cols, ld, mul, nullptr, 0, codes, ldq, scales);
        else
            cols_kernel<BF16, MUL, ALIGNED, 2><<<ct, 512, 0, s>>>(p, rows, cols, ld, mul, nullptr, 0, codes, ldq, scales);
        return hipGetLastError();
    }
    col_max_kernel<BF16, MUL, ALIGNED><<<dim3(ct, (unsigned)chunks), 256, 0, s>>>(p, rows, cols, ld, mul, chunk_rows,
                                                                                partial);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    cols_kernel<BF16, MUL, ALIGNED, 0><<<dim3(ct, (unsigned)((rows + TILE - 1) / TILE)), 256, 0, s>>>(
        p, rows, cols, ld, mul, partial, (int)chunks, codes, ldq, scales);
    return hipGetLastError();
}

// ---------------------------------------------------------------- reconstruction

// four codes a thread and round; a workgroup takes `per` whole rows (rows of up to 2048) or a segment of 4096 of
// one.  A thread requests its four rounds before it writes the first, by streaming stores: 8192 x 14336 to fp32
// 144 -> 85 us (6.9 TB/s; to bf16 52 us, 6.7 TB/s)
constexpr int SEG = 4096;

template <bool BF16>
__device__ __forceinline__ void restore4(uint32_t w, float s, char* d, int64_t left) {
    float x[4];
#pragma unroll
    for (int j = 0; j < 4; j++) x[j] = (float)(int8_t)(w >> (8 * j)) * s;
    if (left >= 4) {
        if (BF16) st8<true>(reinterpret_cast<uint8_t*>(d), pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]));
        else st16<true>(d, __float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
    } else {
        for (int j = 0; j < left; j++) {
            if (BF16) reinterpret_cast<uint16_t*>(d)[j] = (uint16_t)pack_bf16(x[j], x[j]);
            else reinterpret_cast<float*>(d)[j] = x[j];
        }
    }
}

template <bool BF16>
__global__ __launch_bounds__(256) void dequantize_kernel(const int8_t* __restrict__ codes, int64_t ldq,
                                                         const float* __restrict__ scales, int64_t outer, int64_t k,
                                                         char* __restrict__ dst, int64_t ld, int per, Div32 dcols,
                                                         int width) {
    const int64_t row0 = (int64_t)blockIdx.x * per, c0 = (int64_t)blockIdx.y * SEG;
    const int quads = (int)((min((int64_t)width, k - c0) + 3) >> 2);
    const int total = quads * (int)min((int64_t)per, outer - row0);
    for (int i0 = threadIdx.x; i0 < total; i0 += 1024) {
        uint32_t w[4];
        float s[4];
        int r[4];
#pragma unroll
        for (int u = 0; u < 4; u++) {
            const int i = i0 + 256 * u;
            r[u] = per > 1 ? (int)div32((uint32_t)i, dcols) : 0;
            w[u] = 0;
            s[u] = 0.f;
            if (i < total) {
                w[u] = *reinterpret_cast<const uint32_t*>(codes + (row0 + r[u]) * ldq + c0 + 4 * (int64_t)(i - r[u] * quads));
                s[u] = scales[row0 + r[u]];
            }
        }
#pragma unroll
        for (int u = 0; u < 4; u++) {
            const int i = i0 + 256 * u;
            const int64_t c = c0 + 4 * (int64_t)(i - r[u] * quads);
            if (i < total) restore4<BF16>(w[u], s[u], dst + ((row0 + r[u]) * ld + c) * (BF16 ? 2 : 4), k - c);
        }
    }
}

}  // namespace

int64_t quantize_workspace_bytes(int64_t rows, int64_t cols, int axis) {
    return axis == 1 ? 0 : col_chunks(rows, cols) * cols * 4;
}

hipError_t launch_quantize(const void* src, int dtype, int64_t rows, int64_t cols, int64_t ld, int axis,
                           const float* mul, int8_t* codes, int64_t ldq, float* scales, void* ws, hipStream_t s) {
    const bool bf16 = dtype == 1;
    const int64_t es = bf16 ? 2 : 4, lines = axis == 1 ? rows : cols;
    const bool al = reinterpret_cast<uintptr_t>(src) % 16 == 0 && (ld * es) % 16 == 0;
    hipError_t e = hipSuccess;
    for (int64_t l = 0; l < lines && e == hipSuccess; l += PART) {
        const int64_t n = lines - l < PART ? lines - l : PART;
        const char* p = static_cast<const char*>(src) + (axis == 1 ? l * ld : l) * es;
#define CFINT8_ROWS(B, M) launch_rows<B, M>(p, n, cols, ld, mul, codes + l * ldq, ldq, scales + l, s)
#define CFINT8_COLS(B, M, A) launch_cols<B, M, A>(p, rows, n, ld, mul, codes + l * ldq, ldq, scales + l, ws, s)
        if (axis == 1) {
            if (bf16) e = mul ? CFINT8_ROWS(true, true) : CFINT8_ROWS(true, false);
            else e = mul ? CFINT8_ROWS(false, true) : CFINT8_ROWS(false, false);
        } else if (bf16) {
            if (mul) e = al ? CFINT8_COLS(true, true, true) : CFINT8_COLS(true, true, false);
            else e = al ? CFINT8_COLS(true, false, true) : CFINT8_COLS(true, false, false);
        } else {
            if (mul) e = al ? CFINT8_COLS(false, true, true) : CFINT8_COLS(false, true, false);
            else e = al ? CFINT8_COLS(false, false, true) : CFINT8_COLS(false, false, false);
        }
#undef CFINT8_ROWS
#undef CFINT8_COLS
    }
    return e;
}

hipError_t launch_dequantize(const int8_t* codes, int64_t ldq, const float* scales, int64_t outer, int64_t k, void* dst,
                             int dtype, int64_t ld, hipStream_t s) {
    const int width = (int)(k < SEG ? k : SEG);
    const int per = k >= SEG ? 1 : (int)(SEG / k > 64 ? 64 : SEG / k);
    const Div32 d = make_div32((uint32_t)((width + 3) / 4));
    hipError_t e = hipSuccess;
    for (int64_t l = 0; l < outer && e == hipSuccess; l += PART) {
        const int64_t n = outer - l < PART ? outer - l : PART;
        const dim3 grid((unsigned)((n + per - 1) / per), (unsigned)((k + SEG - 1) / SEG));
        const int8_t* q = codes + l * ldq;
        char* p = static_cast<char*>(dst) + l * ld * (dtype == 1 ? 2 : 4);
        if (dtype == 1) dequantize_kernel<true><<<grid, 256, 0, s>>>(q, ldq, scales + l, n, k, p, ld, per, d, width);
        else dequantize_kernel<false><<<grid, 256, 0, s>>>(q, ldq, scales + l, n, k, p, ld, per, d, width);
        e = hipGetLastError();
    }
    return e;
}

}  // namespace cfint8
