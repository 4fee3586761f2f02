// Mixture-of-experts layer for a few tokens with 8-bit weights.
//
// A few tokens against many weights: every taken expert's codes are read once, so the layer is bound by
// memory, and the codes go from memory to the matrix cores as they are.  The other operand of
// v_mfma_i32_16x16x64_i8 is the activation in fixed point: a row's values as integers of 22 bits (bf16) or
// 30 bits (fp32) below a power of two above its largest, split into 3 or 4 signed base-256 digits, one
// product for each digit.  All sums of products are exact int32; the digits' sums meet in fp32.  What lies 2^23 below a
// row's largest is lost to bf16 calls, whose results are rounded to 2^-9: a fourth digit there takes 64 tokens over 128
// experts from 164 to 173 us, one token from 17.2 to 18.5, 8 tokens over 88 experts from 24.5 to 34.8.
//
//   router   logits in 64 bits (they decide, so they are right to the last bit); x into digits
// and, where the tokens' experts are mostly different ones (one token above all),
//   gate_up_one  a workgroup for each (slot, 32 inner columns): ranks the token's logits itself, then dot products of
//                whole rows; h as digits with a power of two for each such slice
//   down_one     a workgroup for each (token, 8 output columns), all its slots
// or else, each expert's codes read once for all its rows,
//   topk     a workgroup for each token: ids and weights
//   gate_up  a workgroup for each (expert, 64 inner columns): h, as digits with a power of two for each 64 of a row
//            (so that no workgroup waits for a whole row's largest value)
//   down     a workgroup for each (expert, 128 output columns): weighted partial rows, one for each slot
//   combine  a token's slots added in order
#include "../../include/cfint8.h"
#include "int8_internal.hpp"
#include "int8_lanes.hpp"
#include "int8_routes.hpp"

namespace cfint8 {

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr int POISON = INT16_MIN;      // exponent of values among which is a NaN or an infinity
constexpr int ROWS = 16;               // token rows of a matrix product
constexpr int UP_COLS = 64;            // inner columns of a gate_up workgroup: h's columns of one exponent
constexpr int DOWN_COLS = 128;         // output columns of a down workgroup
constexpr int WAVES = 4;               // of either

// workspace
struct Layout {
    int64_t logits, xd, xe, hd, he, part, bytes;
};

// exponents of a row of h: one for each 64 columns, an even number
__host__ __device__ constexpr int64_t exponents(int64_t I) { return (I + 2 * UP_COLS - 1) / (2 * UP_COLS) * 2; }

// waves of a gate_up workgroup of the slot path, four inner columns each, which share an exponent there
__host__ __device__ constexpr int one_waves(int P) { return P == 4 ? 4 : 8; }
__host__ __device__ constexpr int64_t one_exponents(int64_t I, int P) { return (I + 4 * one_waves(P) - 1) / (4 * one_waves(P)); }

Layout layout(int64_t T, int64_t E, int64_t topk, int64_t H, int64_t I) {
    Layout l;
    int64_t at = 0;
    auto take = [&](int64_t n) {
        const int64_t r = at;
        at += (n + 255) & ~(int64_t)255;
        return r;
    };
    const int64_t S = T * topk;
    l.logits = take(T * E * 4);
    l.xd = take(T * 4 * H);
    l.xe = take(T * 4);
    l.hd = take(S * 4 * I);
    l.he = take(S * (one_exponents(I, 4) + 2) * 2);   // enough for exponents() too
    l.part = take(S * H * 4);
    l.bytes = at;
    return l;
}

__device__ __forceinline__ float bf16_to_f(uint32_t h) { return __uint_as_float(h << 16); }

__device__ __forceinline__ uint32_t to_bf16(float f) {   // nearest even; NaN stays one
    uint32_t u = __float_as_uint(f);
    if ((u & 0x7FFFFFFFu) > 0x7F800000u) return 0x7FC0u;
    u += 0x7FFFu + ((u >> 16) & 1u);
    return u >> 16;
}

template <bool BF16>
__device__ __forceinline__ void load8(const char* p, int64_t c, float* v) {
    const uint4* q = reinterpret_cast<const uint4*>(p + c * (BF16 ? 2 : 4));
    if (BF16) {
        const uint4 u = q[0];
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; i++) {
            v[2 * i] = bf16_to_f(w[i] & 0xFFFFu);
            v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        }
    } else {
        const uint4 a = q[0], b = q[1];
        const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
        for (int i = 0; i < 8; i++) v[i] = __uint_as_float(w[i]);
    }
}

// exponent e of a row with largest magnitude bits m: values times 2^-e are below 2^22 (3 digits) or 2^30 (4)
template <int P>
__device__ __forceinline__ int digit_exponent(uint32_t m) {
    if (m >= 0x7F800000u) return POISON;
    return __builtin_amdgcn_frexp_expf(__uint_as_float(m)) - (P == 4 ? 30 : 22);
}

// signed digits of a value, digit p in byte p
__device__ __forceinline__ uint32_t digits_of(float v, int e) {
    const int n = e == POISON ? 0 : (int)__builtin_rintf(__builtin_amdgcn_ldexpf(v, -e));
    return ((uint32_t)n + 0x00808080u) ^ 0x00808080u;
}

// digits of 8 values, byte i of out[p] digit p of value i
template <int P>
__device__ __forceinline__ void digits8(const float* v, int e, uint2* out) {
    uint32_t q[8];
#pragma unroll
    for (int i = 0; i < 8; i++) q[i] = digits_of(v[i], e);
#pragma unroll
    for (int p = 0; p < P; p++) {
        uint32_t w[2] = {0, 0};
#pragma unroll
        for (int i = 0; i < 8; i++) w[i >> 2] |= ((q[i] >> (8 * p)) & 0xFFu) << (8 * (i & 3));
        out[p] = make_uint2(w[0], w[1]);
    }
}

__device__ __forceinline__ uint32_t wave_max(uint32_t m) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o));
    return m;
}

__device__ __forceinline__ uint32_t max8(uint32_t m, const float* v) {
#pragma unroll
    for (int i = 0; i < 8; i++) m = max(m, __float_as_uint(v[i]) & 0x7FFFFFFFu);
    return m;
}

template <int P>
__device__ __forceinline__ void put_digits(const float* v, int e, int8_t* dst, int n, int c) {
    uint2 d[P];
    digits8<P>(v, e, d);
#pragma unroll
    for (int p = 0; p < P; p++) *reinterpret_cast<uint2*>(dst + (int64_t)p * n + c) = d[p];
}

// workgroups [0, T): a token's x into digits; then one for each (expert, N tokens), its waves sharing H
template <bool BF16, int P, int N>
__global__ __launch_bounds__(256) void router_kernel(MoeArgs a, int8_t* __restrict__ xd, int* __restrict__ xe,
                                                     float* __restrict__ logits) {
    __shared__ uint32_t top[4];
    __shared__ double part[4][N];
    const int T = (int)a.T, E = (int)a.E, H = (int)a.H, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t es = BF16 ? 2 : 4;
    int b = blockIdx.x;
    if (b < T) {
        const char* src = static_cast<const char*>(a.x) + b * a.ldx * es;
        int8_t* dst = xd + (int64_t)b * P * H;
        uint32_t m = 0;
        for (int c = threadIdx.x * 8; c < H; c += 2048) {
            float v[8];
            load8<BF16>(src, c, v);
            m = max8(m, v);
        }
        m = wave_max(m);
        if (lane == 0) top[wave] = m;
        __syncthreads();
        const int e = digit_exponent<P>(max(max(top[0], top[1]), max(top[2], top[3])));
        for (int c = threadIdx.x * 8; c < H; c += 2048) {
            float v[8];
            load8<BF16>(src, c, v);
            put_digits<P>(v, e, dst, H, c);
        }
        if (threadIdx.x == 0) xe[b] = e;
        return;
    }
    b -= T;
    const int e = b % E, t0 = (b / E) * N, n = min(N, T - t0);
    double s[N] = {};
    const char* r = static_cast<const char*>(a.router) + (int64_t)e * H * es;
    const char* x = static_cast<const char*>(a.x) + t0 * a.ldx * es;
#pragma unroll 2
    for (int c = threadIdx.x * 8; c < H; c += 2048) {
        float w[8];
        load8<BF16>(r, c, w);
#pragma unroll
        for (int t = 0; t < N; t++) {
            float v[8];
            load8<BF16>(x + (t < n ? t : 0) * a.ldx * es, c, v);
#pragma unroll
            for (int i = 0; i < 8; i++) s[t] = __builtin_fma((double)v[i], (double)w[i], s[t]);
        }
    }
    const double sum = N == 4 ? sum4(s[0], s[N == 4 ? 1 : 0], s[N == 4 ? 2 : 0], s[N == 4 ? 3 : 0]) : sum1(s[0]);
    if ((lane & 15) == 0) {
        if (N == 4) part[wave][value_of_row(lane >> 4) % N] = sum;
        else if (lane == 0) part[wave][0] = sum;
    }
    __syncthreads();
    const int t = threadIdx.x;
    if (t < n) logits[(int64_t)(t0 + t) * E + e] = (float)(((part[0][t] + part[1][t]) + part[2][t]) + part[3][t]);
}

// orders logits: NaN below everything, -0 as 0
__device__ __forceinline__ uint32_t order_key(float l) {
    if (l != l) return 0;
    const uint32_t u = __float_as_uint(l + 0.f);
    return u ^ ((u >> 31) ? 0xFFFFFFFFu : 0x80000000u);
}

// how many of a token's experts come before e: larger keys, and equal ones of lower index; keys has E of them, padded
// with zeros to a multiple of 4
__device__ __forceinline__ int rank_of(const uint32_t* keys, int E, int e) {
    const uint32_t k = keys[e];
    int r = 0;
    for (int j = 0; j < E; j += 4) {
        const uint4 q = *reinterpret_cast<const uint4*>(keys + j);
        r += (q.x > k || (q.x == k && j < e)) + (q.y > k || (q.y == k && j + 1 < e)) +
             (q.z > k || (q.z == k && j + 2 < e)) + (q.w > k || (q.w == k && j + 3 < e));
    }
    // the padding's zeros tie with NaN's key only, at indexes past every e
    return r;
}

// ids and weights of token t by N threads (a multiple of 64), its logits' keys in LDS; red has N / 64 + 1 floats
template <int N>
__device__ __forceinline__ void take_topk(const MoeArgs& a, int t, const float* __restrict__ logits,
                                          const uint32_t* keys, float* red) {
    const int E = (int)a.E, k = (int)a.topk, tid = threadIdx.x;
    int32_t* ids = a.ids + (int64_t)t * k;
    float* weights = a.weights + (int64_t)t * k;
    if (a.active && !a.active[t]) {
        for (int j = tid; j < k; j += N) {
            ids[j] = -1;
            weights[j] = 0.f;
        }
        return;
    }
    constexpr int PER = (1024 + N - 1) / N;
    int rank[PER];
#pragma unroll
    for (int i = 0; i < PER; i++) {
        const int e = tid + N * i;
        rank[i] = e < E ? rank_of(keys, E, e) : 1024;
        if (rank[i] == 0) red[0] = logits[(int64_t)t * E + e];
    }
    __syncthreads();
    const float lead = red[0];
    float sum = 0.f, w[PER];
#pragma unroll
    for (int i = 0; i < PER; i++) {
        const int e = tid + N * i;
        w[i] = e < E ? expf(logits[(int64_t)t * E + e] - lead) : 0.f;
        if (!a.renorm || rank[i] < k) sum += w[i];
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
    if ((tid & 63) == 0) red[1 + (tid >> 6)] = sum;
    __syncthreads();
    sum = 0.f;
    for (int i = 0; i < N / 64; i++) sum += red[1 + i];
#pragma unroll
    for (int i = 0; i < PER; i++)
        if (rank[i] < k) {
            ids[rank[i]] = tid + N * i;
            weights[rank[i]] = w[i] / sum;
        }
}

__global__ __launch_bounds__(256) void topk_kernel(MoeArgs a, const float* __restrict__ logits) {
    __shared__ __attribute__((aligned(16))) uint32_t keys[1024];
    __shared__ float red[5];
    const int t = blockIdx.x, E = (int)a.E;
    for (int e = threadIdx.x; e < (E + 3) / 4 * 4; e += 256) keys[e] = e < E ? order_key(logits[(int64_t)t * E + e]) : 0;
    __syncthreads();
    take_topk<256>(a, t, logits, keys, red);
}

// An expert's slots, ascending (an expert is taken at most once by each token), found from ids by every wave for
// itself: no barrier stands between a workgroup's start and its loads.  Returns their number
__device__ __forceinline__ int find_rows(const int32_t* __restrict__ ids, int slots, int e, uint16_t* list) {
    const int lane = threadIdx.x & 63;
    int n = 0;
    for (int s0 = 0; s0 < slots; s0 += 512) {
        int32_t id[8];
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const int s = s0 + 64 * i + lane;
            id[i] = s < slots ? ids[s] : -1;
        }
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const uint64_t b = __ballot(id[i] == e);
            if (id[i] == e) list[n + __popcll(b & ((1ull << lane) - 1))] = (uint16_t)(s0 + 64 * i + lane);
            n += __popcll(b);
        }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    return n;
}

// Which expert a workgroup's first index i stands for: expert i itself where the experts are fewer than the
// slots, else slot i's expert (its rows then begin with slot i, or another index has them); -1 for none
__device__ __forceinline__ int expert_of(const int32_t* __restrict__ ids, int i, int slots, int E) {
    if (E <= slots) return i;
    return ids[i];
}

// Products of 16 rows x 16 NT columns over one of SHARES shares of K, in blocks of 128; use(row digits' fragments,
// codes' fragments, exponents) takes them half a block at a time.  Codes go through LDS: loads of
// 16 lines a quarter of a wave cost the L1 a lookup for each, 64 a kilobyte, copies of whole 128-byte pieces of
// lines 16.  A wave has two slots of its own and copies the next block while it uses this one; the few rows of
// digits come straight to registers, a block ahead as well.
constexpr int TILE = 16 * 128;   // bytes of a tile's block

// line r's 16-byte pieces lie XOR-swizzled by r / 2: 16 lanes that read a piece of 16 lines then cover the 64 banks
__device__ __forceinline__ int swizzle(int row) { return (row >> 1) & 7; }

// codes of up to 16 lines of K bytes, `lines` of them in the matrix
struct Lines {
    const int8_t* p;
    int lines;
};

// The codes come by streaming copies (64 tokens over 128 experts 185 -> 170 us).
// digits: row_offset is where this lane's row (l % 16) begins, or NONE.  EXPS: exponents too, one for each half block
// of a row: exp_offset[v] is where those of row 4 (l / 16) + v begin, or NONE.
constexpr int NONE = 0x40000000;   // past every buffer's end, and so is what is added to it: reads zeros

template <int P, int NT, int SHARES, bool EXPS, class Use>
__device__ __forceinline__ void stream(const int8_t* digits, int digits_bytes, int row_offset, const int16_t* exps,
                                       int exps_bytes, const int (&exp_offset)[4], const Lines (&b)[NT], int K, int share,
                                       char* ring0, char* ring1, Use use) {
    constexpr int SLOT = NT * TILE, LOADS = 2 * NT + 2 * P + (EXPS ? 4 : 0);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lr = lane & 15;
    const int nkb = (K + 127) / 128, mine = (nkb - share + SHARES - 1) / SHARES;
    using lds_ptr = __attribute__((address_space(3))) void*;
    const __amdgpu_buffer_rsrc_t ra = __builtin_amdgcn_make_buffer_rsrc((void*)digits, (short)0, digits_bytes, 0x00020000);
    const __amdgpu_buffer_rsrc_t re = __builtin_amdgcn_make_buffer_rsrc((void*)exps, (short)0, exps_bytes, 0x00020000);
    i32x4 fa[2][2][P];
    int fe[2][4];
    // requests this wave's j-th block; every call issues LOADS loads, past the last block they read nothing
    auto request = [&](int j, char* ring, i32x4 (&f)[2][P], int (&x)[4]) __attribute__((always_inline)) {
        const int k = (share + j * SHARES) * 128;
        const bool in = j < mine;
        int at[2];   // the piece that belongs where this lane writes, of a tile's first and second eight lines
#pragma unroll
        for (int i = 0; i < 2; i++) {
            at[i] = 16 * ((lane & 7) ^ swizzle(8 * i + (lane >> 3)));
            at[i] = k + at[i] < K ? (8 * i + (lane >> 3)) * K + at[i] : NONE;
        }
#pragma unroll
        for (int t = 0; t < NT; t++) {
            const __amdgpu_buffer_rsrc_t rb = __builtin_amdgcn_make_buffer_rsrc(
                (void*)(b[t].p + (in ? k : 0)), (short)0, in ? max(b[t].lines * K - k, 0) : 0, 0x00020000);
#pragma unroll
            for (int i = 0; i < 2; i++)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rb, (lds_ptr)(ring + wave * SLOT + t * TILE + i * 1024), 16,
                                                         at[i], 0, 0, 2);
        }
#pragma unroll
        for (int s = 0; s < 2; s++) {
            const int ks = k + 64 * s + 16 * (lane >> 4);
            const int off = (ks < K ? row_offset : NONE) + ks;
#pragma unroll
            for (int p = 0; p < P; p++)
                f[s][p] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(ra, off + p * K, 0, 0));
        }
        if (EXPS) {
            const int at_k = in ? k / 32 : NONE / 2;
#pragma unroll
            for (int v = 0; v < 4; v++) x[v] = (int)__builtin_amdgcn_raw_buffer_load_b32(re, exp_offset[v] + at_k, 0, 0);
        }
    };
    // a block has landed once only the next one's loads are out; s_waitcnt's vmcnt sits in bits 3:0 and 15:14
    static_assert(LOADS < 64, "vmcnt holds 6 bits");
    constexpr int WAIT = 0x0F70 | (LOADS & 15) | ((LOADS >> 4) << 14);
    auto step = [&](int j, char* now, char* next, i32x4 (&f)[2][P], i32x4 (&g)[2][P], int (&x)[4],
                    int (&y)[4]) __attribute__((always_inline)) {
        __builtin_amdgcn_s_waitcnt(0xC07F);   // the next slot's reads, a step old, are done
        request(j + 1, next, g, y);
        __builtin_amdgcn_s_waitcnt(WAIT);
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
        for (int s = 0; s < 2; s++) {
            i32x4 fb[NT];
            const char* st = now + wave * SLOT + lr * 128 + 16 * ((4 * s + (lane >> 4)) ^ swizzle(lr));
#pragma unroll
            for (int t = 0; t < NT; t++) fb[t] = *reinterpret_cast<const i32x4*>(st + t * TILE);
            int ex[4];
#pragma unroll
            for (int v = 0; v < 4; v++)   // a half block behind K has none: it was never written
                ex[v] = !EXPS || 128 * (share + j * SHARES) + 64 * s >= K ? 0 : s ? x[v] >> 16 : (int16_t)x[v];
            use(f[s], fb, ex);
        }
    };
    request(0, ring0, fa[0], fe[0]);
    for (int j = 0; j < mine; j += 2) {
        step(j, ring0, ring1, fa[0], fa[1], fe[0], fe[1]);
        step(j + 1, ring1, ring0, fa[1], fa[0], fe[1], fe[0]);
    }
    __builtin_amdgcn_s_waitcnt(0x0070);   // no copy and no read is left in flight: the sums take the first slot
}

// element v of a lane's sums with the digits joined
template <int P, int NT>
__device__ __forceinline__ float join(const i32x4 (&acc)[P][NT], int t, int v) {
    float f = (float)acc[P - 1][t][v];
#pragma unroll
    for (int p = P - 2; p >= 0; p--) f = __builtin_fmaf(f, 256.f, (float)acc[p][t][v]);
    return f;
}

// the waves' sums into their first slots: [t][lane], element v of lane l is row 4 (l / 16) + v of column l % 16
template <int NT>
__device__ __forceinline__ void share_sums(const float (&f)[NT][4], char* ring0) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int t = 0; t < NT; t++)
        *reinterpret_cast<float4*>(ring0 + wave * NT * TILE + t * 1024 + 16 * lane) =
            make_float4(f[t][0], f[t][1], f[t][2], f[t][3]);
    __syncthreads();
}

// rows 4 q .. 4 q + 3 of column c of tile t, over the waves that share these columns (every other one from `half`)
template <int NT>
__device__ __forceinline__ void shared_sum(const char* ring0, int half, int t, int q, int c, float (&out)[4]) {
    const char* at = ring0 + t * 1024 + 16 * (16 * q + c);
    float4 s = *reinterpret_cast<const float4*>(at + half * NT * TILE);
#pragma unroll
    for (int w = 2; w < WAVES; w += 2) {
        const float4 v = *reinterpret_cast<const float4*>(at + (half + w) * NT * TILE);
        s.x += v.x;
        s.y += v.y;
        s.z += v.z;
        s.w += v.w;
    }
    out[0] = s.x, out[1] = s.y, out[2] = s.z, out[3] = s.w;
}

// A scale's significand multiplies where its exponent was added before, so that only g, u and y can leave fp32's range,
// not a sum that its scale would have brought back
__device__ __forceinline__ int exponent_of(float s) { return __builtin_amdgcn_frexp_expf(s); }
__device__ __forceinline__ float significand_of(float s) { return __builtin_amdgcn_frexp_mantf(s); }

// f 2^(e + more); NaN where e says so
__device__ __forceinline__ float scaled_by(float f, int e, int more) {
    return e == POISON ? __uint_as_float(0x7FC00000u) : __builtin_amdgcn_ldexpf(f, e + more);
}
__device__ __forceinline__ float row_scaled(float f, int e, float s) {
    return scaled_by(f * significand_of(s), e, exponent_of(s));
}

// Waves of even number take the first 32 columns, the others the last
template <int P>
__global__ __launch_bounds__(64 * WAVES, 2) void gate_up_kernel(MoeArgs a, const int8_t* __restrict__ xd,
                                                                const int* __restrict__ xe, int8_t* __restrict__ hd,
                                                                int16_t* __restrict__ he) {
    constexpr int NT = 4;   // tiles: 2 of gate, 2 of up
    __shared__ uint16_t lists[WAVES][256];
    __shared__ __attribute__((aligned(16))) char ring0[WAVES * NT * TILE], ring1[WAVES * NT * TILE];
    const int T = (int)a.T, E = (int)a.E, k = (int)a.topk, slots = T * k, H = (int)a.H, I = (int)a.I;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int nsl = (I + UP_COLS - 1) / UP_COLS, index = (int)blockIdx.x / nsl;
    uint16_t* rows = lists[wave];
    const int e = expert_of(a.ids, index, slots, E);
    if (e < 0) return;
    const int n = find_rows(a.ids, slots, e, rows);
    if (n == 0 || (E > slots && rows[0] != index)) return;
    const int slice = (int)blockIdx.x % nsl, c0 = slice * UP_COLS, half = wave & 1;
    Lines b[NT];
#pragma unroll
    for (int t = 0; t < NT; t++) {
        const int c = c0 + 32 * half + 16 * (t & 1);   // columns come in sixteens: a tile is there or not
        b[t].lines = c < I ? 16 : 0;
        b[t].p = a.gu + ((int64_t)__builtin_amdgcn_readfirstlane(e) * 2 * I + c + (t >= 2 ? I : 0)) * H;
    }
    for (int r0 = 0; r0 < n; r0 += ROWS) {
        const int r = r0 + (lane & 15);
        i32x4 acc[P][NT] = {};
        const int none[4] = {NONE, NONE, NONE, NONE};
        // what the epilogue multiplies with, on its way before the codes: there a wave takes four rows, a lane a column
        const int c = c0 + lane, q = wave;
        float sg = 0.f, su = 0.f;
        int slot[4] = {}, ex[4] = {};
        if (q < 4 && r0 + 4 * q < n) {
            if (c < I) {
                const float* s = a.gus + (int64_t)e * 2 * I + c;
                sg = s[0], su = s[I];
            }
#pragma unroll
            for (int v = 0; v < 4; v++) {
                slot[v] = rows[min(r0 + 4 * q + v, n - 1)];
                ex[v] = xe[slot[v] / k];
            }
        }
        stream<P, NT, WAVES / 2, false>(
            xd, T * P * H, r < n ? rows[r] / k * P * H : NONE, nullptr, 0, none, b, H, wave >> 1, ring0, ring1,
            [&](const i32x4(&fa)[P], const i32x4(&fb)[NT], const int(&)[4]) __attribute__((always_inline)) {
#pragma unroll
                for (int t = 0; t < NT; t++)
#pragma unroll
                    for (int p = 0; p < P; p++)
                        acc[p][t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fa[p], fb[t], acc[p][t], 0, 0, 0);
            });
        float f[NT][4];
#pragma unroll
        for (int t = 0; t < NT; t++)
#pragma unroll
            for (int v = 0; v < 4; v++) f[t][v] = join<P, NT>(acc, t, v);
        share_sums<NT>(f, ring0);
        if (q < 4 && r0 + 4 * q < n) {
            float g[4], u[4];
            shared_sum<NT>(ring0, lane >> 5, (lane >> 4) & 1, q, lane & 15, g);
            shared_sum<NT>(ring0, lane >> 5, 2 + ((lane >> 4) & 1), q, lane & 15, u);
#pragma unroll
            for (int v = 0; v < 4; v++) {
                if (r0 + 4 * q + v >= n) break;
                const float gv = row_scaled(g[v], ex[v], sg), uv = row_scaled(u[v], ex[v], su);
                const float y = c < I ? gv / (1.f + expf(-gv)) * uv : 0.f;
                const int eh = digit_exponent<P>(wave_max(__float_as_uint(y) & 0x7FFFFFFFu));
                const uint32_t d = digits_of(y, eh);
                int8_t* dst = hd + (int64_t)slot[v] * P * I + c;
                if (c < I)
#pragma unroll
                    for (int p = 0; p < P; p++) dst[(int64_t)p * I] = (int8_t)(d >> (8 * p));
                if (lane == 0) he[slot[v] * exponents(I) + slice] = (int16_t)eh;
            }
        }
        __syncthreads();
    }
}

template <bool BF16>
__device__ __forceinline__ void store4(const MoeArgs& a, int t, int c, const float4& s) {
    char* y = static_cast<char*>(a.y) + (t * a.ldy + c) * (BF16 ? 2 : 4);
    if (BF16) *reinterpret_cast<uint2*>(y) = make_uint2(to_bf16(s.x) | to_bf16(s.y) << 16, to_bf16(s.z) | to_bf16(s.w) << 16);
    else *reinterpret_cast<float4*>(y) = s;
}

template <int P>
__global__ __launch_bounds__(64 * WAVES, 2) void down_kernel(MoeArgs a, const int8_t* __restrict__ hd,
                                                             const int16_t* __restrict__ he, float* __restrict__ part) {
    constexpr int NT = DOWN_COLS / 32, THREADS = 64 * WAVES;
    __shared__ uint16_t lists[WAVES][256];
    __shared__ __attribute__((aligned(16))) char ring0[WAVES * NT * TILE], ring1[WAVES * NT * TILE];
    const int k = (int)a.topk, slots = (int)a.T * k, H = (int)a.H, I = (int)a.I, E = (int)a.E;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = wave & 1;
    const int nsl = (H + DOWN_COLS - 1) / DOWN_COLS, slice = (int)blockIdx.x % nsl, c0 = slice * DOWN_COLS;
    const int index = (int)blockIdx.x / nsl, e = expert_of(a.ids, index, slots, E), row_exps = (int)exponents(I);
    uint16_t* rows = lists[wave];
    int n = e >= 0 ? find_rows(a.ids, slots, e, rows) : 0;
    if (n > 0 && E > slots && rows[0] != index) n = 0;
    Lines b[NT];
#pragma unroll
    for (int t = 0; t < NT; t++) {
        const int c = c0 + 64 * half + 16 * t;
        b[t].lines = c < H ? 16 : 0;
        b[t].p = a.dn + ((int64_t)__builtin_amdgcn_readfirstlane(max(e, 0)) * H + c) * I;
    }
    for (int r0 = 0; r0 < n; r0 += ROWS) {
        const int r = r0 + (lane & 15);
        int exp_offset[4];
#pragma unroll
        for (int v = 0; v < 4; v++) {
            const int q = r0 + 4 * (lane >> 4) + v;
            exp_offset[v] = q < n ? 2 * rows[q] * row_exps : NONE;
        }
        // as in gate_up; here a thread takes a column and four rows, and then the next four
        constexpr int ROUNDS = DOWN_COLS * 4 / THREADS;
        static_assert(THREADS % DOWN_COLS == 0, "a thread keeps its column");
        const int col = threadIdx.x % DOWN_COLS, c = c0 + col;
        int slot[ROUNDS][4];
        float weight[ROUNDS][4];
        const float sd = a.dns[(int64_t)e * H + min(c, H - 1)];   // past the last column it again
#pragma unroll
        for (int i = 0; i < ROUNDS; i++)
#pragma unroll
            for (int v = 0; v < 4; v++) {
                slot[i][v] = rows[min(r0 + 4 * ((int)threadIdx.x / DOWN_COLS + THREADS / DOWN_COLS * i) + v, n - 1)];
                weight[i][v] = a.weights[slot[i][v]];
            }
        float f[NT][4] = {};
        float sc[NT];   // of this lane's columns, for their exponents, which wait for them behind the first codes' request
#pragma unroll
        for (int t = 0; t < NT; t++) sc[t] = a.dns[(int64_t)e * H + min(c0 + 64 * half + 16 * t + (lane & 15), H - 1)];
        stream<P, NT, WAVES / 2, true>(
            hd, slots * P * I, r < n ? rows[r] * P * I : NONE, he, 2 * slots * row_exps, exp_offset, b, I, wave >> 1, ring0,
            ring1, [&](const i32x4(&fa)[P], const i32x4(&fb)[NT], const int(&ex)[4]) __attribute__((always_inline)) {
                const i32x4 zero = {0, 0, 0, 0};
                i32x4 acc[P][NT];
#pragma unroll
                for (int t = 0; t < NT; t++)
#pragma unroll
                    for (int p = 0; p < P; p++)
                        acc[p][t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fa[p], fb[t], zero, 0, 0, 0);
#pragma unroll
                for (int t = 0; t < NT; t++)
#pragma unroll
                    for (int v = 0; v < 4; v++) f[t][v] += scaled_by(join<P, NT>(acc, t, v), ex[v], exponent_of(sc[t]));
            });
        share_sums<NT>(f, ring0);
#pragma unroll
        for (int i = 0; i < ROUNDS; i++) {
            const int q = threadIdx.x / DOWN_COLS + THREADS / DOWN_COLS * i;
            if (r0 + 4 * q >= n || c >= H) continue;
            float s[4];
            shared_sum<NT>(ring0, col >> 6, (col >> 4) & 3, q, col & 15, s);
#pragma unroll
            for (int v = 0; v < 4; v++) {
                if (r0 + 4 * q + v >= n) break;
                const float y = s[v] * significand_of(sd) * weight[i][v];
                part[(int64_t)slot[i][v] * H + c] = y;
            }
        }
        __syncthreads();
    }
}

template <bool BF16>
__global__ __launch_bounds__(256) void combine_kernel(MoeArgs a, const float* __restrict__ part) {
    const int quads = (int)a.H / 4;
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i >= quads * (int)a.T) return;
    const int t = i / quads, c = (i - t * quads) * 4, k = (int)a.topk;
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    if (a.ids[(int64_t)t * k] >= 0)
        for (int j = 0; j < k; j++) {
            const float4 v = *reinterpret_cast<const float4*>(part + ((int64_t)t * k + j) * a.H + c);
            s.x += v.x;
            s.y += v.y;
            s.z += v.z;
            s.w += v.w;
        }
    store4<BF16>(a, t, c, s);
}

// ---------------------------------------------------------------- slot by slot
//
// One token's experts share no weights, so a row of codes meets one row of digits: dot products of whole contiguous rows,
// 16 codes a lane, v_dot4 for each digit, with every load of a workgroup on its way at once.  gate_up: a workgroup for each
// (slot, 32 inner columns), a wave four of gate and of up (fp32's fourth digit needs more registers: 16 columns, so that
// three workgroups fit a unit; 7 tokens, 16 experts of 4096 x 2048 75 -> 70 us).  down: a workgroup for each (token, 8 output
// columns), a wave a slot's 1024 inner columns at a time, so that no workgroup waits for another's sums.  Tokens on the
// same expert read its codes from the L2 that they share.

// digits . codes of a lane's 16
template <int P>
__device__ __forceinline__ void dots(const i32x4 (&d)[P], const i32x4& w, int (&acc)[P]) {
#pragma unroll
    for (int i = 0; i < 4; i++)
#pragma unroll
        for (int p = 0; p < P; p++) acc[p] = __builtin_amdgcn_sdot4(d[p][i], w[i], acc[p], false);
}

template <int P>
__device__ __forceinline__ float join1(const int (&acc)[P]) {
    float f = (float)acc[P - 1];
#pragma unroll
    for (int p = P - 2; p >= 0; p--) f = __builtin_fmaf(f, 256.f, (float)acc[p]);
    return f;
}

// the token's slot-th expert, from its logits: a wave for each eight of 64 candidates counts the logits before theirs
template <int W>
__device__ __forceinline__ int ranked(const float* __restrict__ logits, int E, int slot) {
    __shared__ int expert;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    uint32_t key[RANKED_EXPERTS / 64];
#pragma unroll
    for (int r = 0; r < RANKED_EXPERTS / 64; r++) key[r] = 64 * r + lane < E ? order_key(logits[64 * r + lane]) : 0;
#pragma unroll
    for (int r = 0; r < RANKED_EXPERTS / 64; r++) {
        if (64 * r >= E) break;
#pragma unroll
        for (int i = 0; i < 64 / W; i++) {
            const int from = 64 / W * wave + i, e = 64 * r + from;
            const uint32_t k = (uint32_t)__builtin_amdgcn_readlane((int)key[r], from);
            int before = 0;
#pragma unroll
            for (int q = 0; q < RANKED_EXPERTS / 64; q++)
                if (64 * q < E) before += __popcll(__ballot(key[q] > k || (key[q] == k && 64 * q + lane < e)));
            if (before == slot && e < E && lane == 0) expert = e;
        }
    }
    __syncthreads();
    return __builtin_amdgcn_readfirstlane(expert);
}

template <int P>
__global__ __launch_bounds__(64 * one_waves(P)) void gate_up_one_kernel(MoeArgs a, const int8_t* __restrict__ xd,
                                                          const int* __restrict__ xe, const float* __restrict__ logits,
                                                          int8_t* __restrict__ hd, int16_t* __restrict__ he) {
    constexpr int W = one_waves(P), COLS = 4 * W;
    const int E = (int)a.E, H = (int)a.H, I = (int)a.I, lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int T = (int)a.T, k = (int)a.topk, nsl = (int)one_exponents(I, P), slots = T * k;
    __shared__ __attribute__((aligned(16))) uint32_t keys[RANKED_EXPERTS];
    __shared__ float sums[W + 1], joined[2][COLS];
    const int grid = (nsl + 7) / 8 * 8 * slots;
    if ((int)blockIdx.x >= grid) {   // the last T workgroups: a token's ids and weights for everyone else
        const int t = (int)blockIdx.x - grid, i = threadIdx.x;
        if (i < (E + 3) / 4 * 4) keys[i] = i < E ? order_key(logits[t * E + i]) : 0;
        __syncthreads();
        take_topk<64 * W>(a, t, logits, keys, sums);
        return;
    }
    // workgroups go to the 8 XCDs in turn: all slots of a column slice to one, whose L2 the tokens of an expert share
    const int slot = ((int)blockIdx.x >> 3) % slots, slice = ((int)blockIdx.x >> 3) / slots * 8 + (blockIdx.x & 7), t = slot / k;
    if (slice >= nsl || (a.active && !a.active[t])) return;
    const int e = ranked<W>(logits + t * E, E, slot - t * k), c0 = slice * COLS, cw = c0 + 4 * wave, c = c0 + lane;
    const bool mine = wave == 0 && lane < COLS && c < I;
    const float* s = a.gus + (int64_t)e * 2 * I + c;
    const float sg = mine ? s[0] : 0.f, su = mine ? s[I] : 0.f;
    const int ex = xe[t];
    int acc[8][P] = {};
    if (cw < I) {   // columns come in sixteens
        const int8_t* w = a.gu + ((int64_t)e * 2 * I + cw) * H;
        const __amdgpu_buffer_rsrc_t rg = __builtin_amdgcn_make_buffer_rsrc((void*)w, (short)0, 4 * H, 0x00020000);
        const __amdgpu_buffer_rsrc_t ru =
            __builtin_amdgcn_make_buffer_rsrc((void*)(w + (int64_t)I * H), (short)0, 4 * H, 0x00020000);
        const __amdgpu_buffer_rsrc_t rd = __builtin_amdgcn_make_buffer_rsrc((void*)(xd + (int64_t)t * P * H), (short)0, P * H, 0x00020000);
        for (int k0 = 0; k0 < H; k0 += 2048) {
            i32x4 d[2][P], v[2][8];
#pragma unroll
            for (int x = 0; x < 2; x++) {
                const int k = k0 + 1024 * x + 16 * lane, at = k < H ? k : NONE;
#pragma unroll
                for (int p = 0; p < P; p++)
                    d[x][p] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(rd, at + p * H, 0, 0));
#pragma unroll
                for (int r = 0; r < 4; r++) {
                    v[x][r] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(rg, at + r * H, 0, 0));
                    v[x][4 + r] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(ru, at + r * H, 0, 0));
                }
            }
            __builtin_amdgcn_sched_barrier(0);   // every load goes out before the first is waited for
#pragma unroll
            for (int x = 0; x < 2; x++)
#pragma unroll
                for (int r = 0; r < 8; r++) dots<P>(d[x], v[x][r], acc[r]);
        }
    }
#pragma unroll
    for (int g = 0; g < 2; g++) {
        int sum[P];
#pragma unroll
        for (int p = 0; p < P; p++)
            sum[p] = sum4(acc[4 * g][p], acc[4 * g + 1][p], acc[4 * g + 2][p], acc[4 * g + 3][p]);
        if ((lane & 15) == 0) joined[g][4 * wave + value_of_row(lane >> 4)] = join1<P>(sum);
    }
    __syncthreads();
    if (wave > 0) return;
    float y = 0.f;
    if (mine) {
        const float gv = row_scaled(joined[0][lane], ex, sg), uv = row_scaled(joined[1][lane], ex, su);
        y = gv / (1.f + expf(-gv)) * uv;
    }
    const int eh = digit_exponent<P>(wave_max(__float_as_uint(y) & 0x7FFFFFFFu));
    const uint32_t q = digits_of(y, eh);
    if (mine)
#pragma unroll
        for (int p = 0; p < P; p++) hd[(int64_t)(slot * P + p) * I + c] = (int8_t)(q >> (8 * p));
    if (lane == 0) he[(int64_t)slot * nsl + slice] = (int16_t)eh;
}

template <int P, bool BF16>
__global__ __launch_bounds__(512) void down_one_kernel(MoeArgs a, const int8_t* __restrict__ hd,
                                                       const int16_t* __restrict__ he) {
    constexpr int COLS = 8;
    __shared__ float part[CFINT8_MOE_MAX_TOPK * CFINT8_MOE_MAX_WIDTH / 1024][COLS];
    const int H = (int)a.H, I = (int)a.I, k = (int)a.topk, nch = (I + 1023) / 1024, items = k * nch;
    // as in gate_up, all tokens of a column slice to one XCD
    const int t = ((int)blockIdx.x >> 3) % (int)a.T, c0 = (((int)blockIdx.x >> 3) / (int)a.T * 8 + (blockIdx.x & 7)) * COLS;
    if (c0 >= H) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int row_exps = (int)one_exponents(I, P), col = value_of_row(lane >> 4);   // of the first four
    const bool live = !a.active || a.active[t];
    if (live)
        for (int it = wave; it < items; it += 8) {
            const int slot = t * k + it / nch, e = __builtin_amdgcn_readfirstlane(a.ids[slot]), at = it % nch * 1024 + 16 * lane;
            const __amdgpu_buffer_rsrc_t rw = __builtin_amdgcn_make_buffer_rsrc(
                (void*)(a.dn + ((int64_t)e * H + c0) * I), (short)0, COLS * I, 0x00020000);
            const __amdgpu_buffer_rsrc_t rd =
                __builtin_amdgcn_make_buffer_rsrc((void*)(hd + (int64_t)slot * P * I), (short)0, P * I, 0x00020000);
            const int off = at < I ? at : NONE;
            i32x4 d[P], v[COLS];
#pragma unroll
            for (int r = 0; r < COLS; r++)
                v[r] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(rw, off + r * I, 0, 0));
#pragma unroll
            for (int p = 0; p < P; p++)
                d[p] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(rd, off + p * I, 0, 0));
            const int ex = at < I ? he[slot * row_exps + at / (4 * one_waves(P))] : 0;
            const float* sd = a.dns + (int64_t)e * H + c0 + col;
            const float s0 = sd[0], s1 = sd[4], weight = a.weights[slot];
            __builtin_amdgcn_sched_barrier(0);
            const int e0 = exponent_of(s0), e1 = exponent_of(s1);
            float f[COLS];
#pragma unroll
            for (int r = 0; r < COLS; r++) {
                int acc[P] = {};
                dots<P>(d, v[r], acc);
                f[r] = scaled_by(join1<P>(acc), ex, __builtin_amdgcn_readlane(r < 4 ? e0 : e1, 16 * value_of_row(r & 3)));
            }
            const float y0 = sum4(f[0], f[1], f[2], f[3]) * significand_of(s0) * weight;
            const float y1 = sum4(f[4], f[5], f[6], f[7]) * significand_of(s1) * weight;
            if ((lane & 15) == 0) part[it][col] = y0, part[it][4 + col] = y1;
        }
    __syncthreads();
    if (threadIdx.x >= COLS) return;
    float s = 0.f;
    if (live)
        for (int it = 0; it < items; it++) s += part[it][threadIdx.x];
    const int64_t at = t * a.ldy + c0 + threadIdx.x;
    if (BF16) static_cast<uint16_t*>(a.y)[at] = (uint16_t)to_bf16(s);
    else static_cast<float*>(a.y)[at] = s;
}

template <bool BF16, int P>
hipError_t launch(const MoeArgs& a, hipStream_t s) {
    const Layout l = layout(a.T, a.E, a.topk, a.H, a.I);
    char* w = static_cast<char*>(a.ws);
    float* logits = reinterpret_cast<float*>(w + l.logits);
    int8_t *xd = reinterpret_cast<int8_t*>(w + l.xd), *hd = reinterpret_cast<int8_t*>(w + l.hd);
    int* xe = reinterpret_cast<int*>(w + l.xe);
    int16_t* he = reinterpret_cast<int16_t*>(w + l.he);
    float* part = reinterpret_cast<float*>(w + l.part);
    const int64_t slots = a.T * a.topk, experts = a.E < slots ? a.E : slots;
    const int64_t up = (a.I + UP_COLS - 1) / UP_COLS, down = (a.H + DOWN_COLS - 1) / DOWN_COLS;
    if (a.T == 1) router_kernel<BF16, P, 1><<<(unsigned)(1 + a.E), 256, 0, s>>>(a, xd, xe, logits);
    else router_kernel<BF16, P, 4><<<(unsigned)(a.T + a.E * ((a.T + 3) / 4)), 256, 0, s>>>(a, xd, xe, logits);
    if (by_slots<P>(a.T, a.E, a.topk, a.H, a.I)) {
        const int64_t slices = (one_exponents(a.I, P) + 7) / 8 * 8;
        gate_up_one_kernel<P><<<(unsigned)(slices * slots + a.T), 64 * one_waves(P), 0, s>>>(a, xd, xe, logits, hd, he);
        down_one_kernel<P, BF16><<<(unsigned)((a.H + 63) / 64 * 8 * a.T), 512, 0, s>>>(a, hd, he);
        return hipGetLastError();
    }
    topk_kernel<<<(unsigned)a.T, 256, 0, s>>>(a, logits);
    gate_up_kernel<P><<<(unsigned)(experts * up), 64 * WAVES, 0, s>>>(a, xd, xe, hd, he);
    down_kernel<P><<<(unsigned)(experts * down), 64 * WAVES, 0, s>>>(a, hd, he, part);
    combine_kernel<BF16><<<(unsigned)((a.T * (a.H / 4) + 255) / 256), 256, 0, s>>>(a, part);
    return hipGetLastError();
}

}  // namespace

int64_t moe_workspace_bytes(int64_t T, int64_t E, int64_t topk, int64_t H, int64_t I) {
    return layout(T, E, topk, H, I).bytes;
}

hipError_t launch_moe(const MoeArgs& a, hipStream_t s) {
    return a.bf16 ? launch<true, 3>(a, s) : launch<false, 4>(a, s);
}

}  // namespace cfint8
