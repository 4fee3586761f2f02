// Mixture-of-experts layer for a few tokens with 8-bit weights.
//
// A few tokens against many weights: every taken expert's codes are read once, so the layer is bound by
// memory, and the codes go from memory to the matrix cores as they are.  The other operand of
// v_mfma_i32_16x16x64_i8 is the activation in fixed point: a row's values as integers of 22 bits (bf16) or
// 30 bits (fp32) below a power of two above its largest, split into 3 or 4 signed base-256 digits, one
// product for each digit.  All sums of products are exact int32; the digits' sums meet in fp32.
//
//   router   logits in 64 bits (they decide, so they are right to the last bit), x into digits
//   topk     a wave for each token: ids and weights
//   gate_up  a workgroup for each (expert, 32 inner columns): h in fp32
//   digits   h into digits
//   down     a workgroup for each (expert, 64 output columns): weighted partial rows, one for each slot
//   combine  a token's slots added in order
#include "int8_internal.hpp"

namespace cfint8 {

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr int POISON = INT32_MIN;      // exponent of a row that holds a NaN or an infinity
constexpr int ROWS = 16;               // token rows of a matrix product
constexpr int UP_COLS = 32;            // inner columns of a gate_up workgroup
constexpr int DOWN_COLS = 64;          // output columns of a down workgroup

// workspace
struct Layout {
    int64_t logits, xd, xe, h, hd, he, part, bytes;
};

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
    l.h = take(S * I * 4);
    l.hd = take(S * 4 * I);
    l.he = take(S * 4);
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

// digits of 8 values, byte i of out[p] digit p of value i
template <int P>
__device__ __forceinline__ void digits8(const float* v, int e, uint2* out) {
    uint32_t q[8];
#pragma unroll
    for (int i = 0; i < 8; i++) {
        const int n = e == POISON ? 0 : (int)__builtin_rintf(__builtin_amdgcn_ldexpf(v[i], -e));
        q[i] = ((uint32_t)n + 0x00808080u) ^ 0x00808080u;   // signed digits
    }
#pragma unroll
    for (int p = 0; p < P; p++) {
        uint32_t w[2] = {0, 0};
#pragma unroll
        for (int i = 0; i < 8; i++) w[i >> 2] |= ((q[i] >> (8 * p)) & 0xFFu) << (8 * (i & 3));
        out[p] = make_uint2(w[0], w[1]);
    }
}

__device__ __forceinline__ uint32_t block_max(uint32_t m, uint32_t* red) {   // 256 threads
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o));
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = m;
    __syncthreads();
    return max(max(red[0], red[1]), max(red[2], red[3]));
}

// one row of n (a multiple of 16) values into digits [P][n]
template <bool BF16, int P>
__device__ __forceinline__ void row_digits(const char* src, int n, int8_t* dst, int* exponent, uint32_t* red) {
    uint32_t m = 0;
    for (int c = threadIdx.x * 8; c < n; c += 2048) {
        float v[8];
        load8<BF16>(src, c, v);
#pragma unroll
        for (int i = 0; i < 8; i++) m = max(m, __float_as_uint(v[i]) & 0x7FFFFFFFu);
    }
    const int e = digit_exponent<P>(block_max(m, red));
    for (int c = threadIdx.x * 8; c < n; c += 2048) {
        float v[8];
        uint2 d[P];
        load8<BF16>(src, c, v);
        digits8<P>(v, e, d);
#pragma unroll
        for (int p = 0; p < P; p++) *reinterpret_cast<uint2*>(dst + (int64_t)p * n + c) = d[p];
    }
    if (threadIdx.x == 0) *exponent = e;
}

// workgroups [0, T): a token's x into digits; then (4 experts, one a wave) x (4 tokens)
template <bool BF16, int P>
__global__ __launch_bounds__(256) void router_kernel(MoeArgs a, int8_t* __restrict__ xd, int* __restrict__ xe,
                                                     float* __restrict__ logits) {
    __shared__ uint32_t red[4];
    const int T = (int)a.T, E = (int)a.E, H = (int)a.H;
    const int64_t es = BF16 ? 2 : 4;
    int b = blockIdx.x;
    if (b < T) {
        row_digits<BF16, P>(static_cast<const char*>(a.x) + b * a.ldx * es, H, xd + (int64_t)b * P * H, xe + b, red);
        return;
    }
    b -= T;
    const int eg = (E + 3) / 4;
    const int e = (b % eg) * 4 + (threadIdx.x >> 6), t0 = (b / eg) * 4, lane = threadIdx.x & 63;
    if (e >= E) return;
    double s[4] = {0, 0, 0, 0};
    const char* r = static_cast<const char*>(a.router) + (int64_t)e * H * es;
    for (int c = lane * 8; c < H; c += 512) {
        float w[8];
        load8<BF16>(r, c, w);
#pragma unroll
        for (int t = 0; t < 4; t++) {
            if (t0 + t >= T) break;
            float v[8];
            load8<BF16>(static_cast<const char*>(a.x) + (t0 + t) * a.ldx * es, c, v);
#pragma unroll
            for (int i = 0; i < 8; i++) s[t] = __builtin_fma((double)v[i], (double)w[i], s[t]);
        }
    }
#pragma unroll
    for (int t = 0; t < 4; t++) {
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) s[t] += __shfl_xor(s[t], o);
        if (lane == 0 && t0 + t < T) logits[(int64_t)(t0 + t) * E + e] = (float)s[t];
    }
}

// orders logits: NaN below everything, -0 as 0
__device__ __forceinline__ uint32_t order_key(float l) {
    if (l != l) return 0;
    const uint32_t u = __float_as_uint(l + 0.f);
    return u ^ ((u >> 31) ? 0xFFFFFFFFu : 0x80000000u);
}

// a wave for each token; lane l holds experts l, l + 64, ...
__global__ __launch_bounds__(64) void topk_kernel(MoeArgs a, const float* __restrict__ logits) {
    constexpr int MAX = (int)(1024 / 64);
    const int t = blockIdx.x, lane = threadIdx.x, E = (int)a.E, k = (int)a.topk;
    int32_t* ids = a.ids + (int64_t)t * k;
    float* weights = a.weights + (int64_t)t * k;
    if (a.active && !a.active[t]) {
        for (int j = lane; j < k; j += 64) {
            ids[j] = -1;
            weights[j] = 0.f;
        }
        return;
    }
    float l[MAX];
    uint64_t key[MAX];
#pragma unroll
    for (int i = 0; i < MAX; i++) {
        const int e = lane + 64 * i;
        l[i] = e < E ? logits[(int64_t)t * E + e] : 0.f;
        key[i] = e < E ? ((uint64_t)order_key(l[i]) << 32) | (0xFFFFFFFFu - (uint32_t)e) : 0;
    }
    float lead = 0.f, sum = 0.f, mine = 0.f;
    int my_id = 0;
    for (int j = 0; j < k; j++) {
        uint64_t best = 0;
#pragma unroll
        for (int i = 0; i < MAX; i++) best = max(best, key[i]);
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) best = max(best, (uint64_t)__shfl_xor((unsigned long long)best, o));
        const int e = (int)(0xFFFFFFFFu - (uint32_t)best);
        float le = 0.f;
#pragma unroll
        for (int i = 0; i < MAX; i++)
            if (key[i] == best) {
                key[i] = 0;
                le = l[i];
            }
        le = __shfl(le, e & 63);
        if (j == 0) lead = le;
        const float w = expf(le - lead);
        sum += w;
        if (lane == j) {
            mine = w;
            my_id = e;
        }
    }
    if (!a.renorm) {
        sum = 0.f;
#pragma unroll
        for (int i = 0; i < MAX; i++) sum += lane + 64 * i < E ? expf(l[i] - lead) : 0.f;
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
    }
    if (lane < k) {
        ids[lane] = my_id;
        weights[lane] = mine / sum;
    }
}

// The slots (at most 8192) whose token takes expert e, ascending, in list[]; their number.  All threads
struct Rows {
    uint16_t list[256];   // an expert is taken at most once by each token
    int n;
};

__device__ __forceinline__ void find_rows(const int32_t* __restrict__ ids, int slots, int e, Rows& r) {
    __shared__ int cnt[4], base;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (threadIdx.x == 0) base = 0;
    __syncthreads();
    for (int s0 = 0; s0 < slots; s0 += 256) {
        const int s = s0 + threadIdx.x;
        const bool hit = s < slots && ids[s] == e;
        const uint64_t b = __ballot(hit);
        if (lane == 0) cnt[wave] = __popcll(b);
        __syncthreads();
        int at = base;
        for (int w = 0; w < wave; w++) at += cnt[w];
        if (hit) r.list[at + __popcll(b & ((1ull << lane) - 1))] = (uint16_t)s;
        __syncthreads();
        if (threadIdx.x == 0) base += cnt[0] + cnt[1] + cnt[2] + cnt[3];
        __syncthreads();
    }
    if (threadIdx.x == 0) r.n = base;
    __syncthreads();
}

// Which expert a workgroup's first index stands for: expert i itself where the experts are fewer than the
// slots, else slot i's expert if no earlier slot has it too; -1 for none
__device__ __forceinline__ int expert_of(const int32_t* __restrict__ ids, int i, int slots, int E) {
    if (E <= slots) return i;
    const int e = ids[i];
    if (e < 0) return -1;
    __shared__ int seen;
    if (threadIdx.x == 0) seen = 0;
    __syncthreads();
    for (int s = threadIdx.x; s < i; s += 256)
        if (ids[s] == e) seen = 1;
    __syncthreads();
    return seen ? -1 : e;
}

// digit sums of 16 rows x 16 NT columns over this wave's share of K: lane l holds row (A) or column (B)
// l % 16 at 16 (l / 16) of each 64; a[p] and b[t] point at this lane's line, live: its row exists
template <int P, int NT>
__device__ __forceinline__ void accumulate(const int8_t* a, int64_t plane, bool live, const int8_t* const (&b)[NT],
                                           int K, i32x4 (&acc)[P][NT]) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const i32x4 zero = {0, 0, 0, 0};
#pragma unroll
    for (int p = 0; p < P; p++)
#pragma unroll
        for (int t = 0; t < NT; t++) acc[p][t] = zero;
    for (int k0 = wave * 64; k0 < K; k0 += 256) {
        const int k = k0 + 16 * (lane >> 4);
        i32x4 fa[P], fb[NT];
#pragma unroll
        for (int t = 0; t < NT; t++) fb[t] = k < K ? *reinterpret_cast<const i32x4*>(b[t] + k) : zero;
#pragma unroll
        for (int p = 0; p < P; p++) fa[p] = live && k < K ? *reinterpret_cast<const i32x4*>(a + p * plane + k) : zero;
#pragma unroll
        for (int t = 0; t < NT; t++)
#pragma unroll
            for (int p = 0; p < P; p++)
                acc[p][t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fa[p], fb[t], acc[p][t], 0, 0, 0);
    }
}

// the waves' sums: red[wave][t][column l % 16][row]; the digits meet here
template <int P, int NT>
__device__ __forceinline__ void share(const i32x4 (&acc)[P][NT], float* red) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int t = 0; t < NT; t++)
#pragma unroll
        for (int v = 0; v < 4; v++) {
            float f = (float)acc[P - 1][t][v];
#pragma unroll
            for (int p = P - 2; p >= 0; p--) f = __builtin_fmaf(f, 256.f, (float)acc[p][t][v]);
            red[((wave * NT + t) * 16 + (lane & 15)) * ROWS + 4 * (lane >> 4) + v] = f;
        }
    __syncthreads();
}

// NaN for a poisoned row
__device__ __forceinline__ float row_scaled(float f, int e, float s) {
    return e == POISON ? __uint_as_float(0x7FC00000u) : __builtin_amdgcn_ldexpf(f, e) * s;
}

template <int P>
__global__ __launch_bounds__(256) void gate_up_kernel(MoeArgs a, const int8_t* __restrict__ xd,
                                                      const int* __restrict__ xe, float* __restrict__ h) {
    constexpr int NT = 2 * UP_COLS / 16, HALF = NT / 2;
    __shared__ Rows rows;
    __shared__ __attribute__((aligned(16))) float red[4 * NT * 16 * ROWS];
    const int slots = (int)(a.T * a.topk), H = (int)a.H, I = (int)a.I, lane = threadIdx.x & 63;
    const int nsl = (I + UP_COLS - 1) / UP_COLS;
    const int e = expert_of(a.ids, blockIdx.x / nsl, slots, (int)a.E);
    if (e < 0) return;
    find_rows(a.ids, slots, e, rows);
    const int c0 = (blockIdx.x % nsl) * UP_COLS;
    const int8_t* b[NT];
#pragma unroll
    for (int t = 0; t < NT; t++) {
        const int c = min(c0 + 16 * (t % HALF) + (lane & 15), I - 1) + (t >= HALF ? I : 0);
        b[t] = a.gu + ((int64_t)e * 2 * I + c) * H;
    }
    for (int r0 = 0; r0 < rows.n; r0 += ROWS) {
        const int r = r0 + (lane & 15);
        const bool live = r < rows.n;
        const int8_t* x = xd + (int64_t)(live ? rows.list[r] / (int)a.topk : 0) * P * H;
        i32x4 acc[P][NT];
        accumulate<P, NT>(x, H, live, b, H, acc);
        share<P, NT>(acc, red);
        for (int i = threadIdx.x; i < UP_COLS * ROWS; i += 256) {
            const int row = i / UP_COLS, col = i % UP_COLS;
            if (r0 + row >= rows.n || c0 + col >= I) continue;
            const int at = ((col >> 4) * 16 + (col & 15)) * ROWS + row;
            float g = 0.f, u = 0.f;
#pragma unroll
            for (int w = 0; w < 4; w++) {
                g += red[w * NT * 16 * ROWS + at];
                u += red[(w * NT + HALF) * 16 * ROWS + at];
            }
            const int slot = rows.list[r0 + row], ex = xe[slot / (int)a.topk];
            const float* s = a.gus + (int64_t)e * 2 * I + c0 + col;
            g = row_scaled(g, ex, s[0]);
            u = row_scaled(u, ex, s[I]);
            h[(int64_t)slot * I + c0 + col] = g / (1.f + expf(-g)) * u;
        }
        __syncthreads();
    }
}

template <int P>
__global__ __launch_bounds__(256) void digits_kernel(MoeArgs a, const float* __restrict__ h, int8_t* __restrict__ hd,
                                                     int* __restrict__ he) {
    __shared__ uint32_t red[4];
    const int slot = blockIdx.x;
    if (a.ids[slot] < 0) return;
    row_digits<false, P>(reinterpret_cast<const char*>(h + (int64_t)slot * a.I), (int)a.I, hd + (int64_t)slot * P * a.I,
                         he + slot, red);
}

template <int P>
__global__ __launch_bounds__(256) void down_kernel(MoeArgs a, const int8_t* __restrict__ hd, const int* __restrict__ he,
                                                   float* __restrict__ part) {
    constexpr int NT = DOWN_COLS / 16;
    __shared__ Rows rows;
    __shared__ __attribute__((aligned(16))) float red[4 * NT * 16 * ROWS];
    const int slots = (int)(a.T * a.topk), H = (int)a.H, I = (int)a.I, lane = threadIdx.x & 63;
    const int nsl = (H + DOWN_COLS - 1) / DOWN_COLS;
    const int e = expert_of(a.ids, blockIdx.x / nsl, slots, (int)a.E);
    if (e < 0) return;
    find_rows(a.ids, slots, e, rows);
    const int c0 = (blockIdx.x % nsl) * DOWN_COLS;
    const int8_t* b[NT];
#pragma unroll
    for (int t = 0; t < NT; t++) b[t] = a.dn + ((int64_t)e * H + min(c0 + 16 * t + (lane & 15), H - 1)) * I;
    for (int r0 = 0; r0 < rows.n; r0 += ROWS) {
        const int r = r0 + (lane & 15);
        const bool live = r < rows.n;
        i32x4 acc[P][NT];
        accumulate<P, NT>(hd + (int64_t)(live ? rows.list[r] : 0) * P * I, I, live, b, I, acc);
        share<P, NT>(acc, red);
        for (int i = threadIdx.x; i < DOWN_COLS * ROWS; i += 256) {
            const int row = i / DOWN_COLS, col = i % DOWN_COLS;
            if (r0 + row >= rows.n || c0 + col >= H) continue;
            const int at = col * ROWS + row;
            float f = 0.f;
#pragma unroll
            for (int w = 0; w < 4; w++) f += red[w * NT * 16 * ROWS + at];
            const int slot = rows.list[r0 + row];
            part[(int64_t)slot * H + c0 + col] =
                row_scaled(f, he[slot], a.dns[(int64_t)e * H + c0 + col]) * a.weights[slot];
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
    char* y = static_cast<char*>(a.y) + (t * a.ldy + c) * (BF16 ? 2 : 4);
    if (BF16) *reinterpret_cast<uint2*>(y) = make_uint2(to_bf16(s.x) | to_bf16(s.y) << 16, to_bf16(s.z) | to_bf16(s.w) << 16);
    else *reinterpret_cast<float4*>(y) = s;
}

template <bool BF16, int P>
hipError_t launch(const MoeArgs& a, hipStream_t s) {
    const Layout l = layout(a.T, a.E, a.topk, a.H, a.I);
    char* w = static_cast<char*>(a.ws);
    float* logits = reinterpret_cast<float*>(w + l.logits);
    int8_t *xd = reinterpret_cast<int8_t*>(w + l.xd), *hd = reinterpret_cast<int8_t*>(w + l.hd);
    int *xe = reinterpret_cast<int*>(w + l.xe), *he = reinterpret_cast<int*>(w + l.he);
    float *h = reinterpret_cast<float*>(w + l.h), *part = reinterpret_cast<float*>(w + l.part);
    const int64_t slots = a.T * a.topk, experts = a.E < slots ? a.E : slots;
    const unsigned router = (unsigned)(a.T + ((a.E + 3) / 4) * ((a.T + 3) / 4));
    router_kernel<BF16, P><<<router, 256, 0, s>>>(a, xd, xe, logits);
    topk_kernel<<<(unsigned)a.T, 64, 0, s>>>(a, logits);
    gate_up_kernel<P><<<(unsigned)(experts * ((a.I + UP_COLS - 1) / UP_COLS)), 256, 0, s>>>(a, xd, xe, h);
    digits_kernel<P><<<(unsigned)slots, 256, 0, s>>>(a, h, hd, he);
    down_kernel<P><<<(unsigned)(experts * ((a.H + DOWN_COLS - 1) / DOWN_COLS)), 256, 0, s>>>(a, hd, he, part);
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
