// Product of 8-bit integer codes with a scale for each token and channel on the gfx950 matrix cores.
//
// C[m][n] = (sum_k qa[m][k] qb[n][k]) sa[m] sb[n] + bias[n]: v_mfma_i32_32x32x32_i8 sums exactly, so the
// result depends neither on the tiling nor on the order of K, and every route gives the same C.
//
// tile_kernel: a workgroup of four waves owns a tile of 256 x 256 outputs (down to 64 x 64), a wave a quarter of it.
// K goes in blocks of 128 codes through two to four stages of LDS, filled by buffer-to-LDS loads whose pieces of 16
// codes are swizzled, so that the fragment reads cover all banks.  A block's second half is read under the first
// half's MFMAs, the next block's first half and the copy of a later block go out under the second half's.  A
// 256 x 256 tile needs 192 KB through the LDS a block (reads and copies) for 2048 cycles of MFMA, 75% of its rate;
// smaller wave tiles would need more of it than there is.  At 8192 x 14336 x 4096 (420 us, 2290 TOPS; 430
// to 480 where calls follow each other without a wait) the matrix pipe is busy for 64% of a unit's cycles, at a clock that the
// power limit holds at 1.8 GHz.  C goes past the caches that A and B are read from (streaming stores: 434 -> 415 us; no
// size measured loses more than 3%).
//
// An operand that lies as [K][N] goes to LDS in its own order and is turned by transposing reads on its way to
// registers (4096 x 4096 x 14336 210 us against 235 with a pass that turns it first, 2048 x 2048 x 2048 14.6 against 21).
#include <type_traits>

#include "device_util.hpp"
#include "int8_internal.hpp"
#include "int8_lanes.hpp"
#include "int8_routes.hpp"

namespace cfint8 {

using curvefp::u32x4;

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef int i32x16 __attribute__((ext_vector_type(16)));

// a piece of 16 codes without those past the first `left`
__device__ __forceinline__ i32x4 first_codes(i32x4 v, int left) {
#pragma unroll
    for (int w = 0; w < 4; w++) {
        const int b = left - 4 * w;   // codes of this word
        v[w] = b >= 4 ? v[w] : b <= 0 ? 0 : (int)((uint32_t)v[w] & ((1u << (8 * b)) - 1));
    }
    return v;
}

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {   // nearest even, low half first
    const f32x2 v = {lo, hi};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}

// sum * sa * sb + bias.  The scales' significands multiply the sum and their exponents are applied in one
// step, so nothing leaves fp32's range in between.  Where the scales are moderate (or 0, or NaN) their product is
// normal and sum * (sa * sb) is the same number
__device__ __forceinline__ float scaled_any(int sum, float sa, float sb, float bias) {
    const float m = (float)sum * (__builtin_amdgcn_frexp_mantf(sa) * __builtin_amdgcn_frexp_mantf(sb));
    return __builtin_amdgcn_ldexpf(m, __builtin_amdgcn_frexp_expf(sa) + __builtin_amdgcn_frexp_expf(sb)) + bias;
}

__device__ __forceinline__ bool moderate(float s) {
    return !(fabsf(s) < 0x1p-62f) ? !(fabsf(s) > 0x1p62f) : s == 0.f;
}

template <bool ANY>
__device__ __forceinline__ float scaled(int sum, float sa, float sb, float bias) {
#pragma clang fp contract(off)
    return ANY ? scaled_any(sum, sa, sb, bias) : (float)sum * (sa * sb) + bias;
}

__device__ __forceinline__ i32x2 read_tr(const char* p) {
    return __builtin_amdgcn_ds_read_tr8_b64_v2i32((__attribute__((address_space(3))) i32x2*)p);
}

// 16 bytes of C at a multiple of an element's size
typedef u32x4 u32x4_any __attribute__((aligned(2)));

// LDS written by some lanes of a wave is read by others behind this
__device__ __forceinline__ void wave_exchange() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// Workgroups go to the 8 XCDs round robin, and each XCD has its own L2: XCD x takes the x-th eighth of the
// tiles, in an order that walks groups of 8 tile rows column by column, so that the workgroups resident on an
// XCD share their rows of A and B in its L2.
struct Tile {
    int64_t m0, n0;
    bool valid;
};

__device__ __forceinline__ Tile tile_of(int b, int tiles_m, int tiles_n, int bm, int bn) {
    constexpr int GROUP = 8;
    const int total = tiles_m * tiles_n, share = (total + 7) / 8;
    const int u = (b & 7) * share + (b >> 3);
    Tile t;
    t.valid = u < total && (b >> 3) < share;
    const int g = u / (GROUP * tiles_n), gh = min(GROUP, tiles_m - g * GROUP);
    const int local = u - g * GROUP * tiles_n;
    // the quotients are the same in all lanes but come from vector code: without this every use of them in a
    // buffer descriptor would be a loop over the lanes' values
    t.m0 = (int64_t)__builtin_amdgcn_readfirstlane(g * GROUP + local % gh) * bm;
    t.n0 = (int64_t)__builtin_amdgcn_readfirstlane(local / gh) * bn;
    return t;
}

constexpr int BK = 128;   // codes of a block

// LDS has 64 banks of 4 bytes and serves 16 lanes of a 16-byte read at a time, here the same piece of 16 rows: two
// rows of 128 bytes cover the banks, so the eight rows of equal parity take a place each.  (With row % 8 half of the
// LDS's cycles were conflicts.)
__device__ __forceinline__ int swizzle(int row) { return (row >> 1) & 7; }

// The same for rows of BN bytes that hold B as [k][n]: a transposing read takes, for each half of a wave, 32 bytes of
// eight rows, so these rows' 32-byte pairs of pieces take as many places as 256 bytes have.
template <int BN>
__device__ __forceinline__ int swizzle_kn(int row) { return BN == 256 ? row & 7 : BN == 128 ? (row >> 1) & 3 : (row >> 2) & 1; }

constexpr int gcd(int a, int b) { return b == 0 ? a : gcd(b, a % b); }

// TM, TN: MFMA tiles of 32 that a wave takes along M and N; S: stages; TRANS: b is [K][N]
template <int TM, int TN, int S, bool BF16, bool TRANS>
__global__ __launch_bounds__(256) void tile_kernel(GemmArgs g, int tiles_m, int tiles_n) {
    constexpr int BM = 64 * TM, BN = 64 * TN, WM = 32 * TM, WN = 32 * TN;
    constexpr int PIECES = BK / 16, COPY_ROWS = 1024 / BK;      // of a row; of a 1 KB copy
    constexpr int COPIES_A = BM * BK / 4096, COPIES_B = BN * BK / 4096;   // of a wave
    constexpr int SLICES = BK / 64;                             // 32 codes each, of half a block
    constexpr int MFMAS = TM * TN * SLICES, READS = (TM + (TRANS ? 2 : 1) * TN) * SLICES;   // of half a block
    constexpr int COPIES = COPIES_A + COPIES_B;
    constexpr int HALF = BM * BK;                               // where a stage's B begins
    constexpr int STAGE = HALF + BN * BK;
    __shared__ __attribute__((aligned(16))) char st0[STAGE], st1[STAGE], st2[S > 2 ? STAGE : 16], st3[S > 3 ? STAGE : 16];
    __shared__ __attribute__((aligned(16))) float vec_a[BM], vec_b[BN], vec_bias[BN];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const Tile tile = tile_of((int)blockIdx.x, tiles_m, tiles_n, BM, BN);
    if (!tile.valid) return;
    const int64_t m0 = tile.m0, n0 = tile.n0;
    const int rows_a = (int)min((int64_t)BM, g.M - m0), rows_b = (int)min((int64_t)BN, g.N - n0);
    const int K = (int)g.K, nkb = (K + BK - 1) / BK;

    bool any = false;
    if (tid < BM) {
        const float s = g.as && tid < rows_a ? g.as[m0 + tid] : 1.f;
        vec_a[tid] = s;
        any = !moderate(s);
    }
    if (tid < BN) {
        const float s = g.bs && tid < rows_b ? g.bs[n0 + tid] : 1.f;
        vec_b[tid] = s;
        vec_bias[tid] = g.bias && tid < rows_b ? g.bias[n0 + tid] : 0.f;
        any = any || !moderate(s);
    }
    any = __syncthreads_or(any);

    // copies: a lane brings 16 bytes of its row, the piece that belongs where it writes; a row past the edge and a
    // piece past K lie behind the descriptor's end and arrive as zeros
    using lds_ptr = __attribute__((address_space(3))) void*;
    const int8_t *A = g.a + m0 * g.lda, *B = TRANS ? g.b + n0 : g.b + n0 * g.ldb;
    const int lda = (int)g.lda, ldb = (int)g.ldb, end_a = rows_a * lda, end_b = rows_b * ldb;
    constexpr int PIECES_B = TRANS ? BN / 16 : PIECES, COPY_ROWS_B = 64 / PIECES_B;
    const int row_a = wave * COPIES_A * COPY_ROWS + lane / PIECES, row_b = wave * COPIES_B * COPY_ROWS_B + lane / PIECES_B;
    auto piece = [&](int i, int left) __attribute__((always_inline)) {   // of copy i; a wave's rows start at a multiple of 16
        const int p = 16 * ((lane % PIECES) ^ swizzle(i * COPY_ROWS + lane / PIECES));
        return p < left ? p : 0x40000000;
    };
    auto piece_kn = [&](int i) __attribute__((always_inline)) {   // a wave's rows start at a multiple of 8
        const int p = 16 * ((lane % PIECES_B) ^ (2 * swizzle_kn<BN>(i * COPY_ROWS_B + lane / PIECES_B)));
        return p < rows_b ? p : 0x40000000;
    };
    // past the last block descriptors of no bytes, so that every step counts the same loads
    auto copy = [&](int kb, char* st) __attribute__((always_inline)) {
        const bool in = kb < nkb;
        const int k = in ? kb * BK : 0;
        const __amdgpu_buffer_rsrc_t ra =
            __builtin_amdgcn_make_buffer_rsrc((void*)(A + k), (short)0, in ? end_a - k : 0, 0x00020000);
        const __amdgpu_buffer_rsrc_t rb =
            TRANS ? __builtin_amdgcn_make_buffer_rsrc((void*)(B + (int64_t)k * ldb), (short)0,
                                                      in ? min(K - k, BK) * ldb - (int)n0 : 0, 0x00020000)
                  : __builtin_amdgcn_make_buffer_rsrc((void*)(B + k), (short)0, in ? end_b - k : 0, 0x00020000);
#pragma unroll
        for (int i = 0; i < COPIES_A; i++) {
            const int at = row_a * lda + i * COPY_ROWS * lda + piece(i, K - k);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, (lds_ptr)(st + (wave * COPIES_A + i) * 1024), 16, at, 0, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < COPIES_B; i++) {
            const int at = row_b * ldb + i * COPY_ROWS_B * ldb + (TRANS ? piece_kn(i) : piece(i, K - k));
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rb, (lds_ptr)(st + HALF + (wave * COPIES_B + i) * 1024), 16, at, 0,
                                                     0, 0);
        }
    };
    static_assert((COPIES_A * COPY_ROWS) % 16 == 0 && (COPIES_B * COPY_ROWS_B) % (TRANS ? 8 : 16) == 0,
                  "rows of a wave's copies");
    // K ends inside a piece of block kb, the last: A's codes behind it are cleared (B's then meet zeros; rows of a
    // [k][n] operand behind K are zeros already)
    auto clear_tail = [&](int kb, char* st) __attribute__((always_inline)) {
        if (TRANS || kb != nkb - 1 || K % 16 == 0) return;
        if (tid < BM) {
            const int at = K % BK, p = at >> 4;
            char* r = st + tid * BK + 16 * (p ^ swizzle(tid));
            for (int i = at & 15; i < 16; i++) r[i] = 0;
        }
        __syncthreads();
    };

    const int wm = wave >> 1, wn = wave & 1, lr = lane & 31;
    const int base_a = (wm * WM + lr) * BK, base_b = HALF + (wn * WN + lr) * BK;
    // transposing read: 16 lanes give the addresses of 8 rows of 16 codes, two lanes a row, and get a column of 8 codes
    // each; lanes 16 to 31 take the next 16 columns, lanes 32 to 63 the rows from 16 on, and a second read eight rows more
    const int row_kn = 16 * (lane >> 5) + ((lane & 15) >> 1);
    int at_kn[TN];
    if constexpr (TRANS)
#pragma unroll
        for (int t = 0; t < TN; t++) {
            at_kn[t] = row_kn * BN + 32 * ((wn * TN + t) ^ swizzle_kn<BN>(row_kn)) + 16 * ((lane >> 4) & 1) + 8 * (lane & 1);
            // One offset of unknown origin: as a sum of parts the compiler loses track of which stage is read and waits
            // for the copies into all of them
            asm("" : "+v"(at_kn[t]));
        }
    struct Half {
        i32x4 a[SLICES][TM], b[SLICES][TN];
    };
    auto load_half = [&](Half& f, const char* st, int h) __attribute__((always_inline)) {
#pragma unroll
        for (int s = 0; s < SLICES; s++) {
            const int off = 16 * ((2 * (h * SLICES + s) + (lane >> 5)) ^ swizzle(lr));
#pragma unroll
            for (int t = 0; t < TM; t++) f.a[s][t] = *reinterpret_cast<const i32x4*>(st + base_a + t * 32 * BK + off);
#pragma unroll
            for (int t = 0; t < TN; t++) {
                if constexpr (TRANS) {
                    const char* r = st + at_kn[t];
                    const int at = HALF + (64 * h + 32 * s) * BN;
                    const i32x2 lo = read_tr(r + at), hi = read_tr(r + at + 8 * BN);
                    f.b[s][t] = i32x4{lo.x, lo.y, hi.x, hi.y};
                } else {
                    f.b[s][t] = *reinterpret_cast<const i32x4*>(st + base_b + t * 32 * BK + off);
                }
            }
        }
    };
    i32x16 acc[TM][TN] = {};
    // B is the row operand: a lane then holds four adjacent columns of one row of C
    auto mfma = [&](const Half& f, int x) __attribute__((always_inline)) {
        const int s = x / (TM * TN), i = (x / TN) % TM, j = (i & 1) ? TN - 1 - x % TN : x % TN;
        acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(f.b[s][j], f.a[s][i], acc[i][j], 0, 0, 0);
    };
    constexpr int SG_MFMA = 0x008, SG_VMEM = 0x010, SG_DSR = 0x100;
    // an even mix: GROUPS times (reads, copies, MFMAs)
    constexpr int GROUPS = TRANS ? gcd(gcd(MFMAS, READS), COPIES) : MFMAS < READS ? MFMAS : READS, RG = READS / GROUPS, MG = MFMAS / GROUPS, CG = COPIES / GROUPS;
    auto phase1 = [&](Half& fa, Half& fb, char* st) __attribute__((always_inline)) {
        __builtin_amdgcn_s_waitcnt(0xC07F);   // fa's reads, a phase old
        load_half(fb, st, 1);
#pragma unroll
        for (int x = 0; x < MFMAS; x++) mfma(fa, x);
#pragma unroll
        for (int i = 0; i < GROUPS; i++) {
            __builtin_amdgcn_sched_group_barrier(SG_DSR, RG, 0);
            __builtin_amdgcn_sched_group_barrier(SG_MFMA, MG, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    // every wave is done with its stage, and the next block has landed: only S - 2 newer ones are still out
    // (vmcnt sits in bits 3:0 and 15:14, lgkmcnt in 11:8)
    constexpr int OUT = (S - 2) * COPIES;
    static_assert(OUT < 64, "vmcnt holds 6 bits");
    auto handover = [&]() __attribute__((always_inline)) {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(0x0070 | (OUT & 15) | ((OUT >> 4) << 14));
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    };
    auto phase2 = [&](Half& fa, Half& fb, char* nx, int kb, char* st) __attribute__((always_inline)) {
        copy(kb, st);
        load_half(fa, nx, 0);
#pragma unroll
        for (int x = 0; x < MFMAS; x++) mfma(fb, x);
#pragma unroll
        for (int i = 0; i < GROUPS; i++) {
            __builtin_amdgcn_sched_group_barrier(SG_DSR, RG, 0);
            __builtin_amdgcn_sched_group_barrier(SG_VMEM, CG, 0);
            __builtin_amdgcn_sched_group_barrier(SG_MFMA, MG, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    Half f0, f1;
    auto step = [&](int kb, char* cur, char* nxt) __attribute__((always_inline)) {
        phase1(f0, f1, cur);
        handover();
        clear_tail(kb + 1, nxt);
        phase2(f0, f1, nxt, kb + S, cur);
    };
    // the last block always runs on the last stage: the first ones start behind stage 0 where S does not divide
    char* const st[4] = {st0, st1, st2, st3};
    const int odd = nkb % S;
    auto begin = [&](auto from) __attribute__((always_inline)) {
        constexpr int F = decltype(from)::value;   // the first block's stage
#pragma unroll
        for (int d = 0; d < S; d++) copy(d, st[(F + d) % S]);
        asm volatile("" ::: "memory");
        constexpr int LEFT = (S - 1) * COPIES;
        static_assert(LEFT < 64, "vmcnt holds 6 bits");
        __builtin_amdgcn_s_waitcnt(0x0070 | (LEFT & 15) | ((LEFT >> 4) << 14));
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        clear_tail(0, st[F]);
        load_half(f0, st[F], 0);
#pragma unroll
        for (int d = F; d < S; d++)
            if (F > 0) step(d - F, st[d], st[(d + 1) % S]);
    };
    if (odd == 0) begin(std::integral_constant<int, 0>{});
    else if (S == 2 || odd == 1) begin(std::integral_constant<int, S - 1>{});
    else if (S == 3 || odd == 2) begin(std::integral_constant<int, S == 2 ? 1 : S - 2>{});
    else begin(std::integral_constant<int, S == 4 ? 1 : S - 1>{});
    for (int kb = odd; kb < nkb; kb += S) {
#pragma unroll
        for (int d = 0; d < S; d++) step(kb + d, st[d], st[(d + 1) % S]);
    }
    __builtin_amdgcn_s_waitcnt(0x0070);   // the copies of no bytes

    // Epilogue: 32 rows at a time through LDS of the wave's own, so that C is written in whole rows of the
    // wave's tile, 16 bytes a lane
    __syncthreads();   // every wave is done with the stages
    constexpr int ES = BF16 ? 2 : 4, PITCH = WN * ES + 16, LANES = WN * ES / 16;   // lanes of a row
    static_assert(2 * 32 * PITCH <= STAGE, "two waves' rows fit a stage");
    char* mine = (wm ? st1 : st0) + wn * 32 * PITCH;
    const int64_t mw = m0 + wm * WM, nw = n0 + wn * WN;
    char* C = static_cast<char*>(g.c) + (mw * g.ldc + nw) * ES;
    auto store = [&](auto mode) {
        constexpr bool ANY = decltype(mode)::value;
#pragma unroll
        for (int i = 0; i < TM; i++) {
            const float sa = vec_a[wm * WM + 32 * i + lr];
#pragma unroll
            for (int j = 0; j < TN; j++)
#pragma unroll
                for (int q = 0; q < 4; q++) {
                    const int col = 32 * j + 8 * q + 4 * (lane >> 5);
                    const float4 sb = *reinterpret_cast<const float4*>(&vec_b[wn * WN + col]);
                    const float4 bi = *reinterpret_cast<const float4*>(&vec_bias[wn * WN + col]);
                    const float x = scaled<ANY>(acc[i][j][4 * q], sa, sb.x, bi.x);
                    const float y = scaled<ANY>(acc[i][j][4 * q + 1], sa, sb.y, bi.y);
                    const float z = scaled<ANY>(acc[i][j][4 * q + 2], sa, sb.z, bi.z);
                    const float w = scaled<ANY>(acc[i][j][4 * q + 3], sa, sb.w, bi.w);
                    char* d = mine + lr * PITCH + col * ES;
                    if (BF16) *reinterpret_cast<uint2*>(d) = make_uint2(pack_bf16(x, y), pack_bf16(z, w));
                    else *reinterpret_cast<float4*>(d) = make_float4(x, y, z, w);
                }
            wave_exchange();
#pragma unroll
            for (int r = 0; r < 32; r += 64 / LANES) {
                const int row = r + lane / LANES, col = (lane % LANES) * (16 / ES);
                const u32x4 v = *reinterpret_cast<const u32x4*>(mine + row * PITCH + col * ES);
                if (mw + 32 * i + row >= g.M || nw + col >= g.N) continue;
                char* d = C + ((32 * i + row) * g.ldc + col) * ES;
                if (nw + col + 16 / ES <= g.N) {
                    __builtin_nontemporal_store(v, reinterpret_cast<u32x4_any*>(d));   // any alignment: ldc is the caller's
                } else {
                    for (int k = 0; k < 16 / ES; k++)
                        if (nw + col + k < g.N) {
                            if (BF16) reinterpret_cast<uint16_t*>(d)[k] = (uint16_t)(v[k >> 1] >> (16 * (k & 1)));
                            else reinterpret_cast<uint32_t*>(d)[k] = v[k];
                        }
                }
            }
            wave_exchange();
        }
    };
    if (any) store(std::true_type{});
    else store(std::false_type{});
}

// ---------------------------------------------------------------- few rows

// outputs m .. m + 3 of column n
template <bool BF16>
__device__ __forceinline__ void store_few(const GemmArgs& g, i32x4 s, int64_t m, int64_t n) {
    if (n >= g.N) return;
    const float sb = g.bs ? g.bs[n] : 1.f, bias = g.bias ? g.bias[n] : 0.f;
#pragma unroll
    for (int v = 0; v < 4; v++) {
        if (m + v >= g.M) break;
        const float y = scaled_any(s[v], g.as ? g.as[m + v] : 1.f, sb, bias);
        if (BF16) static_cast<uint16_t*>(g.c)[(m + v) * g.ldc + n] = (uint16_t)pack_bf16(y, y);
        else static_cast<float*>(g.c)[(m + v) * g.ldc + n] = y;
    }
}

// One or two tokens against a weight: bound by the weight's codes.  A wave takes four columns, whose codes are four
// contiguous lines, 16 codes a lane and load, against the tokens' by v_dot4; the next 2048 codes of each are requested
// before these are used.
template <int ROWS, bool BF16, bool STREAMED>
__global__ __launch_bounds__(256) void dot_kernel(GemmArgs g) {
    constexpr int COLS = 4, CHUNKS = 2;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t n0 = ((int64_t)blockIdx.x * 4 + wave) * COLS;
    if (n0 >= g.N) return;
    const int K = (int)g.K, lda = (int)g.lda, ldb = (int)g.ldb, used = (K + 15) & ~15;
    const __amdgpu_buffer_rsrc_t rb = __builtin_amdgcn_make_buffer_rsrc(
        (void*)(g.b + n0 * g.ldb), (short)0, (int)(min((int64_t)COLS, g.N - n0) - 1) * ldb + used, 0x00020000);
    const __amdgpu_buffer_rsrc_t ra =
        __builtin_amdgcn_make_buffer_rsrc((void*)g.a, (short)0, ((int)g.M - 1) * lda + used, 0x00020000);
    struct Chunk {
        i32x4 a[CHUNKS][ROWS], b[CHUNKS][COLS];
    };
    auto request = [&](Chunk& f, int k0) __attribute__((always_inline)) {
#pragma unroll
        for (int x = 0; x < CHUNKS; x++) {
            const int k = k0 + 1024 * x + 16 * lane;
            const int at = k < K ? k : 0x40000000;   // behind the descriptors' ends: zeros
#pragma unroll
            for (int n = 0; n < COLS; n++)
                f.b[x][n] = __builtin_bit_cast(
                    i32x4, __builtin_amdgcn_raw_buffer_load_b128(rb, at + n * ldb, 0, STREAMED ? 2 : 0));
#pragma unroll
            for (int m = 0; m < ROWS; m++)
                f.a[x][m] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(ra, at + m * lda, 0, 0));
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    int acc[ROWS][COLS] = {};
    auto use = [&](Chunk& f, int k0) __attribute__((always_inline)) {
#pragma unroll
        for (int x = 0; x < CHUNKS; x++) {
            if (k0 + 1024 * (x + 1) > K && K % 16 != 0)   // the piece that K ends in: whatever b holds there meets zeros
#pragma unroll
                for (int m = 0; m < ROWS; m++) f.a[x][m] = first_codes(f.a[x][m], K - k0 - 1024 * x - 16 * lane);
#pragma unroll
            for (int m = 0; m < ROWS; m++)
#pragma unroll
                for (int n = 0; n < COLS; n++)
#pragma unroll
                    for (int i = 0; i < 4; i++)
                        acc[m][n] = __builtin_amdgcn_sdot4(f.a[x][m][i], f.b[x][n][i], acc[m][n], false);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    Chunk f0, f1;
    constexpr int STEP = 1024 * CHUNKS;
    request(f0, 0);
    for (int k0 = 0; k0 < K; k0 += 2 * STEP) {
        request(f1, k0 + STEP);
        use(f0, k0);
        request(f0, k0 + 2 * STEP);
        use(f1, k0 + STEP);
    }
    const int64_t n = n0 + value_of_row(lane >> 4);
    i32x4 s = {0, 0, 0, 0};
#pragma unroll
    for (int m = 0; m < ROWS; m++) s[m] = sum4(acc[m][0], acc[m][1], acc[m][2], acc[m][3]);
    if ((lane & 15) == 0) store_few<BF16>(g, s, 0, n);
}

// A weight of 100 MB or more is read past the memory-side cache (256 MB), as it will not be there for the next token
// (1 x 28672 x 8192 36.8 us against 40.5, 1 x 32000 x 4096 22.3 against 23.6; 1 x 14336 x 4096 again and again 12.5 against 11.8)
template <int ROWS>
hipError_t launch_dot(const GemmArgs& g, hipStream_t s) {
    const unsigned grid = (unsigned)((g.N + 15) / 16);
    auto go = [&](auto bf16, auto streamed) {
        dot_kernel<ROWS, decltype(bf16)::value, decltype(streamed)::value><<<grid, 256, 0, s>>>(g);
    };
    if (g.N * g.K >= 100000000) {
        if (g.c_bf16) go(std::true_type{}, std::true_type{});
        else go(std::false_type{}, std::true_type{});
    } else {
        if (g.c_bf16) go(std::true_type{}, std::false_type{});
        else go(std::false_type{}, std::false_type{});
    }
    return hipGetLastError();
}

// A few tokens against a weight: 16 MT x 16 NT outputs a workgroup, K shared out over its waves as above, operands
// through LDS: direct loads of 16 lines a quarter of a wave cost the L1 a lookup for each, 64 a kilobyte (16 x 14336 x
// 4096 waits on them: 19.7 us against 14.1), copies to LDS of whole 128-byte pieces of lines 16.  A wave copies its
// own blocks of 128 codes into two slots of its own, so nothing waits for other waves until the sums meet; more slots
// measured slower (fewer workgroups fit a unit).
template <int MT, int NT, int WAVES, bool BF16>
__global__ __launch_bounds__(64 * WAVES) void few_kernel(GemmArgs g, int tiles_n) {
    constexpr int TILE = 16 * 128, SLOT = (MT + NT) * TILE, COPIES = 2 * (MT + NT);
    __shared__ __attribute__((aligned(16))) char ring0[WAVES * SLOT], ring1[WAVES * SLOT];
    static_assert(MT * NT * 1024 <= SLOT, "a wave's sums fit its slot");
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int tm = __builtin_amdgcn_readfirstlane((int)blockIdx.x / tiles_n), tn = (int)blockIdx.x - tm * tiles_n;
    const int64_t m0 = (int64_t)tm * 16 * MT, n0 = (int64_t)tn * 16 * NT;
    const int K = (int)g.K, nkb = (K + 127) / 128, mine = (nkb - wave + WAVES - 1) / WAVES;
    using lds_ptr = __attribute__((address_space(3))) void*;
    const int8_t *A = g.a + m0 * g.lda, *B = g.b + n0 * g.ldb;
    const int lda = (int)g.lda, ldb = (int)g.ldb;
    const int end_a = (int)min((int64_t)16 * MT, g.M - m0) * lda, end_b = (int)min((int64_t)16 * NT, g.N - n0) * ldb;
    const int row_a = (lane >> 3) * lda, row_b = (lane >> 3) * ldb;
    // this wave's j-th block; past its last one descriptors of no bytes, so that every step counts the same loads
    auto copy = [&](int j, char* ring) {
        const int k = (wave + j * WAVES) * 128;
        const bool in = j < mine;
        const __amdgpu_buffer_rsrc_t ra =
            __builtin_amdgcn_make_buffer_rsrc((void*)(A + (in ? k : 0)), (short)0, in ? end_a - k : 0, 0x00020000);
        const __amdgpu_buffer_rsrc_t rb =
            __builtin_amdgcn_make_buffer_rsrc((void*)(B + (in ? k : 0)), (short)0, in ? end_b - k : 0, 0x00020000);
        int at[2];   // the piece that belongs where this lane writes, of even and of odd copies
#pragma unroll
        for (int i = 0; i < 2; i++) {
            at[i] = 16 * ((lane & 7) ^ swizzle(8 * i + (lane >> 3)));
            at[i] = at[i] < K - k ? at[i] : 0x40000000;
        }
        char* st = ring + wave * SLOT;
#pragma unroll
        for (int i = 0; i < 2 * MT; i++) {
            const int o = row_a + i * 8 * lda + at[i & 1];
            __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, (lds_ptr)(st + i * 1024), 16, o, 0, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < 2 * NT; i++) {
            const int o = row_b + i * 8 * ldb + at[i & 1];
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rb, (lds_ptr)(st + MT * TILE + i * 1024), 16, o, 0, 0, 0);
        }
    };
    i32x4 acc[MT][NT] = {};
    const int lr = lane & 15;
    auto use = [&](int j, const char* ring) {
        const char* st = ring + wave * SLOT;
        const int kb = wave + j * WAVES;
#pragma unroll
        for (int s = 0; s < 2; s++) {
            const int piece = 4 * s + (lane >> 4), off = lr * 128 + 16 * (piece ^ swizzle(lr));
            i32x4 fa[MT], fb[NT];
#pragma unroll
            for (int i = 0; i < MT; i++) fa[i] = *reinterpret_cast<const i32x4*>(st + i * TILE + off);
#pragma unroll
            for (int n = 0; n < NT; n++) fb[n] = *reinterpret_cast<const i32x4*>(st + (MT + n) * TILE + off);
            if (kb == nkb - 1 && K % 16 != 0) {   // K ends inside a piece: A's codes behind it meet B's as zeros
#pragma unroll
                for (int i = 0; i < MT; i++) fa[i] = first_codes(fa[i], K - kb * 128 - 16 * piece);
            }
#pragma unroll
            for (int i = 0; i < MT; i++)
#pragma unroll
                for (int n = 0; n < NT; n++)
                    acc[i][n] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fa[i], fb[n], acc[i][n], 0, 0, 0);
        }
    };
    // a block has landed once only the next one's loads are out; s_waitcnt's vmcnt sits in bits 3:0 and 15:14
    static_assert(COPIES < 64, "vmcnt holds 6 bits");
    constexpr int WAIT = 0x0F70 | (COPIES & 15) | ((COPIES >> 4) << 14);
    auto step = [&](int j, char* now, char* next) {   // next: the slot that the step before this one used
        __builtin_amdgcn_s_waitcnt(0xC07F);           // its reads are done
        copy(j + 1, next);
        __builtin_amdgcn_s_waitcnt(WAIT);
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        use(j, now);
    };
    copy(0, ring0);
    for (int j = 0; j < mine; j += 2) {
        step(j, ring0, ring1);
        step(j + 1, ring1, ring0);
    }
    __builtin_amdgcn_s_waitcnt(0x0070);   // no copy and no read is left in flight: the sums take the first slot
#pragma unroll
    for (int i = 0; i < MT; i++)
#pragma unroll
        for (int j = 0; j < NT; j++)
            *reinterpret_cast<i32x4*>(ring0 + wave * SLOT + (i * NT + j) * 1024 + 16 * lane) = acc[i][j];
    __syncthreads();
    for (int e = tid; e < MT * NT * 64; e += 64 * WAVES) {
        const int t = e >> 6, l = e & 63;
        i32x4 s = {0, 0, 0, 0};
#pragma unroll
        for (int w = 0; w < WAVES; w++) s += *reinterpret_cast<const i32x4*>(ring0 + w * SLOT + 16 * e);
        store_few<BF16>(g, s, m0 + 16 * (t / NT) + 4 * (l >> 4), n0 + 16 * (t % NT) + (l & 15));
    }
}

template <int MT, int NT, int WAVES>
hipError_t launch_few(const GemmArgs& g, hipStream_t s) {
    const int64_t tm = (g.M + 16 * MT - 1) / (16 * MT), tn = (g.N + 16 * NT - 1) / (16 * NT);
    if (g.c_bf16) few_kernel<MT, NT, WAVES, true><<<(unsigned)(tm * tn), 64 * WAVES, 0, s>>>(g, (int)tn);
    else few_kernel<MT, NT, WAVES, false><<<(unsigned)(tm * tn), 64 * WAVES, 0, s>>>(g, (int)tn);
    return hipGetLastError();
}

// ---------------------------------------------------------------- the operand of another product, read transposed

// codes [K][ldb] -> [N][ldt]: tiles of 64 x 64, a thread turns 4 x 4 codes
__global__ __launch_bounds__(256) void transpose_kernel(const int8_t* __restrict__ b, int64_t ldb, int64_t K, int64_t N,
                                                        int8_t* __restrict__ t, int64_t ldt) {
    __shared__ uint32_t tile[64][17];
    const int64_t k0 = (int64_t)blockIdx.y * 64, n0 = (int64_t)blockIdx.x * 64;
    const int x = threadIdx.x & 15, y = threadIdx.x >> 4;
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const int64_t k = k0 + 4 * y + i;
        // whole words: a row of codes is readable up to a multiple of 16
        w[i] = k < K && n0 + 4 * x < N ? *reinterpret_cast<const uint32_t*>(b + k * ldb + n0 + 4 * x) : 0;
    }
    const uint32_t a0 = __builtin_amdgcn_perm(w[1], w[0], 0x05010400u), a1 = __builtin_amdgcn_perm(w[1], w[0], 0x07030602u);
    const uint32_t b0 = __builtin_amdgcn_perm(w[3], w[2], 0x05010400u), b1 = __builtin_amdgcn_perm(w[3], w[2], 0x07030602u);
    tile[4 * x][y] = __builtin_amdgcn_perm(b0, a0, 0x05040100u);
    tile[4 * x + 1][y] = __builtin_amdgcn_perm(b0, a0, 0x07060302u);
    tile[4 * x + 2][y] = __builtin_amdgcn_perm(b1, a1, 0x05040100u);
    tile[4 * x + 3][y] = __builtin_amdgcn_perm(b1, a1, 0x07060302u);
    __syncthreads();
    const int n = threadIdx.x >> 2, q = threadIdx.x & 3;
    if (n0 + n < N && k0 + 16 * q < ldt) {
        const uint32_t* r = &tile[n][4 * q];
        *reinterpret_cast<uint4*>(t + (n0 + n) * ldt + k0 + 16 * q) = make_uint4(r[0], r[1], r[2], r[3]);
    }
}

int64_t ceil_to(int64_t n, int64_t m) { return (n + m - 1) / m * m; }

template <int TM, int TN, int S>
hipError_t launch_tiles(const GemmArgs& g, hipStream_t s) {
    const int64_t tm = (g.M + 64 * TM - 1) / (64 * TM), tn = (g.N + 64 * TN - 1) / (64 * TN);
    const unsigned grid = (unsigned)(((tm * tn + 7) / 8) * 8);
    auto go = [&](auto bf16, auto trans) {
        tile_kernel<TM, TN, S, decltype(bf16)::value, decltype(trans)::value><<<grid, 256, 0, s>>>(g, (int)tm, (int)tn);
    };
    if (g.trans) {
        if (g.c_bf16) go(std::true_type{}, std::true_type{});
        else go(std::false_type{}, std::true_type{});
    } else {
        if (g.c_bf16) go(std::true_type{}, std::false_type{});
        else go(std::false_type{}, std::false_type{});
    }
    return hipGetLastError();
}

hipError_t launch_routed(const GemmArgs& g, hipStream_t s) {
    switch (route_direct(g.M, g.N, g.K, g.trans).kernel) {
        case DOT: return g.M == 1 ? launch_dot<1>(g, s) : launch_dot<2>(g, s);
        case FEW4: return launch_few<1, 1, 4>(g, s);
        case FEW8: return launch_few<1, 1, 8>(g, s);
        case FEW32: return launch_few<2, 2, 4>(g, s);
        case T64: return launch_tiles<1, 1, 4>(g, s);
        case T64_128: return launch_tiles<1, 2, 3>(g, s);
        case T128: return launch_tiles<2, 2, 3>(g, s);
        case T256_128: return launch_tiles<4, 2, 3>(g, s);
        default: return launch_tiles<4, 4, 2>(g, s);
    }
}

}  // namespace

int64_t gemm_workspace_bytes(int64_t M, int64_t N, int64_t K, int trans) {
    return trans && turned(M, N, K) ? N * ceil_to(K, 16) : 0;
}

hipError_t launch_gemm(const GemmArgs& args, hipStream_t s) {
    GemmArgs g = args;
    if (g.trans && turned(g.M, g.N, g.K)) {
        g.trans = 0;
        int8_t* t = static_cast<int8_t*>(g.ws);
        g.b = t;
        g.ldb = ceil_to(g.K, 16);
        const dim3 grid((unsigned)((g.N + 63) / 64), (unsigned)((g.K + 63) / 64));
        transpose_kernel<<<grid, 256, 0, s>>>(args.b, args.ldb, g.K, g.N, t, g.ldb);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    const GemmArgs all = g;
    hipError_t e = hipSuccess;
    for (int64_t m = 0; m < all.M && e == hipSuccess; m += PART)
        for (int64_t n = 0; n < all.N && e == hipSuccess; n += PART) {
            g.M = all.M - m < PART ? all.M - m : PART;
            g.N = all.N - n < PART ? all.N - n : PART;
            g.a = all.a + m * all.lda;
            g.b = all.b + (g.trans ? n : n * all.ldb);
            g.as = all.as ? all.as + m : nullptr;
            g.bs = all.bs ? all.bs + n : nullptr;
            g.bias = all.bias ? all.bias + n : nullptr;
            g.c = static_cast<char*>(all.c) + (m * all.ldc + n) * (all.c_bf16 ? 2 : 4);
            e = launch_routed(g, s);
        }
    return e;
}

}  // namespace cfint8
