// Product of 8-bit integer codes with a scale for each token and channel on the gfx950 matrix cores.
//
// C[m][n] = (sum_k qa[m][k] qb[n][k]) sa[m] sb[n] + bias[n]: v_mfma_i32_32x32x32_i8 sums exactly, so the
// result depends neither on the tiling nor on the order of K, and every route gives the same C.
//
// tile_kernel: a workgroup of four waves owns a tile of 256 x 256 (or 128 x 128) outputs, a wave 128 x 128 (64 x 64) of it.
// K goes in blocks of 128 codes, double-buffered in LDS by buffer-to-LDS loads; rows are 128 bytes with their
// eight 16-byte pieces XOR-swizzled by row % 8 (applied to the addresses that the loads read), so the fragment
// reads of 8 rows cover all banks.  A block's second half is read under the first half's MFMAs, the next
// block's first half and the copy of the block after it go out under the second half's.  A 256 x 256 tile
// needs 192 KB through the LDS a block (reads and copies) for 2048 cycles of MFMA, 75% of its rate;
// smaller wave tiles would need more of it than there is.
#include <type_traits>

#include "device_util.hpp"
#include "int8_internal.hpp"

namespace cfint8 {

using curvefp::u32x4;

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));

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

// WT: MFMA tiles of 32 a wave takes along each side (4 or 2)
template <int WT, bool BF16>
__global__ __launch_bounds__(256) void tile_kernel(GemmArgs g, int tiles_m, int tiles_n) {
    constexpr int BM = 64 * WT, WM = 32 * WT;
    constexpr int HALF = BM * BK;                    // one operand's block
    constexpr int COPIES = HALF / 4096;              // 1 KB copies of a wave for one operand's block
    constexpr int MFMAS = WT * WT * 2, READS = WT * 4;   // of half a block
    __shared__ __attribute__((aligned(16))) char st0[2 * HALF];
    __shared__ __attribute__((aligned(16))) char st1[2 * HALF];
    __shared__ __attribute__((aligned(16))) float vec[3][BM];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const Tile tile = tile_of((int)blockIdx.x, tiles_m, tiles_n, BM, BM);
    if (!tile.valid) return;
    const int64_t m0 = tile.m0, n0 = tile.n0;
    const int rows_a = (int)min((int64_t)BM, g.M - m0), rows_b = (int)min((int64_t)BM, g.N - n0);
    const int K = (int)g.K, nkb = (K + BK - 1) / BK;

    bool any = false;
    if (tid < BM) {
        const float sa = g.as && tid < rows_a ? g.as[m0 + tid] : 1.f, sb = g.bs && tid < rows_b ? g.bs[n0 + tid] : 1.f;
        vec[0][tid] = sa;
        vec[1][tid] = sb;
        vec[2][tid] = g.bias && tid < rows_b ? g.bias[n0 + tid] : 0.f;
        any = !moderate(sa) || !moderate(sb);
    }
    any = __syncthreads_or(any);

    // copies: lane l of a kilobyte brings row l / 8, piece (l % 8) ^ (row % 8); a row past the edge and a piece
    // past K lie behind the descriptor's end and arrive as zeros
    using lds_ptr = __attribute__((address_space(3))) void*;
    const int piece = 16 * ((lane & 7) ^ (lane >> 3));
    const int8_t *A = g.a + m0 * g.lda, *B = g.b + n0 * g.ldb;
    const int end_a = rows_a * (int)g.lda, end_b = rows_b * (int)g.ldb;
    const int row0 = wave * COPIES * 8 + (lane >> 3);
    const int offa = row0 * (int)g.lda, offb = row0 * (int)g.ldb;
    auto copy = [&](int kb, char* st) {
        const int k = kb * BK;
        const __amdgpu_buffer_rsrc_t ra =
            __builtin_amdgcn_make_buffer_rsrc((void*)(A + k), (short)0, end_a - k, 0x00020000);
        const __amdgpu_buffer_rsrc_t rb =
            __builtin_amdgcn_make_buffer_rsrc((void*)(B + k), (short)0, end_b - k, 0x00020000);
        const int at = k + piece < K ? piece : 0x40000000;
#pragma unroll
        for (int i = 0; i < COPIES; i++) {
            const int kbyte = (wave * COPIES + i) * 1024;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, (lds_ptr)(st + kbyte), 16, offa + at + i * 8 * (int)g.lda, 0, 0,
                                                     0);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rb, (lds_ptr)(st + HALF + kbyte), 16, offb + at + i * 8 * (int)g.ldb, 0,
                                                     0, 0);
        }
    };
    // K ends inside a piece: A's codes behind it are cleared (B's then meet zeros)
    auto clear_tail = [&](char* st) {
        if (K % 16 == 0) return;
        if (tid < BM) {
            const int at = K % BK, p = at >> 4;
            char* r = st + tid * BK + 16 * (p ^ (tid & 7));
            for (int i = at & 15; i < 16; i++) r[i] = 0;
        }
        __syncthreads();
    };

    const int wm = wave >> 1, wn = wave & 1, lr = lane & 31;
    const int base_a = (wm * WM + lr) * BK, base_b = HALF + (wn * WM + lr) * BK;
    struct Half {
        i32x4 a[2][WT], b[2][WT];
    };
    auto load_half = [&](Half& f, const char* st, int h) {
#pragma unroll
        for (int s = 0; s < 2; s++) {
            const int off = 16 * ((4 * h + 2 * s + (lane >> 5)) ^ (lr & 7));
#pragma unroll
            for (int t = 0; t < WT; t++) f.a[s][t] = *reinterpret_cast<const i32x4*>(st + base_a + t * 32 * BK + off);
#pragma unroll
            for (int t = 0; t < WT; t++) f.b[s][t] = *reinterpret_cast<const i32x4*>(st + base_b + t * 32 * BK + off);
        }
    };
    i32x16 acc[WT][WT] = {};
    // B is the row operand: a lane then holds four adjacent columns of one row of C
    auto mfma = [&](const Half& f, int x) {
        const int s = x / (WT * WT), i = (x / WT) % WT, j = (i & 1) ? WT - 1 - x % WT : x % WT;
        acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(f.b[s][j], f.a[s][i], acc[i][j], 0, 0, 0);
    };
    constexpr int SG_MFMA = 0x008, SG_VMEM = 0x010, SG_DSR = 0x100;
    constexpr int PER = MFMAS / READS > 0 ? MFMAS / READS : 1;   // MFMAS between two reads
    auto phase1 = [&](Half& fa, Half& fb, char* st) {
        __builtin_amdgcn_s_waitcnt(0xC07F);   // fa's reads, a phase old
        load_half(fb, st, 1);
#pragma unroll
        for (int x = 0; x < MFMAS; x++) mfma(fa, x);
#pragma unroll
        for (int i = 0; i < READS; i++) {
            __builtin_amdgcn_sched_group_barrier(SG_DSR, 1, 0);
            __builtin_amdgcn_sched_group_barrier(SG_MFMA, PER, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    auto handover = [&] {
        __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0): this wave's copies have landed
        __syncthreads();
        __builtin_amdgcn_sched_barrier(0);
    };
    auto phase2 = [&](Half& fa, Half& fb, char* nx, bool more, int kb, char* st) {
        if (more) copy(kb, st);
        load_half(fa, nx, 0);
#pragma unroll
        for (int x = 0; x < MFMAS; x++) mfma(fb, x);
#pragma unroll
        for (int i = 0; i < READS; i++) {
            __builtin_amdgcn_sched_group_barrier(SG_DSR, 1, 0);
            if (more) __builtin_amdgcn_sched_group_barrier(SG_VMEM, 1, 0);
            __builtin_amdgcn_sched_group_barrier(SG_MFMA, PER, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    Half f0, f1;
    auto step = [&](char* cur, char* nxt, int kb) {   // copies block kb into cur once done with it
        phase1(f0, f1, cur);
        handover();
        phase2(f0, f1, nxt, true, kb, cur);
    };
    auto step_before_last = [&](char* cur, char* nxt) {
        phase1(f0, f1, cur);
        handover();
        clear_tail(nxt);
        phase2(f0, f1, nxt, false, 0, cur);
    };
    auto step_last = [&](char* cur) {
        phase1(f0, f1, cur);
#pragma unroll
        for (int x = 0; x < MFMAS; x++) mfma(f1, x);
    };
    // the last two blocks always run on st0 then st1: with an odd number the first goes to st1
    const bool odd = (nkb & 1) != 0;
    char *first = odd ? st1 : st0, *second = odd ? st0 : st1;
    copy(0, first);
    handover();
    if (nkb > 1) copy(1, second);
    else clear_tail(first);
    load_half(f0, first, 0);
    if (nkb == 1) {
        step_last(first);
    } else {
        int s = 0;
        if (odd) {
            step(st1, st0, 2);
            s = 1;
        }
        for (; s + 3 < nkb; s += 2) {
            step(st0, st1, s + 2);
            step(st1, st0, s + 3);
        }
        step_before_last(st0, st1);
        step_last(st1);
    }

    // Epilogue: 32 rows at a time through LDS of the wave's own, so that C is written in whole rows of the
    // wave's tile, 16 bytes a lane
    __syncthreads();   // every wave is done with the stages
    constexpr int ES = BF16 ? 2 : 4, PITCH = WM * ES + 16, LANES = WM * ES / 16;   // lanes of a row
    static_assert(2 * 32 * PITCH <= 2 * HALF, "two waves' rows fit a stage");
    char* mine = (wm ? st1 : st0) + wn * 32 * PITCH;
    const int64_t mw = m0 + wm * WM, nw = n0 + wn * WM;
    char* C = static_cast<char*>(g.c) + (mw * g.ldc + nw) * ES;
    auto store = [&](auto mode) {
        constexpr bool ANY = decltype(mode)::value;
#pragma unroll
        for (int i = 0; i < WT; i++) {
            const float sa = vec[0][wm * WM + 32 * i + lr];
#pragma unroll
            for (int j = 0; j < WT; j++)
#pragma unroll
                for (int q = 0; q < 4; q++) {
                    const int col = 32 * j + 8 * q + 4 * (lane >> 5);
                    const float4 sb = *reinterpret_cast<const float4*>(&vec[1][wn * WM + col]);
                    const float4 bi = *reinterpret_cast<const float4*>(&vec[2][wn * WM + col]);
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
                    __builtin_memcpy(d, &v, 16);   // any alignment: ldc is the caller's
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

template <int WT>
hipError_t launch_tiles(const GemmArgs& g, hipStream_t s) {
    constexpr int BM = 64 * WT;
    const int64_t tm = (g.M + BM - 1) / BM, tn = (g.N + BM - 1) / BM;
    const unsigned grid = (unsigned)(((tm * tn + 7) / 8) * 8);
    if (g.c_bf16) tile_kernel<WT, true><<<grid, 256, 0, s>>>(g, (int)tm, (int)tn);
    else tile_kernel<WT, false><<<grid, 256, 0, s>>>(g, (int)tm, (int)tn);
    return hipGetLastError();
}

}  // namespace

int64_t gemm_workspace_bytes(int64_t, int64_t N, int64_t K, int trans) { return trans ? N * ceil_to(K, 16) : 0; }

hipError_t launch_gemm(const GemmArgs& args, hipStream_t s) {
    GemmArgs g = args;
    if (g.trans) {
        int8_t* t = static_cast<int8_t*>(g.ws);
        g.b = t;
        g.ldb = ceil_to(g.K, 16);
        const dim3 grid((unsigned)((g.N + 63) / 64), (unsigned)((g.K + 63) / 64));
        transpose_kernel<<<grid, 256, 0, s>>>(args.b, args.ldb, g.K, g.N, t, g.ldb);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    const int64_t big = ((g.M + 255) / 256) * ((g.N + 255) / 256);
    return big >= 200 ? launch_tiles<4>(g, s) : launch_tiles<2>(g, s);
}

}  // namespace cfint8
