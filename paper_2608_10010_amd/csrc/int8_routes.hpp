// Which kernels a call's sizes take: host code without HIP.
#pragma once
#include <cstdint>

namespace cfint8 {

constexpr int64_t UNITS = 256;         // compute units
constexpr int RANKED_EXPERTS = 256;    // experts among which the slot-by-slot kernel ranks

// ---------------------------------------------------------------- product

// Route, by estimated time in us.  One or two rows take dot products of whole lines, except where K leaves much of a
// wave's 2048 codes empty and there are workgroups of 16 columns for a part of the units only (1 x 14336 x 4096 12.7 us
// against 13.4 through LDS, 1 x 28672 x 8192 40 against 49, 1 x 1000 x 4096 2.8 against 3.5; 2 x 512 x 512 2.7 against 2.3).
// Up to 16 rows whose 16-column workgroups fit the units at once take these, eight waves where K gives each at least two
// blocks (16 x 4096 x 14336 13.7 us against 17.7 with 32 x 32 tiles; 16 x 1024 x 1024 3.2 us against 2.7 with four), up to
// 32 rows tiles of 32 x 32, which have more of the weight on its way than larger ones (16 x 14336 x 4096 13.9 us against
// 15.8 with 64 x 64, 20 x 10000 x 1000 5.6 against 6.1).  All else goes by the time of a tile's block of 128 codes and what
// a tile costs besides, as measured with one tile on every unit (us; times with K = 4096: 256 x 256 67, 256 x 128 39,
// 128 x 128 23, 64 x 128 15.8, 64 x 64 10.4, 32 x 32 6.6): the smaller tiles spend more on a product but fill the units
// with fewer rows.
enum Kernel { DOT, FEW4, FEW8, FEW32, T64, T64_128, T128, T256_128, T256 };

struct Route {
    Kernel kernel;
    double us;
};

// b [N][K], or [K][N] for the tile kernels
inline Route route_direct(int64_t M, int64_t N, int64_t K, bool trans) {
    auto tiles = [&](int64_t bm, int64_t bn) { return ((M + bm - 1) / bm) * ((N + bn - 1) / bn); };
    const double blocks = (double)((K + 127) / 128);
    if (!trans && M <= 2 && (K >= 2048 || tiles(16, 16) >= 2 * UNITS)) return {DOT, 2.5 + (double)N * (double)K / 5e6};
    if (!trans && M <= 16 && tiles(16, 16) <= UNITS) return {K >= 2048 ? FEW8 : FEW4, 2.5 + 0.07 * blocks};
    auto cost = [&](int64_t bm, int64_t bn, double once, double tile, double block) {
        return once + (double)((tiles(bm, bn) + UNITS - 1) / UNITS) * (tile + block * blocks);
    };
    if (!trans && M <= 32) return {FEW32, cost(32, 32, 2.5, 0.3, 0.11)};
    const Route all[6] = {{FEW32, cost(32, 32, 2.5, 0.3, 0.11)},    {T64, cost(64, 64, 2.0, 0.5, trans ? 0.33 : 0.235)},
                          {T64_128, cost(64, 128, 2.5, 1.0, 0.345)}, {T128, cost(128, 128, 0.0, 4.0, 0.59)},
                          {T256_128, cost(256, 128, 0.0, 6.0, 1.02)}, {T256, cost(256, 256, 0.0, 8.0, 1.83)}};
    int best = trans ? 1 : 0;
    for (int i = best + 1; i < 6; i++)
        if (all[i].us < all[best].us) best = i;
    return all[best];
}

// A [K][N] operand is read as it lies, or turned into the workspace first, which costs a pass over it (at 4.4 TB/s) and a
// launch but leaves the kernels that split K among the waves to few rows: with few columns (16 x 1024 x 4096 9.0 us against
// 12.7 as it lies; 16 x 4096 x 14336 43 against 55, 16 x 4096 x 4096 16.0 against 11.9, 4096 x 4096 x 14336 235 against 210)
inline bool turned(int64_t M, int64_t N, int64_t K) {
    return 3.5 + (double)N * (double)K / 2.2e6 + route_direct(M, N, K, false).us < route_direct(M, N, K, true).us;
}

// ---------------------------------------------------------------- mixture-of-experts layer

// Slot by slot or expert by expert, by estimated time in us: three launches and their latencies, the weights of the
// experts that T tokens take on average at 5.4 TB/s and those that slots share at 6.5, or 6 us for each 512
// workgroups of 32 columns, which rank E logits first (fp32's workgroups have 16 columns and take half as long); or five
// launches and the experts' weights at 5.2 TB/s (fp32: 4.6).  (1 token, 8 of 64 experts of 2048 x 1024: 18 us against 40; 4
// tokens 46 against 52; 12 tokens, 4 of 128 60 against 74; 16 tokens, 8 of 128 of 2048 x 768 107 against 102; 64 tokens, 2
// of 16 103 against 45; fp32, 7 tokens, 2 of 16 of 4096 x 2048 68 against 77.)
template <int P>
inline bool by_slots(int64_t T, int64_t E, int64_t k, int64_t H, int64_t I) {
    if (E > RANKED_EXPERTS) return false;
    const double weights = 3e-6 * (double)H * (double)I, slots = (double)(T * k);   // 1 MB takes 1 us at 1 TB/s
    const double rounds = slots * (double)((I + 31) / 32) / (2.0 * UNITS), chunks = (double)((E + 63) / 64);
    double untaken = 1;
    for (int64_t t = 0; t < T; t++) untaken *= 1 - (double)k / (double)E;
    const double taken = (double)E * (1 - untaken);
    const double read = taken * weights / 5.4 + (slots - taken) * weights / 6.5;
    return 10 + (read > 6 * rounds ? read : 6 * rounds) + 0.6 * rounds * chunks * chunks < 25 + taken * weights / (P == 4 ? 4.6 : 5.2);
}

}  // namespace cfint8
