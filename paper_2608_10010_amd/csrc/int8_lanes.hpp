// Dot products of 8-bit codes by a wave's lanes, for lines that only one or two others meet.
#pragma once
#include <hip/hip_runtime.h>

namespace cfint8 {

// sums over the lanes of four values: lanes 16 i .. of the result hold those of value 0, 2, 1, 3.  Swaps of lanes' halves
// and quarters leave a register for each two and then four values, sixteen lanes are added by rotations
template <class V>
__device__ __forceinline__ V sum4(V a, V b, V c, V d) {
    auto bits = [](V v) { return __builtin_bit_cast(uint32_t, v); };
    auto add = [](uint32_t x, uint32_t y) {
        return __builtin_bit_cast(uint32_t, (V)(__builtin_bit_cast(V, x) + __builtin_bit_cast(V, y)));
    };
    const auto x = __builtin_amdgcn_permlane32_swap(bits(a), bits(b), false, false);
    const auto y = __builtin_amdgcn_permlane32_swap(bits(c), bits(d), false, false);
    const auto z = __builtin_amdgcn_permlane16_swap(add(x[0], x[1]), add(y[0], y[1]), false, false);
    uint32_t s = add(z[0], z[1]);
    s = add(s, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)s, 0x128, 0xF, 0xF, false));
    s = add(s, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)s, 0x124, 0xF, 0xF, false));
    s = add(s, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)s, 0x122, 0xF, 0xF, false));
    s = add(s, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)s, 0x121, 0xF, 0xF, false));
    return __builtin_bit_cast(V, s);
}
// the value that lanes 16 row .. hold
__device__ __forceinline__ int value_of_row(int row) { return row == 1 ? 2 : row == 2 ? 1 : row; }

}  // namespace cfint8
