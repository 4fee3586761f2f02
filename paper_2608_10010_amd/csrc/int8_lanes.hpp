// Dot products of 8-bit codes by a wave's lanes, for lines that only one or two others meet.
#pragma once
#include <hip/hip_runtime.h>

namespace cfint8 {

// a value as 32-bit words, which is what lanes exchange
template <class V>
struct Words {
    uint32_t w[sizeof(V) / 4];
};

// a's upper lanes against b's lower ones (SPAN = 32), or a's odd rows of 16 lanes against b's even ones (16), and added
template <int SPAN, class V>
__device__ __forceinline__ V swap_add(V a, V b) {
    Words<V> x = __builtin_bit_cast(Words<V>, a), y = __builtin_bit_cast(Words<V>, b);
#pragma unroll
    for (int i = 0; i < (int)(sizeof(V) / 4); i++) {
        const auto z = SPAN == 32 ? __builtin_amdgcn_permlane32_swap(x.w[i], y.w[i], false, false)
                                  : __builtin_amdgcn_permlane16_swap(x.w[i], y.w[i], false, false);
        x.w[i] = z[0], y.w[i] = z[1];
    }
    return __builtin_bit_cast(V, x) + __builtin_bit_cast(V, y);
}

// v and that of the lane N further round in its sixteen
template <int N, class V>
__device__ __forceinline__ V rotate_add(V v) {
    Words<V> x = __builtin_bit_cast(Words<V>, v);
#pragma unroll
    for (int i = 0; i < (int)(sizeof(V) / 4); i++)
        x.w[i] = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x.w[i], 0x120 + N, 0xF, 0xF, false);
    return v + __builtin_bit_cast(V, x);
}

// sums over the lanes of four values (int, float, double): lanes 16 i .. of the result hold those of value 0, 2, 1, 3.
// Swaps of lanes' halves and rows leave a register for each two and then four values, sixteen lanes are added by
// rotations: the tree is that of exchanges with lanes 32, 16, 8, 4, 2 and 1 away
template <class V>
__device__ __forceinline__ V sum4(V a, V b, V c, V d) {
    const V s = swap_add<16>(swap_add<32>(a, b), swap_add<32>(c, d));
    return rotate_add<1>(rotate_add<2>(rotate_add<4>(rotate_add<8>(s))));
}
// the sum over the lanes of one, by the same tree
template <class V>
__device__ __forceinline__ V sum1(V a) {
    return sum4(a, a, a, a);
}
// the value that lanes 16 row .. hold
__device__ __forceinline__ int value_of_row(int row) { return row == 1 ? 2 : row == 2 ? 1 : row; }

}  // namespace cfint8
