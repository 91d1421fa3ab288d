// Reductions over neighbouring lanes of a wavefront without a trip through LDS.
#pragma once

#include <hip/hip_runtime.h>

namespace ssm {

template <int CONTROL, class V> __device__ __forceinline__ V exchanged(V v)
{
    static_assert(sizeof(V) == 4, "one register");
    const int x = __builtin_bit_cast(int, v);
    return __builtin_bit_cast(V, __builtin_amdgcn_update_dpp(x, x, CONTROL, 0xf, 0xf, false));
}
// Over groups of 2^lanes neighbouring lanes, the result in all of them: lanes exchange within four, within eight and sixteen by mirroring
// (their fours and eights hold one value by then), rows of sixteen and halves of the wavefront by swaps.
template <class V, class F> __device__ __forceinline__ V over_group(V v, int lanes, F op)
{
    if (lanes >= 1) v = op(v, exchanged<0xb1>(v));           // quad_perm 1 0 3 2
    if (lanes >= 2) v = op(v, exchanged<0x4e>(v));           // quad_perm 2 3 0 1
    if (lanes >= 3) v = op(v, exchanged<0x141>(v));          // row_half_mirror
    if (lanes >= 4) v = op(v, exchanged<0x140>(v));          // row_mirror
    if (lanes >= 5) {
        const unsigned x = __builtin_bit_cast(unsigned, v);
        const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
        const unsigned mine = r[0], other = r[1];            // (a bit cast of r[1] itself reads r[0])
        v = op(__builtin_bit_cast(V, mine), __builtin_bit_cast(V, other));
    }
    if (lanes >= 6) {
        const unsigned x = __builtin_bit_cast(unsigned, v);
        const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
        const unsigned mine = r[0], other = r[1];            // (a bit cast of r[1] itself reads r[0])
        v = op(__builtin_bit_cast(V, mine), __builtin_bit_cast(V, other));
    }
    return v;
}

}  // namespace ssm
