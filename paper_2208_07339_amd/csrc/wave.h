// Sums and ranks over the lanes of a wave.
#pragma once
#include <hip/hip_runtime.h>

namespace llmint8 {

// By the lanes of a row of 16 first, then the rows: a step is one or two instructions, where an exchange through LDS takes the time of
// thirty.
template <int CTRL, int ROWS, class V>
__device__ __forceinline__ V from_lane(V x, V none)
{
    if constexpr (sizeof(V) == 4) {
        return __builtin_bit_cast(V, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, none), __builtin_bit_cast(int, x), CTRL, ROWS, 0xf, false));
    } else {
        typedef int i2 __attribute__((ext_vector_type(2)));
        const i2 n = __builtin_bit_cast(i2, none), v = __builtin_bit_cast(i2, x);
        i2 r;
        r[0] = __builtin_amdgcn_update_dpp(n[0], v[0], CTRL, ROWS, 0xf, false);
        r[1] = __builtin_amdgcn_update_dpp(n[1], v[1], CTRL, ROWS, 0xf, false);
        return __builtin_bit_cast(V, r);
    }
}
// The value of a lane, the same one for all.
template <class V>
__device__ __forceinline__ V lane_of(V x, int lane)
{
    if constexpr (sizeof(V) == 4) {
        return __builtin_bit_cast(V, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), lane));
    } else {
        typedef int i2 __attribute__((ext_vector_type(2)));
        i2 v = __builtin_bit_cast(i2, x);
        v[0] = __builtin_amdgcn_readlane(v[0], lane);
        v[1] = __builtin_amdgcn_readlane(v[1], lane);
        return __builtin_bit_cast(V, v);
    }
}
// f over this lane and those below; all lanes take part.  f(x, none) = x.
template <class V, class F>
__device__ __forceinline__ V wave_upto(V x, V none, F f)
{
    constexpr int SHR = 0x110, BCAST15 = 0x142, BCAST31 = 0x143;  // from the lane that many below; a row's last lane to the next row(s)
    x = f(x, from_lane<SHR | 1, 0xf>(x, none));
    x = f(x, from_lane<SHR | 2, 0xf>(x, none));
    x = f(x, from_lane<SHR | 4, 0xf>(x, none));
    x = f(x, from_lane<SHR | 8, 0xf>(x, none));
    x = f(x, from_lane<BCAST15, 0xa>(x, none));
    x = f(x, from_lane<BCAST31, 0xc>(x, none));
    return x;
}
// f over all lanes, for all
template <class V, class F>
__device__ __forceinline__ V wave_reduce(V x, V none, F f)
{
    return lane_of(wave_upto(x, none, f), 63);
}

// Between a wave's accesses to memory that its lanes share: they are done in order, and so they are to be compiled.
__device__ __forceinline__ void wave_order()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
}

}  // namespace llmint8
