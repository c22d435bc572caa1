// A head of dim / 8 lanes on its way to the cache: what the kernels that store new tokens share.
#pragma once
#include "serving.hpp"
#include "tiles.hpp"

namespace eora {

// 2^e of a block, from its byte
__device__ __forceinline__ float power_of(unsigned byte)
{
    const unsigned low = 127 + SCALE_LEAST, high = 127 + SCALE_MOST;
    return __uint_as_float((byte < low ? low : (byte > high ? high : byte)) << 23);
}

// v plus the value of another lane of its row of 16
template <int CTRL>
__device__ __forceinline__ float plus_dpp(float v)
{
    return v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xF, 0xF, true));
}
// sum over the LPH lanes of a head, in all of them
template <int LPH>
__device__ __forceinline__ float sum_of_head(float v)
{
    v = plus_dpp<0xB1>(v);                                // lanes 1, 0, 3, 2 of each four
    v = plus_dpp<0x4E>(v);                                // lanes 2, 3, 0, 1
    v = plus_dpp<0x141>(v);                               // the eight lanes mirrored: the other four
    if constexpr (LPH >= 16) v = plus_dpp<0x140>(v);      // the sixteen mirrored: the other eight
    if constexpr (LPH >= 32) v += __shfl_xor(v, 16, 64);
    return v;
}

typedef _Float16 h4 __attribute__((ext_vector_type(4)));

}  // namespace eora
