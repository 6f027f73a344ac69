// Sums over the LANES threads that hold a row, for gfx950: 16 or 64 neighbouring lanes, or a whole block of 256 or 1024.  Every
// thread gets the sum, by the same additions.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "tile_math.h"

namespace moshpit {

// v of another lane of the same 16 (CTRL: a DPP control).
template <int CTRL> __device__ __forceinline__ uint32_t lane_from(uint32_t v)
{
    return static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), CTRL, 0xf, 0xf, true));
}
template <int CTRL> __device__ __forceinline__ float lane_from(float v) { return __uint_as_float(lane_from<CTRL>(__float_as_uint(v))); }

template <int LANES> __device__ __forceinline__ float lanes_sum(float v)
{
    static_assert(LANES == 16 || LANES == 64);
    v += lane_from<0xB1>(v);             // the lane's neighbour
    v += lane_from<0x4E>(v);             // the other pair of four
    v += lane_from<0x141>(v);            // the other four of eight
    v += lane_from<0x140>(v);            // the other eight of sixteen
    if constexpr (LANES == 64) {
        const LanePair a = swap16(v, v);
        v = a.first + a.second;
        const LanePair b = swap32(v, v);
        v = b.first + b.second;
    }
    return v;
}

// The largest of a wave's 64 lanes.
__device__ __forceinline__ float lanes_max(float v)
{
    v = fmaxf(v, lane_from<0xB1>(v));
    v = fmaxf(v, lane_from<0x4E>(v));
    v = fmaxf(v, lane_from<0x141>(v));
    v = fmaxf(v, lane_from<0x140>(v));
    const LanePair a = swap16(v, v);
    v = fmaxf(a.first, a.second);
    const LanePair b = swap32(v, v);
    return fmaxf(b.first, b.second);
}

// lds: 16 floats that no thread still reads from the call before the last; a block's threads call it together.
template <int LANES> __device__ __forceinline__ float group_sum(float v, float *lds)
{
    if constexpr (LANES <= 64) return lanes_sum<LANES>(v);
    else {
        v = lanes_sum<64>(v);
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
        __syncthreads();
        v = lds[0];
#pragma unroll
        for (int n = 1; n < LANES / 64; ++n) v += lds[n];
        return v;
    }
}

// Two sums at once; lds: 32 floats.
template <int LANES> __device__ __forceinline__ void group_sums(float &a, float &b, float *lds)
{
    if constexpr (LANES <= 64) {
        a = lanes_sum<LANES>(a);
        b = lanes_sum<LANES>(b);
    } else {
        a = lanes_sum<64>(a);
        b = lanes_sum<64>(b);
        if ((threadIdx.x & 63) == 0) {
            lds[threadIdx.x >> 6] = a;
            lds[16 + (threadIdx.x >> 6)] = b;
        }
        __syncthreads();
        a = lds[0];
        b = lds[16];
#pragma unroll
        for (int n = 1; n < LANES / 64; ++n) {
            a += lds[n];
            b += lds[16 + n];
        }
    }
}

}  // namespace moshpit
