// Short runs of consecutive row elements as binary32 values, for gfx950: whole runs as 128-bit accesses at
// any element address, single elements for the ends of rows.  DT: 0 = binary32, 1 = bfloat16.
#pragma once

#include "row_vec.h"

namespace moshpit {

// Block b of n runs on die b % 8: which of n consecutive pieces of work it takes, so that each die takes a run of them.
__device__ __forceinline__ uint32_t die_run(uint32_t b, uint32_t n)
{
    const uint32_t die = b % 8, each = n / 8, more = n % 8;
    return die * each + (die < more ? die : more) + b / 8;
}

template <int DT> __device__ __forceinline__ float load_one(const void *p)
{
    if constexpr (DT == 0) return *static_cast<const float *>(p);
    else return __uint_as_float(static_cast<uint32_t>(*static_cast<const uint16_t *>(p)) << 16);
}

template <int DT> __device__ __forceinline__ void store_one(void *p, float f)
{
    if constexpr (DT == 0) *static_cast<float *>(p) = f;
    else *static_cast<uint16_t *>(p) = bf16_one(f);
}

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// C elements (4 or 8) from p on.
template <int DT, int C, bool NT = false> __device__ __forceinline__ void load_elems(const char *p, float (&f)[C])
{
    static_assert(C == 4 || C == 8);
    if constexpr (DT == 0) {
#pragma unroll
        for (int k = 0; k < C; k += 4) {
            const f32x4 v = load_vec<NT, f32x4>(p + 4 * k);
            f[k] = v.x; f[k + 1] = v.y; f[k + 2] = v.z; f[k + 3] = v.w;
        }
    } else if constexpr (C == 8) {
        Vec<1, 8>::widen(load_vec<NT, u32x4>(p), f);
    } else {
        const u32x2 v = load_vec<NT, u32x2>(p);
        f[0] = __uint_as_float(v.x << 16); f[1] = __uint_as_float(v.x & 0xffff0000u);
        f[2] = __uint_as_float(v.y << 16); f[3] = __uint_as_float(v.y & 0xffff0000u);
    }
}

template <int DT, int C, bool NT = false> __device__ __forceinline__ void store_elems(char *p, const float (&f)[C])
{
    static_assert(C == 4 || C == 8);
    if constexpr (DT == 0) {
#pragma unroll
        for (int k = 0; k < C; k += 4) store_vec<NT, f32x4>(p + 4 * k, f32x4{f[k], f[k + 1], f[k + 2], f[k + 3]});
    } else if constexpr (C == 8) {
        store_vec<NT, u32x4>(p, Vec<1, 8>::narrow(f));
    } else {
        store_vec<NT, u32x2>(p, u32x2{bf16_pair(f[0], f[1]), bf16_pair(f[2], f[3])});
    }
}

}  // namespace moshpit
