// What the attention kernels share, for gfx950: tiles of rows (keys, values, queries) in LDS, columns (queries or keys) that a wave holds
// in registers, and the two products between them.  A wave's sums are blocks of 32 x 32 in the matrix instructions' layout:
// lane l holds column l % 32, rows 8 * (r / 4) + 4 * (l / 32) + r % 4 for r = 0 .. 15.
//
// Both products of attention have a tile of rows on one side and 32 columns on the other:
//   rows_times      block[row][column] += sum over depth of tile[row][depth] * held[column][depth]          (scores)
//   columns_times   block[depth][column] += sum over rows of tile[row][depth] * weight[row][column]          (sums of rows)
// The weights of the second are blocks of the first as they lie in the lanes: the order of the summed index may be any, as
// long as the tile is read in the same one, so weights never move between lanes.
//
// DT: 0 = binary32, by the binary32 matrix instructions; 1 = bfloat16, weights rounded to bfloat16 for the product.  DP: the depth, rounded up
// to a multiple of 32 (zeros behind it).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "row_elems.h"
#include "tile_math.h"

namespace moshpit {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.693147180559945309417f;

template <int DT> struct Num;
template <> struct Num<0> {
    typedef float lds_t;
    static constexpr int ES = 4, CE = 4;                              // bytes of an element, elements of 16 bytes
};
template <> struct Num<1> {
    typedef uint16_t lds_t;
    static constexpr int ES = 2, CE = 8;
};

constexpr int row_elems_of(int DP) { return DP <= 32 ? 32 : DP <= 64 ? 64 : DP <= 128 ? 128 : 256; }

// Where 16-byte chunk `chunk` of row `row` of a tile with LP elements a row lies, in elements.  Rows are a power of two long, so the chunks
// of a row are stored with their numbers xor a number of the row: 16 consecutive rows' same chunks then lie in different banks (for
// rows_times), and so do 4 consecutive rows' same 64 bytes (for the transposing reads of columns_times).
template <int DT, int LP> __device__ __forceinline__ int chunk_at(int row, int chunk)
{
    constexpr int CE = Num<DT>::CE, CH = LP / CE;
    const int moved = CH >= 16 ? ((row & 3) << 2 | (row >> 2 & 3)) : CH == 8 ? ((row >> 1 & 1) << 2 | (row >> 2 & 3)) : (row >> 2 & 3);
    return row * LP + (chunk ^ moved) * CE;
}

// 16 bytes of a row from p on, of which `left` elements are the row's; zeros behind them.
template <int DT> __device__ __forceinline__ u32x4 load_chunk(const char *p, int left)
{
    constexpr int ES = Num<DT>::ES, CE = Num<DT>::CE;
    if (left >= CE) return load_vec<false, u32x4>(p);
    u32x4 v = {0, 0, 0, 0};
#pragma unroll
    for (int k = 0; k < CE; ++k)
        if (k < left) {
            if constexpr (DT == 0) v[k] = *reinterpret_cast<const uint32_t *>(p + k * ES);
            else v[k / 2] |= static_cast<uint32_t>(*reinterpret_cast<const uint16_t *>(p + k * ES)) << (16 * (k & 1));
        }
    return v;
}

// 32 columns held by a wave: lane l has chunks l / 32, 2 + l / 32, ... of column l % 32.
template <int DT, int DP> struct Held {
    static constexpr int CE = Num<DT>::CE, COUNT = DP / (2 * CE);
    u32x4 v[COUNT];

    // column: this lane's, from its first element on; `depth` elements, none where it is not `there`.
    __device__ __forceinline__ void load(const char *column, bool there, int depth)
    {
        const int half = threadIdx.x >> 5 & 1;
#pragma unroll
        for (int s = 0; s < COUNT; ++s) {
            const int at = (2 * s + half) * CE;
            v[s] = there && at < depth ? load_chunk<DT>(column + at * Num<DT>::ES, depth - at) : u32x4{0, 0, 0, 0};
        }
    }
};

// Rows row0 .. row0 + 31 of the tile times the columns.
template <int DT, int DP> __device__ __forceinline__ f32x16 rows_times(const typename Num<DT>::lds_t *tile, int row0, const Held<DT, DP> &held)
{
    constexpr int LP = row_elems_of(DP);
    const int row = row0 + (threadIdx.x & 31), half = threadIdx.x >> 5 & 1;
    f32x16 sum = {};
#pragma unroll
    for (int s = 0; s < Held<DT, DP>::COUNT; ++s) {
        const u32x4 a = *reinterpret_cast<const u32x4 *>(tile + chunk_at<DT, LP>(row, 2 * s + half));
        if constexpr (DT == 1) sum = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, held.v[s]), sum, 0, 0, 0);
        else
#pragma unroll
            for (int e = 0; e < 4; ++e) sum = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a[e]), __uint_as_float(held.v[s][e]), sum, 0, 0, 0);
    }
    return sum;
}

// Weights of 32 rows as the matrix instructions take them.
template <int DT> struct Weights;
template <> struct Weights<0> {
    f32x16 w;
    __device__ __forceinline__ explicit Weights(const f32x16 &p) : w(p) {}
};
template <> struct Weights<1> {
    u32x4 w[2];
    __device__ __forceinline__ explicit Weights(const f32x16 &p)
    {
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int k = 0; k < 4; ++k) w[t][k] = bf16_pair(p[8 * t + 2 * k], p[8 * t + 2 * k + 1]);
    }
};

// sum + columns col0 .. col0 + 31 of the tile's rows row0 .. row0 + 31, each row times its weight.
template <int DT, int LP>
__device__ __forceinline__ f32x16 columns_times(const typename Num<DT>::lds_t *tile, int row0, int col0, const Weights<DT> &weights, f32x16 sum)
{
    const int lane = threadIdx.x & 63, half = lane >> 5;
    if constexpr (DT == 1) {
        typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
        const int j = lane & 15, row = row0 + 4 * half + (j >> 2), chunk = col0 / 8 + 2 * (lane >> 4 & 1) + (j >> 1 & 1), in = 4 * (j & 1);
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const s16x4 low = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(tile + chunk_at<DT, LP>(row + 16 * t, chunk) + in));
            const s16x4 high = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(tile + chunk_at<DT, LP>(row + 16 * t + 8, chunk) + in));
            const s16x8 a = __builtin_shufflevector(low, high, 0, 1, 2, 3, 4, 5, 6, 7);
            sum = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, weights.w[t]), sum, 0, 0, 0);
        }
    } else {
        const int col = col0 + (lane & 31);
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int row = row0 + 8 * (r >> 2) + 4 * half + (r & 3);
            sum = __builtin_amdgcn_mfma_f32_32x32x2f32(tile[chunk_at<DT, LP>(row, col >> 2) + (col & 3)], weights.w[r], sum, 0, 0, 0);
        }
    }
    return sum;
}

// ROWS rows on their way into a tile by THREADS threads, number `thread` of which this is.
template <int DT, int DP, int ROWS, int THREADS> struct Staged {
    static constexpr int CE = Num<DT>::CE, LP = row_elems_of(DP), CH = LP / CE, COUNT = (ROWS * CH + THREADS - 1) / THREADS;
    static_assert(ROWS * CH % THREADS == 0 || COUNT == 1);            // (of a small tile some threads have nothing)
    u32x4 v[COUNT];

    // rows: the tile's first row, from its first element on; row r is read where bit r of `live` is set and is zeros elsewhere.
    __device__ __forceinline__ void load(const char *rows, int64_t row_bytes, uint64_t live, int depth, int thread)
    {
#pragma unroll
        for (int n = 0; n < COUNT; ++n) {
            const int row = (thread + n * THREADS) / CH, at = (thread + n * THREADS) % CH * CE;
            v[n] = row < ROWS && (live >> row & 1) != 0 && at < depth ? load_chunk<DT>(rows + row * row_bytes + at * Num<DT>::ES, depth - at) : u32x4{0, 0, 0, 0};
        }
    }
    __device__ __forceinline__ void store(typename Num<DT>::lds_t *tile, int thread) const
    {
#pragma unroll
        for (int n = 0; n < COUNT; ++n)
            if (ROWS * CH % THREADS == 0 || thread < ROWS * CH)
                *reinterpret_cast<u32x4 *>(tile + chunk_at<DT, LP>((thread + n * THREADS) / CH, (thread + n * THREADS) % CH)) = v[n];
    }
    // Infinities and NaN to zeros; bit r of what is returned: row r had some among this thread's.
    __device__ __forceinline__ uint64_t clean(int thread)
    {
        uint64_t found = 0;
#pragma unroll
        for (int n = 0; n < COUNT; ++n) {
            bool any = false;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                uint32_t w = v[n][k];
                if constexpr (DT == 0) {
                    if ((w & 0x7f800000u) == 0x7f800000u) w = 0;
                } else {
                    if ((w & 0x7f800000u) == 0x7f800000u) w &= 0xffffu;
                    if ((w & 0x7f80u) == 0x7f80u) w &= 0xffff0000u;
                }
                any = any || w != v[n][k];
                v[n][k] = w;
            }
            if (any) found |= uint64_t(1) << ((thread + n * THREADS) / CH);
        }
        return found;
    }
};

// The column's sums of both halves of the wave.
__device__ __forceinline__ float halves_sum(float v)
{
    const LanePair p = swap32(v, v);
    return p.first + p.second;
}
__device__ __forceinline__ float halves_max(float v)
{
    const LanePair p = swap32(v, v);
    return fmaxf(p.first, p.second);
}

__device__ __forceinline__ int32_t wave_min(int32_t v)
{
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) {
        const int32_t other = __shfl_xor(v, off, 64);
        v = other < v ? other : v;
    }
    return v;
}
__device__ __forceinline__ int32_t wave_max(int32_t v) { return -wave_min(-v); }

// Writes a column's rows (depths col0 .. + 31 of the block) to `to`, its place for depth 0; `depth` elements in all.
template <int DT> __device__ __forceinline__ void store_column(char *to, int col0, int depth, const f32x16 &block, float factor)
{
    constexpr int ES = Num<DT>::ES;
    const int half = threadIdx.x >> 5 & 1;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        const int at = col0 + 8 * g + 4 * half, left = depth - at;
        float f[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) f[k] = block[4 * g + k] * factor;
        if (left >= 4) store_elems<DT, 4>(to + at * ES, f);
        else
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (k < left) store_one<DT>(to + (at + k) * ES, f[k]);
    }
}

}  // namespace moshpit
