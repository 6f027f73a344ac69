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
// Forms:
//   kBf16   bfloat16 matrices; weights are rounded to bfloat16 for their product, the rest is exact before the binary32 sums
//   kParts  binary32 matrices as three bfloat16 parts of 8 significant bits each, six products in place of one: what is left out is below 2^-21 of
//           a product and of its sign, 2^-24.5 of it on average.  At sixteen times the rate of the binary32 matrix instructions, so 2.7 times as fast
//   kF32    binary32 matrices by the binary32 matrix instructions, where the parts of deep heads do not fit the registers
// DP: the depth, rounded up to a multiple of 32 (zeros behind it).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "row_elems.h"
#include "tile_math.h"

namespace moshpit {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.693147180559945309417f;

enum Form { kF32 = 0, kBf16 = 1, kParts = 2 };

template <Form F> struct Num {
    static constexpr int DT = F == kBf16 ? 1 : 0;                     // type of the matrices, as in row_elems.h
    static constexpr int ES = F == kBf16 ? 2 : 4;                     // bytes of their elements
    static constexpr int PARTS = F == kParts ? 3 : 1;
    static constexpr int LS = F == kF32 ? 4 : 2, CE = 16 / LS;        // bytes of an element in LDS, elements of 16 bytes there
    typedef typename std::conditional<F == kF32, float, uint16_t>::type lds_t;
};

// Elements of a tile's row in LDS, and of a tile of `rows` rows, all its parts.
constexpr int row_elems_of(int DP) { return DP <= 32 ? 32 : DP <= 64 ? 64 : DP <= 128 ? 128 : 256; }
template <Form F, int DP> constexpr int tile_elems(int rows) { return Num<F>::PARTS * rows * row_elems_of(DP); }

// Where 16-byte chunk `chunk` of row `row` of a tile with LP elements a row lies, in elements.  Rows are a power of two long, so the chunks
// of a row are stored with their numbers xor a number of the row: 16 consecutive rows' same chunks then lie in different banks (for
// rows_times), and so do 4 consecutive rows' same 64 bytes (for the transposing reads of columns_times).
template <int CH> __device__ __forceinline__ int chunk_shift(int row)
{
    return CH >= 16 ? ((row & 3) << 2 | (row >> 2 & 3)) : CH == 8 ? ((row >> 1 & 1) << 2 | (row >> 2 & 3)) : (row >> 2 & 3);
}
template <Form F, int LP> __device__ __forceinline__ int chunk_at(int row, int chunk)
{
    constexpr int CE = Num<F>::CE;
    return row * LP + (chunk ^ chunk_shift<LP / CE>(row)) * CE;
}

// `count` elements of 4 or 2 bytes from p on that end after `left` of them; zeros behind.
template <int DT, int WORDS> __device__ __forceinline__ void load_words(const char *p, int left, u32x4 (&v)[WORDS])
{
    constexpr int ES = DT == 0 ? 4 : 2, EACH = 16 / ES;
    if (left >= EACH * WORDS) {
#pragma unroll
        for (int q = 0; q < WORDS; ++q) v[q] = load_vec<false, u32x4>(p + 16 * q);
        return;
    }
#pragma unroll
    for (int q = 0; q < WORDS; ++q) {
        v[q] = u32x4{0, 0, 0, 0};
#pragma unroll
        for (int k = 0; k < EACH; ++k)
            if (q * EACH + k < left) {
                if constexpr (DT == 0) v[q][k] = *reinterpret_cast<const uint32_t *>(p + 16 * q + k * ES);
                else v[q][k / 2] |= static_cast<uint32_t>(*reinterpret_cast<const uint16_t *>(p + 16 * q + k * ES)) << (16 * (k & 1));
            }
    }
}

// A unit: the elements of a row that are 16 bytes of a tile's (of each of its parts).
template <Form F> struct Unit {
    static constexpr int WORDS = Num<F>::CE * Num<F>::ES / 16;
    u32x4 v[WORDS];

    __device__ __forceinline__ void load(const char *p, int left) { load_words<Num<F>::DT, WORDS>(p, left, v); }
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int q = 0; q < WORDS; ++q) v[q] = u32x4{0, 0, 0, 0};
    }
};

// Upper halves of two words, a's in the lower half.
__device__ __forceinline__ uint32_t upper_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }

// Two binary32 values as pairs of bfloat16 parts, 8 significant bits each, cut off (so the largest do not round up to infinity).
__device__ __forceinline__ void split_pair(float a, float b, uint32_t (&part)[3])
{
#pragma unroll
    for (int q = 0; q < 3; ++q) {
        const uint32_t u = __float_as_uint(a), w = __float_as_uint(b);
        part[q] = upper_halves(u, w);
        a -= __uint_as_float(u & 0xffff0000u);
        b -= __uint_as_float(w & 0xffff0000u);
    }
}

// A unit's 16 bytes of every part.
template <Form F> __device__ __forceinline__ void parts_of(const Unit<F> &u, u32x4 (&part)[Num<F>::PARTS])
{
    if constexpr (F != kParts) part[0] = u.v[0];
    else
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            uint32_t p[3];
            split_pair(__uint_as_float(u.v[k / 2][2 * (k & 1)]), __uint_as_float(u.v[k / 2][2 * (k & 1) + 1]), p);
#pragma unroll
            for (int q = 0; q < 3; ++q) part[q][k] = p[q];
        }
}

// 32 columns held by a wave: lane l has units l / 32, 2 + l / 32, ... of column l % 32.
template <Form F, int DP> struct Held {
    static constexpr int CE = Num<F>::CE, COUNT = DP / (2 * CE), PARTS = Num<F>::PARTS;
    u32x4 v[PARTS][COUNT];

    // column: this lane's, from its first element on; `depth` elements, none where it is not `there`.
    __device__ __forceinline__ void load(const char *column, bool there, int depth)
    {
        const int half = threadIdx.x >> 5 & 1;
#pragma unroll
        for (int s = 0; s < COUNT; ++s) {
            const int at = (2 * s + half) * CE;
            Unit<F> u;
            u.clear();
            if (there && at < depth) u.load(column + at * Num<F>::ES, depth - at);
            u32x4 part[PARTS];
            parts_of<F>(u, part);
#pragma unroll
            for (int q = 0; q < PARTS; ++q) v[q][s] = part[q];
        }
    }
};

// The sum of products of two columns' elements (both halves' of the wave), in binary32.
template <Form F, int DP> __device__ __forceinline__ float columns_dot(const char *a, const char *b, bool there, int depth)
{
    constexpr int CE = Num<F>::CE, ES = Num<F>::ES, DT = Num<F>::DT;
    const int half = threadIdx.x >> 5 & 1;
    float sum = 0.f;
#pragma unroll
    for (int s = 0; s < DP / (2 * CE); ++s) {
        const int at = (2 * s + half) * CE;
        if (!there || at >= depth) continue;
        Unit<F> x, y;
        x.load(a + at * ES, depth - at);
        y.load(b + at * ES, depth - at);
#pragma unroll
        for (int q = 0; q < Unit<F>::WORDS; ++q)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const uint32_t u = x.v[q][k], w = y.v[q][k];
                if constexpr (DT == 0) sum = fmaf(__uint_as_float(u), __uint_as_float(w), sum);
                else sum = fmaf(__uint_as_float(u & 0xffff0000u), __uint_as_float(w & 0xffff0000u), fmaf(__uint_as_float(u << 16), __uint_as_float(w << 16), sum));
            }
    }
    const LanePair p = swap32(sum, sum);
    return p.first + p.second;
}

// Held columns out of LDS: they are rows 0 .. 31 of a tile.
template <Form F, int DP> struct Aside {
    const uint16_t *tile;                // (of one part: bfloat16)

    __device__ __forceinline__ static void put(const Held<F, DP> &held, uint16_t *into)
    {
#pragma unroll
        for (int s = 0; s < DP / 16; ++s) *reinterpret_cast<u32x4 *>(into + chunk_at<F, row_elems_of(DP)>(threadIdx.x & 31, 2 * s + (threadIdx.x >> 5 & 1))) = held.v[0][s];
    }
};

__device__ __forceinline__ f32x16 mfma_bf16(const u32x4 &a, const u32x4 &b, const f32x16 &c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// Products of parts, the smallest first.  Parts are cut off, so the second is below 2^-7 of its number and the third below 2^-15: the three products that
// are left out come to less than 2 * 2^-22 + 2^-30 of the whole.  (Numbers rounded to their parts would leave out 2^-24 and less, but the largest
// ones then round to infinity.)
constexpr int kTileParts[6] = {2, 1, 0, 1, 0, 0}, kHeldParts[6] = {0, 1, 2, 0, 1, 0};

// v, as a number that the compiler knows nothing of: addresses made of it are made anew where they are used, in an instruction or none, and do not
// take registers from one step to the next (there are dozens, for each of a kernel's tiles).
__device__ __forceinline__ uint32_t afresh(uint32_t v)
{
    asm volatile("" : "+v"(v));
    return v;
}
template <typename T> __device__ __forceinline__ T from_lds(const void *base, uint32_t bytes) { return *reinterpret_cast<const T *>(static_cast<const char *>(base) + bytes); }

// Where row lane % 32 of a tile has chunk lane / 32, in bytes; xor 32 s: chunk 2 s + lane / 32.
template <Form F, int DP> __device__ __forceinline__ uint32_t lane_row()
{
    const int row = threadIdx.x & 31, half = threadIdx.x >> 5 & 1;
    return afresh(static_cast<uint32_t>(chunk_at<F, row_elems_of(DP)>(row, half) * Num<F>::LS));
}

// sum + rows row0 .. row0 + 31 of the tile (ROWS rows a part) times the columns.
template <Form F, int DP, int ROWS>
__device__ __forceinline__ f32x16 rows_times(const typename Num<F>::lds_t *tile, int row0, const Held<F, DP> &held, f32x16 sum = f32x16{})
{
    constexpr int PARTS = Num<F>::PARTS, ROW_BYTES = row_elems_of(DP) * Num<F>::LS;
    const uint32_t at = lane_row<F, DP>();
#pragma unroll
    for (int s = 0; s < Held<F, DP>::COUNT; ++s) {
        u32x4 a[PARTS];
#pragma unroll
        for (int q = 0; q < PARTS; ++q) a[q] = from_lds<u32x4>(tile, (at ^ (32 * s)) + (q * ROWS + row0) * ROW_BYTES);
        if constexpr (F == kBf16) sum = mfma_bf16(a[0], held.v[0][s], sum);
        else if constexpr (F == kParts)
#pragma unroll
            for (int n = 0; n < 6; ++n) sum = mfma_bf16(a[kTileParts[n]], held.v[kHeldParts[n]][s], sum);
        else
#pragma unroll
            for (int e = 0; e < 4; ++e) sum = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a[0][e]), __uint_as_float(held.v[0][s][e]), sum, 0, 0, 0);
    }
    return sum;
}
template <Form F, int DP, int ROWS>
__device__ __forceinline__ f32x16 rows_times(const uint16_t *tile, int row0, const Aside<F, DP> &aside, f32x16 sum = f32x16{})
{
    constexpr int ROW_BYTES = row_elems_of(DP) * 2;
    const uint32_t at = lane_row<F, DP>();
#pragma unroll
    for (int s = 0; s < DP / 16; ++s) sum = mfma_bf16(from_lds<u32x4>(tile, (at ^ (32 * s)) + row0 * ROW_BYTES), from_lds<u32x4>(aside.tile, at ^ (32 * s)), sum);
    return sum;
}

// Weights of 32 rows as the matrix instructions take them.
template <Form F> struct Weights {
    u32x4 w[Num<F>::PARTS][2];
    __device__ __forceinline__ void take(const f32x16 &p)
    {
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if constexpr (F == kBf16) w[0][t][k] = bf16_pair(p[8 * t + 2 * k], p[8 * t + 2 * k + 1]);
                else {
                    uint32_t part[3];
                    split_pair(p[8 * t + 2 * k], p[8 * t + 2 * k + 1], part);
#pragma unroll
                    for (int q = 0; q < 3; ++q) w[q][t][k] = part[q];
                }
            }
    }
};
template <> struct Weights<kF32> {
    f32x16 w;
    __device__ __forceinline__ void take(const f32x16 &p) { w = p; }
};

// sum[m] += columns col0 + 32 m .. + 31 of the tile's rows row0 .. row0 + 31, each row times its weight.
template <Form F, int DP, int ROWS, int BLOCKS>
__device__ __forceinline__ void columns_times(const typename Num<F>::lds_t *tile, int row0, int col0, const Weights<F> &weights, f32x16 (&sum)[BLOCKS])
{
    constexpr int LP = row_elems_of(DP), PARTS = Num<F>::PARTS, ROW_BYTES = LP * Num<F>::LS;
    const int lane = threadIdx.x & 63, half = lane >> 5;
    if constexpr (F != kF32) {
        // A transposing read of 16 lanes takes 4 rows' 16 columns, 8 bytes a lane, and gives lane j column j of all 4.  Two make the 8 rows
        // of a lane; the second's are 8 rows on, where chunks lie xor 2.
        typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
        const int j = lane & 15;
        const uint32_t at = afresh(static_cast<uint32_t>((chunk_at<F, LP>(4 * half + (j >> 2), 2 * (lane >> 4 & 1) + (j >> 1 & 1)) + 4 * (j & 1)) * 2));
#pragma unroll
        for (int m = 0; m < BLOCKS; ++m) {
            const uint32_t low_at = at ^ static_cast<uint32_t>(2 * (col0 + 32 * m)), high_at = low_at ^ 32;
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                u32x4 a[PARTS];
#pragma unroll
                for (int q = 0; q < PARTS; ++q) {
                    const char *part = reinterpret_cast<const char *>(tile) + (q * ROWS + row0 + 16 * t) * ROW_BYTES;
                    const s16x4 low = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(part + low_at));
                    const s16x4 high = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(part + 8 * ROW_BYTES + high_at));
                    a[q] = __builtin_bit_cast(u32x4, __builtin_shufflevector(low, high, 0, 1, 2, 3, 4, 5, 6, 7));
                }
                if constexpr (F == kBf16) sum[m] = mfma_bf16(a[0], weights.w[0][t], sum[m]);
                else
#pragma unroll
                    for (int n = 0; n < 6; ++n) sum[m] = mfma_bf16(a[kTileParts[n]], weights.w[kHeldParts[n]][t], sum[m]);
            }
        }
    } else {
        // (row 8 g + 4 half + e: chunks lie xor (4 e + 2 g + half) % 16)
        const uint32_t at = afresh(static_cast<uint32_t>(4 * half * ROW_BYTES + (((lane >> 2 & 7) ^ half) * 16) + (lane & 3) * 4));
#pragma unroll
        for (int m = 0; m < BLOCKS; ++m)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int g = r >> 2, e = r & 3;
                sum[m] = __builtin_amdgcn_mfma_f32_32x32x2f32(from_lds<float>(tile, (at ^ static_cast<uint32_t>(4 * (col0 + 32 * m)) ^ (16 * (4 * e + 2 * (g & 1)))) + (row0 + 8 * g + e) * ROW_BYTES),
                                                              weights.w[r], sum[m], 0, 0, 0);
            }
    }
}

// ROWS rows on their way into a tile by THREADS threads, number `thread` of which this is.
template <Form F, int DP, int ROWS, int THREADS> struct Staged {
    static constexpr int CE = Num<F>::CE, LP = row_elems_of(DP), CH = LP / CE, COUNT = (ROWS * CH + THREADS - 1) / THREADS;
    static_assert(ROWS * CH % THREADS == 0 || COUNT == 1);            // (of a small tile some threads have nothing)
    Unit<F> unit[COUNT];

    // rows: the tile's first row, from its first element on; row r is read where bit r of `live` is set and is zeros elsewhere.
    __device__ __forceinline__ void load(const char *rows, int64_t row_bytes, uint64_t live, int depth, int thread)
    {
#pragma unroll
        for (int n = 0; n < COUNT; ++n) {
            const int row = (thread + n * THREADS) / CH, at = (thread + n * THREADS) % CH * CE;
            unit[n].clear();
            if (row < ROWS && (live >> row & 1) != 0 && at < depth) unit[n].load(rows + row * row_bytes + at * Num<F>::ES, depth - at);
        }
    }
    __device__ __forceinline__ void store(typename Num<F>::lds_t *tile, int thread) const
    {
#pragma unroll
        for (int n = 0; n < COUNT; ++n) {
            if (ROWS * CH % THREADS != 0 && thread >= ROWS * CH) continue;
            u32x4 part[Num<F>::PARTS];
            parts_of<F>(unit[n], part);
#pragma unroll
            for (int q = 0; q < Num<F>::PARTS; ++q)
                *reinterpret_cast<u32x4 *>(tile + q * ROWS * LP + chunk_at<F, LP>((thread + n * THREADS) / CH, (thread + n * THREADS) % CH)) = part[q];
        }
    }
};

// The same for rows that are whole 16-byte vectors (`chunks` of them), in the type that LDS has them in: from memory into LDS without passing through
// registers, a wave 1 KiB at a time: lane l's 16 bytes to where the wave's begin + 16 * l, so the lane reads the chunk that chunk_at() puts there.
template <Form F, int DP, int ROWS, int THREADS> struct Direct {
    static_assert(F != kParts);
    typedef typename Num<F>::lds_t lds_t;
    static constexpr int CE = Num<F>::CE, LP = row_elems_of(DP), CH = LP / CE, WAVES = THREADS / 64, EACH = 64 / CH, COUNT = ROWS / EACH / WAVES;      // rows of 1 KiB; KiB of a wave
    static_assert(COUNT >= 1 && ROWS % (EACH * WAVES) == 0);

    // Rows 0 .. last of the tile are there to be read; what is in the place of further ones is any row.
    __device__ __forceinline__ static void request(const char *rows, uint32_t row_bytes, int32_t last, int32_t chunks, lds_t *tile)
    {
        typedef __attribute__((address_space(3))) lds_t to_lds_t;
        const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const __amdgpu_buffer_rsrc_t from = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(rows), 0, 0xffffffffu, 0x00027000);
#pragma unroll
        for (int n = 0; n < COUNT; ++n) {
            const int begin = (wave * COUNT + n) * EACH, row = begin + lane / CH, chunk = (lane % CH) ^ chunk_shift<CH>(row);
            const uint32_t at = static_cast<uint32_t>(row < last ? row : last) * row_bytes + (chunk < chunks ? chunk * 16 : 0);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (to_lds_t *)(tile + begin * LP), 16, at, 0, 0, 0);
        }
    }
    // Behind a wait for all that was requested: what is behind the rows' chunks becomes zeros.
    __device__ __forceinline__ static void blank(int32_t chunks, lds_t *tile)
    {
        if (chunks == DP / CE) return;
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
        for (int n = 0; n < COUNT; ++n) {
            const int begin = (wave * COUNT + n) * EACH, chunk = (lane % CH) ^ chunk_shift<CH>(begin + lane / CH);
            if (chunk >= chunks && chunk < DP / CE) *reinterpret_cast<u32x4 *>(tile + begin * LP + lane * CE) = u32x4{0, 0, 0, 0};
        }
    }
    // And rows whose bit in `live` is not set.
    __device__ __forceinline__ static void trim(uint64_t live, lds_t *tile)
    {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
        for (int n = 0; n < COUNT; ++n) {
            const int begin = (wave * COUNT + n) * EACH;
            if ((live >> (begin + lane / CH) & 1) == 0) *reinterpret_cast<u32x4 *>(tile + begin * LP + lane * CE) = u32x4{0, 0, 0, 0};
        }
    }
    __device__ __forceinline__ static void wait() { __builtin_amdgcn_s_waitcnt(0x0f70); }              // vmcnt(0)
};
// Whether a matrix's heads can be read so: whole vectors, and a tile's offsets below 2^31.
inline bool direct_rows(const void *p, int64_t stride, int depth, int dtype)
{
    const int each = dtype == 0 ? 4 : 8;
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride % each == 0 && depth % each == 0 && stride <= (int64_t(1) << 22);
}

// Which tile of which peer's head block number `block` takes.  Tiles with the most work come first for all peers and heads (a peer's sequences may
// be longer than another's, so none is left to a single die), and a tile's blocks of the query heads that share keys go to the
// same die where the peers' heads of keys are a multiple of 8 (block b runs on die b % 8), another one for each tile.
struct Place {
    uint32_t tile;                       // 0: the one with the most work
    int64_t peer;
    int32_t kv_head, member;             // the head of keys, and the query head among those that share it
};
__device__ __forceinline__ Place place_of(uint32_t block, int64_t N, int32_t kv_heads, int32_t members)
{
    const uint32_t units = static_cast<uint32_t>(N) * kv_heads, turn = block / units;
    Place p;
    p.tile = turn / members;
    p.member = static_cast<int32_t>(turn % members);
    uint32_t unit = block % units + p.tile % units;
    unit = unit >= units ? unit - units : unit;
    p.peer = unit / kv_heads;
    p.kv_head = static_cast<int32_t>(unit % kv_heads);
    return p;
}

// Of both halves of the wave, which hold the same columns.
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
    constexpr int ES = DT == 0 ? 4 : 2;
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

// go(form, depth) with the kernels' form and their rounded depth for `depth` elements of type dtype.
template <typename Go> hipError_t by_depth(int dtype, int depth, Go go)
{
    using std::integral_constant;
    auto of_form = [&](auto form, auto deep) {
        if (depth <= 32) return go(form, integral_constant<int, 32>{});
        if (depth <= 64) return go(form, integral_constant<int, 64>{});
        if (depth <= 96) return go(form, integral_constant<int, 96>{});
        if (depth <= 128) return go(form, integral_constant<int, 128>{});
        if (depth <= 192) return go(deep, integral_constant<int, 192>{});
        return go(deep, integral_constant<int, 256>{});
    };
    return dtype == 0 ? of_form(integral_constant<Form, kParts>{}, integral_constant<Form, kF32>{}) : of_form(integral_constant<Form, kBf16>{}, integral_constant<Form, kBf16>{});
}

}  // namespace moshpit
