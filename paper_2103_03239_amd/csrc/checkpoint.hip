// Activations saved in 8 bits and restored, for gfx950 (the form: checkpoint_codes.h).
//
// Bound by HBM: saving reads the activations once and writes a quarter (binary32) or half (bfloat16) of that.
// A lane holds 16 bytes of consecutive elements, so 4 (bfloat16) or 8 neighbouring lanes hold a group of 32 and find its largest
// element with two or three exchanges; a row takes whole groups of lanes.  Activations are read and restored with streaming
// accesses, the codes are written with plain ones: 16 x 4096 x 4096 bfloat16 saved and restored in 242 us, with streaming
// stores of the codes in 265.
#include <hip/hip_runtime.h>

#include "checkpoint_codes.h"
#include "local_ops.h"

namespace moshpit {
namespace {

constexpr int kBlock = 256, kUnits = 4;                // units of a lane
constexpr int unit_elems(int dtype) { return dtype == 0 ? 4 : 8; }

// A unit is 16 bytes of elements of a row; a row takes `row_units` of them, whole groups.
struct Units {
    int64_t rows, width, stride, groups;
    int64_t count;                       // rows * row_units
    uint32_t row_units, magic;           // magic: of a division by row_units < kBlock * kUnits of numbers below twice that
};

// Where a block's units lie: row `row` + `down` and element `at` of it, for unit n of this thread.
struct Span {
    int64_t row;
    uint32_t rest;                       // the block's first unit is number `rest` of its row
    __device__ __forceinline__ explicit Span(const Units &u)
    {
        const int64_t first = int64_t(blockIdx.x) * (kBlock * kUnits);
        row = first / u.row_units;
        rest = static_cast<uint32_t>(first - row * u.row_units);
    }
    template <int VEC> __device__ __forceinline__ void place(const Units &u, int n, uint32_t &down, int32_t &at) const
    {
        const uint32_t unit = rest + n * kBlock + threadIdx.x;
        if (u.row_units >= kBlock * kUnits) down = unit >= u.row_units ? 1 : 0;
        else down = __umulhi(unit, u.magic);
        at = static_cast<int32_t>(unit - down * u.row_units) * VEC;
    }
};

// A unit as it lies in memory; most(): the largest of its elements' bits without the signs.
template <int DT> struct Unit;
template <> struct Unit<0> {
    u32x4 w;
    __device__ __forceinline__ void load(const char *p) { w = load_vec<true, u32x4>(p); }
    __device__ __forceinline__ void put(int k, const char *p) { w[k] = *reinterpret_cast<const uint32_t *>(p); }
    __device__ __forceinline__ void move_down(int n)                  // elements n .. to 0 .., zeros behind them
    {
        w = n == 1 ? u32x4{w[1], w[2], w[3], 0} : n == 2 ? u32x4{w[2], w[3], 0, 0} : u32x4{w[3], 0, 0, 0};
    }
    __device__ __forceinline__ uint32_t most() const
    {
        uint32_t m = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t b = w[k] & 0x7fffffffu;
            m = b > m ? b : m;
        }
        return m;
    }
    __device__ __forceinline__ void widen(float (&f)[4]) const
    {
#pragma unroll
        for (int k = 0; k < 4; ++k) f[k] = __uint_as_float(w[k]);
    }
};
template <> struct Unit<1> {
    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
    u32x4 w;
    __device__ __forceinline__ void load(const char *p) { w = load_vec<true, u32x4>(p); }
    __device__ __forceinline__ void put(int k, const char *p)
    {
        w[k >> 1] |= static_cast<uint32_t>(*reinterpret_cast<const uint16_t *>(p)) << (16 * (k & 1));
    }
    __device__ __forceinline__ void move_down(int n)
    {
        uint64_t low = uint64_t(w[1]) << 32 | w[0], high = uint64_t(w[3]) << 32 | w[2];
        if (n >= 4) {
            low = high;
            high = 0;
        }
        const int bits = 16 * (n & 3);
        if (bits > 0) {
            low = low >> bits | high << (64 - bits);
            high >>= bits;
        }
        w = u32x4{static_cast<uint32_t>(low), static_cast<uint32_t>(low >> 32), static_cast<uint32_t>(high), static_cast<uint32_t>(high >> 32)};
    }
    __device__ __forceinline__ uint32_t most() const                  // two elements at a time
    {
        u16x2 m = {0, 0};
#pragma unroll
        for (int k = 0; k < 4; ++k) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, w[k] & 0x7fff7fffu));
        return static_cast<uint32_t>(m.x > m.y ? m.x : m.y) << 16;
    }
    __device__ __forceinline__ void widen(float (&f)[8]) const { Vec<1, 8>::widen(w, f); }
};

typedef uint16_t half_t __attribute__((aligned(1)));
typedef uint32_t word_t __attribute__((aligned(1)));
typedef u32x2 words_t __attribute__((aligned(1)));
__device__ __forceinline__ void store_codes(int8_t *p, const uint32_t (&w)[1]) { *reinterpret_cast<word_t *>(p) = w[0]; }
__device__ __forceinline__ void store_codes(int8_t *p, const uint32_t (&w)[2]) { *reinterpret_cast<words_t *>(p) = u32x2{w[0], w[1]}; }
template <bool NT> __device__ __forceinline__ void load_codes(const int8_t *p, uint32_t (&w)[1])
{
    w[0] = NT ? __builtin_nontemporal_load(reinterpret_cast<const word_t *>(p)) : *reinterpret_cast<const word_t *>(p);
}
template <bool NT> __device__ __forceinline__ void load_codes(const int8_t *p, uint32_t (&w)[2])
{
    const u32x2 v = NT ? __builtin_nontemporal_load(reinterpret_cast<const words_t *>(p)) : *reinterpret_cast<const words_t *>(p);
    w[0] = v.x;
    w[1] = v.y;
}

template <int DT>
__global__ __launch_bounds__(kBlock) void checkpoint_kernel(const char *__restrict__ x, Units u, int8_t *__restrict__ codes,
                                                            uint8_t *__restrict__ scales)
{
    constexpr int ES = DT == 0 ? 4 : 2, kVec = unit_elems(DT);
    const Span span(u);
    const int32_t width = static_cast<int32_t>(u.width);
    const int64_t rows = u.rows - span.row;
    x += span.row * u.stride * ES;
    codes += span.row * u.width;
    scales += span.row * u.groups;
    const uint32_t stride = static_cast<uint32_t>(u.stride * ES);
    Unit<DT> e[kUnits];
    uint32_t down[kUnits];
    int32_t at[kUnits];
#pragma unroll
    for (int n = 0; n < kUnits; ++n) {
        span.place<kVec>(u, n, down[n], at[n]);
        e[n] = Unit<DT>{};
        if (down[n] >= rows) at[n] = width;
        if (at[n] >= width) continue;
        const char *from = x + uint64_t(down[n]) * stride + at[n] * ES;
        // a row's last elements, where they are no whole unit: the row's last unit's worth moved to their place, one access
        if (at[n] + kVec <= width) e[n].load(from);
        else if (width >= kVec) {
            e[n].load(from - (at[n] + kVec - width) * ES);
            e[n].move_down(at[n] + kVec - width);
        } else
#pragma unroll
            for (int k = 0; k < kVec; ++k)
                if (at[n] + k < width) e[n].put(k, from + k * ES);
    }
#pragma unroll
    for (int n = 0; n < kUnits; ++n) {
        uint32_t most = e[n].most();
#pragma unroll
        for (int off = 1; off < kCheckpointGroup / kVec; off <<= 1) {
            const uint32_t other = __shfl_xor(most, off, 64);
            most = other > most ? other : most;
        }
        if (at[n] >= width) continue;
        const uint32_t byte = scale_byte(most);
        if (threadIdx.x % (kCheckpointGroup / kVec) == 0) scales[uint64_t(down[n]) * static_cast<uint32_t>(u.groups) + at[n] / static_cast<int32_t>(kCheckpointGroup)] = static_cast<uint8_t>(byte);
        float f[kVec];
        e[n].widen(f);
        uint32_t w[kVec / 4] = {};
        if (byte != kScaleNaN) {
            if (byte == kScaleTop) keep_finite(f);
            const float factor = to_code_factor(byte);
#pragma unroll
            for (int k = 0; k < kVec / 4; ++k) w[k] = pack_codes(f + 4 * k, factor);
        }
        int8_t *to = codes + uint64_t(down[n]) * static_cast<uint32_t>(width) + at[n];
        if (at[n] + kVec <= width) store_codes(to, w);
        else {                                                        // 4, 2 and 1 codes as there are
            const int left = width - at[n];
            uint32_t v = w[0];
            if (left & 4) {
                *reinterpret_cast<word_t *>(to) = v;
                to += 4;
                v = w[kVec / 4 - 1];
            }
            if (left & 2) {
                *reinterpret_cast<half_t *>(to) = static_cast<uint16_t>(v);
                to += 2;
                v >>= 16;
            }
            if (left & 1) *to = static_cast<int8_t>(v);
        }
    }
}

// LINES: the rows of the codes are whole cache lines, which a wave reads for good; elsewhere two waves share some.  16 x 4096 x
// 4096 bfloat16 saved and restored with streaming loads of the codes in 242 us, with plain ones in 281; 64 x 8000 x 115
// binary32 in 144 and 124.
template <int DT, bool LINES>
__global__ __launch_bounds__(kBlock) void restore_kernel(const int8_t *__restrict__ codes, const uint8_t *__restrict__ scales, Units u,
                                                         char *__restrict__ out)
{
    constexpr int ES = DT == 0 ? 4 : 2, kVec = unit_elems(DT);
    const Span span(u);
    const int32_t width = static_cast<int32_t>(u.width);
    const int64_t rows = u.rows - span.row;
    out += span.row * u.stride * ES;
    codes += span.row * u.width;
    scales += span.row * u.groups;
    const uint32_t stride = static_cast<uint32_t>(u.stride * ES);
    uint32_t w[kUnits][kVec / 4];
    uint32_t byte[kUnits], down[kUnits];
    int32_t at[kUnits];
#pragma unroll
    for (int n = 0; n < kUnits; ++n) {
        span.place<kVec>(u, n, down[n], at[n]);
#pragma unroll
        for (int k = 0; k < kVec / 4; ++k) w[n][k] = 0;
        byte[n] = 0;
        if (down[n] >= rows) at[n] = width;
        if (at[n] >= width) continue;
        const int8_t *from = codes + uint64_t(down[n]) * static_cast<uint32_t>(width) + at[n];
        byte[n] = scales[uint64_t(down[n]) * static_cast<uint32_t>(u.groups) + at[n] / static_cast<int32_t>(kCheckpointGroup)];
        if (at[n] + kVec <= width) load_codes<LINES>(from, w[n]);
        else
#pragma unroll
            for (int k = 0; k < kVec; ++k)
                if (at[n] + k < width) w[n][k >> 2] |= (static_cast<uint32_t>(from[k]) & 0xffu) << (8 * (k & 3));
    }
#pragma unroll
    for (int n = 0; n < kUnits; ++n) {
        if (at[n] >= width) continue;
        const float factor = to_value_factor(byte[n]);
        float f[kVec];
#pragma unroll
        for (int k = 0; k < kVec; ++k) f[k] = factor * code_of(w[n][k >> 2], k & 3);
        char *to = out + uint64_t(down[n]) * stride + at[n] * ES;
        if (at[n] + kVec <= width) store_elems<DT, kVec, true>(to, f);
        else
            for (int k = 0; k < kVec; ++k)
                if (at[n] + k < width) store_one<DT>(to + k * ES, f[k]);
    }
}

Units units_of(int dtype, int64_t rows, int64_t width, int64_t stride)
{
    Units u{rows, width, stride, checkpoint_groups(width), 0, 0, 0};
    u.row_units = static_cast<uint32_t>(kCheckpointGroup / unit_elems(dtype) * u.groups);
    u.magic = static_cast<uint32_t>((uint64_t(1) << 32) / u.row_units + 1);      // (exact below 2^32 / row_units)
    u.count = rows * u.row_units;
    return u;
}

int64_t blocks_of(const Units &u) { return (u.count + kBlock * kUnits - 1) / (kBlock * kUnits); }

}  // namespace

hipError_t launch_checkpoint(const void *x, int dtype, int64_t rows, int64_t width, int64_t stride, int8_t *codes, uint8_t *scales,
                             hipStream_t stream)
{
    if (rows == 0) return hipSuccess;
    const Units u = units_of(dtype, rows, width, stride);
    if (!launchable(blocks_of(u), kBlock)) return hipErrorInvalidConfiguration;
    const uint32_t blocks = static_cast<uint32_t>(blocks_of(u));
    (dtype == 0 ? checkpoint_kernel<0> : checkpoint_kernel<1>)<<<blocks, kBlock, 0, stream>>>(static_cast<const char *>(x), u, codes, scales);
    return hipGetLastError();
}

hipError_t launch_checkpoint_restore(const int8_t *codes, const uint8_t *scales, int64_t rows, int64_t width, void *out, int dtype,
                                     int64_t stride, hipStream_t stream)
{
    if (rows == 0) return hipSuccess;
    const Units u = units_of(dtype, rows, width, stride);
    if (!launchable(blocks_of(u), kBlock)) return hipErrorInvalidConfiguration;
    const uint32_t blocks = static_cast<uint32_t>(blocks_of(u));
    const bool lines = width % 128 == 0 && reinterpret_cast<uintptr_t>(codes) % 128 == 0;
    (dtype == 0 ? (lines ? restore_kernel<0, true> : restore_kernel<0, false>) : (lines ? restore_kernel<1, true> : restore_kernel<1, false>))<<<blocks, kBlock, 0, stream>>>(codes, scales, u, static_cast<char *>(out));
    return hipGetLastError();
}

}  // namespace moshpit
