// Activations saved in 8 bits and restored, for gfx950 (the form: checkpoint_codes.h).
//
// Bound by HBM: saving reads the activations once and writes a quarter (binary32) or half (bfloat16) of that.
// A lane holds 8 consecutive elements, so 4 neighbouring lanes hold a group of 32 and find its largest element
// with two exchanges; a row takes whole groups of lanes.
#include <hip/hip_runtime.h>

#include "checkpoint_codes.h"
#include "local_ops.h"

namespace moshpit {
namespace {

constexpr int kBlock = 256, kVec = 8, kUnits = 4;      // elements of a lane at a time; such units of a lane

// A unit is 8 elements of a row; a row takes `row_units` of them, a multiple of 4.
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
    __device__ __forceinline__ void place(const Units &u, int n, uint32_t &down, int32_t &at) const
    {
        const uint32_t unit = rest + n * kBlock + threadIdx.x;
        if (u.row_units >= kBlock * kUnits) down = unit >= u.row_units ? 1 : 0;
        else down = __umulhi(unit, u.magic);
        at = static_cast<int32_t>(unit - down * u.row_units) * kVec;
    }
};

// 8 elements as they lie in memory; most(): the largest of their bits without the signs.
template <int DT> struct Elems8;
template <> struct Elems8<0> {
    u32x4 w[2];
    __device__ __forceinline__ void load(const char *p)
    {
        w[0] = load_vec<false, u32x4>(p);                             // (the two halves share cache lines: no streaming hint)
        w[1] = load_vec<false, u32x4>(p + 16);
    }
    __device__ __forceinline__ void put(int k, const char *p) { w[k >> 2][k & 3] = *reinterpret_cast<const uint32_t *>(p); }
    __device__ __forceinline__ void move_down(int n)                  // elements n .. 7 to 0 .., zeros behind them
    {
#pragma unroll
        for (int by = 4; by > 0; by /= 2)
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const uint32_t from = k + by < 8 ? w[(k + by) >> 2 & 1][(k + by) & 3] : 0u;
                w[k >> 2][k & 3] = n & by ? from : w[k >> 2][k & 3];
            }
    }
    __device__ __forceinline__ uint32_t most() const
    {
        uint32_t m = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const uint32_t b = w[k >> 2][k & 3] & 0x7fffffffu;
            m = b > m ? b : m;
        }
        return m;
    }
    __device__ __forceinline__ void widen(float (&f)[8]) const
    {
#pragma unroll
        for (int k = 0; k < 8; ++k) f[k] = __uint_as_float(w[k >> 2][k & 3]);
    }
};
template <> struct Elems8<1> {
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

template <int DT>
__global__ __launch_bounds__(kBlock) void checkpoint_kernel(const char *__restrict__ x, Units u, int8_t *__restrict__ codes,
                                                            uint8_t *__restrict__ scales)
{
    constexpr int ES = DT == 0 ? 4 : 2;
    const Span span(u);
    const int32_t width = static_cast<int32_t>(u.width);
    const int64_t rows = u.rows - span.row;
    x += span.row * u.stride * ES;
    codes += span.row * u.width;
    scales += span.row * u.groups;
    const uint32_t stride = static_cast<uint32_t>(u.stride * ES);
    Elems8<DT> e[kUnits];
    uint32_t down[kUnits];
    int32_t at[kUnits];
#pragma unroll
    for (int n = 0; n < kUnits; ++n) {
        span.place(u, n, down[n], at[n]);
        e[n] = Elems8<DT>{};
        if (down[n] >= rows) at[n] = width;
        if (at[n] >= width) continue;
        const char *from = x + uint64_t(down[n]) * stride + at[n] * ES;
        // a row's last elements, where they are no whole unit: the row's last 8 moved to their place, so that one access does
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
        for (int off = 1; off < 4; off <<= 1) {
            const uint32_t other = __shfl_xor(most, off, 64);
            most = other > most ? other : most;
        }
        if (at[n] >= width) continue;
        const uint32_t byte = scale_byte(most);
        if ((threadIdx.x & 3) == 0) scales[uint64_t(down[n]) * static_cast<uint32_t>(u.groups) + at[n] / static_cast<int32_t>(kCheckpointGroup)] = static_cast<uint8_t>(byte);
        float f[kVec];
        e[n].widen(f);
        u32x2 w = {0, 0};
        if (byte != kScaleNaN) {
            const float factor = to_code_factor(byte);
            w = u32x2{pack_codes(f, factor), pack_codes(f + 4, factor)};
        }
        int8_t *to = codes + uint64_t(down[n]) * static_cast<uint32_t>(width) + at[n];
        if (at[n] + kVec <= width) {
            typedef u32x2 any_t __attribute__((aligned(1)));
            __builtin_nontemporal_store(w, reinterpret_cast<any_t *>(to));
        } else {                                                      // 4, 2 and 1 codes as there are
            typedef uint32_t word_t __attribute__((aligned(1)));
            typedef uint16_t half_t __attribute__((aligned(1)));
            const int left = width - at[n];
            uint32_t v = w.x;
            if (left & 4) {
                *reinterpret_cast<word_t *>(to) = v;
                to += 4;
                v = w.y;
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

template <int DT>
__global__ __launch_bounds__(kBlock) void restore_kernel(const int8_t *__restrict__ codes, const uint8_t *__restrict__ scales, Units u,
                                                         char *__restrict__ out)
{
    constexpr int ES = DT == 0 ? 4 : 2;
    const Span span(u);
    const int32_t width = static_cast<int32_t>(u.width);
    const int64_t rows = u.rows - span.row;
    out += span.row * u.stride * ES;
    codes += span.row * u.width;
    scales += span.row * u.groups;
    const uint32_t stride = static_cast<uint32_t>(u.stride * ES);
    u32x2 w[kUnits];
    uint32_t byte[kUnits], down[kUnits];
    int32_t at[kUnits];
#pragma unroll
    for (int n = 0; n < kUnits; ++n) {
        span.place(u, n, down[n], at[n]);
        w[n] = u32x2{0, 0};
        byte[n] = 0;
        if (down[n] >= rows) at[n] = width;
        if (at[n] >= width) continue;
        const int8_t *from = codes + uint64_t(down[n]) * static_cast<uint32_t>(width) + at[n];
        byte[n] = scales[uint64_t(down[n]) * static_cast<uint32_t>(u.groups) + at[n] / static_cast<int32_t>(kCheckpointGroup)];
        if (at[n] + kVec <= width) {
            typedef u32x2 any_t __attribute__((aligned(1)));
            w[n] = __builtin_nontemporal_load(reinterpret_cast<const any_t *>(from));
        } else
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
        if (at[n] + kVec <= width) store_elems<DT, kVec, DT == 1>(to, f);
        else
            for (int k = 0; k < kVec; ++k)
                if (at[n] + k < width) store_one<DT>(to + k * ES, f[k]);
    }
}

Units units_of(int64_t rows, int64_t width, int64_t stride)
{
    Units u{rows, width, stride, checkpoint_groups(width), 0, 0, 0};
    u.row_units = static_cast<uint32_t>(4 * u.groups);
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
    const Units u = units_of(rows, width, stride);
    if (!launchable(blocks_of(u), kBlock)) return hipErrorInvalidConfiguration;
    const uint32_t blocks = static_cast<uint32_t>(blocks_of(u));
    (dtype == 0 ? checkpoint_kernel<0> : checkpoint_kernel<1>)<<<blocks, kBlock, 0, stream>>>(static_cast<const char *>(x), u, codes, scales);
    return hipGetLastError();
}

hipError_t launch_checkpoint_restore(const int8_t *codes, const uint8_t *scales, int64_t rows, int64_t width, void *out, int dtype,
                                     int64_t stride, hipStream_t stream)
{
    if (rows == 0) return hipSuccess;
    const Units u = units_of(rows, width, stride);
    if (!launchable(blocks_of(u), kBlock)) return hipErrorInvalidConfiguration;
    const uint32_t blocks = static_cast<uint32_t>(blocks_of(u));
    (dtype == 0 ? restore_kernel<0> : restore_kernel<1>)<<<blocks, kBlock, 0, stream>>>(codes, scales, u, static_cast<char *>(out));
    return hipGetLastError();
}

}  // namespace moshpit
