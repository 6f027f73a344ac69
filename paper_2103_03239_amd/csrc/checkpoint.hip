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
    uint32_t row_units;
};

__device__ __forceinline__ void unit_place(const Units &u, int64_t unit, int64_t &row, int64_t &at)
{
    row = unit / u.row_units;
    at = (unit - row * u.row_units) * kVec;
}

template <int DT>
__global__ __launch_bounds__(kBlock) void checkpoint_kernel(const char *__restrict__ x, Units u, int8_t *__restrict__ codes,
                                                            uint8_t *__restrict__ scales)
{
    constexpr int ES = DT == 0 ? 4 : 2;
    const int64_t first = int64_t(blockIdx.x) * (kBlock * kUnits) + threadIdx.x;
    float f[kUnits][kVec];
    int64_t row[kUnits], at[kUnits];
#pragma unroll
    for (int n = 0; n < kUnits; ++n) {
        const int64_t unit = first + n * kBlock;
        unit_place(u, unit, row[n], at[n]);
#pragma unroll
        for (int k = 0; k < kVec; ++k) f[n][k] = 0.f;
        if (unit >= u.count) {
            at[n] = u.width;
            continue;
        }
        const char *from = x + (row[n] * u.stride + at[n]) * ES;
        if (at[n] + kVec <= u.width) load_elems<DT, kVec>(from, f[n]);
        else
            for (int k = 0; k < kVec; ++k)
                if (at[n] + k < u.width) f[n][k] = load_one<DT>(from + k * ES);
    }
#pragma unroll
    for (int n = 0; n < kUnits; ++n) {
        uint32_t most = 0;
#pragma unroll
        for (int k = 0; k < kVec; ++k) {
            const uint32_t bits = __float_as_uint(f[n][k]) & 0x7fffffffu;
            most = bits > most ? bits : most;
        }
#pragma unroll
        for (int off = 1; off < 4; off <<= 1) {
            const uint32_t other = __shfl_xor(most, off, 64);
            most = other > most ? other : most;
        }
        if (at[n] >= u.width) continue;
        const uint32_t byte = scale_byte(most);
        if ((threadIdx.x & 3) == 0) scales[row[n] * u.groups + at[n] / kCheckpointGroup] = static_cast<uint8_t>(byte);
        const float factor = byte == kScaleNaN ? 0.f : to_code_factor(byte);
        if (byte == kScaleNaN)
            for (int k = 0; k < kVec; ++k) f[n][k] = 0.f;
        const u32x2 w = {pack_codes(f[n], factor), pack_codes(f[n] + 4, factor)};
        int8_t *to = codes + row[n] * u.width + at[n];
        if (at[n] + kVec <= u.width) {
            typedef u32x2 any_t __attribute__((aligned(1)));
            *reinterpret_cast<any_t *>(to) = w;
        } else
            for (int k = 0; k < kVec; ++k)
                if (at[n] + k < u.width) to[k] = static_cast<int8_t>(w[k >> 2] >> (8 * (k & 3)));
    }
}

template <int DT>
__global__ __launch_bounds__(kBlock) void restore_kernel(const int8_t *__restrict__ codes, const uint8_t *__restrict__ scales, Units u,
                                                         char *__restrict__ out)
{
    constexpr int ES = DT == 0 ? 4 : 2;
    const int64_t first = int64_t(blockIdx.x) * (kBlock * kUnits) + threadIdx.x;
    u32x2 w[kUnits];
    uint32_t byte[kUnits];
    int64_t row[kUnits], at[kUnits];
#pragma unroll
    for (int n = 0; n < kUnits; ++n) {
        const int64_t unit = first + n * kBlock;
        unit_place(u, unit, row[n], at[n]);
        w[n] = u32x2{0, 0};
        byte[n] = 0;
        if (unit >= u.count || at[n] >= u.width) {
            at[n] = u.width;
            continue;
        }
        const int8_t *from = codes + row[n] * u.width + at[n];
        byte[n] = scales[row[n] * u.groups + at[n] / kCheckpointGroup];
        if (at[n] + kVec <= u.width) {
            typedef u32x2 any_t __attribute__((aligned(1)));
            w[n] = *reinterpret_cast<const any_t *>(from);
        } else
            for (int k = 0; k < kVec; ++k)
                if (at[n] + k < u.width) w[n][k >> 2] |= (static_cast<uint32_t>(from[k]) & 0xffu) << (8 * (k & 3));
    }
#pragma unroll
    for (int n = 0; n < kUnits; ++n) {
        if (at[n] >= u.width) continue;
        const float factor = to_value_factor(byte[n]);
        float f[kVec];
#pragma unroll
        for (int k = 0; k < kVec; ++k) f[k] = factor * code_of(w[n][k >> 2], k & 3);
        char *to = out + (row[n] * u.stride + at[n]) * ES;
        if (at[n] + kVec <= u.width) store_elems<DT, kVec>(to, f);
        else
            for (int k = 0; k < kVec; ++k)
                if (at[n] + k < u.width) store_one<DT>(to + k * ES, f[k]);
    }
}

Units units_of(int64_t rows, int64_t width, int64_t stride)
{
    Units u{rows, width, stride, checkpoint_groups(width), 0, 0};
    u.row_units = static_cast<uint32_t>(4 * u.groups);
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
