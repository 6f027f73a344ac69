// Dropout with a mask that is drawn and never stored, onto a residual or alone, for gfx950:
//   out = residual + (kept ? x * 2^16 / (2^16 - cut) : 0),   cut = round(p * 2^16)
// Element c of row n (all peers' rows in a row) is kept when bits 16 (c % 4) .. + 15 of
//   mix(mix(mix(seed + K1 (step + 1)) + K2 (n + 1)) ^ (c / 4))
// are at least cut, mix being the library's mixer (mix64.h).  The backward pass is the same call on the gradient.
//
// Bound by HBM with the mixer close behind: 8 elements take two words and a row's key, six 64-bit products.  A thread takes
// kUnits units of 8 elements, kBlock units apart; a block's units lie one behind the other over the rows.  16 x 4096 rows of 4096 in bfloat16
// onto a residual: 256 us, 6.3 TB/s.
#include <hip/hip_runtime.h>

#include "local_ops.h"
#include "mix64.h"
#include "row_elems.h"

namespace moshpit {
namespace {

constexpr int kBlock = 256, kUnits = 4, kUnit = 8;
constexpr uint64_t kStepFactor = 0xE7037ED1A0B428DBull, kRowFactor = 0x8EBC6AF09C88C6E3ull;

template <int DT, bool RESIDUAL>
__global__ __launch_bounds__(kBlock) void dropout_kernel(DropoutArgs a, uint32_t row_units)
{
    constexpr int ES = DT == 0 ? 4 : 2;
    const int64_t first = int64_t(blockIdx.x) * (kBlock * kUnits), first_row = first / row_units;
    const uint32_t rest = static_cast<uint32_t>(first - first_row * row_units);
    const uint64_t base = mix64(a.seed + kStepFactor * ((a.step ? *a.step : 0) + 1));
    const int32_t width = static_cast<int32_t>(a.width);
    float f[kUnits][kUnit], r[kUnits][kUnit];
    int64_t row[kUnits];
    int32_t at[kUnits], left[kUnits];
#pragma unroll
    for (int n = 0; n < kUnits; ++n) {
        const uint32_t unit = rest + n * kBlock + threadIdx.x, down = unit / row_units;      // (rest < row_units <= 2^20)
        row[n] = first_row + down;
        at[n] = static_cast<int32_t>(unit - down * row_units) * kUnit;
        left[n] = row[n] < a.rows ? width - at[n] : 0;
        if (left[n] <= 0) continue;
        const char *x = a.x + (row[n] * a.x_stride + at[n]) * ES, *y = a.residual + (row[n] * a.residual_stride + at[n]) * ES;
        if (left[n] >= kUnit) {
            load_elems<DT, kUnit, true>(x, f[n]);
            if constexpr (RESIDUAL) load_elems<DT, kUnit, true>(y, r[n]);
        } else
#pragma unroll
            for (int k = 0; k < kUnit; ++k)
                if (k < left[n]) {
                    f[n][k] = load_one<DT>(x + k * ES);
                    if constexpr (RESIDUAL) r[n][k] = load_one<DT>(y + k * ES);
                }
    }
#pragma unroll
    for (int n = 0; n < kUnits; ++n) {
        if (left[n] <= 0) continue;
        const uint64_t key = mix64(base + kRowFactor * static_cast<uint64_t>(row[n] + 1));
        float out[kUnit];
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const uint64_t word = mix64(key ^ static_cast<uint64_t>(at[n] / 4 + q));
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const uint32_t bits = static_cast<uint32_t>(word >> (16 * k)) & 0xffffu;
                const float v = bits >= a.cut ? f[n][4 * q + k] * a.factor : 0.f;
                out[4 * q + k] = RESIDUAL ? r[n][4 * q + k] + v : v;
            }
        }
        char *to = a.out + (row[n] * a.out_stride + at[n]) * ES;
        if (left[n] >= kUnit) store_elems<DT, kUnit, true>(to, out);
        else
#pragma unroll
            for (int k = 0; k < kUnit; ++k)
                if (k < left[n]) store_one<DT>(to + k * ES, out[k]);
    }
}

int64_t blocks_of(const DropoutArgs &a) { return (a.rows * ((a.width + kUnit - 1) / kUnit) + kBlock * kUnits - 1) / (kBlock * kUnits); }

}  // namespace

bool dropout_fits(const DropoutArgs &a) { return launchable(blocks_of(a), kBlock); }

hipError_t launch_dropout(const DropoutArgs &a, int dtype, hipStream_t stream)
{
    if (a.rows == 0) return hipSuccess;
    const uint32_t row_units = static_cast<uint32_t>((a.width + kUnit - 1) / kUnit);
    auto kernel = dtype == 0 ? (a.residual ? dropout_kernel<0, true> : dropout_kernel<0, false>) : (a.residual ? dropout_kernel<1, true> : dropout_kernel<1, false>);
    kernel<<<static_cast<uint32_t>(blocks_of(a)), kBlock, 0, stream>>>(a, row_units);
    return hipGetLastError();
}

}  // namespace moshpit
