// Root-mean-square norm of h = x + residual (or of h = x) with a gain of every peer's own, and its backward pass, for gfx950:
//   y = x^ g,   x^ = h r,   r = (mean(h^2) + eps)^(-1/2)
//   dx = r (u - x^ mean(u x^)) + dh,   u = g dy,          dg_i = sum over t of dy x^
// in binary32 (h not rounded before the norm), each result rounded once; y also in the 8-bit form of checkpoint_codes.h,
// from the values that are stored.
//
// Bound by HBM.  A row lies in the registers of LANES threads, U units of 8 elements each, from its sums to its results, so it is
// read once.  A block takes rows of one peer, whose gain it holds, and in the backward pass the sums of the gain's
// gradient: a thread meets the same columns in every row.  The blocks' sums are joined by a second kernel, in order.
// Rows of more than 16384 elements are read twice, in the backward pass three times (sums, the gain's gradient by columns, results): 4 x 4000 rows of
// 20000 in bfloat16 with a residual: 731 us and 1365 (of 16384: 415, 413).  16 x 4096 rows of 4096 in bfloat16: forward with residual and 8-bit output 418 us, 5.8 TB/s;
// backward with a residual's gradient 407 us, 5.3 TB/s.
#include <hip/hip_runtime.h>

#include "checkpoint_codes.h"
#include "local_ops.h"
#include "row_sums.h"

namespace moshpit {
namespace {

constexpr int kUnit = 8;
constexpr int kBlock = 256;              // of the join, and the fewest threads of a block that takes rows
constexpr int64_t kMostHeld = 16384;     // elements of a row that registers hold

template <int LANES> constexpr int threads_of() { return LANES > kBlock ? LANES : kBlock; }

// Unit at p, of which `left` elements (1 and more) are the row's; zeros behind them.
template <int DT> __device__ __forceinline__ void load_unit(const char *p, int left, float (&f)[kUnit])
{
    constexpr int ES = DT == 0 ? 4 : 2;
    if (left >= kUnit) load_elems<DT, kUnit, true>(p, f);
    else
#pragma unroll
        for (int k = 0; k < kUnit; ++k) f[k] = k < left ? load_one<DT>(p + k * ES) : 0.f;
}
template <int DT, bool NT = true> __device__ __forceinline__ void store_unit(char *p, int left, const float (&f)[kUnit])
{
    constexpr int ES = DT == 0 ? 4 : 2;
    if (left >= kUnit) store_elems<DT, kUnit, NT>(p, f);
    else
#pragma unroll
        for (int k = 0; k < kUnit; ++k)
            if (k < left) store_one<DT>(p + k * ES, f[k]);
}

// f as it is stored.
template <int DT> __device__ __forceinline__ void round_unit(float (&f)[kUnit])
{
    if constexpr (DT == 1) Vec<1, 8>::widen(Vec<1, 8>::narrow(f), f);
}

typedef u32x2 codes_t __attribute__((aligned(1)));

// Codes of a unit, whose 32 elements with one scale lie in 4 neighbouring lanes (zeros behind the row's end), all of them here.
__device__ __forceinline__ void save_unit(float (&f)[kUnit], int64_t at, int left, int8_t *codes, uint8_t *scales)
{
    uint32_t most = 0;
#pragma unroll
    for (int k = 0; k < kUnit; ++k) {
        const uint32_t b = __float_as_uint(f[k]) & 0x7fffffffu;
        most = b > most ? b : most;
    }
#pragma unroll
    for (int off = 1; off < 4; off <<= 1) {
        const uint32_t other = off == 1 ? lane_from<0xB1>(most) : lane_from<0x4E>(most);
        most = other > most ? other : most;
    }
    if (left <= 0) return;
    const uint32_t byte = scale_byte(most);
    if (threadIdx.x % 4 == 0) scales[at / kCheckpointGroup] = static_cast<uint8_t>(byte);
    uint32_t w[2] = {0, 0};
    if (byte != kScaleNaN) {
        if (byte == kScaleTop) keep_finite(f);
        const float factor = to_code_factor(byte);
        w[0] = pack_codes(f, factor);
        w[1] = pack_codes(f + 4, factor);
    }
    if (left >= kUnit) *reinterpret_cast<codes_t *>(codes + at) = u32x2{w[0], w[1]};
    else
#pragma unroll
        for (int k = 0; k < kUnit; ++k)
            if (k < left) codes[at + k] = static_cast<int8_t>(w[k / 4] >> (8 * (k & 3)));
}

// What a row's results are made with: x^ = (h factor) inverse, 1 / root mean square = (inverse root) root (each a factor of its own), root^2 = factor and
//   inverse = (mean((h factor)^2) + eps factor^2)^(-1/2).
// factor is 1 but where mean(h^2) + eps passes binary32, or is so small that squares lose bits below the normal numbers.  With 2^-96 the largest elements'
// squares are 2^64 and the sum of 2^23 of them 2^87 (elements that it takes below the normal numbers are off by 2^-95 of the row's root mean square
// and less); with 2^96 elements that were 2^-38 at most stay below 2^58, and the smallest, 2^-149, square to 2^-106.
struct Size {
    float factor, inverse, root;
};
constexpr float kTooSmall = 0x1p-100f;   // (squares' lost bits: 2^-150 each, 2^-50 of it)

// Of a row that LANES threads share: sum(factor) is the sum over it of (h factor)^2, in every one of them.
template <int LANES, typename Sum> __device__ __forceinline__ Size size_of(float share, float eps, Sum sum)
{
    const float mean = fmaf(sum(1.f), share, eps);
    Size s{1.f, rsqrtf(mean), 1.f};
    if (__builtin_expect(!(mean < INFINITY) || mean < kTooSmall, 0)) { // (the same in every thread of the row)
        s.root = mean < kTooSmall ? 0x1p48f : 0x1p-48f;
        s.factor = s.root * s.root;
        s.inverse = rsqrtf(fmaf(sum(s.factor), share, eps * s.factor * s.factor));
    }
    if constexpr (LANES >= 64)                                         // (they take no vector registers: 16 x 4096 rows of 4096 in bfloat16, backward: 407 us, 490 with them)
        for (float *v : {&s.factor, &s.inverse, &s.root}) *v = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(*v)));
    return s;
}

template <int DT, int ST, int LANES, int U>
__global__ __launch_bounds__(threads_of<LANES>())
void norm_kernel(NormArgs a, int64_t rows_each, int64_t parts)
{
    constexpr int ES = DT == 0 ? 4 : 2, GS = ST == 0 ? 4 : 2, SLOTS = threads_of<LANES>() / LANES;
    __shared__ float scratch[2][16];
    const int lane = threadIdx.x % LANES, slot = threadIdx.x / LANES;
    const int64_t peer = blockIdx.x / parts, begin = (blockIdx.x % parts) * rows_each;
    const int64_t end = begin + rows_each < a.T ? begin + rows_each : a.T;
    const int32_t width = static_cast<int32_t>(a.width);
    const char *gain = a.gain + peer * a.gain_stride * GS;
    float g[U][kUnit];
    int32_t at[U], left[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        at[u] = (u * LANES + lane) * kUnit;
        left[u] = width - at[u];
        if (left[u] > 0) load_unit<ST>(gain + int64_t(at[u]) * GS, left[u], g[u]);
    }
    const float share = 1.f / static_cast<float>(width);
    int phase = 0;
    for (int64_t t = begin + slot; t < end; t += SLOTS) {              // (one slot, where the threads of a row wait for each other)
        const int64_t row = peer * a.T + t;
        float h[U][kUnit];
#pragma unroll
        for (int u = 0; u < U; ++u) {
#pragma unroll
            for (int k = 0; k < kUnit; ++k) h[u][k] = 0.f;
            if (left[u] > 0) load_unit<DT>(a.x + (row * a.x_stride + at[u]) * ES, left[u], h[u]);
        }
        if (a.residual)
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (left[u] > 0) {
                    float r[kUnit];
                    load_unit<DT>(a.residual + (row * a.residual_stride + at[u]) * ES, left[u], r);
#pragma unroll
                    for (int k = 0; k < kUnit; ++k) h[u][k] += r[k];
                }
        const Size s = size_of<LANES>(share, a.eps, [&](float factor) {
            float sum = 0.f;
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int k = 0; k < kUnit; ++k) sum = fmaf(h[u][k] * factor, h[u][k] * factor, sum);
            return group_sum<LANES>(sum, scratch[phase ^= 1]);
        });
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (left[u] > 0 && a.total) store_unit<DT>(a.total + (row * a.total_stride + at[u]) * ES, left[u], h[u]);
            if (left[u] > 0) {
#pragma unroll
                for (int k = 0; k < kUnit; ++k) h[u][k] = h[u][k] * s.factor * s.inverse * g[u][k];
                round_unit<DT>(h[u]);
                if (left[u] < kUnit)
#pragma unroll
                    for (int k = 0; k < kUnit; ++k) h[u][k] = k < left[u] ? h[u][k] : 0.f;
                store_unit<DT>(a.out + (row * a.out_stride + at[u]) * ES, left[u], h[u]);
            }
            if (a.codes) save_unit(h[u], at[u], left[u], a.codes + row * a.width, a.scales + row * checkpoint_groups(a.width));
        }
    }
}

// Rows that registers do not hold, a block each: sums, then results, h from memory both times.
template <int DT, int ST>
__global__ __launch_bounds__(1024) void wide_norm_kernel(NormArgs a)
{
    constexpr int ES = DT == 0 ? 4 : 2, GS = ST == 0 ? 4 : 2;
    __shared__ float scratch[2][16];
    const int64_t row = blockIdx.x;
    const char *gain = a.gain + row / a.T * a.gain_stride * GS, *x = a.x + row * a.x_stride * ES;
    const char *residual = a.residual ? a.residual + row * a.residual_stride * ES : nullptr;
    const int32_t width = static_cast<int32_t>(a.width), last = (width + 4 * kUnit - 1) / (4 * kUnit) * (4 * kUnit);   // (whole groups of lanes)
    auto load = [&](int32_t at, float (&h)[kUnit]) {
        load_unit<DT>(x + int64_t(at) * ES, width - at, h);
        if (residual) {
            float r[kUnit];
            load_unit<DT>(residual + int64_t(at) * ES, width - at, r);
#pragma unroll
            for (int k = 0; k < kUnit; ++k) h[k] += r[k];
        }
    };
    int phase = 0;
    const Size s = size_of<1024>(1.f / static_cast<float>(width), a.eps, [&](float factor) {
        float sum = 0.f, h[kUnit];
        for (int32_t at = threadIdx.x * kUnit; at < width; at += 1024 * kUnit) {
            load(at, h);
#pragma unroll
            for (int k = 0; k < kUnit; ++k) sum = fmaf(h[k] * factor, h[k] * factor, sum);
        }
        return group_sum<1024>(sum, scratch[phase ^= 1]);
    });
    for (int32_t at = threadIdx.x * kUnit; at < last; at += 1024 * kUnit) {
        float h[kUnit] = {}, g[kUnit];
        const int32_t left = width - at;
        if (left > 0) {
            load(at, h);
            load_unit<ST>(gain + int64_t(at) * GS, left, g);
            if (a.total) store_unit<DT>(a.total + (row * a.total_stride + at) * ES, left, h);
#pragma unroll
            for (int k = 0; k < kUnit; ++k) h[k] = k < left ? h[k] * s.factor * s.inverse * g[k] : 0.f;
            round_unit<DT>(h);
            store_unit<DT>(a.out + (row * a.out_stride + at) * ES, left, h);
        }
        if (a.codes) save_unit(h, at, left, a.codes + row * a.width, a.scales + row * checkpoint_groups(a.width));
    }
}

// sums: [N][parts][width], the gain's gradient over the rows of a block, which takes every parts-th one, so that the blocks that run at the same time read
// neighbouring rows (4 x 30000 rows of 1000 in bfloat16: 189 us, by pieces of consecutive rows 218).
template <int DT, int ST, int LANES, int U>
__global__ __launch_bounds__(threads_of<LANES>())
void norm_grad_kernel(NormGradArgs a, int64_t parts, float *__restrict__ sums)
{
    constexpr int ES = DT == 0 ? 4 : 2, GS = ST == 0 ? 4 : 2, SLOTS = threads_of<LANES>() / LANES;
    __shared__ float scratch[2][32];
    const int lane = threadIdx.x % LANES, slot = threadIdx.x / LANES;
    const int64_t peer = blockIdx.x / parts, part = blockIdx.x % parts;
    const int32_t width = static_cast<int32_t>(a.width);
    const char *gain = a.gain + peer * a.gain_stride * GS;
    float g[U][kUnit], dg[U][kUnit];
    int32_t at[U], left[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        at[u] = (u * LANES + lane) * kUnit;
        left[u] = width - at[u];
#pragma unroll
        for (int k = 0; k < kUnit; ++k) g[u][k] = dg[u][k] = 0.f;
        if (left[u] > 0) load_unit<ST>(gain + int64_t(at[u]) * GS, left[u], g[u]);
    }
    const float share = 1.f / static_cast<float>(width);
    int phase = 0;
    for (int64_t t = part * SLOTS + slot; t < a.T; t += parts * SLOTS) {      // (SLOTS > 1: within a wave or less, no barrier in the loop)
        const int64_t row = peer * a.T + t;
        float h[U][kUnit], dy[U][kUnit], product = 0.f;
#pragma unroll
        for (int u = 0; u < U; ++u) {
#pragma unroll
            for (int k = 0; k < kUnit; ++k) h[u][k] = dy[u][k] = 0.f;
            if (left[u] > 0) {
                load_unit<DT>(a.x + (row * a.x_stride + at[u]) * ES, left[u], h[u]);
                load_unit<DT>(a.dy + (row * a.dy_stride + at[u]) * ES, left[u], dy[u]);
            }
        }
        const Size s = size_of<LANES>(share, a.eps, [&](float factor) {
            float square = 0.f;
            product = 0.f;
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int k = 0; k < kUnit; ++k) {
                    const float v = h[u][k] * factor;
                    square = fmaf(v, v, square);
                    product = fmaf(dy[u][k] * g[u][k], v, product);
                }
            group_sums<LANES>(square, product, scratch[phase ^= 1]);
            return square;
        });
        const float mean = product * share * s.inverse, outer = s.inverse * s.root;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (left[u] <= 0) continue;
            float d[kUnit];
            if (a.dtotal) load_unit<DT>(a.dtotal + (row * a.dtotal_stride + at[u]) * ES, left[u], d);
#pragma unroll
            for (int k = 0; k < kUnit; ++k) {
                const float v = h[u][k] * s.factor * s.inverse;
                dg[u][k] = fmaf(dy[u][k], v, dg[u][k]);
                const float e = outer * ((dy[u][k] * g[u][k] - v * mean) * s.root);
                d[k] = a.dtotal ? d[k] + e : e;
            }
            store_unit<DT>(a.dx + (row * a.dx_stride + at[u]) * ES, left[u], d);
        }
    }
    float *to = sums + blockIdx.x * a.width;
    if constexpr (SLOTS == 1) {
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (left[u] > 0) store_unit<0, false>(reinterpret_cast<char *>(to + at[u]), left[u], dg[u]);
    } else {                             // the block's slots, in order
        __shared__ float all[SLOTS][U * LANES * kUnit];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int k = 0; k < kUnit; ++k) all[slot][at[u] + k] = dg[u][k];
        __syncthreads();
        for (int32_t c = threadIdx.x; c < width; c += threads_of<LANES>()) {
            float sum = all[0][c];
#pragma unroll
            for (int n = 1; n < SLOTS; ++n) sum += all[n][c];
            to[c] = sum;
        }
    }
}

// Rows that registers do not hold: factor, inverse, mean(u x^) and root of a row, by a block.
template <int DT, int ST>
__global__ __launch_bounds__(1024) void wide_norm_sums_kernel(NormGradArgs a, float4 *__restrict__ found)
{
    constexpr int ES = DT == 0 ? 4 : 2, GS = ST == 0 ? 4 : 2;
    __shared__ float scratch[2][32];
    const int64_t row = blockIdx.x;
    const char *gain = a.gain + row / a.T * a.gain_stride * GS, *x = a.x + row * a.x_stride * ES, *dy = a.dy + row * a.dy_stride * ES;
    const int32_t width = static_cast<int32_t>(a.width);
    float product = 0.f;
    int phase = 0;
    const float share = 1.f / static_cast<float>(width);
    const Size s = size_of<1024>(share, a.eps, [&](float factor) {
        float square = 0.f;
        product = 0.f;
        for (int32_t at = threadIdx.x * kUnit; at < width; at += 1024 * kUnit) {
            float h[kUnit], d[kUnit], g[kUnit];
            load_unit<DT>(x + int64_t(at) * ES, width - at, h);
            load_unit<DT>(dy + int64_t(at) * ES, width - at, d);
            load_unit<ST>(gain + int64_t(at) * GS, width - at, g);
#pragma unroll
            for (int k = 0; k < kUnit; ++k) {
                const float v = h[k] * factor;
                square = fmaf(v, v, square);
                product = fmaf(d[k] * g[k], v, product);
            }
        }
        group_sums<1024>(square, product, scratch[phase ^= 1]);
        return square;
    });
    if (threadIdx.x == 0) found[row] = float4{s.factor, s.inverse, product * share * s.inverse, s.root};
}

// Their gain's gradient: a thread has a column, and adds up the rows of a part.
template <int DT>
__global__ __launch_bounds__(kBlock) void wide_gain_kernel(NormGradArgs a, const float4 *__restrict__ found, int64_t rows_each, int64_t parts,
                                                           float *__restrict__ sums)
{
    constexpr int ES = DT == 0 ? 4 : 2;
    const int64_t tiles = (a.width + kBlock - 1) / kBlock, c = blockIdx.x % tiles * kBlock + threadIdx.x, part = blockIdx.x / tiles;
    if (c >= a.width) return;
    const int64_t peer = part / parts, begin = part % parts * rows_each, end = begin + rows_each < a.T ? begin + rows_each : a.T;
    float sum = 0.f;
#pragma unroll 4
    for (int64_t row = peer * a.T + begin; row < peer * a.T + end; ++row) {
        const float4 s = found[row];
        sum = fmaf(load_one<DT>(a.dy + (row * a.dy_stride + c) * ES), load_one<DT>(a.x + (row * a.x_stride + c) * ES) * s.x * s.y, sum);
    }
    sums[part * a.width + c] = sum;
}

// And their input's.
template <int DT, int ST>
__global__ __launch_bounds__(1024) void wide_norm_grad_kernel(NormGradArgs a, const float4 *__restrict__ found)
{
    constexpr int ES = DT == 0 ? 4 : 2, GS = ST == 0 ? 4 : 2;
    const int64_t row = blockIdx.x;
    const char *gain = a.gain + row / a.T * a.gain_stride * GS;
    const int32_t width = static_cast<int32_t>(a.width);
    const float4 s = found[row];
    for (int32_t at = threadIdx.x * kUnit; at < width; at += 1024 * kUnit) {
        float h[kUnit], d[kUnit], g[kUnit], more[kUnit] = {};
        load_unit<DT>(a.x + (row * a.x_stride + at) * ES, width - at, h);
        load_unit<DT>(a.dy + (row * a.dy_stride + at) * ES, width - at, d);
        load_unit<ST>(gain + int64_t(at) * GS, width - at, g);
        if (a.dtotal) load_unit<DT>(a.dtotal + (row * a.dtotal_stride + at) * ES, width - at, more);
#pragma unroll
        for (int k = 0; k < kUnit; ++k) {
            const float e = s.y * s.w * ((d[k] * g[k] - h[k] * s.x * s.y * s.z) * s.w);
            d[k] = a.dtotal ? more[k] + e : e;
        }
        store_unit<DT>(a.dx + (row * a.dx_stride + at) * ES, width - at, d);
    }
}

// grad_i[c] = [grad_i[c] +] the parts' sums, added in order within each of 8 shares of them and then over the shares.
template <int ST, bool ADD>
__global__ __launch_bounds__(kBlock) void gain_join_kernel(const float *__restrict__ sums, int64_t parts, int64_t width, int64_t peer_stride,
                                                           char *__restrict__ base)
{
    constexpr int GS = ST == 0 ? 4 : 2, SHARES = 8, COLS = kBlock / SHARES;
    __shared__ float share[SHARES][COLS];
    const int64_t tiles = (width + COLS - 1) / COLS, peer = blockIdx.x / tiles, c = blockIdx.x % tiles * COLS + threadIdx.x % COLS;
    const int s = threadIdx.x / COLS;
    const int64_t each = (parts + SHARES - 1) / SHARES, begin = s * each, end = begin + each < parts ? begin + each : parts;
    float sum = 0.f;
    if (c < width) {
        const float *from = sums + peer * parts * width + c;
        for (int64_t p = begin; p < end; p += 8) {                     // eight requested at a time
            float v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = p + k < end ? from[(p + k) * width] : 0.f;
#pragma unroll
            for (int k = 0; k < 8; ++k) sum += v[k];
        }
    }
    share[s][threadIdx.x % COLS] = sum;
    __syncthreads();
    if (s != 0 || c >= width) return;
#pragma unroll
    for (int n = 1; n < SHARES; ++n) sum += share[n][threadIdx.x];
    char *at = base + (peer * peer_stride + c) * GS;
    store_one<ST>(at, ADD ? load_one<ST>(at) + sum : sum);
}

// How many threads hold a row, and units each: the fewest that 16 to 1024 threads can.
struct Shape {
    int lanes, units;
};
Shape shape_of(int64_t width)
{
    const int64_t units = (width + kUnit - 1) / kUnit;
    return units <= 16 ? Shape{16, 1} : units <= 32 ? Shape{16, 2} : units <= 64 ? Shape{64, 1} : units <= 128 ? Shape{64, 2} : units <= 256 ? Shape{256, 1}
         : units <= 512 ? Shape{256, 2} : units <= 1024 ? Shape{256, 4} : Shape{1024, 2};
}

// Rows of a block: all the same number of turns of its slots, enough blocks for the chip.
struct Parts {
    int64_t each, parts;                 // rows of a part, parts of a peer
};
Parts parts_of(int64_t N, int64_t T, int slots, int64_t blocks)
{
    const int64_t turns = (T + slots - 1) / slots, want = blocks / N > 1 ? blocks / N : 1;
    const int64_t each = turns > 0 ? (turns + want - 1) / want * slots : slots;
    return Parts{each, T > 0 ? (T + each - 1) / each : 1};
}
int slots_of(const Shape &s) { return s.lanes >= kBlock ? 1 : kBlock / s.lanes; }
// Blocks a compute unit.  A block reads its gain once: 16 x 4096 rows of 4096 in bfloat16 with a binary32 gain, residual and 8-bit output (and its
// restoring) in 546 us, with 8 blocks in 630, with 256 in 565.  In the backward pass it leaves its sums, too: 407 us with 8, 397 with 16, 431 with 32, but
// 4 x 8000 rows of 8192 in 584, 620 and 689, 4 x 30000 rows of 1000 in 189, 202 and 218.
int64_t blocks_wanted(int compute_units, const Shape &s) { return int64_t(compute_units) * (s.lanes > kBlock ? 4 : 64); }
int64_t grad_blocks_wanted(int compute_units, const Shape &s) { return int64_t(compute_units) * (s.lanes > kBlock ? 4 : 8); }
Parts grad_parts(int64_t N, int64_t T, int64_t width, int compute_units)
{
    if (width > kMostHeld) return parts_of(N, T, 1, 2 * compute_units / ((width + kBlock - 1) / kBlock) + 1);
    const Shape s = shape_of(width);
    return parts_of(N, T, slots_of(s), grad_blocks_wanted(compute_units, s));
}

template <typename Go> hipError_t by_shape(const Shape &s, Go go)
{
    using std::integral_constant;
#define SHAPE(L, W) \
    if (s.lanes == L && s.units == W) return go(integral_constant<int, L>{}, integral_constant<int, W>{})
    SHAPE(16, 1);
    SHAPE(16, 2);
    SHAPE(64, 1);
    SHAPE(64, 2);
    SHAPE(256, 1);
    SHAPE(256, 2);
    SHAPE(256, 4);
#undef SHAPE
    return go(integral_constant<int, 1024>{}, integral_constant<int, 2>{});
}
template <typename Go> hipError_t by_types(int dtype, int state_dtype, Go go)
{
    using std::integral_constant;
    if (dtype == 0) return state_dtype == 0 ? go(integral_constant<int, 0>{}, integral_constant<int, 0>{}) : go(integral_constant<int, 0>{}, integral_constant<int, 1>{});
    return state_dtype == 0 ? go(integral_constant<int, 1>{}, integral_constant<int, 0>{}) : go(integral_constant<int, 1>{}, integral_constant<int, 1>{});
}

}  // namespace

bool norm_fits(int64_t N, int64_t T, int64_t width)
{
    return launchable(width > kMostHeld ? N * T : N, 1024) && launchable(N * ((width + 31) / 32), kBlock);
}

hipError_t launch_norm(const NormArgs &a, int dtype, int state_dtype, int compute_units, hipStream_t stream)
{
    if (a.T == 0) return hipSuccess;
    return by_types(dtype, state_dtype, [&](auto dt, auto st) {
        constexpr int DT = decltype(dt)::value, ST = decltype(st)::value;
        if (a.width > kMostHeld) {
            wide_norm_kernel<DT, ST><<<static_cast<uint32_t>(a.N * a.T), 1024, 0, stream>>>(a);
            return hipGetLastError();
        }
        const Shape s = shape_of(a.width);
        const Parts p = parts_of(a.N, a.T, slots_of(s), blocks_wanted(compute_units, s));
        return by_shape(s, [&](auto lanes, auto units) {
            constexpr int LANES = decltype(lanes)::value, U = decltype(units)::value;
            norm_kernel<DT, ST, LANES, U><<<static_cast<uint32_t>(a.N * p.parts), threads_of<LANES>(), 0, stream>>>(a, p.each, p.parts);
            return hipGetLastError();
        });
    });
}

int64_t norm_grad_work_bytes(int64_t N, int64_t T, int64_t width, int compute_units)
{
    const int64_t sums = (4 * N * grad_parts(N, T, width, compute_units).parts * width + 15) / 16 * 16;
    return sums + (width > kMostHeld ? int64_t(sizeof(float4)) * N * T : 0);
}

hipError_t launch_norm_grad(const NormGradArgs &a, int dtype, int state_dtype, bool accumulate, char *grad, int64_t grad_stride, void *work,
                            int compute_units, hipStream_t stream)
{
    const Parts p = grad_parts(a.N, a.T, a.width, compute_units);
    float *sums = static_cast<float *>(work);
    return by_types(dtype, state_dtype, [&](auto dt, auto st) {
        constexpr int DT = decltype(dt)::value, ST = decltype(st)::value;
        hipError_t e = hipSuccess;
        if (a.width > kMostHeld) {
            float4 *found = reinterpret_cast<float4 *>(static_cast<char *>(work) + (4 * a.N * p.parts * a.width + 15) / 16 * 16);
            const uint32_t rows = static_cast<uint32_t>(a.N * a.T), tiles = static_cast<uint32_t>((a.width + kBlock - 1) / kBlock * a.N * p.parts);
            if (rows > 0) wide_norm_sums_kernel<DT, ST><<<rows, 1024, 0, stream>>>(a, found);
            wide_gain_kernel<DT><<<tiles, kBlock, 0, stream>>>(a, found, p.each, p.parts, sums);
            if (rows > 0) wide_norm_grad_kernel<DT, ST><<<rows, 1024, 0, stream>>>(a, found);
            e = hipGetLastError();
        } else
            e = by_shape(shape_of(a.width), [&](auto lanes, auto units) {
                constexpr int LANES = decltype(lanes)::value, U = decltype(units)::value;
                norm_grad_kernel<DT, ST, LANES, U><<<static_cast<uint32_t>(a.N * p.parts), threads_of<LANES>(), 0, stream>>>(a, p.parts, sums);
                return hipGetLastError();
            });
        if (e != hipSuccess) return e;
        const uint32_t blocks = static_cast<uint32_t>((a.width + 31) / 32 * a.N);
        if (accumulate) gain_join_kernel<ST, true><<<blocks, kBlock, 0, stream>>>(sums, p.parts, a.width, grad_stride, grad);
        else gain_join_kernel<ST, false><<<blocks, kBlock, 0, stream>>>(sums, p.parts, a.width, grad_stride, grad);
        return hipGetLastError();
    });
}

}  // namespace moshpit
