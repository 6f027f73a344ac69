// The gradient of a linear layer's weights, for every peer, from the layer's input saved in 8 bits, for gfx950:
//   grad_i[o][c] = sum over t of dy[i * T + t][o] * x[i * T + t][c],   x = code * 2^e (checkpoint_codes.h)
//
// A matrix product whose summed index, the token, is the slow one of both operands.  Tiles of kTokens tokens are
// staged through LDS as they lie in memory, [token][column] in bfloat16, and the transposing LDS reads of gfx950
// hand the matrix instructions their operands, 8 tokens of a column to a lane.  The codes become bfloat16 on their
// way into LDS, which is exact.  A binary32 dy is staged as three bfloat16 parts (8 significant bits each, exact
// down to 2^-133), whose products with x are exact in binary32: three matrix instructions in place of one, at five
// times the rate of the binary32 ones.  Sums are binary32.
#include <hip/hip_runtime.h>

#include "checkpoint_codes.h"
#include "local_ops.h"

namespace moshpit {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kBlock = 256, kTileO = 128, kTileI = 128, kTokens = 32;
// LDS row of a tile: 64 bytes more than 256, so that the 4 token rows a transposing read takes at a time lie in
// different banks (they would all lie in the same ones otherwise)
constexpr int kRowElems = 128 + 32;

struct Split {
    int32_t tiles_o, tiles_i, parts;     // tiles of a peer's matrix; parts of its tokens
    int64_t tokens;                      // tokens of a part, a multiple of kTokens
};

// 8 tokens of a column for each lane: lane l gets column l % 32 and tokens 8 * (l / 32) .. + 7 of the 16 from `tile` on.
__device__ __forceinline__ bf16x8 operand(const uint16_t *tile)
{
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    const int lane = threadIdx.x & 63, j = lane & 15;
    const uint16_t *at = tile + (8 * (lane >> 5) + (j >> 2)) * kRowElems + 16 * ((lane >> 4) & 1) + 4 * (j & 3);
    const s16x4 low = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)at);
    const s16x4 high = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(at + 4 * kRowElems));
    typedef short s16x8 __attribute__((ext_vector_type(8)));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(low, high, 0, 1, 2, 3, 4, 5, 6, 7));
}

// f as a sum of bfloat16 values: all of it, or its upper 8 significant bits, the next 8 and the last 8 (cut off, so that
// the largest binary32 values do not round up to infinity).  An infinity or NaN is all in the first part.
template <int PARTS> __device__ __forceinline__ void split_parts(float f, float (&part)[PARTS])
{
    if constexpr (PARTS == 1) part[0] = f;
    else {
        const uint32_t bits = __float_as_uint(f);
        const bool finite = (bits & 0x7f800000u) != 0x7f800000u;
        part[0] = finite ? __uint_as_float(bits & 0xffff0000u) : f;
        const float rest = finite ? f - part[0] : 0.f;
        part[1] = __uint_as_float(__float_as_uint(rest) & 0xffff0000u);
        part[2] = rest - part[1];
    }
}

template <int YT, int ST, bool ADD, bool PARTIAL>
__global__ __launch_bounds__(kBlock) void weight_grad_kernel(const char *__restrict__ dy, const int8_t *__restrict__ codes,
                                                             const uint8_t *__restrict__ scales, WeightGradGeom g, Split s, char *__restrict__ base,
                                                             float *__restrict__ partials)
{
    constexpr int EY = YT == 0 ? 4 : 2, PARTS = YT == 0 ? 3 : 1;
    __shared__ __attribute__((aligned(16))) uint16_t lds_y[PARTS][kTokens * kRowElems];
    __shared__ __attribute__((aligned(16))) uint16_t lds_x[kTokens * kRowElems];
    uint32_t b = blockIdx.x;
    const int32_t ti = b % s.tiles_i;
    b /= s.tiles_i;
    const int32_t to = b % s.tiles_o;
    b /= s.tiles_o;
    const int32_t part = b % s.parts;
    const int64_t peer = b / s.parts;
    const int64_t o0 = int64_t(to) * kTileO, c0 = int64_t(ti) * kTileI;
    const int64_t t_begin = part * s.tokens, t_end = t_begin + s.tokens < g.T ? t_begin + s.tokens : g.T;
    const int64_t groups = checkpoint_groups(g.ins);

    // this thread's share of a tile: 8 outputs of tokens y_row and y_row + 16, 16 codes of token x_row
    const int y_row = threadIdx.x >> 4, y_col = (threadIdx.x & 15) * 8;
    const int x_row = threadIdx.x >> 3, x_col = (threadIdx.x & 7) * 16;
    const bool y_whole = o0 + y_col + 8 <= g.outs, x_whole = c0 + x_col + 16 <= g.ins;
    float y[2][8];
    u32x4 x;
    uint32_t byte;
    auto load = [&](int64_t t0) {
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            const int64_t t = t0 + y_row + 16 * n;
#pragma unroll
            for (int k = 0; k < 8; ++k) y[n][k] = 0.f;
            if (t >= t_end) continue;
            const char *from = dy + ((peer * g.T + t) * g.dy_stride + o0 + y_col) * EY;
            if (y_whole) load_elems<YT, 8>(from, y[n]);
            else
                for (int k = 0; k < 8; ++k)
                    if (o0 + y_col + k < g.outs) y[n][k] = load_one<YT>(from + k * EY);
        }
        const int64_t t = t0 + x_row;
        x = u32x4{0, 0, 0, 0};
        byte = 1;
        if (t >= t_end || c0 + x_col >= g.ins) return;
        const int64_t row = peer * g.T + t;
        const int8_t *from = codes + row * g.ins + c0 + x_col;
        byte = scales[row * groups + (c0 + x_col) / kCheckpointGroup];
        if (x_whole) {
            typedef u32x4 any_t __attribute__((aligned(1)));
            x = *reinterpret_cast<const any_t *>(from);
        } else {
            for (int k = 0; k < 16; ++k)
                if (c0 + x_col + k < g.ins) x[k >> 2] |= (static_cast<uint32_t>(from[k]) & 0xffu) << (8 * (k & 3));
        }
    };
    auto to_lds = [&]() {
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            float parts[PARTS][8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                float p[PARTS];
                split_parts<PARTS>(y[n][k], p);
#pragma unroll
                for (int q = 0; q < PARTS; ++q) parts[q][k] = p[q];
            }
#pragma unroll
            for (int q = 0; q < PARTS; ++q)
                *reinterpret_cast<u32x4 *>(lds_y[q] + (y_row + 16 * n) * kRowElems + y_col) = Vec<1, 8>::narrow(parts[q]);
        }
        const float factor = to_value_factor(byte);
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            float f[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) f[k] = factor * code_of(x[2 * n + (k >> 2)], k & 3);
            *reinterpret_cast<u32x4 *>(lds_x + x_row * kRowElems + x_col + 8 * n) = Vec<1, 8>::narrow(f);
        }
    };

    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int wo = (wave >> 1) * 64, wi = (wave & 1) * 64;
    f32x16 acc[2][2] = {};
    if (t_begin < t_end) load(t_begin);
    for (int64_t t0 = t_begin; t0 < t_end; t0 += kTokens) {
        to_lds();
        __syncthreads();
        if (t0 + kTokens < t_end) load(t0 + kTokens);
#pragma unroll
        for (int k0 = 0; k0 < kTokens; k0 += 16) {
            bf16x8 xi[2];
#pragma unroll
            for (int n = 0; n < 2; ++n) xi[n] = operand(lds_x + k0 * kRowElems + wi + 32 * n);
#pragma unroll
            for (int q = PARTS - 1; q >= 0; --q)
#pragma unroll
                for (int m = 0; m < 2; ++m) {
                    const bf16x8 yo = operand(lds_y[q] + k0 * kRowElems + wo + 32 * m);
#pragma unroll
                    for (int n = 0; n < 2; ++n) acc[m][n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(yo, xi[n], acc[m][n], 0, 0, 0);
                }
        }
        __syncthreads();
    }
    constexpr int ES = ST == 0 ? 4 : 2;
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int k = 0; k < 16; ++k) {
                const int64_t o = o0 + wo + 32 * m + 8 * (k >> 2) + 4 * (lane >> 5) + (k & 3), c = c0 + wi + 32 * n + (lane & 31);
                if (o >= g.outs || c >= g.ins) continue;
                if constexpr (PARTIAL) partials[((part * g.N + peer) * g.outs + o) * g.ins + c] = acc[m][n][k];
                else {
                    char *at = base + (peer * g.peer_stride + o * g.ins + c) * ES;
                    store_one<ST>(at, ADD ? load_one<ST>(at) + acc[m][n][k] : acc[m][n][k]);
                }
            }
}

// The parts of every sum, added in the order of their tokens.
template <int ST, bool ADD>
__global__ __launch_bounds__(kBlock) void weight_grad_join_kernel(const float *__restrict__ partials, int32_t parts, int64_t N, int64_t count,
                                                                  int64_t peer_stride, char *__restrict__ base)
{
    constexpr int ES = ST == 0 ? 4 : 2;
    const int64_t all = N * count;
    for (int64_t k = int64_t(blockIdx.x) * kBlock + threadIdx.x; k < all; k += int64_t(gridDim.x) * kBlock) {
        float sum = 0.f;
        for (int32_t p = 0; p < parts; ++p) sum += partials[p * all + k];
        char *at = base + ((k / count) * peer_stride + k % count) * ES;
        store_one<ST>(at, ADD ? load_one<ST>(at) + sum : sum);
    }
}

Split split_of(const WeightGradGeom &g, int compute_units)
{
    Split s;
    s.tiles_o = static_cast<int32_t>((g.outs + kTileO - 1) / kTileO);
    s.tiles_i = static_cast<int32_t>((g.ins + kTileI - 1) / kTileI);
    const int64_t tiles = g.N * s.tiles_o * s.tiles_i, steps = (g.T + kTokens - 1) / kTokens;
    // parts of at least 8 steps until every compute unit has two blocks
    int64_t parts = 2 * compute_units / tiles;
    if (parts > steps / 8) parts = steps / 8;
    if (parts < 1) parts = 1;
    const int64_t each = (steps + parts - 1) / parts;
    s.tokens = (each > 0 ? each : 1) * kTokens;
    s.parts = static_cast<int32_t>(steps > 0 ? (steps + each - 1) / each : 1);
    return s;
}

template <int YT, int ST, bool ADD>
void launch(const void *dy, const int8_t *codes, const uint8_t *scales, const WeightGradGeom &g, void *base, float *work, const Split &s,
            hipStream_t stream)
{
    const uint32_t blocks = static_cast<uint32_t>(g.N * s.parts * s.tiles_o * s.tiles_i);
    const char *from = static_cast<const char *>(dy);
    char *to = static_cast<char *>(base);
    if (s.parts == 1) {
        weight_grad_kernel<YT, ST, ADD, false><<<blocks, kBlock, 0, stream>>>(from, codes, scales, g, s, to, nullptr);
        return;
    }
    weight_grad_kernel<YT, 0, false, true><<<blocks, kBlock, 0, stream>>>(from, codes, scales, g, s, nullptr, work);
    const int64_t count = g.outs * g.ins, join_blocks = (g.N * count + kBlock - 1) / kBlock;
    weight_grad_join_kernel<ST, ADD><<<static_cast<uint32_t>(join_blocks < 8192 ? join_blocks : 8192), kBlock, 0, stream>>>(work, s.parts, g.N, count,
                                                                                                                            g.peer_stride, to);
}

}  // namespace

bool weight_grad_fits(const WeightGradGeom &g)
{
    const int64_t tiles_o = (g.outs + kTileO - 1) / kTileO, tiles_i = (g.ins + kTileI - 1) / kTileI;
    return tiles_o * tiles_i <= 0xffffffffLL / kBlock / g.N;                     // (more than one part only where that is few)
}

int64_t weight_grad_work_bytes(const WeightGradGeom &g, int dy_dtype, int compute_units)
{
    const Split s = split_of(g, compute_units);
    return s.parts == 1 ? 0 : 4 * s.parts * g.N * g.outs * g.ins;
}

hipError_t launch_weight_grad(const void *dy, int dy_dtype, const int8_t *codes, const uint8_t *scales, const WeightGradGeom &g, void *base,
                              int state_dtype, bool accumulate, void *work, int compute_units, hipStream_t stream)
{
    const Split s = split_of(g, compute_units);
    auto go = [&](auto add) {
        constexpr bool ADD = decltype(add)::value;
        auto f = dy_dtype == 0 ? (state_dtype == 0 ? launch<0, 0, ADD> : launch<0, 1, ADD>) : (state_dtype == 0 ? launch<1, 0, ADD> : launch<1, 1, ADD>);
        f(dy, codes, scales, g, base, static_cast<float *>(work), s, stream);
    };
    if (accumulate) go(std::true_type{});
    else go(std::false_type{});
    return hipGetLastError();
}

}  // namespace moshpit
