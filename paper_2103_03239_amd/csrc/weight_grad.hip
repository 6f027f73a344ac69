// The gradient of a linear layer's weights, for every peer, from the layer's input saved in 8 bits, for gfx950:
//   grad_i[o][c] = sum over t of dy[i * T + t][o] * x[i * T + t][c],   x = code * 2^e (checkpoint_codes.h)
//
// A matrix product whose summed index, the token, is the slow one of both operands.  Tiles of kTokens tokens are
// staged through LDS as they lie in memory, [token][column] in bfloat16, and the transposing LDS reads of gfx950
// hand the matrix instructions their operands, 8 tokens of a column to a lane.  The codes become bfloat16 on their
// way into LDS, which is exact.  A binary32 dy is staged as three bfloat16 parts (8 significant bits each, exact
// down to 2^-133), whose products with x are exact in binary32: three matrix instructions in place of one, at sixteen
// times the rate of the binary32 ones.  Sums are binary32.
//
// Bound by the matrix cores where the matrices are large, and by what feeds them: 16 matrices of 1024 x 4096 from 4096
// tokens of bfloat16 dy in 501 to 535 us by card, 1030 to 1100 TFLOP/s of the 1301 that a plain bfloat16 product reaches.  dy
// through registers on its way into LDS takes 6 % longer (613 against 578 us on one card, back to back).  The codes go through
// registers, since they become bfloat16 on the way.
#include <hip/hip_runtime.h>

#include "checkpoint_codes.h"
#include "local_ops.h"
#include "moshpit_internal.h"

namespace moshpit {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kBlock = 256;              // of the join

// How the sums of a matrix are tiled: WO x WI waves a block, MO x MI blocks of 32 x 32 sums a wave, K tokens a step.
template <int WO_, int WI_, int MO_, int MI_, int K_> struct Tile {
    static constexpr int WO = WO_, WI = WI_, MO = MO_, MI = MI_, K = K_;
    static constexpr int O = 32 * WO * MO, I = 32 * WI * MI, THREADS = 64 * WO * WI;
};

struct Split {
    int32_t tiles_o, tiles_i, parts;     // tiles of a peer's matrix; parts of its tokens
    int64_t tokens;                      // tokens of a part, a multiple of the tokens of a step
};

// A tile in LDS: rows of tokens, C columns in bfloat16.  A transposing read takes 64 bytes of 4 token rows at a time; a row is a
// whole number of times as long as all banks together, so the 64-byte chunks of row t are stored with their number xor
// t % 4, and the four rows' lie in different banks.
template <int C> __device__ __forceinline__ uint32_t lds_at(int row, int col)
{
    return static_cast<uint32_t>(row * C + ((col >> 5 ^ (row & 3)) << 5) + (col & 31));
}

// 8 tokens of a column for each lane: lane l gets column l % 32 of the 32 from `col` on and tokens 8 * (l / 32) .. + 7 of the 16
// from `row` on (both multiples of 32 and 16).
template <int C> __device__ __forceinline__ bf16x8 operand(const uint16_t *tile, int row, int col)
{
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    const int lane = threadIdx.x & 63, j = lane & 15;
    const uint16_t *at = tile + lds_at<C>(8 * (lane >> 5) + (j >> 2), col + 16 * ((lane >> 4) & 1) + 4 * (j & 3)) + row * C;
    const s16x4 low = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)at);
    const s16x4 high = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(at + 4 * C));
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

// A 128-bit value moved down by `bytes` (0 .. 16 and more), zeros from above.
__device__ __forceinline__ u32x4 moved_down(const u32x4 &v, int bytes)
{
    uint64_t low = uint64_t(v[1]) << 32 | v[0], high = uint64_t(v[3]) << 32 | v[2];
    if (bytes >= 8) {
        low = high;
        high = 0;
        bytes -= 8;
    }
    if (bytes >= 8) low = bytes = 0;
    if (bytes > 0) {
        low = low >> (8 * bytes) | high << (64 - 8 * bytes);
        high >>= 8 * bytes;
    }
    return u32x4{static_cast<uint32_t>(low), static_cast<uint32_t>(low >> 32), static_cast<uint32_t>(high), static_cast<uint32_t>(high >> 32)};
}

// What a thread has in flight of a step's tiles: 8 outputs of YN tokens as they lie in memory, 16 codes of XN tokens and their scale
// bytes.  Columns beyond a row's end: the thread reads the row's last ones instead and moves them to their place on the way into LDS;
// tokens beyond the last: it reads the last one and puts zeros into LDS.
//
// DIRECT: dy goes from memory into LDS without passing through registers, a wave 1 KiB at a time: lane l's 16 bytes to where the wave's
// rows begin + 16 * l, so the lane reads the columns that lds_at() puts there.  Columns beyond the row's end are read as the tile's
// first ones (their sums are not stored), tokens beyond the last as the last one and then overwritten with zeros.
template <int YT, typename T, bool DIRECT> struct Staged {
    static constexpr int PARTS = YT == 0 ? 3 : 1, EY = YT == 0 ? 4 : 2;
    static constexpr int TO = T::O, TI = T::I, K = T::K;
    static constexpr int Y_THREADS = TO / 8, YR = T::THREADS / Y_THREADS, YN = K / YR;        // threads of a token, tokens at a time, times
    static constexpr int X_THREADS = TI / 16, XR = T::THREADS / X_THREADS, XN = K / XR;
    static constexpr int YH = DIRECT ? 0 : YN;                                 // of them through registers
    u32x4 y[YH > 0 ? YH : 1][EY / 2], x[XN];
    uint32_t byte[XN];

    struct Place {
        const char *y;                   // the part's first token: its outputs, codes and scales
        const int8_t *x;
        const uint8_t *scale;
        int64_t y_step, x_step, scale_step;     // bytes from a token to the next
        uint32_t y_at, x_at, scale_at;   // this thread's, from there on
        uint32_t y_from, x_from, scale_from;    // the same without the token
        int32_t y_over, x_over;          // columns this thread's were moved back
        bool whole;                      // no thread's were
    };
    __device__ __forceinline__ static int y_row() { return threadIdx.x / Y_THREADS; }
    __device__ __forceinline__ static int y_col() { return threadIdx.x % Y_THREADS * 8; }
    __device__ __forceinline__ static int x_row() { return threadIdx.x / X_THREADS; }
    __device__ __forceinline__ static int x_col() { return threadIdx.x % X_THREADS * 16; }

    // y_left, x_left: columns of the matrix from the tile's first on (the matrix has at least 8 and 16).
    __device__ __forceinline__ static void place_thread(Place &p, int64_t y_left, int64_t x_left, int64_t o0, int64_t c0)
    {
        p.whole = y_left >= TO && x_left >= TI;
        const int32_t yl = y_left < TO ? static_cast<int32_t>(y_left) : TO, xl = x_left < TI ? static_cast<int32_t>(x_left) : TI;
        p.y_over = y_col() + 8 > yl ? y_col() + 8 - yl : 0;
        p.x_over = x_col() + 16 > xl ? x_col() + 16 - xl : 0;
        const int32_t yc = y_col() - p.y_over, xc = x_col() - p.x_over;         // (may be before the tile, not before the row)
        if constexpr (DIRECT) {
            const int32_t col = ((y_col() >> 5 ^ (y_row() & 3)) << 5) + (y_col() & 31);
            p.y_from = static_cast<uint32_t>((o0 + (col < yl ? col : 0)) * EY);
        } else
            p.y_from = static_cast<uint32_t>((o0 + yc) * EY);
        p.x_from = static_cast<uint32_t>(c0 + xc);
        p.scale_from = static_cast<uint32_t>((c0 + (x_col() < xl ? x_col() : xl - 1)) / kCheckpointGroup);
        p.y_at = p.y_from + static_cast<uint32_t>(y_row() * p.y_step);
        p.x_at = p.x_from + static_cast<uint32_t>(x_row() * p.x_step);
        p.scale_at = p.scale_from + static_cast<uint32_t>(x_row() * p.scale_step);
    }

    // dy of the step whose first token is number t of the part's `count`, on its way into LDS.  FULL: the step is known to have K tokens.
    template <bool FULL> __device__ __forceinline__ static void direct_y(const Place &p, int64_t t, int64_t count, uint16_t *lds_y)
    {
        typedef __attribute__((address_space(3))) uint16_t lds_u16;
        static_assert(YR % 4 == 0 && 64 % Y_THREADS == 0 && YT == 1);           // (rows of a thread have the same number mod 4)
        const int wave_row = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * (64 / Y_THREADS);
        const __amdgpu_buffer_rsrc_t from = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(p.y + t * p.y_step), 0, 0xffffffffu, 0x00027000);
#pragma unroll
        for (int n = 0; n < YN; ++n) {
            uint32_t at = p.y_at, down = static_cast<uint32_t>(YR * n * p.y_step);       // below 2^31: K rows of up to 2^25 bytes
            if constexpr (!FULL) {
                const int64_t row = t + y_row() + YR * n < count ? y_row() + YR * n : count - 1 - t;
                at = p.y_from + static_cast<uint32_t>(row) * static_cast<uint32_t>(p.y_step);
                down = 0;
            }
            __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (lds_u16 *)(lds_y + (wave_row + YR * n) * TO), 16, at, down, 0, 0);
        }
    }
    // All that this wave requested with direct_y() is in LDS; tokens from number `left` on become zeros.
    template <bool FULL> __device__ __forceinline__ static void direct_done(int64_t left, uint16_t *lds_y)
    {
        __builtin_amdgcn_s_waitcnt(0x0f70);                                     // vmcnt(0)
        if (!FULL && left < K) {
#pragma unroll
            for (int n = 0; n < YN; ++n)
                if (y_row() + YR * n >= left) *reinterpret_cast<u32x4 *>(lds_y + (y_row() + YR * n) * TO + y_col()) = u32x4{0, 0, 0, 0};
        }
    }

    // The step whose first token is number t of the part's `count`.
    __device__ __forceinline__ void load(const Place &p, int64_t t, int64_t count)
    {
        typedef u32x4 any_t __attribute__((aligned(1)));
        if (t + K <= count) {
#pragma unroll
            for (int n = 0; n < YH; ++n) {
                const char *from = p.y + (t + YR * n) * p.y_step + p.y_at;
#pragma unroll
                for (int q = 0; q < EY / 2; ++q) y[n][q] = *reinterpret_cast<const any_t *>(from + 16 * q);
            }
#pragma unroll
            for (int n = 0; n < XN; ++n) {
                x[n] = *reinterpret_cast<const any_t *>(p.x + (t + XR * n) * p.x_step + p.x_at);
                byte[n] = *(p.scale + (t + XR * n) * p.scale_step + p.scale_at);
            }
            return;
        }
        const int32_t left = static_cast<int32_t>(count - t);                   // 1 .. K - 1
#pragma unroll
        for (int n = 0; n < YH; ++n) {
            const int32_t row = y_row() + YR * n < left ? y_row() + YR * n : left - 1;
            const char *from = p.y + t * p.y_step + (int64_t(row) * p.y_step + p.y_from);
#pragma unroll
            for (int q = 0; q < EY / 2; ++q) y[n][q] = *reinterpret_cast<const any_t *>(from + 16 * q);
        }
#pragma unroll
        for (int n = 0; n < XN; ++n) {
            const int32_t row = x_row() + XR * n < left ? x_row() + XR * n : left - 1;
            x[n] = *reinterpret_cast<const any_t *>(p.x + t * p.x_step + (int64_t(row) * p.x_step + p.x_from));
            byte[n] = (p.scale + t * p.scale_step)[row * p.scale_step + p.scale_from];
        }
    }
    // Before the step goes into LDS, where its tile or tokens are not whole.  left: tokens from the step's first on.
    __device__ __forceinline__ void trim(const Place &p, int64_t left)
    {
        if (!p.whole) {
#pragma unroll
            for (int n = 0; n < YH; ++n) {
                if constexpr (YT == 1) y[n][0] = moved_down(y[n][0], 2 * p.y_over);
                else {
                    const int over = p.y_over < 8 ? p.y_over : 8;               // 8 values of 4 bytes: 4 and more move a vector down
                    const u32x4 none = {0, 0, 0, 0}, low = over >= 4 ? (over >= 8 ? none : y[n][1]) : y[n][0], high = over >= 4 ? none : y[n][1];
                    const int by = over & 3;
                    u32x4 a, b;
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        a[k] = by == 0 ? low[k] : by == 1 ? (k < 3 ? low[(k + 1) & 3] : high[0]) : by == 2 ? (k < 2 ? low[(k + 2) & 3] : high[(k + 2) & 3])
                                                                                                 : (k < 1 ? low[3] : high[(k + 3) & 3]);
                        b[k] = by == 0 ? high[k] : k + by < 4 ? high[by == 1 ? (k + 1) & 3 : by == 2 ? (k + 2) & 3 : (k + 3) & 3] : 0u;
                    }
                    y[n][0] = a;
                    y[n][1] = b;
                }
            }
#pragma unroll
            for (int n = 0; n < XN; ++n) x[n] = moved_down(x[n], p.x_over);
        }
        if (left < K) {
#pragma unroll
            for (int n = 0; n < YH; ++n)
                if (y_row() + YR * n >= left)
#pragma unroll
                    for (int q = 0; q < EY / 2; ++q) y[n][q] = u32x4{0, 0, 0, 0};
#pragma unroll
            for (int n = 0; n < XN; ++n)
                if (x_row() + XR * n >= left) {
                    x[n] = u32x4{0, 0, 0, 0};
                    byte[n] = 1;
                }
        }
    }

    // Nothing of the codes and scales is waited for before this point.
    __device__ __forceinline__ void wanted()
    {
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int n = 0; n < XN; ++n) asm volatile("" : "+v"(x[n]), "+v"(byte[n]));
    }

    // Outputs of times n: into LDS, in parts.
    __device__ __forceinline__ void store_y(int n, uint16_t *lds_y) const
    {
        const uint32_t at = lds_at<TO>(y_row() + YR * n, y_col());
        if constexpr (YT == 1) *reinterpret_cast<u32x4 *>(lds_y + at) = y[n][0];
        else {
            float part[PARTS][8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                float f[PARTS];
                split_parts<PARTS>(__uint_as_float(y[n][k / 4][k & 3]), f);
#pragma unroll
                for (int q = 0; q < PARTS; ++q) part[q][k] = f[q];
            }
#pragma unroll
            for (int q = 0; q < PARTS; ++q) *reinterpret_cast<u32x4 *>(lds_y + q * K * TO + at) = Vec<1, 8>::narrow(part[q]);
        }
    }
    // Codes of times n as bfloat16 values, code * 2^e.  (Signed bytes convert in one instruction each; unsigned ones, with 128 * 2^e taken
    // off in a fused multiply-add, would take as many and have no 128 * 2^e for the largest groups.)  The two writes meet in the banks;
    // choosing by lane which half goes first avoids that and costs more: 568 us instead of 550 for 16 x 1024 x 4096 from 4096 tokens.
    __device__ __forceinline__ void store_x(int n, uint16_t *lds_x) const
    {
        const float factor = to_value_factor(byte[n]);
        u32x4 half[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float f[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) f[k] = factor * code_of(x[n][2 * h + k / 4], k & 3);
            half[h] = Vec<1, 8>::narrow(f);
        }
        const int row = x_row() + XR * n, col = x_col();
        *reinterpret_cast<u32x4 *>(lds_x + lds_at<TI>(row, col)) = half[0];
        *reinterpret_cast<u32x4 *>(lds_x + lds_at<TI>(row, col) + 8) = half[1];
    }
};

template <int YT, int ST, bool ADD, bool PARTIAL, typename T, bool DIRECT>
__global__ __launch_bounds__(T::THREADS, 2)
void weight_grad_kernel(const char *__restrict__ dy, const int8_t *__restrict__ codes, const uint8_t *__restrict__ scales, WeightGradGeom g,
                        Split s, char *__restrict__ base, float *__restrict__ partials)
{
    using St = Staged<YT, T, DIRECT>;
    constexpr int PARTS = St::PARTS, TO = T::O, TI = T::I, K = T::K, MO = T::MO, MI = T::MI, STEPS = K / 16;
    constexpr int Y_ELEMS = PARTS * K * TO, ELEMS = Y_ELEMS + K * TI;
    // Two buffers of a step's tiles.  With DIRECT they are four variables: an access to one does not wait for what is on its way
    // into another.
    __shared__ __attribute__((aligned(16))) uint16_t y_even[DIRECT ? Y_ELEMS : 2 * ELEMS];
    __shared__ __attribute__((aligned(16))) uint16_t y_odd[DIRECT ? Y_ELEMS : 8];
    __shared__ __attribute__((aligned(16))) uint16_t x_even[DIRECT ? K * TI : 8];
    __shared__ __attribute__((aligned(16))) uint16_t x_odd[DIRECT ? K * TI : 8];

    // a die takes a run of tiles, so that the tiles of a peer share its operands in the die's cache
    uint32_t b = die_run(blockIdx.x, gridDim.x);
    const int32_t ti = b % s.tiles_i;
    b /= s.tiles_i;
    const int32_t to = b % s.tiles_o;
    b /= s.tiles_o;
    const int32_t part = b % s.parts;
    const int64_t peer = b / s.parts;
    const int64_t o0 = int64_t(to) * TO, c0 = int64_t(ti) * TI;
    const int64_t t_begin = part * s.tokens, count = t_begin + s.tokens < g.T ? s.tokens : g.T - t_begin;
    const int64_t groups = checkpoint_groups(g.ins), row0 = peer * g.T + t_begin;

    typename St::Place place;
    place.y_step = g.dy_stride * St::EY;
    place.x_step = g.ins;
    place.scale_step = groups;
    place.y = dy + row0 * place.y_step;
    place.x = codes + row0 * place.x_step;
    place.scale = scales + row0 * groups;
    St::place_thread(place, g.outs - o0, g.ins - c0, o0, c0);

    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int wo = wave / T::WI * 32 * MO, wi = wave % T::WI * 32 * MI;
    f32x16 acc[MO][MI] = {};
    // The products of a step are taken in UNITS of MO * MI matrix instructions: 16 tokens and one part of dy.  A unit's operands
    // are read from LDS before the products of the unit before it.  Step k + 1's tiles go into the other buffer between the
    // products of the second half of step k, and step k + 2's are requested right after.
    constexpr int UNITS = STEPS * PARTS, LATE = UNITS / 2;
    St st;
    bf16x8 xi[2][MI], yo[2][MO];
    auto read = [&](const uint16_t *lds_y, const uint16_t *lds_x, int u) {
        const uint16_t *tile_y = lds_y + (PARTS - 1 - u % PARTS) * K * TO;
        const int k = u / PARTS;
        if (u % PARTS == 0)
#pragma unroll
            for (int n = 0; n < MI; ++n) xi[k & 1][n] = operand<TI>(lds_x, 16 * k, wi + 32 * n);
#pragma unroll
        for (int m = 0; m < MO; ++m) yo[u & 1][m] = operand<TO>(tile_y, 16 * k, wo + 32 * m);
    };
    auto multiply = [&](int u) {
#pragma unroll
        for (int m = 0; m < MO; ++m)
#pragma unroll
            for (int n = 0; n < MI; ++n)
                acc[m][n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(yo[u & 1][m], xi[u / PARTS & 1][n], acc[m][n], 0, 0, 0);
    };
    auto to_lds = [&](uint16_t *lds_y, uint16_t *lds_x, int part, int parts) {
#pragma unroll
        for (int n = part * St::YH / parts; n < (part + 1) * St::YH / parts; ++n) st.store_y(n, lds_y);
#pragma unroll
        for (int n = part * St::XN / parts; n < (part + 1) * St::XN / parts; ++n) st.store_x(n, lds_x);
    };
    int64_t t = 0;
    if (count > 0) {
        if constexpr (DIRECT) St::template direct_y<false>(place, 0, count, y_even);
        st.load(place, 0, count);
        st.trim(place, count);
        to_lds(y_even, DIRECT ? x_even : y_even + Y_ELEMS, 0, 1);
        if constexpr (DIRECT) St::template direct_done<false>(count, y_even);
        if (K < count) st.load(place, K, count);
        __syncthreads();
    }
    // step t's products from `now`, step t + K's tiles into `next`
    auto step = [&](auto full, const uint16_t *y_now, const uint16_t *x_now, uint16_t *y_next, uint16_t *x_next) {
        constexpr bool FULL = decltype(full)::value;
        if constexpr (DIRECT) St::template direct_y<FULL>(place, t + K, count, y_next);
        if constexpr (DIRECT) __builtin_amdgcn_sched_barrier(0);                // (requested now, not when the products are through)
        read(y_now, x_now, 0);
#pragma unroll
        for (int u = 0; u < UNITS; ++u) {
            if constexpr (DIRECT)
                if (u == LATE) st.wanted();
            if (!FULL && u == LATE && (!place.whole || t + 2 * K > count)) st.trim(place, count - t - K);
            if (u + 1 < UNITS) read(y_now, x_now, u + 1);
            multiply(u);
            if (u >= LATE) to_lds(y_next, x_next, u - LATE, UNITS - LATE);
        }
        if constexpr (DIRECT) St::template direct_done<FULL>(count - t - K, y_next);
        if (t + 2 * K < count) st.load(place, t + 2 * K, count);
        __syncthreads();
        t += K;
    };
    const uint16_t *y_last = y_even, *x_last = x_even;
    if constexpr (DIRECT) {              // (two steps by name: which variable an access meets has to be known where it stands)
        while (t + 3 * K <= count) {
            step(std::true_type{}, y_even, x_even, y_odd, x_odd);
            step(std::true_type{}, y_odd, x_odd, y_even, x_even);
        }
        const bool odd_whole = t + 2 * K <= count;
        if (odd_whole) step(std::true_type{}, y_even, x_even, y_odd, x_odd);
        bool odd = odd_whole;
        if (t + K < count) {
            step(std::false_type{}, odd ? y_odd : y_even, odd ? x_odd : x_even, odd ? y_even : y_odd, odd ? x_even : x_odd);
            odd = !odd;
        }
        y_last = odd ? y_odd : y_even;
        x_last = odd ? x_odd : x_even;
    } else {
        uint32_t now = 0;
        for (; t + K < count; now = ELEMS - now)
            step(std::false_type{}, y_even + now, y_even + now + Y_ELEMS, y_even + (ELEMS - now), y_even + (ELEMS - now) + Y_ELEMS);
        y_last = y_even + now;
        x_last = y_last + Y_ELEMS;
    }
    if (count > 0) {
        read(y_last, x_last, 0);
#pragma unroll
        for (int u = 0; u < UNITS; ++u) {
            if (u + 1 < UNITS) read(y_last, x_last, u + 1);
            __builtin_amdgcn_sched_barrier(0);
            multiply(u);
        }
    }
    // lane l holds column l % 32 of a 32 x 32 block, rows 8 * (k / 4) + 4 * (l / 32) + k % 4
    constexpr int ES = PARTIAL || ST == 0 ? 4 : 2;
    char *out = PARTIAL ? reinterpret_cast<char *>(partials + (part * g.N + peer) * g.outs * g.ins) : base + peer * g.peer_stride * ES;
    const int32_t o_left = static_cast<int32_t>(g.outs - o0 < TO ? g.outs - o0 : TO) - wo - 4 * (lane >> 5);
    const int32_t c_left = static_cast<int32_t>(g.ins - c0 < TI ? g.ins - c0 : TI) - wi - (lane & 31);
    const uint32_t lane_at = static_cast<uint32_t>((4 * (lane >> 5) * g.ins + (lane & 31)) * ES);
    out += ((o0 + wo) * g.ins + c0 + wi) * ES;
#pragma unroll
    for (int m = 0; m < MO; ++m)
#pragma unroll
        for (int n = 0; n < MI; ++n) {
            if (32 * n >= c_left) continue;
#pragma unroll
            for (int k = 0; k < 16; ++k) {
                const int row = 32 * m + 8 * (k >> 2) + (k & 3);
                if (row >= o_left) continue;
                char *at = out + (row * g.ins + 32 * n) * ES + lane_at;
                if constexpr (PARTIAL) *reinterpret_cast<float *>(at) = acc[m][n][k];
                else store_one<ST>(at, ADD ? load_one<ST>(at) + acc[m][n][k] : acc[m][n][k]);
            }
            __builtin_amdgcn_sched_barrier(0);                       // (sums of other blocks not requested yet)
        }
}

// Matrices of fewer than 8 outputs or 16 inputs, by one thread a sum: less than a tile's vectors.
template <int YT, int ST, bool ADD>
__global__ __launch_bounds__(kBlock) void thin_weight_grad_kernel(const char *__restrict__ dy, const int8_t *__restrict__ codes,
                                                                  const uint8_t *__restrict__ scales, WeightGradGeom g, char *__restrict__ base)
{
    constexpr int EY = YT == 0 ? 4 : 2, ES = ST == 0 ? 4 : 2;
    const int64_t k = int64_t(blockIdx.x) * kBlock + threadIdx.x, sums = g.outs * g.ins;
    if (k >= g.N * sums) return;
    const int64_t peer = k / sums, o = k % sums / g.ins, c = k % g.ins, groups = checkpoint_groups(g.ins);
    float sum = 0.f;
#pragma unroll 4
    for (int64_t t = peer * g.T; t < (peer + 1) * g.T; ++t)
        sum = fmaf(load_one<YT>(dy + (t * g.dy_stride + o) * EY),
                   to_value_factor(scales[t * groups + c / kCheckpointGroup]) * static_cast<float>(codes[t * g.ins + c]), sum);
    char *at = base + (peer * g.peer_stride + k % sums) * ES;
    store_one<ST>(at, ADD ? load_one<ST>(at) + sum : sum);
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
        for (int32_t p = 0; p < parts; p += 8) {                      // eight requested at a time
            float v[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) v[u] = p + u < parts ? partials[(p + u) * all + k] : 0.f;
#pragma unroll
            for (int u = 0; u < 8; ++u) sum += v[u];
        }
        char *at = base + ((k / count) * peer_stride + k % count) * ES;
        store_one<ST>(at, ADD ? load_one<ST>(at) + sum : sum);
    }
}

// Which tile: 256 x 256 sums read half as much LDS for a product as 128 x 128, where enough of them are there to fill the chip and
// they do not reach far beyond the matrix (64 matrices of 2496 x 32 from 902 tokens in bfloat16: 73 us with the small ones, 107 with the wide).
bool wide_tiles(const WeightGradGeom &g, int compute_units)
{
    auto sums = [&](int64_t tile) { return ((g.outs + tile - 1) / tile) * ((g.ins + tile - 1) / tile) * tile * tile; };
    return g.N * sums(256) / (256 * 256) >= compute_units && 4 * sums(256) <= 5 * sums(128);
}

Split split_of(const WeightGradGeom &g, int dy_dtype, int compute_units)
{
    const bool wide = wide_tiles(g, compute_units);
    const int64_t tile = wide ? 256 : 128, step = wide && dy_dtype != 0 ? 64 : 32;
    Split s;
    s.tiles_o = static_cast<int32_t>((g.outs + tile - 1) / tile);
    s.tiles_i = static_cast<int32_t>((g.ins + tile - 1) / tile);
    const int64_t tiles = g.N * s.tiles_o * s.tiles_i, steps = (g.T + step - 1) / step;
    // Parts of at least 8 steps until every compute unit has two blocks.  A step of binary32 takes 1 to 2 us, three times one of bfloat16, the
    // join about 4: where the sums are few, 4 steps there (2 x 393 x 68 from 371 tokens: 13.6 us, with 8 23.5; 16 x 256 x 256 from 300:
    // 18.0 and 16.1; in bfloat16 2 x 392 x 64 from 371: 12.7 and 10.0).
    const int64_t least = dy_dtype == 0 && g.N * g.outs * g.ins <= (1 << 19) ? 4 : 8;
    int64_t parts = wide ? 1 : 2 * compute_units / tiles;
    if (parts > steps / least) parts = steps / least;
    if (parts < 1) parts = 1;
    const int64_t each = (steps + parts - 1) / parts;
    s.tokens = (each > 0 ? each : 1) * step;
    s.parts = static_cast<int32_t>(steps > 0 ? (steps + each - 1) / each : 1);
    return s;
}

template <int YT, int ST, bool ADD, bool PARTIAL>
hipError_t launch_products(const char *dy, const int8_t *codes, const uint8_t *scales, const WeightGradGeom &g, char *base, float *work, const Split &s,
                           bool wide, hipStream_t stream)
{
    constexpr int WIDE_K = YT == 0 ? 32 : 64, NARROW_K = 32;
    const uint32_t blocks = static_cast<uint32_t>(g.N * s.parts * s.tiles_o * s.tiles_i);
    auto go = [&](auto kernel, int threads) {
        kernel<<<blocks, threads, 0, stream>>>(dy, codes, scales, g, s, base, work);
        return hipGetLastError();
    };
    // dy straight into LDS where its rows are whole 16-byte vectors: 16 x 1024 x 2048 from 1024 tokens in 84 us (through registers 93),
    // 16 x 1000 x 1008 from 4096 in 129 (147), 2 x 1024 x 1024 from 4096 in 41 (43); 64 x 512 x 3584 from 64, a single step, in 101 (100)
    if constexpr (YT == 1)
        if ((reinterpret_cast<uintptr_t>(dy) & 15) == 0 && g.dy_stride % 8 == 0 && g.outs % 8 == 0 && g.ins % 16 == 0) {
            if constexpr (!PARTIAL)
                if (wide) return go(weight_grad_kernel<YT, ST, ADD, false, Tile<2, 4, 4, 2, WIDE_K>, true>, 512);
            return go(weight_grad_kernel<YT, ST, ADD, PARTIAL, Tile<2, 2, 2, 2, NARROW_K>, true>, 256);
        }
    if constexpr (!PARTIAL)
        if (wide) return go(weight_grad_kernel<YT, ST, ADD, false, Tile<2, 4, 4, 2, WIDE_K>, false>, 512);
    return go(weight_grad_kernel<YT, ST, ADD, PARTIAL, Tile<2, 2, 2, 2, NARROW_K>, false>, 256);
}

template <int YT, int ST, bool ADD>
hipError_t launch(const void *dy, const int8_t *codes, const uint8_t *scales, const WeightGradGeom &g, void *base, float *work, const Split &s,
                  bool wide, hipStream_t stream)
{
    const char *from = static_cast<const char *>(dy);
    char *to = static_cast<char *>(base);
    if (g.outs < 8 || g.ins < 16) {
        thin_weight_grad_kernel<YT, ST, ADD><<<static_cast<uint32_t>((g.N * g.outs * g.ins + kBlock - 1) / kBlock), kBlock, 0, stream>>>(
            from, codes, scales, g, to);
        return hipGetLastError();
    }
    if (s.parts == 1) return launch_products<YT, ST, ADD, false>(from, codes, scales, g, to, nullptr, s, wide, stream);
    const hipError_t e = launch_products<YT, 0, false, true>(from, codes, scales, g, nullptr, work, s, wide, stream);
    if (e != hipSuccess) return e;
    const int64_t count = g.outs * g.ins, join_blocks = (g.N * count + kBlock - 1) / kBlock;
    weight_grad_join_kernel<ST, ADD><<<static_cast<uint32_t>(join_blocks < 8192 ? join_blocks : 8192), kBlock, 0, stream>>>(work, s.parts, g.N, count,
                                                                                                                            g.peer_stride, to);
    return hipGetLastError();
}

}  // namespace

bool weight_grad_fits(const WeightGradGeom &g)
{
    return (g.outs < 8 || g.ins < 16 ? (g.outs * g.ins + kBlock) / kBlock : ((g.outs + 127) / 128) * ((g.ins + 127) / 128)) <= 0xffffffffLL / kBlock / g.N;       // (more than one part only where that is few)
}

int64_t weight_grad_work_bytes(const WeightGradGeom &g, int dy_dtype, int compute_units)
{
    const Split s = split_of(g, dy_dtype, compute_units);
    return s.parts == 1 || g.outs < 8 || g.ins < 16 ? 0 : 4 * s.parts * g.N * g.outs * g.ins;
}

hipError_t launch_weight_grad(const void *dy, int dy_dtype, const int8_t *codes, const uint8_t *scales, const WeightGradGeom &g, void *base,
                              int state_dtype, bool accumulate, void *work, int compute_units, hipStream_t stream)
{
    const Split s = split_of(g, dy_dtype, compute_units);
    const bool wide = wide_tiles(g, compute_units);
    auto go = [&](auto add) {
        constexpr bool ADD = decltype(add)::value;
        auto f = dy_dtype == 0 ? (state_dtype == 0 ? launch<0, 0, ADD> : launch<0, 1, ADD>) : (state_dtype == 0 ? launch<1, 0, ADD> : launch<1, 1, ADD>);
        return f(dy, codes, scales, g, base, static_cast<float *>(work), s, wide, stream);
    };
    return accumulate ? go(std::true_type{}) : go(std::false_type{});
}

}  // namespace moshpit
