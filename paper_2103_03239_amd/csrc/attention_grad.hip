// The backward pass of causal attention over packed sequences, for gfx950.  With p_ij = exp(s_ij - lse_i), s = scale q . k:
//   dp_ij = dout_i . v_j,   delta_i = dout_i . out_i,   ds_ij = p_ij (dp_ij - delta_i)
//   dv_j = sum_i p_ij dout_i,   dk_j = scale sum_i ds_ij q_i,   dq_i = scale sum_j ds_ij k_j
// with the sums over i also over the query heads that share the keys.
//
// Every sum has an order of its own that no other block takes part in, so there are no atomics and a call repeats to the bit; the price is
// that p and dp are made twice, 14 multiplications a pair and depth instead of 10.  Three kernels:
//   delta    delta_i, and of every tile of queries the range of `first` (which tiles a key is to be met with)
//   keys     a wave holds 32 keys and values as columns and goes over the queries that see them: blocks [query][key], dk and dv [depth][key]
//   queries  a wave holds 32 queries and their dout as columns and goes over the keys they see: blocks [key][query], dq [depth][query]
#include <hip/hip_runtime.h>

#include "attention_tile.h"
#include "local_ops.h"

namespace moshpit {
namespace {

constexpr int kThreads = 256, kWaves = 4;
constexpr int kStat = 32;                                // queries of a tile whose range of `first` is kept

struct Range {
    int32_t lo, hi;                      // smallest and largest `first` of the queries that hold a token; lo = INT32_MAX: none does
};

// delta of a row's heads by 16 lanes each, 4 rows and heads a wave; the ranges by the blocks behind them.
template <int DT>
__global__ __launch_bounds__(kThreads) void delta_kernel(AttentionGradArgs a, float *__restrict__ delta, Range *__restrict__ ranges, int64_t delta_blocks)
{
    constexpr int ES = Num<DT>::ES;
    const int lane = threadIdx.x & 15;
    if (blockIdx.x >= delta_blocks) {
        const int64_t stats = (a.T + kStat - 1) / kStat, n = (blockIdx.x - delta_blocks) * (kThreads / 16) + threadIdx.x / 16;
        if (n >= a.N * stats) return;
        const int64_t peer = n / stats;
        const int32_t begin = static_cast<int32_t>(n % stats) * kStat;
        Range r{INT32_MAX, -1};
        for (int k = lane; k < kStat; k += 16) {
            const int32_t i = begin + k, f = i < a.T ? a.first[peer * a.T + i] : -1;
            if (f < 0 || f > i) continue;
            r.lo = f < r.lo ? f : r.lo;
            r.hi = f > r.hi ? f : r.hi;
        }
#pragma unroll
        for (int off = 1; off < 16; off <<= 1) {
            const int32_t lo = __shfl_xor(r.lo, off, 64), hi = __shfl_xor(r.hi, off, 64);
            r.lo = lo < r.lo ? lo : r.lo;
            r.hi = hi > r.hi ? hi : r.hi;
        }
        if (lane == 0) ranges[n] = r;
        return;
    }
    const int64_t n = int64_t(blockIdx.x) * (kThreads / 16) + threadIdx.x / 16, row = n / a.heads, head = n % a.heads;
    if (row >= a.N * a.T) return;
    const char *out = a.out + (row * a.out_stride + head * a.depth) * ES, *dout = a.dout + (row * a.dout_stride + head * a.depth) * ES;
    float sum = 0.f;
    for (int at = lane * 8; at < a.depth; at += 128) {
        float x[8], y[8];
        if (at + 8 <= a.depth) {
            load_elems<DT, 8>(out + at * ES, x);
            load_elems<DT, 8>(dout + at * ES, y);
        } else
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                x[k] = at + k < a.depth ? load_one<DT>(out + (at + k) * ES) : 0.f;
                y[k] = at + k < a.depth ? load_one<DT>(dout + (at + k) * ES) : 0.f;
            }
#pragma unroll
        for (int k = 0; k < 8; ++k) sum = fmaf(x[k], y[k], sum);
    }
#pragma unroll
    for (int off = 1; off < 16; off <<= 1) sum += __shfl_xor(sum, off, 64);
    if (lane == 0) delta[(row / a.T * a.heads + head) * a.T + row % a.T] = sum;
}

// How a launch of the kernel for keys is cut: `parts` of the queries and heads that a block of keys meets, sums of a part apart, and
// `slices` of DA depths of dk and dv.
struct KeysPlan {
    uint32_t tiles;
    int32_t parts;
};

// Depths of dk and dv that a block's sums have: all up to 128, as registers allow.
template <int DT, int DP> constexpr int sum_depths() { return DP <= 128 ? DP : DT == 0 ? 64 : 128; }

template <int DT, int DP>
__global__ __launch_bounds__(kThreads, DP > 128 || (DT == 0 && DP > 64) ? 1 : 2)
void keys_grad_kernel(AttentionGradArgs a, KeysPlan plan, const float *__restrict__ delta, const Range *__restrict__ ranges, float *__restrict__ partials)
{
    constexpr int ES = Num<DT>::ES, ROWS = kStat, LP = row_elems_of(DP), DA = sum_depths<DT, DP>(), BLOCKS = DA / 32, SLICES = DP / DA;
    typedef typename Num<DT>::lds_t lds_t;
    __shared__ __attribute__((aligned(16))) lds_t queries[2][ROWS * LP], douts[2][ROWS * LP];
    __shared__ __attribute__((aligned(16))) float lses[2][ROWS], deltas[2][ROWS];
    __shared__ __attribute__((aligned(16))) int32_t firsts[2][ROWS];

    uint32_t b = die_run(blockIdx.x, gridDim.x);
    const int32_t slice = b % SLICES;
    b /= SLICES;
    const uint32_t tile = b % plan.tiles;                              // (the first ones, which the most queries see, first)
    b /= plan.tiles;
    const int32_t part = b % plan.parts;
    b /= plan.parts;
    const int32_t kv_head = b % a.kv_heads, group = a.heads / a.kv_heads, lane = threadIdx.x & 63, half = lane >> 5, wave = threadIdx.x >> 6;
    const int64_t peer = b / a.kv_heads, row0 = peer * a.T;
    const int32_t T = static_cast<int32_t>(a.T), begin = static_cast<int32_t>(tile * (32 * kWaves)), wave_begin = begin + 32 * wave, j = wave_begin + (lane & 31);
    const int32_t *first = a.first + row0;
    auto begin_of = [&](int32_t i) {
        const int32_t f = i < T ? first[i] : -1;
        return f <= i ? f : -1;
    };
    const bool there = begin_of(j) >= 0;

    Held<DT, DP> k, v;
    k.load(a.k + ((row0 + j) * a.k_stride + int64_t(kv_head) * a.depth) * ES, there, a.depth);
    v.load(a.v + ((row0 + j) * a.v_stride + int64_t(kv_head) * a.depth) * ES, there, a.depth);
    f32x16 dk[BLOCKS] = {}, dv[BLOCKS] = {};

    // The tiles of queries that see one of the block's keys, each for the heads of the group: numbers part, part + parts, ... of them.
    const int32_t last = begin + 32 * kWaves - 1, stats = (T + ROWS - 1) / ROWS;
    const Range *range = ranges + peer * stats;
    int32_t base = begin / ROWS, turn = 0, at = -1, head = 0;          // the tiles looked at from, the item's tile and head
    uint64_t left = 0;
    Range r{};
    auto look = [&] {
        const int32_t n = base + lane;
        r = n < stats ? range[n] : Range{INT32_MAX, -1};
        left = __ballot(r.lo <= last);
    };
    look();
    auto advance = [&]() -> bool {                                     // to the next item of this part; false: there is none
        for (;;) {
            if (at >= 0 && ++head < group) {
                if (turn++ % plan.parts == part) return true;
                continue;
            }
            while (left == 0) {
                base += 64;
                if (base >= stats) return false;
                look();
            }
            at = base + __builtin_ctzll(left);
            left &= left - 1;
            head = -1;
        }
    };
    Staged<DT, DP, ROWS, kThreads> q_next, d_next;
    float lse_next = 0.f, delta_next = 0.f;
    int32_t first_next = -1;
    auto request = [&] {
        const int32_t i = at * ROWS + (threadIdx.x & (ROWS - 1)), h = kv_head * group + head;
        first_next = begin_of(i);
        const uint64_t live = __ballot(first_next >= 0) & 0xffffffffull;
        q_next.load(a.q + ((row0 + at * ROWS) * a.q_stride + int64_t(h) * a.depth) * ES, a.q_stride * ES, live, a.depth, threadIdx.x);
        d_next.load(a.dout + ((row0 + at * ROWS) * a.dout_stride + int64_t(h) * a.depth) * ES, a.dout_stride * ES, live, a.depth, threadIdx.x);
        const int64_t n = (peer * a.heads + h) * a.T + i;
        lse_next = first_next >= 0 ? a.lse[n] * kLog2e : INFINITY;    // (a query without a token: weights of 0)
        delta_next = first_next >= 0 ? delta[n] : 0.f;
    };
    auto fill = [&](int into) {
        q_next.store(queries[into], threadIdx.x);
        d_next.store(douts[into], threadIdx.x);
        if (threadIdx.x < ROWS) {
            lses[into][threadIdx.x] = lse_next;
            deltas[into][threadIdx.x] = delta_next;
            firsts[into][threadIdx.x] = first_next;
        }
    };
    int now = 0;
    bool more = advance();
    if (more) {
        request();
        fill(0);
    }
    while (more) {
        const int32_t i0 = at * ROWS;
        const int32_t lo = __shfl(r.lo, at - base, 64), hi = __shfl(r.hi, at - base, 64);
        more = advance();
        __syncthreads();
        if (more) request();
        if (lo <= wave_begin + 31 && i0 + ROWS > wave_begin) {
            f32x16 p = rows_times<DT, DP>(queries[now], 0, k);
            f32x16 ds = rows_times<DT, DP>(douts[now], 0, v);
            const bool whole = i0 >= wave_begin + 31 && hi <= wave_begin;
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const f32x4 l = *reinterpret_cast<const f32x4 *>(&lses[now][8 * g + 4 * half]), d = *reinterpret_cast<const f32x4 *>(&deltas[now][8 * g + 4 * half]);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    p[4 * g + e] = __builtin_amdgcn_exp2f(fmaf(p[4 * g + e], a.scale, -l[e]));
                    ds[4 * g + e] = p[4 * g + e] * (ds[4 * g + e] - d[e]);
                }
            }
            if (!whole) {
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const u32x4 f = *reinterpret_cast<const u32x4 *>(&firsts[now][8 * g + 4 * half]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int32_t i = i0 + 8 * g + 4 * half + e, from = static_cast<int32_t>(f[e]);
                        const bool sees = from >= 0 && from <= j && j <= i;
                        p[4 * g + e] = sees ? p[4 * g + e] : 0.f;
                        ds[4 * g + e] = sees ? ds[4 * g + e] : 0.f;
                    }
                }
            }
            const Weights<DT> wp(p), ws(ds);
#pragma unroll
            for (int m = 0; m < BLOCKS; ++m) {
                dv[m] = columns_times<DT, LP>(douts[now], 0, slice * DA + 32 * m, wp, dv[m]);
                dk[m] = columns_times<DT, LP>(queries[now], 0, slice * DA + 32 * m, ws, dk[m]);
            }
        }
        now ^= 1;
        if (more) fill(now);
    }
    if (j >= T) return;
    const float factor = a.scale * kLn2;                               // (a.scale: times log2 e)
    const int64_t width = int64_t(a.kv_heads) * a.depth, column = int64_t(kv_head) * a.depth;
    if (!there)
#pragma unroll
        for (int m = 0; m < BLOCKS; ++m) dk[m] = dv[m] = f32x16{};
    if (plan.parts == 1) {
#pragma unroll
        for (int m = 0; m < BLOCKS; ++m) {
            store_column<DT>(a.dk + ((row0 + j) * a.dk_stride + column) * ES, slice * DA + 32 * m, a.depth, dk[m], factor);
            store_column<DT>(a.dv + ((row0 + j) * a.dv_stride + column) * ES, slice * DA + 32 * m, a.depth, dv[m], 1.f);
        }
    } else {
        char *to = reinterpret_cast<char *>(partials + ((int64_t(part) * a.N * a.T + row0 + j) * 2 * width + column));
#pragma unroll
        for (int m = 0; m < BLOCKS; ++m) {
            store_column<0>(to, slice * DA + 32 * m, a.depth, dk[m], factor);
            store_column<0>(to + width * 4, slice * DA + 32 * m, a.depth, dv[m], 1.f);
        }
    }
}

// The parts of dk and dv, in order.
template <int DT>
__global__ __launch_bounds__(kThreads) void keys_join_kernel(AttentionGradArgs a, int32_t parts, const float *__restrict__ partials)
{
    constexpr int ES = Num<DT>::ES;
    const int64_t width = int64_t(a.kv_heads) * a.depth, all = a.N * a.T * 2 * width;
    for (int64_t n = int64_t(blockIdx.x) * kThreads + threadIdx.x; n < all; n += int64_t(gridDim.x) * kThreads) {
        float sum = 0.f;
        for (int32_t p = 0; p < parts; p += 4) {                      // four requested at a time
            float v[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) v[u] = p + u < parts ? partials[(p + u) * all + n] : 0.f;
#pragma unroll
            for (int u = 0; u < 4; ++u) sum += v[u];
        }
        const int64_t row = n / (2 * width), c = n % (2 * width);
        if (c < width) store_one<DT>(a.dk + (row * a.dk_stride + c) * ES, sum);
        else store_one<DT>(a.dv + (row * a.dv_stride + c - width) * ES, sum);
    }
}

template <int DT, int DP>
__global__ __launch_bounds__(kThreads, DP > 128 || (DT == 0 && DP > 64) ? 1 : 2)
void queries_grad_kernel(AttentionGradArgs a, uint32_t tiles, const float *__restrict__ delta)
{
    constexpr int ES = Num<DT>::ES, ROWS = 32, LP = row_elems_of(DP), BLOCKS = DP / 32;
    typedef typename Num<DT>::lds_t lds_t;
    __shared__ __attribute__((aligned(16))) lds_t keys[2][ROWS * LP], values[2][ROWS * LP];
    __shared__ int32_t ends[2][kWaves];

    uint32_t b = die_run(blockIdx.x, gridDim.x);
    const uint32_t tile = tiles - 1 - b % tiles;
    b /= tiles;
    const int32_t head = b % a.heads, kv_head = head / (a.heads / a.kv_heads), lane = threadIdx.x & 63, half = lane >> 5, wave = threadIdx.x >> 6;
    const int64_t peer = b / a.heads, row0 = peer * a.T;
    const int32_t T = static_cast<int32_t>(a.T), i = static_cast<int32_t>(tile * (32 * kWaves) + wave * 32 + (lane & 31));
    const int32_t *first = a.first + row0;
    auto begin_of = [&](int32_t n) {
        const int32_t f = n < T ? first[n] : -1;
        return f <= n ? f : -1;
    };
    const int32_t mine = begin_of(i);
    const bool there = mine >= 0;
    const int32_t lo = there ? mine : INT32_MAX, hi = there ? i : -1;
    const int32_t wave_lo = wave_min(lo), wave_hi = wave_max(hi), all_from = wave_max(there ? mine : -1), all_to = wave_min(there ? i : INT32_MAX);
    if (lane == 0) {
        ends[0][wave] = wave_lo;
        ends[1][wave] = wave_hi;
    }
    __syncthreads();
    int32_t from = ends[0][0], to = ends[1][0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) {
        from = ends[0][w] < from ? ends[0][w] : from;
        to = ends[1][w] > to ? ends[1][w] : to;
    }
    Held<DT, DP> q, d;
    q.load(a.q + ((row0 + i) * a.q_stride + int64_t(head) * a.depth) * ES, there, a.depth);
    d.load(a.dout + ((row0 + i) * a.dout_stride + int64_t(head) * a.depth) * ES, there, a.depth);
    const int64_t n = (peer * a.heads + head) * a.T + i;
    const float lse = there ? a.lse[n] * kLog2e : INFINITY, off = there ? delta[n] : 0.f;
    f32x16 dq[BLOCKS] = {};
    const char *k_rows = a.k + (row0 * a.k_stride + int64_t(kv_head) * a.depth) * ES, *v_rows = a.v + (row0 * a.v_stride + int64_t(kv_head) * a.depth) * ES;
    const int64_t k_bytes = a.k_stride * ES, v_bytes = a.v_stride * ES;
    auto live_of = [&](int32_t f) { return __ballot(f >= 0) & 0xffffffffull; };
    if (from <= to) {
        Staged<DT, DP, ROWS, kThreads> k_next, v_next;
        uint64_t live = live_of(begin_of(from + (lane & 31))), live_next = 0;
        int32_t begin_next = from + ROWS <= to ? begin_of(from + ROWS + (lane & 31)) : -1;
        int now = 0;
        k_next.load(k_rows + from * k_bytes, k_bytes, live, a.depth, threadIdx.x);
        v_next.load(v_rows + from * v_bytes, v_bytes, live, a.depth, threadIdx.x);
        k_next.store(keys[0], threadIdx.x);
        v_next.store(values[0], threadIdx.x);
        for (int32_t at = from; at <= to; at += ROWS, now ^= 1, live = live_next) {
            __syncthreads();
            const bool more = at + ROWS <= to;
            if (more) {
                live_next = live_of(begin_next);
                k_next.load(k_rows + (at + ROWS) * k_bytes, k_bytes, live_next, a.depth, threadIdx.x);
                v_next.load(v_rows + (at + ROWS) * v_bytes, v_bytes, live_next, a.depth, threadIdx.x);
                begin_next = at + 2 * ROWS <= to ? begin_of(at + 2 * ROWS + (lane & 31)) : -1;
            }
            if (at <= wave_hi && at + ROWS > wave_lo) {
                const f32x16 s = rows_times<DT, DP>(keys[now], 0, q);
                f32x16 ds = rows_times<DT, DP>(values[now], 0, d);
#pragma unroll
                for (int r = 0; r < 16; ++r) ds[r] = __builtin_amdgcn_exp2f(fmaf(s[r], a.scale, -lse)) * (ds[r] - off);
                const bool whole = at >= all_from && at + ROWS - 1 <= all_to && live == 0xffffffffull;
                if (!whole) {
                    const int32_t low = there ? lo - at - 4 * half : INT32_MAX / 2;
                    const uint32_t span = there ? static_cast<uint32_t>(hi - lo) : 0u;
                    const uint32_t seen = static_cast<uint32_t>(live) >> (4 * half);
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const int32_t j = 8 * (r >> 2) + (r & 3);
                        ds[r] = static_cast<uint32_t>(j - low) <= span && (seen >> j & 1) != 0 ? ds[r] : 0.f;
                    }
                }
                const Weights<DT> w(ds);
#pragma unroll
                for (int m = 0; m < BLOCKS; ++m) dq[m] = columns_times<DT, LP>(keys[now], 0, 32 * m, w, dq[m]);
            }
            if (more) {
                k_next.store(keys[now ^ 1], threadIdx.x);
                v_next.store(values[now ^ 1], threadIdx.x);
            }
        }
    }
    if (i >= T) return;
    char *to_row = a.dq + ((row0 + i) * a.dq_stride + int64_t(head) * a.depth) * ES;
#pragma unroll
    for (int m = 0; m < BLOCKS; ++m) {
        if (!there) dq[m] = f32x16{};
        store_column<DT>(to_row, 32 * m, a.depth, dq[m], a.scale * kLn2);
    }
}

int depth_of(int depth) { return depth <= 32 ? 32 : depth <= 64 ? 64 : depth <= 128 ? 128 : 256; }

int slices_of(int dtype, int depth) { return depth_of(depth) <= 128 ? 1 : dtype == 0 ? 4 : 2; }

int64_t tiles_of(const AttentionGradArgs &a) { return (a.T + 32 * kWaves - 1) / (32 * kWaves); }
int64_t stats_of(const AttentionGradArgs &a) { return (a.T + kStat - 1) / kStat; }

KeysPlan keys_plan(const AttentionGradArgs &a, int dtype, int compute_units)
{
    KeysPlan p;
    p.tiles = static_cast<uint32_t>(tiles_of(a));
    const int64_t blocks = a.N * a.kv_heads * tiles_of(a) * slices_of(dtype, a.depth), group = a.heads / a.kv_heads;
    // the parts that fill the chip, at least a tile of queries for all heads of the group, and 8 parts at most
    int64_t parts = blocks > 0 ? 2 * int64_t(compute_units) / blocks : 1;
    if (parts > 8) parts = 8;
    if (parts > group * stats_of(a)) parts = group * stats_of(a);
    p.parts = static_cast<int32_t>(parts < 1 ? 1 : parts);
    return p;
}

int64_t round_up(int64_t n) { return (n + 255) / 256 * 256; }

}  // namespace

bool attention_grad_fits(const AttentionGradArgs &a, int dtype)
{
    const int64_t delta_blocks = (a.N * a.T * a.heads + 15) / 16 + (a.N * stats_of(a) + 15) / 16;
    return launchable(delta_blocks, kThreads) && launchable(a.N * a.heads * tiles_of(a) * slices_of(dtype, a.depth), kThreads);
}

int64_t attention_grad_work_bytes(const AttentionGradArgs &a, int dtype, int compute_units)
{
    const KeysPlan p = keys_plan(a, dtype, compute_units);
    const int64_t sums = p.parts > 1 ? 4 * p.parts * a.N * a.T * 2 * a.kv_heads * a.depth : 0;
    return round_up(4 * a.N * a.heads * a.T) + round_up(int64_t(sizeof(Range)) * a.N * stats_of(a)) + sums;
}

hipError_t launch_attention_grad(const AttentionGradArgs &given, int dtype, void *work, int compute_units, hipStream_t stream)
{
    AttentionGradArgs a = given;
    if (a.T == 0) return hipSuccess;
    const KeysPlan p = keys_plan(a, dtype, compute_units);
    a.scale *= kLog2e;
    float *delta = static_cast<float *>(work);
    Range *ranges = reinterpret_cast<Range *>(static_cast<char *>(work) + round_up(4 * a.N * a.heads * a.T));
    float *partials = reinterpret_cast<float *>(reinterpret_cast<char *>(ranges) + round_up(int64_t(sizeof(Range)) * a.N * stats_of(a)));
    const int64_t delta_blocks = (a.N * a.T * a.heads + 15) / 16, range_blocks = (a.N * stats_of(a) + 15) / 16;
    (dtype == 0 ? delta_kernel<0> : delta_kernel<1>)<<<static_cast<uint32_t>(delta_blocks + range_blocks), kThreads, 0, stream>>>(a, delta, ranges, delta_blocks);
    auto of = [&](auto dt, auto dp) {
        constexpr int DT = decltype(dt)::value, DP = decltype(dp)::value;
        const uint32_t slices = DP / sum_depths<DT, DP>();
        keys_grad_kernel<DT, DP><<<static_cast<uint32_t>(a.N * a.kv_heads * p.tiles * p.parts) * slices, kThreads, 0, stream>>>(a, p, delta, ranges, partials);
        if (p.parts > 1) {
            const int64_t blocks = (a.N * a.T * 2 * a.kv_heads * a.depth + kThreads - 1) / kThreads;
            keys_join_kernel<DT><<<static_cast<uint32_t>(blocks < 4096 ? blocks : 4096), kThreads, 0, stream>>>(a, p.parts, partials);
        }
        queries_grad_kernel<DT, DP><<<static_cast<uint32_t>(a.N * a.heads * p.tiles), kThreads, 0, stream>>>(a, p.tiles, delta);
        return hipGetLastError();
    };
    using std::integral_constant;
    auto of_type = [&](auto dt) {
        switch (depth_of(a.depth)) {
        case 32: return of(dt, integral_constant<int, 32>{});
        case 64: return of(dt, integral_constant<int, 64>{});
        case 128: return of(dt, integral_constant<int, 128>{});
        default: return of(dt, integral_constant<int, 256>{});
        }
    };
    return dtype == 0 ? of_type(integral_constant<int, 0>{}) : of_type(integral_constant<int, 1>{});
}

}  // namespace moshpit
