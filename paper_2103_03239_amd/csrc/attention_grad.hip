// The backward pass of causal attention over packed sequences, for gfx950.  With p_ij = exp(s_ij - lse_i), s = scale q . k:
//   dp_ij = dout_i . v_j,   delta_i = dout_i . out_i,   ds_ij = p_ij (dp_ij - delta_i)
//   dv_j = sum_i p_ij dout_i,   dk_j = scale sum_i ds_ij q_i,   dq_i = scale sum_j ds_ij k_j
// with the sums over i also over the query heads that share the keys.
//
// Every sum has an order of its own that no other block takes part in, so there are no atomics and a call repeats to the bit; the price is
// that p and dp are made twice, 14 multiplications a pair and depth instead of 10 (in bfloat16 two more, see queries_grad_kernel).  Three kernels:
//   ranges   of every tile of queries the range of `first` (which tiles a key is to be met with)
//   queries  a wave holds 32 queries and their dout as columns and goes over the keys they see: blocks [key][query], dq [depth][query]; and delta_i, which
//            the columns hold both factors of
//   keys     a wave holds 32 keys and values as columns and goes over the queries that see them: blocks [query][key], dk and dv [depth][key]
// Bound by registers: the columns and the sums leave two waves a SIMD, which the exponentials and roundings of one hide badly behind the
// products of the other (matrix cores busy for 22 % of the time in the one, 25 in the other; vector instructions 37 and 32).  16 x 8 heads of 64, 4 heads of
// keys, 4096 tokens in bfloat16: queries 273 us, keys 258 us (forward 139 us).  What spills: keys' kernel for bfloat16 heads of 128 (7 registers; 122 where
// heads are not whole vectors), queries' kernel for such heads of 96 (44) and 256 (244), both for binary32 heads of 256 and, not whole vectors, of 192.
#include <hip/hip_runtime.h>

#include "attention_tile.h"
#include "local_ops.h"

namespace moshpit {
namespace {

constexpr int kThreads = 256, kWaves = 4, kColumns = 32 * kWaves;     // columns of a block: keys or queries
// Queries of a tile of keys_grad_kernel, whose range of `first` is kept.
template <Form F, int DP> constexpr int query_rows() { return F == kBf16 && DP <= 64 ? 64 : 32; }
int query_rows_of(int dtype, int depth) { return dtype != 0 && depth <= 64 ? 64 : 32; }

struct Range {
    int32_t lo, hi;                      // smallest and largest `first` of the queries that hold a token; lo = INT32_MAX: none does
};

// The ranges, 16 lanes each.
__global__ __launch_bounds__(kThreads) void ranges_kernel(AttentionGradArgs a, Range *__restrict__ ranges, int32_t rows)
{
    const int lane = threadIdx.x & 15;
    const int64_t stats = (a.T + rows - 1) / rows, n = int64_t(blockIdx.x) * (kThreads / 16) + threadIdx.x / 16;
    if (n >= a.N * stats) return;
    const int64_t peer = n / stats;
    const int32_t begin = static_cast<int32_t>(n % stats) * rows;
    Range r{INT32_MAX, -1};
    for (int k = lane; k < rows; k += 16) {
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
}

// How a launch of the kernel for keys is cut: `parts` of the queries and heads that a block of keys meets, sums of a part apart, and
// `slices` of sum_depths() depths of dk and dv.
struct KeysPlan {
    uint32_t tiles;
    int32_t parts;
};

// Depths of dk and dv that a block's sums have: all up to 128, as registers allow.
template <Form F, int DP> constexpr int sum_depths() { return DP <= 128 ? DP : F == kF32 ? 64 : DP == 192 ? 96 : 128; }

// SIMD waves a SIMD; ASIDE: the values stay in LDS (registers do not hold them beside the keys and the sums); DIRECT: rows go straight into LDS.
template <Form F, int DP, int SIMD, bool ASIDE, bool DIRECT>
__global__ __launch_bounds__(kThreads, SIMD)
void keys_grad_kernel(AttentionGradArgs a, KeysPlan plan, const float *__restrict__ delta, const Range *__restrict__ ranges, float *__restrict__ partials)
{
    constexpr int ES = Num<F>::ES, DT = Num<F>::DT, ROWS = query_rows<F, DP>(), DA = sum_depths<F, DP>(), BLOCKS = DA / 32, SLICES = DP / DA, ELEMS = tile_elems<F, DP>(ROWS);
    constexpr uint64_t ALL = ROWS == 64 ? ~uint64_t(0) : 0xffffffffull;
    typedef Direct<(DIRECT ? F : kBf16), (DIRECT ? DP : 128), ROWS, kThreads> Straight;
    typedef typename Num<F>::lds_t lds_t;
    __shared__ __attribute__((aligned(16))) lds_t q_even[ELEMS], q_odd[ELEMS], d_even[ELEMS], d_odd[ELEMS], aside[ASIDE ? tile_elems<F, DP>(kColumns) : 8];
    __shared__ __attribute__((aligned(16))) float lses[2][ROWS], deltas[2][ROWS];
    __shared__ __attribute__((aligned(16))) int32_t firsts[2][ROWS];

    const int32_t group = a.heads / a.kv_heads, lane = threadIdx.x & 63, half = lane >> 5, wave = threadIdx.x >> 6;
    const Place place = place_of(blockIdx.x, a.N, a.kv_heads, plan.parts * SLICES);    // (the first tiles are seen by the most queries)
    const int32_t part = place.member / SLICES, slice = place.member % SLICES, kv_head = place.kv_head;
    const int64_t peer = place.peer, row0 = peer * a.T;
    const int32_t T = static_cast<int32_t>(a.T), begin = static_cast<int32_t>(place.tile * kColumns), j = begin + 32 * wave + (lane & 31);
    const int32_t wave_begin = __builtin_amdgcn_readfirstlane(begin + 32 * wave);
    const int32_t *first = a.first + row0;
    auto begin_of = [&](int32_t i) {
        const int32_t f = i < T ? first[i] : -1;
        return f <= i ? f : -1;
    };
    const bool there = begin_of(j) >= 0;

    Held<F, DP> k, v;
    k.load(a.k + ((row0 + j) * a.k_stride + int64_t(kv_head) * a.depth) * ES, there, a.depth);
    v.load(a.v + ((row0 + j) * a.v_stride + int64_t(kv_head) * a.depth) * ES, there, a.depth);
    if constexpr (ASIDE) Aside<F, DP>::put(v, aside + 32 * wave * row_elems_of(DP));
    f32x16 dk[BLOCKS] = {}, dv[BLOCKS] = {};

    // The tiles of queries that see one of the block's keys, each for the heads of the group: numbers part, part + parts, ... of them.
    struct Item {
        int32_t tile, member, lo, hi;
    };
    const int32_t last = begin + kColumns - 1, stats = (T + ROWS - 1) / ROWS;
    const Range *range = ranges + peer * stats;
    int32_t base = begin / ROWS, turn = 0;                             // the tiles looked at from
    uint64_t left = 0;
    Range r{};
    auto look = [&] {
        const int32_t n = base + lane;
        r = n < stats ? range[n] : Range{INT32_MAX, -1};
        left = __ballot(r.lo <= last);
    };
    look();
    Item item{-1, 0, 0, 0};
    auto advance = [&]() -> bool {                                     // to the next item of this part; false: there is none
        for (;;) {
            if (item.tile >= 0 && ++item.member < group) {
                const bool mine = turn == part;
                turn = turn + 1 == plan.parts ? 0 : turn + 1;
                if (mine) return true;
                continue;
            }
            while (left == 0) {
                base += 64;
                if (base >= stats) return false;
                look();
            }
            const int32_t n = __builtin_ctzll(left);
            left &= left - 1;
            item = Item{base + n, -1, __builtin_amdgcn_readlane(r.lo, n), __builtin_amdgcn_readlane(r.hi, n)};
        }
    };
    typename std::conditional<DIRECT, char, Staged<F, DP, ROWS, kThreads>>::type q_next, d_next;
    float lse_next = 0.f, delta_next = 0.f;
    int32_t first_next = -1;
    uint64_t live_next = 0;
    auto request = [&](lds_t *q_into, lds_t *d_into) __attribute__((always_inline)) {
        const int32_t i0 = item.tile * ROWS, i = i0 + (threadIdx.x & (ROWS - 1)), h = kv_head * group + item.member;
        const char *q = a.q + ((row0 + i0) * a.q_stride + int64_t(h) * a.depth) * ES, *d = a.dout + ((row0 + i0) * a.dout_stride + int64_t(h) * a.depth) * ES;
        first_next = begin_of(i);
        const int64_t n = (peer * a.heads + h) * a.T + (i < T ? i : T - 1);
        lse_next = a.lse[n] * kLog2e;
        delta_next = delta[n];
        if constexpr (DIRECT) {
            Straight::request(q, static_cast<uint32_t>(a.q_stride * ES), T - 1 - i0, a.depth / Num<F>::CE, q_into);
            Straight::request(d, static_cast<uint32_t>(a.dout_stride * ES), T - 1 - i0, a.depth / Num<F>::CE, d_into);
            __builtin_amdgcn_sched_barrier(0);
        }
        live_next = __ballot(first_next >= 0) & ALL;
        if constexpr (!DIRECT) {
            q_next.load(q, a.q_stride * ES, live_next, a.depth, threadIdx.x);
            d_next.load(d, a.dout_stride * ES, live_next, a.depth, threadIdx.x);
        }
    };
    auto fill = [&](lds_t *q_into, lds_t *d_into, int into) __attribute__((always_inline)) {
        if constexpr (DIRECT) {
            Straight::wait();
            Straight::blank(a.depth / Num<F>::CE, q_into);
            Straight::blank(a.depth / Num<F>::CE, d_into);
            if (live_next != ALL) {
                Straight::trim(live_next, q_into);
                Straight::trim(live_next, d_into);
            }
        } else {
            q_next.store(q_into, threadIdx.x);
            d_next.store(d_into, threadIdx.x);
        }
        if (threadIdx.x < ROWS) {
            lses[into][threadIdx.x] = first_next >= 0 ? -lse_next : -INFINITY;     // (a query without a token: weights of 0)
            deltas[into][threadIdx.x] = first_next >= 0 ? -delta_next : 0.f;
            firsts[into][threadIdx.x] = first_next;
        }
    };
    auto step = [&](const lds_t *queries, const lds_t *douts, int now, lds_t *q_into, lds_t *d_into) __attribute__((always_inline)) {
        const Item it = item;
        const bool more = advance();
        __syncthreads();
        if (more) request(q_into, d_into);
#pragma unroll
        for (int n = 0; n < ROWS / 32; ++n) {
            const int32_t i0 = it.tile * ROWS + 32 * n;
            if (it.lo > wave_begin + 31 || i0 + 32 <= wave_begin) continue;
            f32x16 p = rows_times<F, DP, ROWS>(queries, 32 * n, k), ds;
#pragma unroll
            for (int g = 0; g < 4; ++g) {                              // (dp - delta: the sums begin with -delta)
                const f32x4 d = *reinterpret_cast<const f32x4 *>(&deltas[now][32 * n + 8 * g + 4 * half]);
#pragma unroll
                for (int e = 0; e < 4; ++e) ds[4 * g + e] = d[e];
            }
            if constexpr (ASIDE) ds = rows_times<F, DP, ROWS>(douts, 32 * n, Aside<F, DP>{aside + 32 * wave * row_elems_of(DP)}, ds);
            else ds = rows_times<F, DP, ROWS>(douts, 32 * n, v, ds);
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const f32x4 l = *reinterpret_cast<const f32x4 *>(&lses[now][32 * n + 8 * g + 4 * half]);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    p[4 * g + e] = __builtin_amdgcn_exp2f(fmaf(p[4 * g + e], a.scale, l[e]));
                    ds[4 * g + e] *= p[4 * g + e];
                }
            }
            if (i0 < wave_begin + 31 || it.hi > wave_begin) {
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const u32x4 f = *reinterpret_cast<const u32x4 *>(&firsts[now][32 * n + 8 * g + 4 * half]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int32_t i = i0 + 8 * g + 4 * half + e, from = static_cast<int32_t>(f[e]);
                        const bool sees = from >= 0 && from <= j && j <= i;
                        p[4 * g + e] = sees ? p[4 * g + e] : 0.f;
                        ds[4 * g + e] = sees ? ds[4 * g + e] : 0.f;
                    }
                }
            }
            Weights<F> w;
            w.take(p);
            columns_times<F, DP, ROWS>(douts, 32 * n, slice * DA, w, dv);
            w.take(ds);
            columns_times<F, DP, ROWS>(queries, 32 * n, slice * DA, w, dk);
        }
        if (more) fill(q_into, d_into, now ^ 1);
        return more;
    };
    if (advance()) {
        request(q_even, d_even);
        fill(q_even, d_even, 0);
        for (;;) {
            if (!step(q_even, d_even, 0, q_odd, d_odd)) break;
            if (!step(q_odd, d_odd, 1, q_even, d_even)) break;
        }
    }
    if (j >= T) return;
    const float factor = there ? a.scale * kLn2 : 0.f;                 // (a.scale: times log2 e)
    const int64_t width = int64_t(a.kv_heads) * a.depth, column = int64_t(kv_head) * a.depth;
#pragma unroll
    for (int m = 0; m < BLOCKS; ++m) {
        if (!there) dk[m] = dv[m] = f32x16{};
        const int at = slice * DA + 32 * m;
        if (plan.parts == 1) {
            store_column<DT>(a.dk + ((row0 + j) * a.dk_stride + column) * ES, at, a.depth, dk[m], factor);
            store_column<DT>(a.dv + ((row0 + j) * a.dv_stride + column) * ES, at, a.depth, dv[m], 1.f);
        } else {
            char *to = reinterpret_cast<char *>(partials + ((int64_t(part) * a.N * a.T + row0 + j) * 2 * width + column));
            store_column<0>(to, at, a.depth, dk[m], factor);
            store_column<0>(to + width * 4, at, a.depth, dv[m], 1.f);
        }
    }
}

// The parts of dk and dv, in order.
template <int DT>
__global__ __launch_bounds__(kThreads) void keys_join_kernel(AttentionGradArgs a, int32_t parts, const float *__restrict__ partials)
{
    constexpr int ES = DT == 0 ? 4 : 2;
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

// ROWS keys a tile; SIMD, DIRECT as above.
template <Form F, int DP, int ROWS, int SIMD, bool DIRECT>
__global__ __launch_bounds__(kThreads, SIMD)
void queries_grad_kernel(AttentionGradArgs a, uint32_t tiles, float *__restrict__ delta)
{
    constexpr int ES = Num<F>::ES, DT = Num<F>::DT, BLOCKS = DP / 32, ELEMS = tile_elems<F, DP>(ROWS);
    constexpr uint64_t ALL = ROWS == 64 ? ~uint64_t(0) : 0xffffffffull;
    typedef Direct<(DIRECT ? F : kBf16), (DIRECT ? DP : 128), (DIRECT ? ROWS : 64), kThreads> Straight;
    typedef typename Num<F>::lds_t lds_t;
    __shared__ __attribute__((aligned(16))) lds_t k_even[ELEMS], k_odd[ELEMS], v_even[ELEMS], v_odd[ELEMS];
    __shared__ int32_t ends[2][kWaves];

    const int32_t group = a.heads / a.kv_heads, lane = threadIdx.x & 63, half = lane >> 5, wave = threadIdx.x >> 6;
    const Place place = place_of(blockIdx.x, a.N, a.kv_heads, group);
    const uint32_t tile = tiles - 1 - place.tile;
    const int32_t kv_head = place.kv_head, head = kv_head * group + place.member;
    const int64_t peer = place.peer, row0 = peer * a.T;
    const int32_t T = static_cast<int32_t>(a.T), i = static_cast<int32_t>(tile * kColumns) + wave * 32 + (lane & 31);
    const int32_t *first = a.first + row0;
    auto begin_of = [&](int32_t n) {
        const int32_t f = n < T ? first[n] : -1;
        return f <= n ? f : -1;
    };
    const int32_t lo = begin_of(i);
    const bool there = lo >= 0;
    const int32_t wave_lo = __builtin_amdgcn_readfirstlane(wave_min(there ? lo : INT32_MAX)), wave_hi = __builtin_amdgcn_readfirstlane(wave_max(there ? i : -1));
    const int32_t all_from = __builtin_amdgcn_readfirstlane(wave_max(there ? lo : -1)), all_to = __builtin_amdgcn_readfirstlane(wave_min(there ? i : INT32_MAX));
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
    from = __builtin_amdgcn_readfirstlane(from);
    to = __builtin_amdgcn_readfirstlane(to);
    Held<F, DP> q, d;
    q.load(a.q + ((row0 + i) * a.q_stride + int64_t(head) * a.depth) * ES, there, a.depth);
    d.load(a.dout + ((row0 + i) * a.dout_stride + int64_t(head) * a.depth) * ES, there, a.depth);
    const int64_t n = (peer * a.heads + head) * a.T + i;
    const float lse = there ? a.lse[n] * kLog2e : INFINITY;
    const float off = columns_dot<F, DP>(a.out + ((row0 + i) * a.out_stride + int64_t(head) * a.depth) * ES,
                                         a.dout + ((row0 + i) * a.dout_stride + int64_t(head) * a.depth) * ES, there, a.depth);
    float drift = 0.f;
    // delta from out as it was rounded (bfloat16) is off by 2^-9 of its terms, which would bring dq that much of the keys' mean, beside few keys more than
    // all other roundings (windows of 4 tokens: dq off by 3.0e-3, so 2.3e-3).  sum ds over the keys, 0 in truth, is how much it is off: mean, the keys' sum
    // by p, is taken from dq so many times.  (16 x 8 heads of 64, 4096 tokens: a training step in 665 us, without 614.)
    f32x16 dq[BLOCKS] = {}, mean[F == kBf16 ? BLOCKS : 1] = {};
    const char *k_rows = a.k + (row0 * a.k_stride + int64_t(kv_head) * a.depth) * ES, *v_rows = a.v + (row0 * a.v_stride + int64_t(kv_head) * a.depth) * ES;
    const int64_t k_bytes = a.k_stride * ES, v_bytes = a.v_stride * ES;
    auto begins_at = [&](int32_t at) { return at <= to ? begin_of(at + lane) : -1; };
    auto live_of = [&](int32_t f) { return __ballot(f >= 0) & ALL; };
    if (from <= to) {
        typename std::conditional<DIRECT, char, Staged<F, DP, ROWS, kThreads>>::type k_next, v_next;
        auto request = [&](int32_t at, uint64_t live, lds_t *k_into, lds_t *v_into) __attribute__((always_inline)) {
            if constexpr (DIRECT) {
                Straight::request(k_rows + at * k_bytes, static_cast<uint32_t>(k_bytes), T - 1 - at, a.depth / Num<F>::CE, k_into);
                Straight::request(v_rows + at * v_bytes, static_cast<uint32_t>(v_bytes), T - 1 - at, a.depth / Num<F>::CE, v_into);
            } else {
                k_next.load(k_rows + at * k_bytes, k_bytes, live, a.depth, threadIdx.x);
                v_next.load(v_rows + at * v_bytes, v_bytes, live, a.depth, threadIdx.x);
            }
        };
        auto fill = [&](uint64_t live, lds_t *k_into, lds_t *v_into) __attribute__((always_inline)) {
            if constexpr (DIRECT) {
                Straight::wait();
                Straight::blank(a.depth / Num<F>::CE, k_into);
                Straight::blank(a.depth / Num<F>::CE, v_into);
                if (live != ALL) Straight::trim(live, k_into);         // (values without a token meet a weight that is taken as 0)
            } else {
                k_next.store(k_into, threadIdx.x);
                v_next.store(v_into, threadIdx.x);
            }
        };
        uint64_t live = live_of(begins_at(from)), live_next = 0;
        int32_t begin_next = begins_at(from + ROWS), at = from;
        request(from, live, k_even, v_even);
        fill(live, k_even, v_even);
        auto step = [&](const lds_t *keys, const lds_t *values, lds_t *k_into, lds_t *v_into) __attribute__((always_inline)) {
            __syncthreads();
            const bool more = at + ROWS <= to;
            if (more) {
                live_next = live_of(begin_next);
                request(at + ROWS, live_next, k_into, v_into);
                begin_next = begins_at(at + 2 * ROWS);
                if constexpr (DIRECT) __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int n = 0; n < ROWS / 32; ++n) {
                const int32_t j0 = at + 32 * n;
                if (j0 > wave_hi || j0 + 32 <= wave_lo) continue;
                const f32x16 s = rows_times<F, DP, ROWS>(keys, 32 * n, q);
                f32x16 ds = rows_times<F, DP, ROWS>(values, 32 * n, d), p;
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    p[r] = __builtin_amdgcn_exp2f(fmaf(s[r], a.scale, -lse));
                    ds[r] = p[r] * (ds[r] - off);
                }
                const uint32_t seen = static_cast<uint32_t>(live >> (32 * n));
                if (j0 < all_from || j0 + 31 > all_to || seen != 0xffffffffu) {
                    const int32_t low = there ? lo - j0 - 4 * half : INT32_MAX / 2;
                    const uint32_t span = there ? static_cast<uint32_t>(i - lo) : 0u, mine = seen >> (4 * half);
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const int32_t j = 8 * (r >> 2) + (r & 3);
                        const bool sees = static_cast<uint32_t>(j - low) <= span && (mine >> j & 1) != 0;
                        ds[r] = sees ? ds[r] : 0.f;
                        if constexpr (F == kBf16) p[r] = sees ? p[r] : 0.f;
                    }
                }
                Weights<F> w;
                w.take(ds);
                columns_times<F, DP, ROWS>(keys, 32 * n, 0, w, dq);
                if constexpr (F == kBf16) {
#pragma unroll
                    for (int r = 0; r < 16; ++r) drift += ds[r];
                    w.take(p);
                    columns_times<F, DP, ROWS>(keys, 32 * n, 0, w, mean);
                }
            }
            if (more) fill(live_next, k_into, v_into);
            live = live_next;
            at += ROWS;
            return more;
        };
        for (;;) {
            if (!step(k_even, v_even, k_odd, v_odd)) break;
            if (!step(k_odd, v_odd, k_even, v_even)) break;
        }
    }
    if constexpr (F == kBf16) drift = halves_sum(drift);
    if (there && half == 0) delta[n] = off + drift;
    if (i >= T) return;
    char *to_row = a.dq + ((row0 + i) * a.dq_stride + int64_t(head) * a.depth) * ES;
#pragma unroll
    for (int m = 0; m < BLOCKS; ++m) {
        if constexpr (F == kBf16)
#pragma unroll
            for (int r = 0; r < 16; ++r) dq[m][r] = fmaf(-drift, mean[m][r], dq[m][r]);
        if (!there) dq[m] = f32x16{};
        store_column<DT>(to_row, 32 * m, a.depth, dq[m], a.scale * kLn2);
    }
}

int slices_of(int dtype, int depth) { return depth <= 128 ? 1 : dtype != 0 ? 2 : depth <= 192 ? 3 : 4; }

int64_t tiles_of(const AttentionGradArgs &a) { return (a.T + kColumns - 1) / kColumns; }
int64_t stats_of(const AttentionGradArgs &a, int dtype) { return (a.T + query_rows_of(dtype, a.depth) - 1) / query_rows_of(dtype, a.depth); }

// Blocks of the kernels a compute unit, as their registers allow.
int waves_of(int dtype, int depth) { return dtype == 0 || depth > 128 ? 1 : 2; }

KeysPlan keys_plan(const AttentionGradArgs &a, int dtype, int compute_units)
{
    KeysPlan p;
    p.tiles = static_cast<uint32_t>(tiles_of(a));
    const int64_t blocks = a.N * a.kv_heads * tiles_of(a) * slices_of(dtype, a.depth), group = a.heads / a.kv_heads;
    // A block goes over all queries that see its keys, the first keys' over the most, so there are to be twice as many as run at once, in up to 8
    // parts of at least a tile of queries: 2 x 2 x 64 tiles of 128 keys, groups of 4 heads of 64, 8192 tokens: the backward pass in 657 us, with half as
    // many parts in 816, with twice as many in 689; 4 x 4 x 32 of 128, groups of 2: 564, 710, 582.
    const int64_t at_once = int64_t(compute_units) * (waves_of(dtype, a.depth));
    int64_t parts = blocks > 0 ? (2 * at_once + blocks - 1) / blocks : 1;
    if (parts > 8) parts = 8;
    if (parts > group * stats_of(a, dtype)) parts = group * stats_of(a, dtype);
    p.parts = static_cast<int32_t>(parts < 1 ? 1 : parts);
    return p;
}

int64_t round_up(int64_t n) { return (n + 255) / 256 * 256; }

}  // namespace

bool attention_grad_fits(const AttentionGradArgs &a, int dtype)
{
    return launchable((a.N * stats_of(a, dtype) + 15) / 16, kThreads) && launchable(a.N * a.heads * tiles_of(a) * slices_of(dtype, a.depth), kThreads);
}

int64_t attention_grad_work_bytes(const AttentionGradArgs &a, int dtype, int compute_units)
{
    const KeysPlan p = keys_plan(a, dtype, compute_units);
    const int64_t sums = p.parts > 1 ? 4 * p.parts * a.N * a.T * 2 * a.kv_heads * a.depth : 0;
    return round_up(4 * a.N * a.heads * a.T) + round_up(int64_t(sizeof(Range)) * a.N * stats_of(a, dtype)) + sums;
}

hipError_t launch_attention_grad(const AttentionGradArgs &given, int dtype, void *work, int compute_units, hipStream_t stream)
{
    AttentionGradArgs a = given;
    if (a.T == 0) return hipSuccess;
    const KeysPlan p = keys_plan(a, dtype, compute_units);
    a.scale *= kLog2e;
    float *delta = static_cast<float *>(work);
    Range *ranges = reinterpret_cast<Range *>(static_cast<char *>(work) + round_up(4 * a.N * a.heads * a.T));
    float *partials = reinterpret_cast<float *>(reinterpret_cast<char *>(ranges) + round_up(int64_t(sizeof(Range)) * a.N * stats_of(a, dtype)));
    ranges_kernel<<<static_cast<uint32_t>((a.N * stats_of(a, dtype) + 15) / 16), kThreads, 0, stream>>>(a, ranges, query_rows_of(dtype, a.depth));
    const bool q_direct = direct_rows(a.q, a.q_stride, a.depth, dtype) && direct_rows(a.dout, a.dout_stride, a.depth, dtype);
    const bool k_direct = direct_rows(a.k, a.k_stride, a.depth, dtype) && direct_rows(a.v, a.v_stride, a.depth, dtype);
    auto of = [&](auto form, auto dp) {
        constexpr Form F = decltype(form)::value;
        constexpr int DP = decltype(dp)::value, DT = Num<F>::DT, SIMD = DP > 128 || F == kParts ? 1 : 2;
        // (bfloat16 heads of 128: with the keys' mean the sums of dq leave one wave a SIMD; two spill: 4 x 8 heads, 4096 tokens: 631 us, 654; of 96: 511, 448)
        constexpr int Q_SIMD = DP > 96 ? 1 : SIMD;
        constexpr bool ASIDE = F == kBf16 && DP == 128, STRAIGHT = F != kParts && DP > 32;
        const uint32_t key_blocks = static_cast<uint32_t>(a.N * a.kv_heads * p.tiles * p.parts) * (DP / sum_depths<F, DP>()), query_blocks = static_cast<uint32_t>(a.N * a.heads * p.tiles);
        constexpr int ROWS = F == kBf16 && DP <= 128 ? 64 : 32;
        if (STRAIGHT && k_direct) queries_grad_kernel<F, DP, ROWS, Q_SIMD, STRAIGHT><<<query_blocks, kThreads, 0, stream>>>(a, p.tiles, delta);
        else queries_grad_kernel<F, DP, ROWS, Q_SIMD, false><<<query_blocks, kThreads, 0, stream>>>(a, p.tiles, delta);
        if (STRAIGHT && q_direct) keys_grad_kernel<F, DP, SIMD, ASIDE, STRAIGHT><<<key_blocks, kThreads, 0, stream>>>(a, p, delta, ranges, partials);
        else keys_grad_kernel<F, DP, SIMD, ASIDE, false><<<key_blocks, kThreads, 0, stream>>>(a, p, delta, ranges, partials);
        if (p.parts > 1) {
            const int64_t blocks = (a.N * a.T * 2 * a.kv_heads * a.depth + kThreads - 1) / kThreads;
            keys_join_kernel<DT><<<static_cast<uint32_t>(blocks < 4096 ? blocks : 4096), kThreads, 0, stream>>>(a, p.parts, partials);
        }
        return hipGetLastError();
    };
    return by_depth(dtype, a.depth, of);
}

}  // namespace moshpit
