// Causal attention over packed sequences, and attention of new tokens over a cache, for gfx950.  For query i of a head with key j:
//   s_ij = scale q_i . k_j,   out_i = sum_j exp(s_ij - lse_i) v_j,   lse_i = log sum_j exp s_ij
// over the keys first_i <= j <= i of places that hold a token (cached: over a span's rows up to the query's own).
//
// One pass over the keys with running largest and sum.  A wave holds 32 queries as columns; tiles of keys and values lie in LDS, two of each, the
// next ones on their way through registers.  Scores come as blocks [key][query] (attention_tile.h), so a query's largest and sum are
// taken within a lane and once between the two halves of the wave, and the weights go into the second product where they lie.
// Sums are rescaled only where a query's largest score has grown by more than 2^8 (weights stay below 2^8, in binary32).
//
// A weight of 0 times a value that is no number is no number, so a sequence's infinities would reach others that share its tiles.  Rows
// of places without a token are never read.  For the rest the block looks at its results: where they are not finite, it goes over its
// keys again with such values taken out of the tiles, and adds each to the queries that see its row.
#include <hip/hip_runtime.h>

#include "attention_tile.h"
#include "local_ops.h"

namespace moshpit {
namespace {

constexpr int kThreads = 256, kWaves = 4;
constexpr float kSlack = 8.f;                            // by how many powers of two weights may pass 1

// Rows of a tile: 64 where four tiles of them fit 64 KiB.
template <int DT, int DP> constexpr int tile_rows() { return 4 * 64 * row_elems_of(DP) * Num<DT>::ES <= 65536 ? 64 : 32; }

// Waves of a block of cached_kernel: four where their tiles fit 64 KiB.
template <int DT, int DP> constexpr int cached_waves() { return 4 * 2 * 32 * row_elems_of(DP) * Num<DT>::ES <= 65536 ? 4 : 2; }

// A wave's queries (columns) and their sums so far.
template <int DT, int DP> struct Queries {
    static constexpr int BLOCKS = DP / 32;
    Held<DT, DP> q;
    f32x16 sum[BLOCKS];
    float top, total;                    // top: what scores * scale log2 e are taken from (-inf: none yet); total: of this half's weights

    __device__ __forceinline__ void clear()
    {
        top = -INFINITY;
        total = 0.f;
#pragma unroll
        for (int m = 0; m < BLOCKS; ++m) sum[m] = f32x16{};
    }

    // Scores of ROWS keys to weights; `largest` of them (this half's).
    template <int N> __device__ __forceinline__ void weigh(f32x16 (&s)[N], float scale)
    {
        float most = s[0][0];
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int r = 0; r < 16; ++r) most = fmaxf(most, s[n][r]);
        most = halves_max(most) * scale;
        if (__any(most > top + kSlack)) {
            const float now = fmaxf(top, most), factor = now == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(top - now);
            top = now;
            total *= factor;
#pragma unroll
            for (int m = 0; m < BLOCKS; ++m)
#pragma unroll
                for (int r = 0; r < 16; ++r) sum[m][r] *= factor;
        }
        const float from = top == -INFINITY ? 0.f : top;
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[n][r] = __builtin_amdgcn_exp2f(fmaf(s[n][r], scale, -from));
                total += s[n][r];
            }
    }

    // Values that are no numbers of the rows in `odd` (bits: rows of the tile), which are zeros in the tile, from memory.
    template <int N>
    __device__ void add_odd(const f32x16 (&weight)[N], uint64_t odd, const char *values, int64_t row_bytes, int depth)
    {
        const int half = threadIdx.x >> 5 & 1;
        while (odd) {
            const int row = __builtin_ctzll(odd);
            odd &= odd - 1;
            float w = 0.f;
#pragma unroll
            for (int n = 0; n < N; ++n)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (row / 32 == n && (row >> 3 & 3) == r / 4 && (row & 3) == r % 4) w = weight[n][r];
            const LanePair both = swap32(w, w);
            w = (row & 4) ? both.second : both.first;
            const char *value = values + row * row_bytes;
#pragma unroll
            for (int m = 0; m < BLOCKS; ++m)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int at = 32 * m + 8 * (r >> 2) + 4 * half + (r & 3);
                    if (at >= depth) continue;
                    const float v = load_one<DT>(value + at * Num<DT>::ES);
                    if (!(fabsf(v) < INFINITY) && w != 0.f) sum[m][r] += w * v;
                }
        }
    }

    __device__ __forceinline__ bool finite() const
    {
        float all = 0.f;                                               // (0 * x is 0 for numbers alone)
#pragma unroll
        for (int m = 0; m < BLOCKS; ++m)
#pragma unroll
            for (int r = 0; r < 16; ++r) all = fmaf(sum[m][r], 0.f, all);
        return all == 0.f;
    }
};

template <int DT, int DP, int WAVES_A_SIMD>
__global__ __launch_bounds__(kThreads, WAVES_A_SIMD)
void attention_kernel(AttentionArgs a)
{
    constexpr int ES = Num<DT>::ES, ROWS = tile_rows<DT, DP>(), N = ROWS / 32, LP = row_elems_of(DP), BLOCKS = DP / 32;
    typedef typename Num<DT>::lds_t lds_t;
    __shared__ __attribute__((aligned(16))) lds_t keys[2][ROWS * LP], values[2][ROWS * LP];
    __shared__ int32_t ends[2][kWaves];
    __shared__ unsigned long long odd_rows[2];

    uint32_t b = die_run(blockIdx.x, gridDim.x);
    const uint32_t tile = a.tiles - 1 - b % a.tiles;                   // (the last ones, which see the most keys, first)
    b /= a.tiles;
    const int32_t head = b % a.heads, kv_head = head / (a.heads / a.kv_heads), lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t peer = b / a.heads, row0 = peer * a.T;
    const int32_t T = static_cast<int32_t>(a.T), i = static_cast<int32_t>(tile * (32 * kWaves) + wave * 32 + (lane & 31));
    const int32_t *first = a.first + row0;
    auto begin_of = [&](int32_t j) {                                   // -1: no token
        const int32_t f = j < T ? first[j] : -1;
        return f <= j ? f : -1;
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

    Queries<DT, DP> x;
    x.q.load(a.q + ((row0 + i) * a.q_stride + int64_t(head) * a.depth) * ES, there, a.depth);
    const char *k_rows = a.k + (row0 * a.k_stride + int64_t(kv_head) * a.depth) * ES, *v_rows = a.v + (row0 * a.v_stride + int64_t(kv_head) * a.depth) * ES;
    const int64_t k_bytes = a.k_stride * ES, v_bytes = a.v_stride * ES;
    auto live_of = [&](int32_t begin) { return __ballot(begin >= 0) & (ROWS == 64 ? ~uint64_t(0) : 0xffffffffull); };

    auto pass = [&](auto careful) {
        constexpr bool CAREFUL = decltype(careful)::value;
        x.clear();
        if (to < from) return;
        Staged<DT, DP, ROWS, kThreads> k_next, v_next;
        uint64_t live = live_of(begin_of(from + lane)), live_next = 0;
        int32_t begin_next = from + ROWS <= to ? begin_of(from + ROWS + lane) : -1;
        int now = 0;
        auto fill = [&](int into) {
            if constexpr (CAREFUL) {
                if (threadIdx.x == 0) odd_rows[into] = 0;
                __syncthreads();
                const uint64_t odd = v_next.clean(threadIdx.x);
                if (odd) atomicOr(&odd_rows[into], static_cast<unsigned long long>(odd));
            }
            k_next.store(keys[into], threadIdx.x);
            v_next.store(values[into], threadIdx.x);
        };
        k_next.load(k_rows + from * k_bytes, k_bytes, live, a.depth, threadIdx.x);
        v_next.load(v_rows + from * v_bytes, v_bytes, live, a.depth, threadIdx.x);
        fill(0);
        for (int32_t at = from; at <= to; at += ROWS, now ^= 1, live = live_next) {
            __syncthreads();
            const bool more = at + ROWS <= to;
            if (more) {
                live_next = live_of(begin_next);
                k_next.load(k_rows + (at + ROWS) * k_bytes, k_bytes, live_next, a.depth, threadIdx.x);
                v_next.load(v_rows + (at + ROWS) * v_bytes, v_bytes, live_next, a.depth, threadIdx.x);
                begin_next = at + 2 * ROWS <= to ? begin_of(at + 2 * ROWS + lane) : -1;
            }
            if (at <= wave_hi && at + ROWS > wave_lo) {
                f32x16 s[N];
#pragma unroll
                for (int n = 0; n < N; ++n) s[n] = rows_times<DT, DP>(keys[now], 32 * n, x.q);
                const bool whole = at >= all_from && at + ROWS - 1 <= all_to && live == (ROWS == 64 ? ~uint64_t(0) : 0xffffffffull);
                if (!whole) {
                    const int half = lane >> 5;
                    const int32_t low = there ? lo - at - 4 * half : INT32_MAX / 2;
                    const uint32_t span = there ? static_cast<uint32_t>(hi - lo) : 0u;
                    const uint64_t seen = live >> (4 * half);
#pragma unroll
                    for (int n = 0; n < N; ++n)
#pragma unroll
                        for (int r = 0; r < 16; ++r) {
                            const int32_t j = 32 * n + 8 * (r >> 2) + (r & 3);
                            const bool sees = static_cast<uint32_t>(j - low) <= span && (seen >> j & 1) != 0;
                            s[n][r] = sees ? s[n][r] : -INFINITY;
                        }
                }
                x.weigh(s, a.scale);
#pragma unroll
                for (int n = 0; n < N; ++n) {
                    const Weights<DT> w(s[n]);
#pragma unroll
                    for (int m = 0; m < BLOCKS; ++m) x.sum[m] = columns_times<DT, LP>(values[now], 32 * n, 32 * m, w, x.sum[m]);
                }
                if constexpr (CAREFUL) x.add_odd(s, odd_rows[now], v_rows + at * v_bytes, v_bytes, a.depth);
            }
            if (more) fill(now ^ 1);
        }
    };
    pass(std::false_type{});
    if (__syncthreads_or(there && !x.finite())) pass(std::true_type{});

    if (i >= T) return;
    const float total = halves_sum(x.total);
    char *out = a.out + ((row0 + i) * a.out_stride + int64_t(head) * a.depth) * ES;
    if (lane < 32 && a.lse) a.lse[(peer * a.heads + head) * a.T + i] = there ? (x.top + __builtin_amdgcn_logf(total)) * kLn2 : 0.f;
    const float share = 1.f / total;
#pragma unroll
    for (int m = 0; m < BLOCKS; ++m) {
        if (!there) x.sum[m] = f32x16{};
        store_column<DT>(out, 32 * m, a.depth, x.sum[m], there ? share : 0.f);
    }
}

// Tokens' queries against a span of keys.  A block has one sequence, one head of keys and a share of the span; its waves take tiles of 32 keys in turn,
// each its own in LDS, for the same 32 columns: the queries of the heads that share the keys, of the new tokens one after the other.
template <int DT, int DP, int WAVES>
__global__ __launch_bounds__(64 * WAVES, DT == 0 && DP > 128 ? 1 : 2)
void cached_kernel(CachedArgs a, float *__restrict__ partials)
{
    constexpr int ES = Num<DT>::ES, LP = row_elems_of(DP), BLOCKS = DP / 32;
    typedef typename Num<DT>::lds_t lds_t;
    __shared__ __attribute__((aligned(16))) lds_t all[WAVES][2 * 32 * LP];
    __shared__ float tops[WAVES][32], totals[WAVES][32];

    uint32_t b = die_run(blockIdx.x, gridDim.x);
    const int32_t split = b % a.splits;
    b /= a.splits;
    const int32_t col_tile = b % a.col_tiles;
    b /= a.col_tiles;
    const int32_t kv_head = b % a.kv_heads;
    b /= a.kv_heads;
    const int32_t seq = b % a.seqs, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
    const int64_t peer = b / a.seqs;
    const int32_t group = a.heads / a.kv_heads, column = col_tile * 32 + (lane & 31), token = column / group, head = kv_head * group + column % group;
    const bool there = token < a.fresh;
    const int32_t n_keys = static_cast<int32_t>(a.n_keys);
    int32_t begin = a.spans[2 * (peer * a.seqs + seq)], end = a.spans[2 * (peer * a.seqs + seq) + 1];
    begin = begin < 0 ? 0 : begin > n_keys ? n_keys : begin;
    end = end > n_keys ? n_keys : end;
    const int32_t count = end > begin ? end - begin : 0;
    const int32_t each = static_cast<int32_t>((count + 32u * WAVES * a.splits - 1) / (32u * WAVES * a.splits)) * (32 * WAVES);
    const int32_t to = int64_t(split + 1) * each < count ? (split + 1) * each : count;    // (keys by their number in the span)
    const int32_t sees = there ? count - (a.fresh - 1 - token) : 0;                       // how many of them this query does
    const int32_t all_see = count - (a.fresh - 1);

    Queries<DT, DP> x;
    const int64_t row = (peer * a.seqs + seq) * a.fresh + token;
    x.q.load(a.q + (row * a.q_stride + int64_t(head) * a.depth) * ES, there, a.depth);
    x.clear();
    const char *k_rows = a.k + ((peer * a.n_keys + begin) * a.k_stride + int64_t(kv_head) * a.depth) * ES;
    const char *v_rows = a.v + ((peer * a.n_keys + begin) * a.v_stride + int64_t(kv_head) * a.depth) * ES;
    const int64_t k_bytes = a.k_stride * ES, v_bytes = a.v_stride * ES;
    lds_t *keys = all[wave], *values = keys + 32 * LP;
    auto live_of = [&](int32_t at) { return at + 32 <= to ? 0xffffffffull : (uint64_t(1) << (to - at)) - 1; };
    int32_t at = split * each + 32 * wave;
    Staged<DT, DP, 32, 64> k_next, v_next;
    if (at < to) {
        k_next.load(k_rows + at * k_bytes, k_bytes, live_of(at), a.depth, lane);
        v_next.load(v_rows + at * v_bytes, v_bytes, live_of(at), a.depth, lane);
    }
    auto settle = [] {                                                 // LDS of a wave: what was written before is read behind it
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    };
    for (; at < to; at += 32 * WAVES) {
        settle();
        k_next.store(keys, lane);
        v_next.store(values, lane);
        settle();
        const int32_t next = at + 32 * WAVES;
        if (next < to) {
            k_next.load(k_rows + next * k_bytes, k_bytes, live_of(next), a.depth, lane);
            v_next.load(v_rows + next * v_bytes, v_bytes, live_of(next), a.depth, lane);
        }
        f32x16 s[1] = {rows_times<DT, DP>(keys, 0, x.q)};
        if (at + 32 > to || at + 32 > all_see) {
            const int32_t seen = (sees < to ? sees : to) - at - 4 * half;
#pragma unroll
            for (int r = 0; r < 16; ++r) s[0][r] = 8 * (r >> 2) + (r & 3) < seen ? s[0][r] : -INFINITY;
        }
        x.weigh(s, a.scale);
        const Weights<DT> w(s[0]);
#pragma unroll
        for (int m = 0; m < BLOCKS; ++m) x.sum[m] = columns_times<DT, LP>(values, 0, 32 * m, w, x.sum[m]);
    }

    // the waves' sums, in order
    x.total = halves_sum(x.total);
    if (lane < 32) {
        tops[wave][lane] = x.top;
        totals[wave][lane] = x.total;
    }
    __syncthreads();
    float top = tops[0][lane & 31], total = 0.f;
#pragma unroll
    for (int w = 1; w < WAVES; ++w) top = fmaxf(top, tops[w][lane & 31]);
    auto factor_of = [&](float t) { return t == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(t - top); };
#pragma unroll
    for (int w = 0; w < WAVES; ++w) total += totals[w][lane & 31] * factor_of(tops[w][lane & 31]);
    const float factor = factor_of(x.top);
    // a wave at a time adds its sums to block 32 * m of [depth][column] in LDS
    float *joined = reinterpret_cast<float *>(all);
    static_assert(sizeof(all) >= 32 * DP * sizeof(float));
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        if (wave == w)
#pragma unroll
            for (int m = 0; m < BLOCKS; ++m)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    float *p = joined + (32 * m + 8 * (r >> 2) + 4 * half + (r & 3)) * 32 + (lane & 31);
                    const float v = x.top == -INFINITY ? 0.f : x.sum[m][r] * factor;
                    *p = w == 0 ? v : *p + v;
                }
        __syncthreads();
    }
        const int32_t columns = a.fresh * group - col_tile * 32 < 32 ? a.fresh * group - col_tile * 32 : 32;
    for (int32_t n = threadIdx.x; n < columns * a.depth; n += 64 * WAVES) {
        const int32_t c = n / a.depth, d = n % a.depth, t = (col_tile * 32 + c) / group, h = kv_head * group + (col_tile * 32 + c) % group;
        const int64_t r = (peer * a.seqs + seq) * a.fresh + t;
        const float v = joined[d * 32 + c];
        if (a.splits == 1) {
            float sum = 0.f, most = tops[0][c];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) most = fmaxf(most, tops[w][c]);
#pragma unroll
            for (int w = 0; w < WAVES; ++w) sum += tops[w][c] == -INFINITY ? 0.f : totals[w][c] * __builtin_amdgcn_exp2f(tops[w][c] - most);
            store_one<DT>(a.out + (r * a.out_stride + int64_t(h) * a.depth + d) * ES, most == -INFINITY ? 0.f : v / sum);
        } else
            partials[((r * a.heads + h) * a.splits + split) * (a.depth + 2) + 2 + d] = v;
    }
    if (a.splits > 1 && wave == 0 && half == 0 && there) {
        float *p = partials + ((row * a.heads + head) * a.splits + split) * (a.depth + 2);
        p[0] = top;
        p[1] = total;
    }
}

// The shares of a span, in order: a wave has a query of a head.
template <int DT>
__global__ __launch_bounds__(kThreads) void cached_join_kernel(CachedArgs a, const float *__restrict__ partials, int64_t rows)
{
    constexpr int ES = Num<DT>::ES;
    const int64_t n = int64_t(blockIdx.x) * kWaves + (threadIdx.x >> 6);
    if (n >= rows * a.heads) return;
    const int64_t row = n / a.heads, head = n % a.heads;
    const int lane = threadIdx.x & 63;
    const float *p = partials + n * a.splits * (a.depth + 2);
    float top = -INFINITY;
    for (int s = 0; s < a.splits; ++s) top = fmaxf(top, p[s * (a.depth + 2)]);
    char *out = a.out + (row * a.out_stride + head * a.depth) * ES;
    for (int d = lane; d < a.depth; d += 64) {
        float sum = 0.f, total = 0.f;
        for (int s = 0; s < a.splits; ++s) {
            const float *q = p + s * (a.depth + 2);
            if (q[0] == -INFINITY) continue;
            const float f = __builtin_amdgcn_exp2f(q[0] - top);
            total = fmaf(q[1], f, total);
            sum = fmaf(q[2 + d], f, sum);
        }
        store_one<DT>(out + d * ES, top == -INFINITY ? 0.f : sum / total);
    }
}

template <typename Go> hipError_t by_depth(int dtype, int depth, Go go)
{
    using std::integral_constant;
    auto of_type = [&](auto dt) {
        if (depth <= 32) return go(dt, integral_constant<int, 32>{});
        if (depth <= 64) return go(dt, integral_constant<int, 64>{});
        if (depth <= 128) return go(dt, integral_constant<int, 128>{});
        return go(dt, integral_constant<int, 256>{});
    };
    return dtype == 0 ? of_type(integral_constant<int, 0>{}) : of_type(integral_constant<int, 1>{});
}

int64_t attention_blocks(const AttentionArgs &a) { return a.N * a.heads * ((a.T + 32 * kWaves - 1) / (32 * kWaves)); }

}  // namespace

bool attention_fits(const AttentionArgs &a) { return launchable(attention_blocks(a), kThreads); }

hipError_t launch_attention(AttentionArgs a, int dtype, hipStream_t stream)
{
    if (a.T == 0) return hipSuccess;
    a.tiles = static_cast<uint32_t>((a.T + 32 * kWaves - 1) / (32 * kWaves));
    a.scale *= kLog2e;
    return by_depth(dtype, a.depth, [&](auto dt, auto dp) {
        constexpr int DT = decltype(dt)::value, DP = decltype(dp)::value;
        attention_kernel<DT, DP, (DP > 128 ? 1 : 2)><<<static_cast<uint32_t>(attention_blocks(a)), kThreads, 0, stream>>>(a);
        return hipGetLastError();
    });
}

// Shares of a span: enough blocks for the chip, 512 keys each and more where the keys of a peer are even over its sequences.
CachedPlan cached_plan(const CachedArgs &a, int compute_units)
{
    CachedPlan p;
    p.col_tiles = (a.fresh * (a.heads / a.kv_heads) + 31) / 32;
    const int64_t blocks = a.N * a.seqs * a.kv_heads * p.col_tiles;
    const int64_t most = blocks > 0 ? 4 * int64_t(compute_units) / blocks : 1, use = (a.n_keys + 511) / 512;
    const int64_t splits = most < use ? most : use;
    p.splits = static_cast<int32_t>(splits < 1 ? 1 : splits);
    p.work_bytes = p.splits > 1 ? 4 * a.N * a.seqs * a.fresh * a.heads * p.splits * (a.depth + 2) : 0;
    p.fits = launchable(blocks * p.splits, kThreads) && launchable(a.N * a.seqs * a.fresh * a.heads, 64);
    return p;
}

hipError_t launch_cached(CachedArgs a, int dtype, const CachedPlan &p, void *work, hipStream_t stream)
{
    const int64_t rows = a.N * a.seqs * a.fresh;
    if (rows == 0) return hipSuccess;
    a.col_tiles = p.col_tiles;
    a.splits = p.splits;
    a.scale *= kLog2e;
    float *partials = static_cast<float *>(work);
    const hipError_t e = by_depth(dtype, a.depth, [&](auto dt, auto dp) {
        constexpr int DT = decltype(dt)::value, DP = decltype(dp)::value;
        constexpr int WAVES = cached_waves<DT, DP>();
        cached_kernel<DT, DP, WAVES><<<static_cast<uint32_t>(a.N * a.seqs * a.kv_heads * p.col_tiles * p.splits), 64 * WAVES, 0, stream>>>(a, partials);
        return hipGetLastError();
    });
    if (e != hipSuccess || p.splits == 1) return e;
    const uint32_t blocks = static_cast<uint32_t>((rows * a.heads + kWaves - 1) / kWaves);
    (dtype == 0 ? cached_join_kernel<0> : cached_join_kernel<1>)<<<blocks, kThreads, 0, stream>>>(a, partials, rows);
    return hipGetLastError();
}

}  // namespace moshpit
