// Causal attention over packed sequences, and attention of new tokens over a cache, for gfx950.  For query i of a head with key j:
//   s_ij = scale q_i . k_j,   out_i = sum_j exp(s_ij - lse_i) v_j,   lse_i = log sum_j exp s_ij
// over the keys first_i <= j <= i of places that hold a token (cached: over a span's rows up to the query's own).
//
// One pass over the keys with running largest and sum.  A wave holds 32 queries as columns; tiles of keys and values lie in LDS, two of each (binary32 heads
// deeper than 64: one, where two blocks are to run beside each other).  The next ones go straight into LDS where heads are whole vectors of the type that it
// has them in, else through registers.  Scores come as blocks [key][query] (attention_tile.h), so a query's largest and sum are
// taken within a lane and once between the two halves of the wave, and the weights go into the second product where they lie.
// Sums are rescaled only where a query's largest score has grown by more than 2^8 (weights stay below 2^8, in binary32).
//
// A weight of 0 times a value that is no number is no number, so a sequence's infinities would reach others that share its tiles.  Rows
// of places without a token are zeros in the tiles.  For the rest a wave looks at its results: a query whose weights are numbers and whose sums are
// not is taken again, key by key over those that it sees (and of binary32 ones in parts, one whose weights are not).  That is slow: 8192 tokens of 4 heads
// of 128 in bfloat16 in 103 ms where the first value has an infinity; a NaN in the key in the middle of 4096 of 80 in binary32: 7 ms.
//
// Prompts are bound by what follows on what: an exponential, a maximum and a rounding for each pair beside its 4 depth multiplications, which a wave
// makes one after the other, and two waves a SIMD (heads of 128) that nothing keeps half a step apart.  Heads of 128 in bfloat16: matrix cores busy for 42 % of
// the time, vector instructions for 46, neither full; of 64, four waves a SIMD: 21 and 54.  2 x 16 heads of 128, 4 heads of keys,
// 8192 tokens in two sequences a peer: 367 us, 0.88 PFLOP/s over the pairs that are seen; 16 x 8 heads of 64, 4 of keys, 4096 tokens in 8 sequences: 139 us.
// One new token is bound by the reads of the cache: 4 x 8
// sequences of up to 16384, 4 heads of keys of 128 in bfloat16, in 145 us, 4.9 TB/s, of which about 20 us are the start, the longest span's end and
// the join; 5 new tokens of each: 160 us.
#include <hip/hip_runtime.h>

#include "attention_tile.h"
#include "local_ops.h"
#include "row_sums.h"

namespace moshpit {
namespace {

constexpr int kThreads = 256, kWaves = 4, kQueries = 32 * kWaves;     // of a block
constexpr float kSlack = 8.f;                            // by how many powers of two weights may pass 1

// A wave's 32 queries (columns) and their sums so far.
template <Form F, int DP> struct Queries {
    static constexpr int BLOCKS = DP / 32;
    Held<F, DP> q;
    f32x16 sum[BLOCKS];
    float top, total;                    // top: what scores * scale log2 e are taken from (-inf: none yet); total: of this half's weights

    __device__ __forceinline__ void clear()
    {
        top = -INFINITY;
        total = 0.f;
#pragma unroll
        for (int m = 0; m < BLOCKS; ++m) sum[m] = f32x16{};
    }

    // Scores of 32 * N keys, from the tile's first row on.
    template <int ROWS, int N> __device__ __forceinline__ void score(const typename Num<F>::lds_t *keys, f32x16 (&s)[N]) const
    {
#pragma unroll
        for (int n = 0; n < N; ++n) s[n] = rows_times<F, DP, ROWS>(keys, 32 * n, q);
    }
    template <int N> __device__ __forceinline__ static float largest(const f32x16 (&s)[N])
    {
        float most = s[0][0];
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int r = 0; r < 16; ++r) most = fmaxf(most, s[n][r]);
        return most;
    }
    // Before weights are taken from scores of which `most` is the largest (of this half's).
    __device__ __forceinline__ void rescale(float most, float scale)
    {
        most = halves_max(most) * scale;
        if (!__any(most > top + kSlack)) return;
        const float now = fmaxf(top, most), factor = now == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(top - now);
        top = now;
        total *= factor;
#pragma unroll
        for (int m = 0; m < BLOCKS; ++m)
#pragma unroll
            for (int r = 0; r < 16; ++r) sum[m][r] *= factor;
    }
    __device__ __forceinline__ void weigh(f32x16 &s, float scale, Weights<F> &w)
    {
        const float from = top == -INFINITY ? 0.f : top;
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], scale, -from));
        w.take(s);
#pragma unroll
        for (int r = 0; r < 16; ++r) total += s[r];                   // (not as rounded for the product: the log-sum is a binary32 result)
    }
    // sum += rows row0 .. + 31 of the tile of values (ROWS rows) times their weights
    template <int ROWS> __device__ __forceinline__ void add(const typename Num<F>::lds_t *values, int row0, const Weights<F> &w)
    {
        columns_times<F, DP, ROWS>(values, row0, 0, w, sum);
    }
    // What scores of 32 * N keys bring, whose values the tile holds.
    template <int ROWS, int N> __device__ __forceinline__ void take(f32x16 (&s)[N], float scale, const typename Num<F>::lds_t *values)
    {
#pragma unroll
        for (int n = 0; n < N; ++n) {
            Weights<F> w;
            weigh(s[n], scale, w);
            add<ROWS>(values, 32 * n, w);
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

// The sum of products of `depth` elements, in order.
template <int DT> __device__ __forceinline__ float dot(const char *x, const char *y, int32_t depth)
{
    constexpr int ES = DT == 0 ? 4 : 2;
    float s = 0.f;
    int32_t d = 0;
    for (; d + 4 <= depth; d += 4) {
        float f[4], g[4];
        load_elems<DT, 4>(x + d * ES, f);
        load_elems<DT, 4>(y + d * ES, g);
#pragma unroll
        for (int e = 0; e < 4; ++e) s = fmaf(f[e], g[e], s);
    }
    for (; d < depth; ++d) s = fmaf(load_one<DT>(x + d * ES), load_one<DT>(y + d * ES), s);
    return s;
}

// One query's result by a wave, key by key over those that it sees, where values that are no numbers have come into its sums or finite ones have passed
// binary32: with weights from its log-sum, which add up to 1.  lse: its log2-sum, or NaN where scores of three parts were no numbers (an infinity
// times parts of 0 is none, also where the score is -inf, a weight of 0): then it is found first, and where it is no number either, nothing more is read.
template <int DT> __device__ __forceinline__ void attend_alone(const AttentionArgs &a, int64_t peer, int32_t head, int32_t i, int32_t lo, float lse)
{
    constexpr int ES = DT == 0 ? 4 : 2, MOST = 256 / 64;
    const int32_t lane = threadIdx.x & 63, kv_head = head / (a.heads / a.kv_heads);
    const int64_t row0 = peer * a.T;
    const char *q = a.q + ((row0 + i) * a.q_stride + int64_t(head) * a.depth) * ES;
    auto score = [&](int32_t j) {                                      // -inf: not seen
        const int32_t f = j <= i ? a.first[row0 + j] : -1;
        if (f < 0 || f > j) return -INFINITY;
        const char *k = a.k + ((row0 + j) * a.k_stride + int64_t(kv_head) * a.depth) * ES;
        return dot<DT>(q, k, a.depth) * a.scale;
    };
    if (DT == 0 && lse != lse) {
        float top = -INFINITY, total = 0.f;
        for (int32_t j0 = lo; j0 <= i; j0 += 64) {
            const float s = score(j0 + lane);
            if (!__all(s < INFINITY)) {                                // NaN or +inf: no weight is a number
                total = NAN;
                break;
            }
            const float now = lanes_max(fmaxf(top, s));
            if (now == -INFINITY) continue;
            total = fmaf(total, __builtin_amdgcn_exp2f(top - now), lanes_sum<64>(__builtin_amdgcn_exp2f(s - now)));
            top = now;
        }
        lse = top + __builtin_amdgcn_logf(total);
    }
    const bool numbers = fabsf(lse) < INFINITY;
    float sum[MOST] = {};
    for (int32_t j0 = lo; j0 <= i && numbers; j0 += 64) {
        const float w = __builtin_amdgcn_exp2f(score(j0 + lane) - lse);
        for (uint64_t left = __ballot(w != 0.f); left; left &= left - 1) {
            const int32_t n = __builtin_ctzll(left);
            const float one = __shfl(w, n, 64);
            const char *v = a.v + ((row0 + j0 + n) * a.v_stride + int64_t(kv_head) * a.depth) * ES;
#pragma unroll
            for (int t = 0; t < MOST; ++t)
                if (lane + 64 * t < a.depth) sum[t] = fmaf(one, load_one<DT>(v + (lane + 64 * t) * ES), sum[t]);
        }
    }
    char *out = a.out + ((row0 + i) * a.out_stride + int64_t(head) * a.depth) * ES;
#pragma unroll
    for (int t = 0; t < MOST; ++t)
        if (lane + 64 * t < a.depth) store_one<DT>(out + (lane + 64 * t) * ES, numbers ? sum[t] : NAN);
    if (lane == 0 && a.lse) a.lse[(peer * a.heads + head) * a.T + i] = lse * kLn2;
}

// ROWS keys a tile, JOINT blocks of 32 keys at a time, SIMD waves a SIMD, DIRECT: rows go straight into LDS.
template <Form F, int DP, int ROWS, int JOINT, int SIMD, bool DIRECT>
__global__ __launch_bounds__(kThreads, SIMD)
void attention_kernel(AttentionArgs a)
{
    constexpr int ES = Num<F>::ES, DT = Num<F>::DT, BLOCKS = DP / 32, N = JOINT, ELEMS = tile_elems<F, DP>(ROWS);
    constexpr uint64_t ALL = ROWS == 64 ? ~uint64_t(0) : 0xffffffffull;
    constexpr bool TWO = F != kParts || DP <= 64 || SIMD == 1;         // two buffers of a tile, or one (the launch says where)
    typedef Direct<(DIRECT ? F : kBf16), (DIRECT ? DP : 128), (DIRECT ? ROWS : 64), kThreads> Straight;
    typedef typename Num<F>::lds_t lds_t;
    // (four variables: an access to one does not wait for what is on its way into another)
    __shared__ __attribute__((aligned(16))) lds_t k_even[ELEMS], k_odd[TWO ? ELEMS : 8], v_even[ELEMS], v_odd[TWO ? ELEMS : 8];
    __shared__ int32_t ends[2][kWaves];

    const int32_t group = a.heads / a.kv_heads, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5;
    const Place p = place_of(blockIdx.x, a.N, a.kv_heads, group);
    const uint32_t tile = a.tiles - 1 - p.tile;                        // (the last ones see the most keys)
    const int32_t kv_head = p.kv_head, head = kv_head * group + p.member;
    const int64_t peer = p.peer, row0 = peer * a.T;
    const int32_t T = static_cast<int32_t>(a.T), wave_first = static_cast<int32_t>(tile * kQueries) + wave * 32, i = wave_first + (lane & 31);
    const int32_t *first = a.first + row0;
    auto begin_of = [&](int32_t j) {                                   // -1: no token
        const int32_t f = j < T ? first[j] : -1;
        return f <= j ? f : -1;
    };
    const int32_t lo = begin_of(i);
    const bool there = lo >= 0;
    Queries<F, DP> x;
    x.q.load(a.q + ((row0 + i) * a.q_stride + int64_t(head) * a.depth) * ES, there, a.depth);
    // keys wave_lo .. wave_hi are seen by some query, all_from .. all_to by all of them that hold a token
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

    const char *k_rows = a.k + (row0 * a.k_stride + int64_t(kv_head) * a.depth) * ES, *v_rows = a.v + (row0 * a.v_stride + int64_t(kv_head) * a.depth) * ES;
    const int64_t k_bytes = a.k_stride * ES, v_bytes = a.v_stride * ES;
    auto begins_at = [&](int32_t at) { return at <= to ? begin_of(at + lane) : -1; };
    auto live_of = [&](int32_t begin) { return __ballot(begin >= 0) & ALL; };

    x.clear();
    if (from <= to) {
        typename std::conditional<DIRECT, char, Staged<F, DP, ROWS, kThreads>>::type k_next, v_next;
        auto request = [&](auto &next, const char *rows, int64_t bytes, int32_t at, uint64_t live, lds_t *into) __attribute__((always_inline)) {
            if constexpr (DIRECT) Straight::request(rows + at * bytes, static_cast<uint32_t>(bytes), T - 1 - at, a.depth / Num<F>::CE, into);
            else next.load(rows + at * bytes, bytes, live, a.depth, threadIdx.x);
        };
        auto put = [&](auto &next, lds_t *into) __attribute__((always_inline)) {
            if constexpr (!DIRECT) next.store(into, threadIdx.x);
        };
        auto landed = [&](uint64_t v_live, lds_t *k_into, lds_t *v_into) __attribute__((always_inline)) {      // (keys without a token get no weight, their values are zeros)
            if constexpr (DIRECT) {
                Straight::wait();
                Straight::blank(a.depth / Num<F>::CE, k_into);
                Straight::blank(a.depth / Num<F>::CE, v_into);
                if (v_live != ALL) Straight::trim(v_live, v_into);
            }
        };
        uint64_t live = live_of(begins_at(from)), live_next = 0;
        int32_t begin_next = begins_at(from + ROWS), at = from;
        request(k_next, k_rows, k_bytes, from, live, k_even);
        request(v_next, v_rows, v_bytes, from, live, v_even);
        put(k_next, k_even);
        put(v_next, v_even);
        landed(live, k_even, v_even);
        // The tile that begins at `at`; the next one goes into the other two.  False: it was the last.
        auto step = [&](const lds_t *keys, const lds_t *values, lds_t *k_into, lds_t *v_into) __attribute__((always_inline)) {
            __syncthreads();
            const bool more = at + ROWS <= to;
            if (more) {
                live_next = live_of(begin_next);
                request(k_next, k_rows, k_bytes, at + ROWS, live_next, k_into);
                request(v_next, v_rows, v_bytes, at + ROWS, live_next, v_into);
                begin_next = begins_at(at + 2 * ROWS);
                if constexpr (DIRECT) __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int n0 = 0; n0 < ROWS / 32; n0 += N) {
                const int32_t j0 = at + 32 * n0;
                if (j0 > wave_hi || j0 + 32 * N <= wave_lo) continue;
                f32x16 s[N];
                x.template score<ROWS>(keys + 32 * n0 * row_elems_of(DP), s);
                const uint64_t seen = live >> (32 * n0), all = N == 2 ? ~uint64_t(0) : 0xffffffffull;
                if (j0 < all_from || j0 + 32 * N - 1 > all_to || (seen & all) != all) {
                    const int32_t low = there ? lo - j0 - 4 * half : INT32_MAX / 2;
                    const uint32_t span = there ? static_cast<uint32_t>(i - lo) : 0u;
                    const uint64_t mine = seen >> (4 * half);
#pragma unroll
                    for (int n = 0; n < N; ++n)
#pragma unroll
                        for (int r = 0; r < 16; ++r) {
                            const int32_t j = 32 * n + 8 * (r >> 2) + (r & 3);
                            s[n][r] = static_cast<uint32_t>(j - low) <= span && (mine >> j & 1) != 0 ? s[n][r] : -INFINITY;
                        }
                }
                x.rescale(x.largest(s), a.scale);
                x.template take<ROWS>(s, a.scale, values + 32 * n0 * row_elems_of(DP));
            }
            if (more) {
                if constexpr (!TWO) __syncthreads();
                put(k_next, k_into);
                put(v_next, v_into);
                landed(live_next, k_into, v_into);
            }
            live = live_next;
            at += ROWS;
            return more;
        };
        for (;;) {
            if (!step(k_even, v_even, TWO ? k_odd : k_even, TWO ? v_odd : v_even)) break;
            if constexpr (TWO)
                if (!step(k_odd, v_odd, k_even, v_even)) break;
        }
    }

    const float total = halves_sum(x.total), share = 1.f / total, lse = x.top + __builtin_amdgcn_logf(total);
    char *out = a.out + ((row0 + i) * a.out_stride + int64_t(head) * a.depth) * ES;
    // weights that are numbers, but sums that are not, or scores of parts that are not
    const uint64_t halves = __ballot(there && (F == kParts && lse != lse ? true : fabsf(lse) < INFINITY && !x.finite()));
    const uint32_t spoilt = static_cast<uint32_t>(halves) | static_cast<uint32_t>(halves >> 32);
    if (i < T && (spoilt >> (lane & 31) & 1) == 0) {
        if (half == 0 && a.lse) a.lse[(peer * a.heads + head) * a.T + i] = there ? lse * kLn2 : 0.f;
#pragma unroll
        for (int m = 0; m < BLOCKS; ++m) {
            if (!there) x.sum[m] = f32x16{};
            store_column<DT>(out, 32 * m, a.depth, x.sum[m], there ? share : 0.f);
        }
    }
    // (told that it is rare, or registers go to its loops: a cache's heads of 256 in binary32: 410 us, 523)
    for (uint32_t left = spoilt; __builtin_expect(left != 0, 0); left &= left - 1) {
        const int32_t n = __builtin_ctz(left);
        attend_alone<DT>(a, peer, head, wave_first + n, __shfl(lo, n, 64), __shfl(lse, n, 64));
    }
}

// Tokens' queries against a span of keys.  A block has one sequence, one head of keys and a share of the span; its waves take tiles of 32 keys in turn,
// for the same 32 columns: the queries of the heads that share the keys, of the new tokens one after the other.  Nobody waits for
// anybody before the end.
// How many rows the sequence has in the cache, and the first.
__device__ __forceinline__ int32_t span_of(const CachedArgs &a, int64_t seq, int32_t &begin)
{
    const int32_t n_keys = static_cast<int32_t>(a.n_keys), first = a.spans[2 * seq], last = a.spans[2 * seq + 1], end = last > n_keys ? n_keys : last;
    begin = first < 0 ? 0 : first > n_keys ? n_keys : first;
    return end > begin ? end - begin : 0;
}
struct Share {
    int64_t peer, row;                   // row: of this lane's query
    int32_t split, kv_head, col_tile, seq, group, head, from, to, sees, all_see;      // keys of the share, by their number in the span
    bool there;
    const char *k_rows, *v_rows;         // key 0

    __device__ __forceinline__ Share(const CachedArgs &a, int es)
    {
        uint32_t b = blockIdx.x;
        kv_head = b % a.kv_heads;                                      // (neighbours in memory run at the same time)
        b /= a.kv_heads;
        col_tile = b % a.col_tiles;
        b /= a.col_tiles;
        seq = b % a.seqs;
        b /= a.seqs;
        peer = b % static_cast<uint32_t>(a.N);
        split = static_cast<int32_t>(b / static_cast<uint32_t>(a.N));
        group = a.heads / a.kv_heads;
        const int32_t column = col_tile * 32 + (threadIdx.x & 31), token = column / group;
        int32_t begin;
        head = kv_head * group + column - token * group;
        there = token < a.fresh;
        row = (peer * a.seqs + seq) * a.fresh + token;
        const int32_t count = span_of(a, peer * a.seqs + seq, begin);
        const int32_t each = static_cast<int32_t>((count + 32u * kWaves * a.splits - 1) / (32u * kWaves * a.splits)) * (32 * kWaves);
        from = split * each;
        to = int64_t(split + 1) * each < count ? (split + 1) * each : count;
        sees = there ? count - (a.fresh - 1 - token) : 0;             // how many of the span's keys this query does
        all_see = count - (a.fresh - 1);
        k_rows = a.k + ((peer * a.n_keys + begin) * a.k_stride + int64_t(kv_head) * a.depth) * es;
        v_rows = a.v + ((peer * a.n_keys + begin) * a.v_stride + int64_t(kv_head) * a.depth) * es;
    }
    // Scores of keys j0 .. j0 + 31 that the queries do not see become -inf.
    __device__ __forceinline__ void mask(f32x16 &s, int32_t j0) const
    {
        if (j0 + 32 <= to && j0 + 32 <= all_see) return;
        const int32_t seen = (sees < to ? sees : to) - j0 - 4 * (threadIdx.x >> 5 & 1);
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = 8 * (r >> 2) + (r & 3) < seen ? s[r] : -INFINITY;
    }
};

// This lane's elements of a query's sums by a wave again, for the same reasons and in the same manner as attend_alone, key by key over those that the query
// sees.  Both halves of a column take part.
template <int DT, int BLOCKS>
__device__ __forceinline__ void attend_again(const CachedArgs &a, const Share &share, int32_t wave, int32_t half, float &top, float &total, f32x16 (&sum)[BLOCKS])
{
    constexpr int ES = DT == 0 ? 4 : 2;
    const char *q = a.q + (share.row * a.q_stride + int64_t(share.head) * a.depth) * ES;
    const int32_t end = share.sees < share.to ? share.sees : share.to;
    auto each = [&](auto go) {                                         // go(key, score), for as long as it is true
        for (int32_t at = share.from + 32 * wave; at < end; at += 32 * kWaves)
            for (int32_t j = at; j < end && j < at + 32; ++j) {
                const char *k = share.k_rows + j * a.k_stride * ES;
                if (!go(j, dot<DT>(q, k, a.depth) * a.scale)) return;
            }
    };
#pragma unroll
    for (int m = 0; m < BLOCKS; ++m) sum[m] = f32x16{};
    if (DT == 0 && total != total) {
        top = -INFINITY;
        total = 0.f;
        each([&](int32_t, float s) {
            if (!(s < INFINITY)) {                                     // NaN or +inf: no weight is a number
                top = -INFINITY;
                total = NAN;
                return false;
            }
            if (s == -INFINITY) return true;
            const float now = fmaxf(top, s);
            total = fmaf(total, __builtin_amdgcn_exp2f(top - now), __builtin_amdgcn_exp2f(s - now));
            top = now;
            return true;
        });
        if (top == -INFINITY) return;
    }
    top += __builtin_amdgcn_logf(total);
    total = 0.f;
    each([&](int32_t j, float s) {
        const float w = __builtin_amdgcn_exp2f(s - top);
        if (w == 0.f) return true;
        total += w;
#pragma unroll
        for (int m = 0; m < BLOCKS; ++m)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int32_t d = 32 * m + 8 * (r >> 2) + 4 * half + (r & 3);
                if (d < a.depth) sum[m][r] = fmaf(w, load_one<DT>(share.v_rows + (j * a.v_stride + d) * ES), sum[m][r]);
            }
        return true;
    });
}

// A wave has one tile in LDS, keys and values by turns, and the one after it on its way in registers.  (Four tiles a wave, straight into LDS, bring
// nothing: 4 x 8 sequences of up to 16384, 4 heads of keys of 128 in bfloat16, in 155 us against 147.  Nor do equal shares of all sequences' keys, whatever
// their lengths: 141 us, and 33 against 23 for two sequences of 16000 and one head of keys.)
template <Form F, int DP, int SIMD>
__global__ __launch_bounds__(kThreads, SIMD)
void cached_kernel(CachedArgs a, float *__restrict__ partials)
{
    constexpr int ES = Num<F>::ES, DT = Num<F>::DT, BLOCKS = DP / 32, ELEMS = tile_elems<F, DP>(32);
    typedef typename Num<F>::lds_t lds_t;
    __shared__ __attribute__((aligned(16))) lds_t tiles[kWaves][ELEMS];
    __shared__ float tops[kWaves][32], totals[kWaves][32], block_total[32];
    const Share share(a, ES);
    const int32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
    const int64_t k_bytes = a.k_stride * ES, v_bytes = a.v_stride * ES;
    lds_t *tile = tiles[wave];
    auto live_of = [&](int32_t at) { return at + 32 <= share.to ? 0xffffffffull : (uint64_t(1) << (share.to - at)) - 1; };
    Queries<F, DP> x;
    int32_t at = share.from + 32 * wave;
    Staged<F, DP, 32, 64> next;
    if (at < share.to) next.load(share.k_rows + at * k_bytes, k_bytes, live_of(at), a.depth, lane);
    x.q.load(a.q + (share.row * a.q_stride + int64_t(share.head) * a.depth) * ES, share.there, a.depth);
    x.clear();
    auto put = [&] {                                                   // into the wave's own tile: written behind what was read, read behind what is written
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        next.store(tile, lane);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    };
    for (; at < share.to; at += 32 * kWaves) {
        put();
        next.load(share.v_rows + at * v_bytes, v_bytes, live_of(at), a.depth, lane);
        f32x16 s[1];
        x.template score<32>(tile, s);
        share.mask(s[0], at);
        x.rescale(x.largest(s), a.scale);
        Weights<F> w;
        x.weigh(s[0], a.scale, w);
        put();
        const int32_t after = at + 32 * kWaves;
        if (after < share.to) next.load(share.k_rows + after * k_bytes, k_bytes, live_of(after), a.depth, lane);
        x.template add<32>(tile, 0, w);
    }

    // the waves' sums, in order
    x.total = halves_sum(x.total);
    const uint64_t halves = __ballot(share.there && (F == kParts && x.total != x.total ? true : fabsf(x.top) < INFINITY && fabsf(x.total) < INFINITY && !x.finite()));
    if (__builtin_expect(((halves | halves >> 32) >> (lane & 31) & 1) != 0, 0)) attend_again<DT>(a, share, wave, half, x.top, x.total, x.sum);
    if (half == 0) {
        tops[wave][lane] = x.top;
        totals[wave][lane] = x.total;
    }
    __syncthreads();
    float top = tops[0][lane & 31], total = 0.f;
#pragma unroll
    for (int w = 1; w < kWaves; ++w) top = fmaxf(top, tops[w][lane & 31]);
    // (a quarter: four waves' sums together pass binary32 only where one of them does)
    auto factor_of = [&](float t) { return t == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(t - top) * (1.f / kWaves); };
#pragma unroll
    for (int w = 0; w < kWaves; ++w) total += totals[w][lane & 31] * factor_of(tops[w][lane & 31]);
    const float factor = factor_of(x.top);
    // Eight columns at a time, [wave][depth][9], in the place of the tiles (which no wave needs any more).
    constexpr int SOME = 8, PLACE = SOME + 1;
    float *joined = reinterpret_cast<float *>(tiles);
    static_assert(sizeof(tiles) >= kWaves * DP * PLACE * sizeof(float));
    const int32_t first = share.col_tile * 32, columns = a.fresh * share.group - first < 32 ? a.fresh * share.group - first : 32;
    for (int32_t c0 = 0; c0 < columns; c0 += SOME) {
        if (c0 > 0) __syncthreads();
        const int32_t mine = (lane & 31) - c0;
        if (mine >= 0 && mine < SOME)
#pragma unroll
            for (int m = 0; m < BLOCKS; ++m)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    joined[(wave * DP + 32 * m + 8 * (r >> 2) + 4 * half + (r & 3)) * PLACE + mine] = x.top == -INFINITY ? 0.f : x.sum[m][r] * factor;
        if (c0 == 0 && wave == 0 && half == 0) block_total[lane] = total;
        __syncthreads();
        const int32_t some = columns - c0 < SOME ? columns - c0 : SOME;
        for (int32_t n = threadIdx.x; n < some * a.depth; n += kThreads) {
            const int32_t c = n / a.depth, d = n - c * a.depth, column = first + c0 + c, t = column / share.group, h = share.kv_head * share.group + column - t * share.group;
            const int64_t r = (share.peer * a.seqs + share.seq) * a.fresh + t;
            float v = joined[d * PLACE + c];
#pragma unroll
            for (int w = 1; w < kWaves; ++w) v += joined[(w * DP + d) * PLACE + c];
            if (a.splits == 1) store_one<DT>(a.out + (r * a.out_stride + int64_t(h) * a.depth + d) * ES, share.all_see + t > 0 ? v / block_total[c0 + c] : 0.f);
            else partials[((r * a.heads + h) * a.splits + share.split) * a.depth + d] = v;
        }
    }
    if (a.splits > 1 && wave == 0 && half == 0 && share.there) {
        const int64_t shares = a.N * a.seqs * a.fresh * a.heads * a.splits;
        float *p = partials + shares * a.depth + (share.row * a.heads + share.head) * a.splits + share.split;
        p[0] = top;
        p[shares] = total;
    }
}

// The shares of a span, in order: a wave has a query of a head, a lane the top and total of one share (of several, where there are more than 64).
template <int DT>
__global__ __launch_bounds__(kThreads) void cached_join_kernel(CachedArgs a, const float *__restrict__ partials, int64_t rows)
{
    constexpr int ES = DT == 0 ? 4 : 2, MOST = 256 / 64;
    const int64_t n = int64_t(blockIdx.x) * kWaves + (threadIdx.x >> 6);
    if (n >= rows * a.heads) return;
    const int64_t row = n / a.heads, head = n % a.heads, shares = rows * a.heads * a.splits;
    const int lane = threadIdx.x & 63;
    const float *tops = partials + shares * a.depth + n * a.splits, *totals = tops + shares, *sums = partials + n * a.splits * a.depth;
    float top = -INFINITY, sum[MOST] = {}, total = 0.f;
    const float less = __uint_as_float((127u - (32 - __clz(a.splits - 1))) << 23);     // 2^-n <= 1 / splits, as above
    for (int s = lane; s < a.splits; s += 64) top = fmaxf(top, tops[s]);
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor(top, off, 64));
    for (int s0 = 0; s0 < a.splits; s0 += 64) {
        const int left = a.splits - s0 < 64 ? a.splits - s0 : 64;
        float mine = -INFINITY, part = 0.f;
        if (lane < left) {
            mine = tops[s0 + lane];
            part = totals[s0 + lane];
        }
        const float factor = mine == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mine - top) * less;
        for (int s = 0; s < left; s += 4) {                            // four shares requested at a time
            float v[4][MOST];
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int t = 0; t < MOST; ++t) v[u][t] = s + u < left && lane + 64 * t < a.depth ? sums[int64_t(s0 + s + u) * a.depth + lane + 64 * t] : 0.f;
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const float f = __shfl(factor, (s + u) & 63, 64), p = __shfl(part, (s + u) & 63, 64);
                if (s + u >= left) continue;
                total = fmaf(p, f, total);
#pragma unroll
                for (int t = 0; t < MOST; ++t) sum[t] = fmaf(v[u][t], f, sum[t]);
            }
        }
    }
    int32_t begin;
    const bool some = span_of(a, row / a.fresh, begin) > a.fresh - 1 - row % a.fresh;
    char *out = a.out + (row * a.out_stride + head * a.depth) * ES;
#pragma unroll
    for (int t = 0; t < MOST; ++t)
        if (lane + 64 * t < a.depth) store_one<DT>(out + (lane + 64 * t) * ES, some ? sum[t] / total : 0.f);
}

int64_t attention_blocks(const AttentionArgs &a) { return a.N * a.heads * ((a.T + kQueries - 1) / kQueries); }

}  // namespace

bool attention_fits(const AttentionArgs &a) { return launchable(attention_blocks(a), kThreads); }

hipError_t launch_attention(AttentionArgs a, int dtype, int compute_units, hipStream_t stream)
{
    if (a.T == 0) return hipSuccess;
    a.scale *= kLog2e;
    a.tiles = static_cast<uint32_t>((a.T + kQueries - 1) / kQueries);
    const uint32_t blocks = static_cast<uint32_t>(attention_blocks(a));
    return by_depth(dtype, a.depth, [&](auto form, auto dp) {
        constexpr Form F = decltype(form)::value;
        constexpr int DP = decltype(dp)::value;
        // bfloat16: two blocks of keys at a time (2 x 16 heads of 128, 8192 tokens: 430 us, one at a time 454), up to a depth of 64 one, with four waves a
        // SIMD (16 x 8 heads of 64, 4096 tokens: 138 us, two at a time with three waves 150)
        const bool direct = F != kParts && direct_rows(a.k, a.k_stride, a.depth, dtype) && direct_rows(a.v, a.v_stride, a.depth, dtype);
        if constexpr (F == kParts) {
            // binary32 deeper than 64: one buffer of a tile and two blocks a compute unit (4 x 8 heads, 4000 tokens, depth 80: 323 us, depth 128: 570; two
            // buffers and one block 509, 631).  Deeper than 96 that spills, and two buffers pay for as long as there are not more than two blocks for
            // each compute unit (4 x 4 heads of 128, 500 tokens: 56 us, one buffer 71; 4 x 16 heads, 1000 tokens: 132, 143; 4000 tokens: above)
            if constexpr (DP > 96)
                if (blocks <= 2 * static_cast<uint32_t>(compute_units)) {
                    attention_kernel<F, DP, 32, 1, 1, false><<<blocks, kThreads, 0, stream>>>(a);
                    return hipGetLastError();
                }
            attention_kernel<F, DP, 32, 1, 2, false><<<blocks, kThreads, 0, stream>>>(a);
        }
        else if constexpr (DP > 128) {
            if (direct) attention_kernel<F, DP, 32, 1, 1, true><<<blocks, kThreads, 0, stream>>>(a);
            else attention_kernel<F, DP, 32, 1, 1, false><<<blocks, kThreads, 0, stream>>>(a);
        } else {
            constexpr int JOINT = DP <= 64 ? 1 : 2, SIMD = DP <= 64 ? 4 : 2;
            if (direct) attention_kernel<F, DP, 64, JOINT, SIMD, true><<<blocks, kThreads, 0, stream>>>(a);
            else attention_kernel<F, DP, 64, JOINT, (DP <= 64 ? 3 : 2), false><<<blocks, kThreads, 0, stream>>>(a);
        }
        return hipGetLastError();
    });
}

// Blocks of cached_kernel a compute unit, as its registers allow.  The deepest heads hold a tile on its way, the queries and the sums in more than there are:
// 84 of 256 in bfloat16 spill, 205 of 192 and 799 of 256 in binary32 (4 x 8 sequences, 4 heads of keys, caches of 8192 in bfloat16 and 4096 in binary32: of 192
// 144 us and 242, of 256 374 and 410).
constexpr int cached_waves(Form f, int dp) { return f == kBf16 && dp <= 128 ? 2 : 1; }

// Shares of a span: twice the blocks that run at once, and 512 keys each and more where the keys of a peer are one sequence's.
CachedPlan cached_plan(const CachedArgs &a, int dtype, int compute_units)
{
    CachedPlan p;
    p.col_tiles = (a.fresh * (a.heads / a.kv_heads) + 31) / 32;
    const int64_t blocks = a.N * a.seqs * a.kv_heads * p.col_tiles, at_once = int64_t(compute_units) * cached_waves(dtype == 0 ? kF32 : kBf16, a.depth);
    const int64_t most = blocks > 0 ? 2 * at_once / blocks : 1, use = (a.n_keys + 511) / 512;
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
    const hipError_t e = by_depth(dtype, a.depth, [&](auto form, auto dp) {
        constexpr Form F = decltype(form)::value;
        constexpr int DP = decltype(dp)::value;
        const uint32_t blocks = static_cast<uint32_t>(a.N * a.seqs * a.kv_heads * p.col_tiles * p.splits);
        cached_kernel<F, DP, cached_waves(F, DP)><<<blocks, kThreads, 0, stream>>>(a, partials);
        return hipGetLastError();
    });
    if (e != hipSuccess || p.splits == 1) return e;
    const uint32_t join_blocks = static_cast<uint32_t>((rows * a.heads + kWaves - 1) / kWaves);
    (dtype == 0 ? cached_join_kernel<0> : cached_join_kernel<1>)<<<join_blocks, kThreads, 0, stream>>>(a, partials, rows);
    return hipGetLastError();
}

}  // namespace moshpit
