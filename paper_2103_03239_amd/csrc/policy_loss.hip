// The clipped policy loss with a KL term, from logits, and the logits' gradient, for gfx950.  For a row z of
// logits, its token a and weight w:
//   lp = z_a - log sum_j exp z_j,  r = exp(lp - old),  k = exp(ref - lp) - (ref - lp) - 1
//   loss = w * (kl_coef * k - min(A r, A clip(r, 1 - clip_low, 1 + clip_high)))
//   d loss / d lp = s = w * (kl_coef * (1 - exp(ref - lp)) - [A r <= A clip(r)] A r)
//   d loss / d z_j = s * ([j = a] - exp(z_j - m) / sum exp(z - m)),   m = max z
// in binary32 throughout, the gradient rounded once.  A row without weight or token is not read: its gradient
// and log-probability are zeros.
//
// Bound by HBM: a row is read once and its gradient written once, so a block holds a whole row in registers
// (VECS vectors of 16 bytes a thread) from the first pass (largest element and sum of exponentials, by thread,
// wave and block) to the second (gradient).  Rows that do not fit, and few rows, are cut into slices: a first
// kernel leaves (largest, sum) of every slice, a second joins them and writes the gradient, its second
// read of the logits coming from the caches where they are small.  16384 bfloat16 rows of 50001, 0.7 of
// them with a token, in 487 to 499 us, 5.7 TB/s; log-probabilities alone of 8192 binary32 rows of 30000 in 161 us, 6.1 TB/s.
#include <hip/hip_runtime.h>

#include "local_ops.h"
#include "row_elems.h"

namespace moshpit {
namespace {

constexpr float kLog2e = 1.44269504088896340736f;

// exp(x - m), m finite or x = m = -inf excluded by the caller
__device__ __forceinline__ float exp_above(float x, float m) { return __builtin_amdgcn_exp2f((x - m) * kLog2e); }

// The largest element of a set and the sum of exp(x - largest) over it; {-inf, 0} of nothing.
struct TopSum {
    float top, sum;
};
__device__ __forceinline__ TopSum join(const TopSum &a, const TopSum &b)
{
    const float top = fmaxf(a.top, b.top);
    // a set whose largest element is -inf has the sum 0 (nothing) or its number of elements (all -inf): exp(-inf - top) = 0
    // counts neither where the other one is finite, and where both are -inf the sums add as they are
    const float fa = a.top == top ? 1.f : exp_above(a.top, top), fb = b.top == top ? 1.f : exp_above(b.top, top);
    // (a NaN anywhere stays in the sum: fmaxf drops it from the tops)
    return {top, a.sum * fa + b.sum * fb};
}

// v of a lane further down the wave (CTRL: a DPP control), `old` where there is none.
template <int CTRL, int ROWS> __device__ __forceinline__ float from_lane(float old, float v)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, old), __builtin_bit_cast(int, v), CTRL, ROWS, 0xf, false));
}
// A whole wave's largest value and sum, in the same order every time: within rows of 16 lanes, then across them.
__device__ __forceinline__ float wave_top(float v)
{
    v = fmaxf(v, from_lane<0x111, 0xf>(-INFINITY, v));
    v = fmaxf(v, from_lane<0x112, 0xf>(-INFINITY, v));
    v = fmaxf(v, from_lane<0x114, 0xf>(-INFINITY, v));
    v = fmaxf(v, from_lane<0x118, 0xf>(-INFINITY, v));
    v = fmaxf(v, from_lane<0x142, 0xa>(-INFINITY, v));
    v = fmaxf(v, from_lane<0x143, 0xc>(-INFINITY, v));
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
}
__device__ __forceinline__ float wave_sum(float v)
{
    v += from_lane<0x111, 0xf>(0.f, v);
    v += from_lane<0x112, 0xf>(0.f, v);
    v += from_lane<0x114, 0xf>(0.f, v);
    v += from_lane<0x118, 0xf>(0.f, v);
    v += from_lane<0x142, 0xa>(0.f, v);
    v += from_lane<0x143, 0xc>(0.f, v);
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
}
__device__ __forceinline__ TopSum wave_join(const TopSum &t)
{
    const float top = wave_top(t.top);
    return {top, wave_sum(t.sum * (t.top == top ? 1.f : exp_above(t.top, top)))};
}

// The first wave gets the block's.
template <int THREADS>
__device__ __forceinline__ TopSum block_join(TopSum t)
{
    constexpr int WAVES = THREADS / 64;
    __shared__ TopSum of_wave[WAVES];
    t = wave_join(t);
    if constexpr (WAVES > 1) {
        if ((threadIdx.x & 63) == 0) of_wave[threadIdx.x >> 6] = t;
        __syncthreads();
        if (threadIdx.x < 64) t = wave_join(threadIdx.x < WAVES ? of_wave[threadIdx.x] : TopSum{-INFINITY, 0.f});
    }
    return t;
}

// A wave's accesses begin with a cache line where the block has threads enough for the up to 126 single elements around them: 16
// x 1024 rows of 50001 bfloat16 logits in 498 us, at 16-byte boundaries in 540.
constexpr int line_of(int threads) { return threads >= 128 ? 128 : 16; }

// Elements [begin, end) of a row as whole vectors, the first at a multiple of ALIGN bytes, and single elements around them.
template <int DT, int ALIGN = 16> struct Slice {
    static constexpr int ES = DT == 0 ? 4 : 2, VE = 16 / ES;
    const char *vectors;                 // the first whole vector
    int32_t count;                       // whole vectors
    int32_t head, tail;                  // single elements before and after them
    __device__ __forceinline__ Slice(const char *from, int64_t n)
    {
        const uint32_t phase = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(from)) % ALIGN / ES;
        head = phase ? ALIGN / ES - static_cast<int32_t>(phase) : 0;
        if (head > n) head = static_cast<int32_t>(n);
        vectors = from + head * ES;
        count = static_cast<int32_t>((n - head) / VE);
        tail = static_cast<int32_t>(n - head - int64_t(count) * VE);
    }
    // element of single number k, 0 <= k < head + tail, from the slice's first one on
    __device__ __forceinline__ int64_t single(int k) const { return k < head ? k : int64_t(count) * VE + k; }
};

template <int DT> __device__ __forceinline__ void widen_vec(const u32x4 &m, float (&f)[16 / (DT == 0 ? 4 : 2)])
{
    if constexpr (DT == 0) {
#pragma unroll
        for (int k = 0; k < 4; ++k) f[k] = __uint_as_float(m[k]);
    } else Vec<1, 8>::widen(m, f);
}

template <int VE> __device__ __forceinline__ float largest(const float (&f)[VE])
{
    float top = f[0];
#pragma unroll
    for (int k = 1; k < VE; ++k) top = fmaxf(top, f[k]);
    return top;
}

// The sum of exp(f - m).  The difference comes first: -m log2 e in a fused multiply-add would be off by 2^-24 of its own size, which
// grows with an offset common to the row, and infinite for m near the type's lowest value, as a mask may be.
template <int VE> __device__ __forceinline__ float sum_exp(const float (&f)[VE], float m)
{
    float e[VE];
#pragma unroll
    for (int k = 0; k < VE; ++k) e[k] = exp_above(f[k], m);
#pragma unroll
    for (int w = VE / 2; w > 0; w /= 2)
#pragma unroll
        for (int k = 0; k < w; ++k) e[k] += e[k + w];
    return e[0];
}
// What is taken from values whose largest is `top`: of -inf alone nothing, so that exp(-inf) = 0.
__device__ __forceinline__ float base_of(float top) { return top == -INFINITY ? 0.f : top; }

template <int VE> __device__ __forceinline__ void add_values(TopSum &t, const float (&f)[VE])
{
    const float top = largest(f);
    if (top > t.top) {
        t.sum *= t.top == -INFINITY ? 0.f : exp_above(t.top, top);
        t.top = top;
    }
    t.sum += sum_exp(f, base_of(t.top));
}

// What was made of these registers is not to be kept for the next pass over them: the row as it came is all there is room for.
template <int N> __device__ __forceinline__ void keep_packed(u32x4 (&held)[N])
{
#pragma unroll
    for (int v = 0; v < N; ++v) asm volatile("" : "+v"(held[v]));
}

struct RowPlace {
    int64_t vocab, stride;
};

// What a row adds to its peer's sums: loss, w k, w [clipped].
struct RowTerms {
    float loss, kl, clipped;
};

// exp(x) - 1 - x, given exp(x) - 1.  Near 0 the difference has few of its terms' digits (none at 1e-4, and a policy starts as its own
// reference) and may come out negative: within 1/2 the series x^2 / 2 (1 + x / 3 (1 + x / 4 (...))), which ends below 2^-28 of it.
__device__ __forceinline__ float above_tangent(float x, float exp_less_1)
{
    if (!(fabsf(x) < 0.5f)) return exp_less_1 - x;
    float s = 1.f;
#pragma unroll
    for (int n = 10; n >= 3; --n) s = fmaf(x * (1.f / static_cast<float>(n)), s, 1.f);
    return 0.5f * x * x * s;
}

// From a row's log-probability: its terms and d loss / d lp.
__device__ __forceinline__ float row_terms(const PolicyTerms &p, int64_t row, float w, float lp, RowTerms &terms)
{
    const float A = p.advantage[row], r = expf(lp - p.old_logp[row]);
    const float low = 1.f - p.clip_low, high = 1.f + p.clip_high;
    const float plain = A * r, cut = A * (r < low ? low : r > high ? high : r);
    const bool clipped = plain > cut;
    float k = 0.f, dk = 0.f;
    if (p.ref_logp) {
        const float off = p.ref_logp[row] - lp, e = expm1f(off);
        k = above_tangent(off, e);
        dk = -e;
    }
    // (with the coefficient 0 k is a statistic alone: 0 times an infinite one would be NaN)
    const float kl = p.kl_coef != 0.f ? p.kl_coef * k : 0.f, dkl = p.kl_coef != 0.f ? p.kl_coef * dk : 0.f;
    terms.loss = w * (kl - (clipped ? cut : plain));
    terms.kl = w * k;
    terms.clipped = clipped ? w : 0.f;
    return w * (dkl - (clipped ? 0.f : plain));
}

// Where a row's log-probability and terms go: the terms wait for the others of the peer, or are the peer's sums already (T = 1).
struct RowOut {
    float *logp, *stats;                 // stats: of peers with one row each, or nullptr
    RowTerms *terms;
    __device__ __forceinline__ void put(int64_t row, float lp, const RowTerms &t) const
    {
        logp[row] = lp;
        if (stats) {
            stats[3 * row] = t.loss;
            stats[3 * row + 1] = t.kl;
            stats[3 * row + 2] = t.clipped;
        } else terms[row] = t;
    }
};

template <int DT, int THREADS>
__device__ __forceinline__ void store_zeros(char *grad, int64_t n)
{
    constexpr int ES = DT == 0 ? 4 : 2;
    const Slice<DT, line_of(THREADS)> s(grad, n);
    for (int v = threadIdx.x; v < s.count; v += THREADS)
        store_vec<true, u32x4>(const_cast<char *>(s.vectors) + int64_t(v) * 16, u32x4{0, 0, 0, 0});
    for (int k = threadIdx.x; k < s.head + s.tail; k += THREADS) store_one<DT>(grad + s.single(k) * ES, 0.f);
}

// A row by THREADS threads, in registers; rows of 64 threads four to a block.  The gradient may take the logits' place (here and
// below): every element is read before it is written, by the same thread.
constexpr int rows_of_block(int threads) { return threads == 64 ? 4 : 1; }

template <int DT, int THREADS, int VECS>
__global__ __launch_bounds__(THREADS * rows_of_block(THREADS), VECS == 8 ? 8 : 4)
void policy_row_kernel(const char *logits, int64_t rows, RowPlace at, const int32_t *__restrict__ tokens, PolicyTerms p, char *grad,
                       int64_t grad_stride, RowOut out)
{
    constexpr int ES = DT == 0 ? 4 : 2, VE = 16 / ES, ALIGN = line_of(THREADS);
    // runs of rows for each die: 16 x 1600 rows of 32768 bfloat16 logits, a power of two apart, in 574 us, row by row in 647
    const int64_t row = int64_t(die_run(blockIdx.x, gridDim.x)) * rows_of_block(THREADS) + threadIdx.y;
    if (row >= rows) return;
    const float w = p.weight[row];
    const int64_t token = tokens[row];
    char *to = grad + row * grad_stride * ES;
    if (w == 0.f || token < 0 || token >= at.vocab) {
        store_zeros<DT, THREADS>(to, at.vocab);
        if (threadIdx.x == 0) out.put(row, 0.f, RowTerms{0.f, 0.f, 0.f});
        return;
    }
    const char *from = logits + row * at.stride * ES;
    const Slice<DT, ALIGN> s(from, at.vocab);
    const float z_token = load_one<DT>(from + token * ES);
    u32x4 held[VECS];
    float single = -INFINITY;
#pragma unroll
    for (int v = 0; v < VECS; ++v) {
        const int32_t i = v * THREADS + threadIdx.x;
        if (i < s.count) held[v] = load_vec<true, u32x4>(s.vectors + int64_t(i) * 16);
    }
    if (static_cast<int32_t>(threadIdx.x) < s.head + s.tail) single = load_one<DT>(from + s.single(threadIdx.x) * ES);
    // first this thread's largest value, then its sum: its values are all here
    TopSum t{single, 0.f};
#pragma unroll
    for (int v = 0; v < VECS; ++v) {
        if (v * THREADS + static_cast<int32_t>(threadIdx.x) >= s.count) continue;
        float f[VE];
        widen_vec<DT>(held[v], f);
        t.top = fmaxf(t.top, largest(f));
    }
    keep_packed(held);
    const float own_base = base_of(t.top);
    t.sum = exp_above(single, own_base);
#pragma unroll
    for (int v = 0; v < VECS; ++v) {
        if (v * THREADS + static_cast<int32_t>(threadIdx.x) >= s.count) continue;
        float f[VE];
        widen_vec<DT>(held[v], f);
        t.sum += sum_exp(f, own_base);
    }
    keep_packed(held);
    t = block_join<THREADS>(t);
    float slope, factor, top;
    if (threadIdx.x < 64) {                                           // (the same for all its lanes)
        const float lp = z_token - t.top - logf(t.sum);
        RowTerms mine;
        slope = row_terms(p, row, w, lp, mine);
        factor = -slope / t.sum;
        top = t.top;                                                  // (a row of -inf alone: NaN)
        if (threadIdx.x == 0) out.put(row, lp, mine);
    }
    if constexpr (THREADS > 64) {
        __shared__ float of_row[3];
        if (threadIdx.x == 0) {
            of_row[0] = slope;
            of_row[1] = factor;
            of_row[2] = top;
        }
        __syncthreads();
        slope = of_row[0];
        factor = of_row[1];
        top = of_row[2];
    }
    const int32_t token_vec = static_cast<int32_t>((token - s.head) >> (DT == 0 ? 2 : 3));       // (may be none of the whole ones)
    const int32_t token_elem = static_cast<int32_t>(token - s.head) & (VE - 1);
#pragma unroll
    for (int v = 0; v < VECS; ++v) {
        const int32_t i = v * THREADS + threadIdx.x;
        if (i >= s.count) continue;
        float f[VE];
        widen_vec<DT>(held[v], f);
#pragma unroll
        for (int k = 0; k < VE; ++k) f[k] = factor * exp_above(f[k], top);
        if (i == token_vec) {
#pragma unroll
            for (int k = 0; k < VE; ++k)
                if (k == token_elem) f[k] += slope;
        }
        store_elems<DT, VE, true>(to + (s.head + i * VE) * ES, f);
    }
    if (static_cast<int32_t>(threadIdx.x) < s.head + s.tail) {
        const int64_t e = s.single(threadIdx.x);
        store_one<DT>(to + e * ES, factor * exp_above(single, top) + (token == e ? slope : 0.f));
    }
}

// Short rows, up to 2 KiB: a wave takes kShort of them, finds each one's largest value and sum, does the arithmetic of their terms
// side by side, a row a lane, and writes the gradients.  (A wave a row spends more on the terms than on the row.)
constexpr int kShort = 8, kShortVecs = 2;

template <int DT, bool GRAD>
__global__ __launch_bounds__(256, 4)
void short_rows_kernel(const char *logits, int64_t rows, RowPlace at, const int32_t *__restrict__ tokens, PolicyTerms p, char *grad,
                       int64_t grad_stride, RowOut out)
{
    constexpr int ES = DT == 0 ? 4 : 2, VE = 16 / ES;
    const int lane = threadIdx.x & 63;
    const int64_t first = (int64_t(blockIdx.x) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6)) * kShort;
    if (first >= rows) return;
    const int count = rows - first < kShort ? static_cast<int>(rows - first) : kShort;
    // lane r looks after row first + r
    const int64_t own = first + (lane < count ? lane : 0);
    const int32_t token = tokens[own];
    const float w = GRAD ? p.weight[own] : 1.f;
    const bool live = lane < count && w != 0.f && token >= 0 && token < at.vocab;
    const uint64_t alive = __ballot(live);
    const float z_token = live ? load_one<DT>(logits + (own * at.stride + token) * ES) : 0.f;
    u32x4 held[kShort][kShortVecs];
    float single[kShort];
#pragma unroll
    for (int r = 0; r < kShort; ++r) {
        single[r] = -INFINITY;
        if (!(alive >> r & 1)) continue;
        const char *from = logits + (first + r) * at.stride * ES;
        const Slice<DT> s(from, at.vocab);
#pragma unroll
        for (int v = 0; v < kShortVecs; ++v)
            if (v * 64 + lane < s.count) held[r][v] = load_vec<true, u32x4>(s.vectors + (v * 64 + lane) * 16);
        if (lane < s.head + s.tail) single[r] = load_one<DT>(from + s.single(lane) * ES);
    }
    TopSum mine{0.f, 1.f};
#pragma unroll
    for (int r = 0; r < kShort; ++r) {
        if (!(alive >> r & 1)) continue;
        const Slice<DT> s(logits + (first + r) * at.stride * ES, at.vocab);
        float f[kShortVecs][VE], top = single[r];
#pragma unroll
        for (int v = 0; v < kShortVecs; ++v) {
            if (v * 64 + lane >= s.count) continue;
            widen_vec<DT>(held[r][v], f[v]);
            top = fmaxf(top, largest(f[v]));
        }
        top = wave_top(top);
        const float base = base_of(top);
        float sum = exp_above(single[r], base);
#pragma unroll
        for (int v = 0; v < kShortVecs; ++v)
            if (v * 64 + lane < s.count) sum += sum_exp(f[v], base);
        sum = wave_sum(sum);
        if (lane == r) mine = TopSum{top, sum};
        if constexpr (GRAD) keep_packed(held[r]);
    }
    const float lp = live ? z_token - mine.top - logf(mine.sum) : 0.f;
    RowTerms terms{0.f, 0.f, 0.f};
    float slope = 0.f;
    if constexpr (GRAD) {
        if (live) slope = row_terms(p, own, w, lp, terms);
        if (lane < count) out.put(own, lp, terms);
    } else if (lane < count) out.logp[own] = lp;
    if constexpr (!GRAD) return;
    const float factor = -slope / mine.sum;
    auto lane_value = [](float v, int r) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), r)); };
#pragma unroll
    for (int r = 0; r < kShort; ++r) {
        if (r >= count) break;
        char *to = grad + (first + r) * grad_stride * ES;
        if (!(alive >> r & 1)) {
            const Slice<DT> s(to, at.vocab);
            for (int v = lane; v < s.count; v += 64) store_vec<true, u32x4>(const_cast<char *>(s.vectors) + v * 16, u32x4{0, 0, 0, 0});
            if (lane < s.head + s.tail) store_one<DT>(to + s.single(lane) * ES, 0.f);
            continue;
        }
        const Slice<DT> s(logits + (first + r) * at.stride * ES, at.vocab);
        const float row_slope = lane_value(slope, r), row_factor = lane_value(factor, r), row_top = lane_value(mine.top, r);
        const int32_t row_token = __builtin_amdgcn_readlane(token, r);
#pragma unroll
        for (int v = 0; v < kShortVecs; ++v) {
            const int32_t i = v * 64 + lane;
            if (i >= s.count) continue;
            float f[VE];
            widen_vec<DT>(held[r][v], f);
            const int32_t e = s.head + i * VE;
#pragma unroll
            for (int k = 0; k < VE; ++k) f[k] = row_factor * exp_above(f[k], row_top) + (row_token == e + k ? row_slope : 0.f);
            store_elems<DT, VE, true>(to + e * ES, f);
        }
        if (lane < s.head + s.tail) {
            const int64_t e = s.single(lane);
            store_one<DT>(to + e * ES, row_factor * exp_above(single[r], row_top) + (row_token == e ? row_slope : 0.f));
        }
    }
}

constexpr int64_t kShortBytes = kShortVecs * 64 * 16;

// Rows cut into slices: block b works on slice b % slices of row b / slices.
struct Cut {
    int32_t slices;
    int64_t length;                      // elements of a slice
};

template <int DT, int THREADS>
__global__ __launch_bounds__(THREADS * rows_of_block(THREADS))
void slice_sum_kernel(const char *__restrict__ logits, int64_t rows, RowPlace at, Cut cut, const int32_t *__restrict__ tokens,
                      const float *__restrict__ weight, TopSum *__restrict__ sums, float *__restrict__ z_token, float *__restrict__ logp)
{
    constexpr int ES = DT == 0 ? 4 : 2, VE = 16 / ES, kBatch = 8;
    const int64_t block = int64_t(blockIdx.x) * rows_of_block(THREADS) + threadIdx.y;       // (rows of 64 threads are not cut)
    const int64_t row = THREADS == 64 ? block : block / cut.slices;
    if (row >= rows) return;
    const int32_t slice = THREADS == 64 ? 0 : blockIdx.x % static_cast<uint32_t>(cut.slices);
    const int64_t token = tokens[row];
    const bool live = (!weight || weight[row] != 0.f) && token >= 0 && token < at.vocab;
    if (!live) {
        if (logp && slice == 0 && threadIdx.x == 0) logp[row] = 0.f;
        return;
    }
    const int64_t begin = slice * cut.length, end = begin + cut.length < at.vocab ? begin + cut.length : at.vocab;
    const char *from = logits + (row * at.stride + begin) * ES;
    const Slice<DT, line_of(THREADS)> s(from, end - begin);
    TopSum t{-INFINITY, 0.f};
    for (int k = threadIdx.x; k < s.head + s.tail; k += THREADS) t = join(t, TopSum{load_one<DT>(from + s.single(k) * ES), 1.f});
    for (int32_t i0 = threadIdx.x; i0 < s.count; i0 += THREADS * kBatch) {
        u32x4 m[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u)
            if (i0 + u * THREADS < s.count) m[u] = load_vec<false, u32x4>(s.vectors + int64_t(i0 + u * THREADS) * 16);
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            if (i0 + u * THREADS >= s.count) continue;
            float f[VE];
            widen_vec<DT>(m[u], f);
            add_values(t, f);
        }
    }
    t = block_join<THREADS>(t);
    if (threadIdx.x != 0) return;
    if (!z_token) {
        logp[row] = load_one<DT>(logits + (row * at.stride + token) * ES) - t.top - logf(t.sum);
        return;
    }
    sums[block] = t;
    if (slice == 0) z_token[row] = load_one<DT>(logits + (row * at.stride + token) * ES);
}

// The slices of a row joined, by a wave.
__device__ __forceinline__ TopSum joined(const TopSum *__restrict__ sums, int32_t slices)
{
    TopSum t{-INFINITY, 0.f};
    for (int32_t k = threadIdx.x & 63; k < slices; k += 64) t = join(t, sums[k]);
    return wave_join(t);
}

template <int DT, int THREADS>
__global__ __launch_bounds__(THREADS) void policy_slice_kernel(const char *logits, RowPlace at, Cut cut, const int32_t *__restrict__ tokens,
                                                               PolicyTerms p, const TopSum *__restrict__ sums, const float *__restrict__ z_token, char *grad, int64_t grad_stride,
                                                               RowOut out)
{
    constexpr int ES = DT == 0 ? 4 : 2, VE = 16 / ES, kBatch = 4;
    const int64_t row = blockIdx.x / static_cast<uint32_t>(cut.slices);
    const int32_t slice = blockIdx.x % static_cast<uint32_t>(cut.slices);
    const float w = p.weight[row];
    const int64_t token = tokens[row];
    const int64_t begin = slice * cut.length, end = begin + cut.length < at.vocab ? begin + cut.length : at.vocab;
    char *to = grad + (row * grad_stride + begin) * ES;
    if (w == 0.f || token < 0 || token >= at.vocab) {
        store_zeros<DT, THREADS>(to, end - begin);
        if (slice == 0 && threadIdx.x == 0) out.put(row, 0.f, RowTerms{0.f, 0.f, 0.f});
        return;
    }
    const TopSum t = joined(sums + row * cut.slices, cut.slices);
    const float lp = z_token[row] - t.top - logf(t.sum);             // (kept aside: another block's gradient may be in the logit's place by now)
    RowTerms mine;
    const float slope = row_terms(p, row, w, lp, mine);
    if (slice == 0 && threadIdx.x == 0) out.put(row, lp, mine);
    const float factor = -slope / t.sum;
    const char *from = logits + (row * at.stride + begin) * ES;
    const Slice<DT, line_of(THREADS)> s(from, end - begin);
    for (int32_t i0 = threadIdx.x; i0 < s.count; i0 += THREADS * kBatch) {
        u32x4 m[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u)
            if (i0 + u * THREADS < s.count) m[u] = load_vec<false, u32x4>(s.vectors + int64_t(i0 + u * THREADS) * 16);
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            const int32_t i = i0 + u * THREADS;
            if (i >= s.count) continue;
            float f[VE];
            widen_vec<DT>(m[u], f);
            const int64_t e = s.head + int64_t(i) * VE;
#pragma unroll
            for (int k = 0; k < VE; ++k) f[k] = factor * exp_above(f[k], t.top);
            if (token >= begin + e && token < begin + e + VE) {
#pragma unroll
                for (int k = 0; k < VE; ++k)
                    if (token == begin + e + k) f[k] += slope;
            }
            store_elems<DT, VE, true>(to + e * ES, f);
        }
    }
    for (int k = threadIdx.x; k < s.head + s.tail; k += THREADS) {
        const int64_t e = s.single(k);
        store_one<DT>(to + e * ES, factor * exp_above(load_one<DT>(from + e * ES), t.top) + (token == begin + e ? slope : 0.f));
    }
}

__global__ __launch_bounds__(64) void logp_join_kernel(const TopSum *__restrict__ sums, const float *__restrict__ z_token, int32_t slices,
                                                       const int32_t *__restrict__ tokens, int64_t vocab, float *__restrict__ logp)
{
    const int64_t row = blockIdx.x, token = tokens[row];
    if (token < 0 || token >= vocab) return;                         // (written by the kernel before)
    const TopSum t = joined(sums + row * slices, slices);
    if (threadIdx.x == 0) logp[row] = z_token[row] - t.top - logf(t.sum);
}

// The terms of a peer's rows, summed in binary64 in an order that depends on T alone.  A thread requests four rows' terms before
// it adds the first: one block is bound by the latency of its loads.  Threads by what a loss with rows of 64 entries took with 64, 256
// and 1024: 256 peers of 100 rows 19.8, 19.9 and 20.6 us, 256 of 1024 105.6, 102.8 and 103.2, 4 of 8192 44.3, 24.2 and 20.3.
constexpr int kStatsThreads = 1024;

__global__ __launch_bounds__(kStatsThreads) void policy_stats_kernel(const RowTerms *__restrict__ terms, int64_t T, float *__restrict__ stats)
{
    __shared__ double of_wave[kStatsThreads / 64][3];
    const RowTerms *mine = terms + int64_t(blockIdx.x) * T;
    const int32_t step = blockDim.x;
    double sum[3] = {0.0, 0.0, 0.0};
    for (int64_t t0 = threadIdx.x; t0 < T; t0 += 4 * step) {
        RowTerms v[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) v[u] = t0 + u * step < T ? mine[t0 + u * step] : RowTerms{0.f, 0.f, 0.f};
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            sum[0] += v[u].loss;
            sum[1] += v[u].kl;
            sum[2] += v[u].clipped;
        }
    }
#pragma unroll
    for (int q = 0; q < 3; ++q) {
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) sum[q] += __shfl_down(sum[q], off, 64);
        if ((threadIdx.x & 63) == 0) of_wave[threadIdx.x >> 6][q] = sum[q];
    }
    __syncthreads();
    if (threadIdx.x < 3) {
        double all = 0.0;
        for (int w = 0; w < step / 64; ++w) all += of_wave[w][threadIdx.x];
        stats[int64_t(blockIdx.x) * 3 + threadIdx.x] = static_cast<float>(all);
    }
}

// ---- launches ----------------------------------------------------------------

constexpr int kSliceThreads = 256;
constexpr int64_t kRowBytes = 1024 * 16 * 16;         // what a block of 1024 threads holds

int64_t elem_size(int dtype) { return dtype == 0 ? 4 : 2; }

// Slices of a row: enough blocks for the chip, at least 16 KiB each.
Cut cut_of(int64_t rows, int64_t vocab, int dtype, int compute_units)
{
    const int64_t want = (4 * compute_units + rows - 1) / rows, most = (vocab * elem_size(dtype) + 16383) / 16384;
    int64_t slices = want < most ? want : most;
    if (slices < 1) slices = 1;
    Cut cut;
    cut.length = ((vocab + slices - 1) / slices + 7) / 8 * 8;
    cut.slices = static_cast<int32_t>((vocab + cut.length - 1) / cut.length);
    return cut;
}

struct Work {
    int64_t terms, z_token, sums, bytes;
};
Work layout(int64_t rows, const Cut &cut)
{
    Work w;
    w.terms = 0;
    w.z_token = w.terms + static_cast<int64_t>(sizeof(RowTerms)) * rows;
    w.sums = (w.z_token + 4 * rows + 15) / 16 * 16;
    w.bytes = w.sums + static_cast<int64_t>(sizeof(TopSum)) * rows * cut.slices;
    return w;
}

template <int DT>
void launch_policy(const void *logits, int64_t rows, int64_t vocab, int64_t stride, const int32_t *tokens, const PolicyTerms &p, void *grad,
                   int64_t grad_stride, float *logp, float *stats, char *work, int compute_units, hipStream_t stream)
{
    const Cut cut = cut_of(rows, vocab, DT, compute_units);
    const Work w = layout(rows, cut);
    const RowPlace at{vocab, stride};
    const char *from = static_cast<const char *>(logits);
    char *to = static_cast<char *>(grad);
    const RowOut out{logp, stats, reinterpret_cast<RowTerms *>(work + w.terms)};
    const int64_t bytes = vocab * elem_size(DT);
    if (bytes <= kRowBytes) {
        auto go = [&](auto kernel, int threads) {
            const int each = rows_of_block(threads);
            kernel<<<static_cast<uint32_t>((rows + each - 1) / each), dim3(threads, each), 0, stream>>>(from, rows, at, tokens, p, to, grad_stride, out);
        };
        if (bytes <= kShortBytes && rows >= 16 * compute_units)
            short_rows_kernel<DT, true><<<static_cast<uint32_t>((rows + 4 * kShort - 1) / (4 * kShort)), 256, 0, stream>>>(from, rows, at, tokens, p, to,
                                                                                                                       grad_stride, out);
        else if (bytes <= 64 * 8 * 16) go(policy_row_kernel<DT, 64, 8>, 64);
        else if (bytes <= 128 * 8 * 16) go(policy_row_kernel<DT, 128, 8>, 128);
        else if (bytes <= 256 * 8 * 16) go(policy_row_kernel<DT, 256, 8>, 256);
        else if (bytes <= 512 * 8 * 16) go(policy_row_kernel<DT, 512, 8>, 512);
        else if (bytes <= 1024 * 8 * 16) go(policy_row_kernel<DT, 1024, 8>, 1024);
        else go(policy_row_kernel<DT, 1024, 16>, 1024);
        return;
    }
    TopSum *sums = reinterpret_cast<TopSum *>(work + w.sums);
    float *z = reinterpret_cast<float *>(work + w.z_token);
    const uint32_t blocks = static_cast<uint32_t>(rows * cut.slices);
    slice_sum_kernel<DT, kSliceThreads><<<blocks, kSliceThreads, 0, stream>>>(from, rows, at, cut, tokens, p.weight, sums, z, nullptr);
    policy_slice_kernel<DT, kSliceThreads><<<blocks, kSliceThreads, 0, stream>>>(from, at, cut, tokens, p, sums, z, to, grad_stride, out);
}

}  // namespace

int64_t policy_work_bytes(int64_t N, int64_t T, int64_t vocab, int dtype, int compute_units)
{
    return N * T == 0 ? 0 : layout(N * T, cut_of(N * T, vocab, dtype, compute_units)).bytes;
}

hipError_t launch_policy_loss(const void *logits, int dtype, int64_t N, int64_t T, int64_t vocab, int64_t stride, const int32_t *tokens,
                              const PolicyTerms &p, void *grad, int64_t grad_stride, float *logp, float *stats, void *work,
                              int compute_units, hipStream_t stream)
{
    char *at = static_cast<char *>(work);
    if (!launchable(N * T, 1024) && !launchable(N * T, (vocab * elem_size(dtype) + 127) / 128 + 63)) return hipErrorInvalidConfiguration;
    if (T > 0)
        (dtype == 0 ? launch_policy<0> : launch_policy<1>)(logits, N * T, vocab, stride, tokens, p, grad, grad_stride, logp, T == 1 ? stats : nullptr, at,
                                                           compute_units, stream);
    if (T != 1) policy_stats_kernel<<<static_cast<uint32_t>(N), T <= 256 ? 64 : T <= 1024 ? 256 : kStatsThreads, 0, stream>>>(reinterpret_cast<const RowTerms *>(at), T, stats);
    return hipGetLastError();
}

hipError_t launch_token_logp(const void *logits, int dtype, int64_t rows, int64_t vocab, int64_t stride, const int32_t *tokens, float *logp,
                             void *work, int compute_units, hipStream_t stream)
{
    if (rows == 0) return hipSuccess;
    if (!launchable(rows, kSliceThreads)) return hipErrorInvalidConfiguration;
    const Cut cut = cut_of(rows, vocab, dtype, compute_units);
    const Work w = layout(rows, cut);
    TopSum *sums = reinterpret_cast<TopSum *>(static_cast<char *>(work) + w.sums);
    float *z = cut.slices > 1 ? reinterpret_cast<float *>(static_cast<char *>(work) + w.z_token) : nullptr;
    if (vocab * elem_size(dtype) <= kShortBytes && rows >= 16 * compute_units) {
        (dtype == 0 ? short_rows_kernel<0, false> : short_rows_kernel<1, false>)<<<static_cast<uint32_t>((rows + 4 * kShort - 1) / (4 * kShort)), 256, 0, stream>>>(
            static_cast<const char *>(logits), rows, RowPlace{vocab, stride}, tokens, PolicyTerms{}, nullptr, 0, RowOut{logp, nullptr, nullptr});
        return hipGetLastError();
    }
    // rows of up to 8 KiB by a wave, four to a block
    const int threads = cut.slices == 1 && vocab * elem_size(dtype) <= 8192 ? 64 : kSliceThreads, each = rows_of_block(threads);
    auto kernel = threads == 64 ? (dtype == 0 ? slice_sum_kernel<0, 64> : slice_sum_kernel<1, 64>)
                                : (dtype == 0 ? slice_sum_kernel<0, kSliceThreads> : slice_sum_kernel<1, kSliceThreads>);
    kernel<<<static_cast<uint32_t>((rows * cut.slices + each - 1) / each), dim3(threads, each), 0, stream>>>(
        static_cast<const char *>(logits), rows, RowPlace{vocab, stride}, cut, tokens, nullptr, sums, z, logp);
    if (cut.slices > 1) logp_join_kernel<<<static_cast<uint32_t>(rows), 64, 0, stream>>>(sums, z, cut.slices, tokens, vocab, logp);
    return hipGetLastError();
}

}  // namespace moshpit
