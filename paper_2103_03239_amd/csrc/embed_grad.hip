// The gradient of the peers' embedding tables for gfx950:
//   grad_i[v][:] = scale * sum over t with tokens[i][t] == v of dy[i][t][:]      (binary32 sums, rounded once)
// for every row v of every table (rows without a token: zeros, or untouched where the gradient is added).
//
// Tokens first: each peer's places are sorted by token, stably (a radix sort, up to 8 bits a pass), so that the
// places of a row lie side by side in ascending order.  Meanwhile other blocks of the same launch clear the tables:
// most rows of a vocabulary have no token, and a plain fill writes them at 6.8 TB/s, while waves that each
// write the empty rows between their own reached 4.7 (64 tables of 30000 x 128 binary32).
// Then the sums.  The sorted places are cut into shares of kShare, one to a wave and column slice; a cut moves to the
// start of its row where the row has at most 63 places.  A row that is still cut leaves a partial sum per share, and
// a last kernel adds those in ascending order.  Which sums are formed and in which order follows from the
// sizes and tokens alone.
//
// Bound by HBM: dy is read once, the tables' gradient is written once (rows with tokens twice).  64 tables of 30000 x 128
// binary32 from 4096 places each in 207 us (1.03 GB written and read at least: 5.0 TB/s), 4 of 32000 x 1024 from 65536
// in 196 us.
#include <hip/hip_runtime.h>

#include "local_ops.h"
#include "row_elems.h"

namespace moshpit {
namespace {

// ---- places sorted by token --------------------------------------------------

constexpr int kBins = 256;

struct SortPlan {
    int32_t T, passes, bits;             // bits of a pass
    uint32_t vocab;
    uint32_t tiles;                      // of a peer; block b works on tile b % tiles of peer b / tiles
    uint32_t sort_blocks;                // blocks beyond these clear the tables
};

__device__ __forceinline__ uint32_t sort_key(const int32_t *__restrict__ tokens, int64_t at, uint32_t vocab)
{
    const uint32_t k = static_cast<uint32_t>(tokens[at]);
    return k < vocab ? k : vocab;                                // places without a token come last
}

// The lanes of a wave see each other's LDS accesses before this point from here on.
__device__ __forceinline__ void wave_order()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// The sums of v over the lanes up to each.
__device__ __forceinline__ uint32_t upto_lane(uint32_t v)
{
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);    // within rows of 16 lanes: 1, 2, 4 and 8 lanes down
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);    // the last lane of rows 0 and 2 to rows 1 and 3
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);    // lane 31 to rows 2 and 3
    return v;
}

// Where each of a block's items goes within the block when they are ordered by the `bits` (up to 8) bits of their key from
// `shift` on, stably.  Item i of lane l of wave w is number w * 64 * ITEMS + i * 64 + l of the block.
// count: LDS, (waves + 1) * kBins; afterwards count[waves * kBins + b] is where bin b begins in the block.
template <int THREADS, int ITEMS>
__device__ __forceinline__ void block_rank(const uint32_t (&key)[ITEMS], int shift, int bits, uint32_t *count, uint32_t (&rank)[ITEMS])
{
    constexpr int WAVES = THREADS / 64;
    const uint32_t bins = (1u << bits) - 1;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int b = threadIdx.x; b < WAVES * kBins; b += THREADS) count[b] = 0;
    __syncthreads();
    uint32_t *mine = count + wave * kBins;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const uint32_t digit = (key[i] >> shift) & bins;
        uint32_t low = ~0u, high = ~0u;                               // lanes whose digit is this one's
#pragma unroll
        for (int b = 0; b < 8; ++b) {                                 // (bits beyond `bits` are 0 in every lane)
            const uint64_t has = __ballot((digit >> b) & 1);
            const uint32_t mine_has = 0u - ((digit >> b) & 1);
            low &= ~(static_cast<uint32_t>(has) ^ mine_has);
            high &= ~(static_cast<uint32_t>(has >> 32) ^ mine_has);
        }
        const uint32_t below = __builtin_amdgcn_mbcnt_hi(high, __builtin_amdgcn_mbcnt_lo(low, 0));
        const uint32_t before = mine[digit];
        rank[i] = before + below;
        wave_order();                                            // every lane has read before one adds
        if (below == 0) mine[digit] = before + static_cast<uint32_t>(__popc(low) + __popc(high));
        wave_order();
    }
    __syncthreads();
    uint32_t *start = count + WAVES * kBins;
    for (int b = threadIdx.x; b < kBins; b += THREADS) {
        uint32_t sum = 0;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const uint32_t c = count[w * kBins + b];
            count[w * kBins + b] = sum;
            sum += c;
        }
        start[b] = sum;
    }
    __syncthreads();
    if (wave == 0) {                                             // exclusive sums over the 256 bins, 4 a lane
        uint32_t c[4], sum = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            c[k] = sum;
            sum += start[lane * 4 + k];
        }
        const uint32_t upto = upto_lane(sum);
#pragma unroll
        for (int k = 0; k < 4; ++k) start[lane * 4 + k] = upto - sum + c[k];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const uint32_t digit = (key[i] >> shift) & bins;
        rank[i] += mine[digit] + start[digit];
    }
}

// What the blocks beyond the sort's do: zeros to the tables, 16 bytes a thread (more of them write in a wider window of
// memory at a time: 983 MB in 160 us, with 4 or 16 vectors a thread in 165 to 168).
struct Fill {
    char *base;
    int64_t peer_bytes, table_bytes;     // from table to table; of a table
    uint32_t blocks;                     // of a table
    uint32_t first;                      // block of all tables that this launch begins with
};

template <int THREADS> __device__ __forceinline__ void fill_zeros(const Fill &f, uint32_t block)
{
    block += f.first;
    const int64_t begin = int64_t(block % f.blocks) * (16 * THREADS);
    char *table = f.base + int64_t(block / f.blocks) * f.peer_bytes;
    // whole vectors at 16-byte boundaries; the few bytes at the table's ends by elements
    const uint32_t phase = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(table)) % 16;
    const int64_t head = phase ? 16 - phase : 0;
    const int64_t at = begin + head + int64_t(threadIdx.x) * 16;
    if (at + 16 <= f.table_bytes) store_vec<true, u32x4>(table + at, u32x4{0, 0, 0, 0});
    else
        for (int64_t e = at; e < f.table_bytes; e += 2) *reinterpret_cast<uint16_t *>(table + e) = 0;
    if (begin == 0 && threadIdx.x < head / 2 && threadIdx.x * 2 < f.table_bytes) *reinterpret_cast<uint16_t *>(table + 2 * threadIdx.x) = 0;
}

// All passes of a peer's sort by one block, T <= THREADS * ITEMS.
template <int THREADS, int ITEMS>
__global__ __launch_bounds__(THREADS) void sort_block_kernel(const int32_t *__restrict__ tokens, SortPlan p, uint32_t *__restrict__ keys,
                                                             int32_t *__restrict__ places, Fill fill)
{
    if (blockIdx.x >= p.sort_blocks) return fill_zeros<THREADS>(fill, blockIdx.x - p.sort_blocks);
    __shared__ uint32_t count[(THREADS / 64 + 1) * kBins];
    __shared__ uint32_t swap_key[THREADS * ITEMS];
    __shared__ uint16_t swap_place[THREADS * ITEMS];
    const int64_t row = int64_t(blockIdx.x) * p.T;
    const int base = (threadIdx.x >> 6) * 64 * ITEMS + (threadIdx.x & 63);
    uint32_t key[ITEMS], rank[ITEMS];
    uint16_t place[ITEMS];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const int at = base + i * 64;
        key[i] = at < p.T ? sort_key(tokens, row + at, p.vocab) : 0xffffffffu;      // (last in every pass, behind the row's own)
        place[i] = static_cast<uint16_t>(at);
    }
    for (int pass = 0; pass < p.passes; ++pass) {
        block_rank<THREADS, ITEMS>(key, p.bits * pass, p.bits, count, rank);
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            swap_key[rank[i]] = key[i];
            swap_place[rank[i]] = place[i];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            key[i] = swap_key[base + i * 64];
            place[i] = swap_place[base + i * 64];
        }
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const int at = base + i * 64;
        if (at >= p.T) continue;
        keys[row + at] = key[i];
        places[row + at] = place[i];
    }
}

// Longer rows: tiles of kTile places, for each pass the bins' sizes per tile, where each (bin, tile) begins,
// then every item to its place.
constexpr int kTileThreads = 256, kTileItems = 16, kTile = kTileThreads * kTileItems;

__device__ __forceinline__ uint32_t pass_key(const int32_t *__restrict__ tokens, const uint32_t *__restrict__ keys, int64_t at, uint32_t vocab)
{
    return keys ? keys[at] : sort_key(tokens, at, vocab);
}

__global__ __launch_bounds__(kTileThreads) void sort_count_kernel(const int32_t *__restrict__ tokens, const uint32_t *__restrict__ keys,
                                                                   SortPlan p, int shift, uint32_t *__restrict__ bins, Fill fill)
{
    if (blockIdx.x >= p.sort_blocks) return fill_zeros<kTileThreads>(fill, blockIdx.x - p.sort_blocks);
    __shared__ uint32_t count[kBins];
    const uint32_t peer = blockIdx.x / p.tiles, tile = blockIdx.x % p.tiles;
    const int64_t row = int64_t(peer) * p.T;
    for (int b = threadIdx.x; b < kBins; b += kTileThreads) count[b] = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kTileItems; ++i) {
        const int64_t at = int64_t(tile) * kTile + i * kTileThreads + threadIdx.x;
        if (at < p.T) atomicAdd(&count[(pass_key(tokens, keys, row + at, p.vocab) >> shift) & ((1u << p.bits) - 1)], 1u);
    }
    __syncthreads();
    uint32_t *mine = bins + int64_t(peer) * kBins * p.tiles;
    for (int b = threadIdx.x; b < kBins; b += kTileThreads) mine[int64_t(b) * p.tiles + tile] = count[b];
}

// Exclusive sums of a peer's kBins * tiles counts, in place, by one block.
__global__ __launch_bounds__(1024) void sort_scan_kernel(uint32_t *__restrict__ bins, int64_t count)
{
    __shared__ uint32_t wave_sum[16];
    uint32_t *mine = bins + int64_t(blockIdx.x) * count;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t before = 0;
    for (int64_t k0 = 0; k0 < count; k0 += 4096) {
        const int64_t k = k0 + 4 * threadIdx.x;
        uint32_t v[4], sum = 0;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const uint32_t c = k + u < count ? mine[k + u] : 0;
            v[u] = sum;
            sum += c;
        }
        const uint32_t upto = upto_lane(sum);
        if (lane == 63) wave_sum[wave] = upto;
        __syncthreads();
        uint32_t waves_before = 0, all = 0;
#pragma unroll
        for (int w = 0; w < 16; ++w) {
            if (w < wave) waves_before += wave_sum[w];
            all += wave_sum[w];
        }
        const uint32_t first = before + waves_before + upto - sum;
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (k + u < count) mine[k + u] = first + v[u];
        before += all;
        __syncthreads();
    }
}

__global__ __launch_bounds__(kTileThreads) void sort_move_kernel(const int32_t *__restrict__ tokens, const uint32_t *__restrict__ keys,
                                                                  const int32_t *__restrict__ places, SortPlan p, int shift,
                                                                  const uint32_t *__restrict__ bins, uint32_t *__restrict__ keys_out,
                                                                  int32_t *__restrict__ places_out, Fill fill)
{
    if (blockIdx.x >= p.sort_blocks) return fill_zeros<kTileThreads>(fill, blockIdx.x - p.sort_blocks);
    __shared__ uint32_t count[(kTileThreads / 64 + 1) * kBins];
    __shared__ uint32_t goes_to[kBins];
    const uint32_t peer = blockIdx.x / p.tiles, tile = blockIdx.x % p.tiles;
    const int64_t row = int64_t(peer) * p.T;
    const int64_t base = int64_t(tile) * kTile + (threadIdx.x >> 6) * 64 * kTileItems + (threadIdx.x & 63);
    const uint32_t *mine = bins + int64_t(peer) * kBins * p.tiles;
    uint32_t key[kTileItems], rank[kTileItems];
#pragma unroll
    for (int i = 0; i < kTileItems; ++i) {
        const int64_t at = base + i * 64;
        key[i] = at < p.T ? pass_key(tokens, keys, row + at, p.vocab) : 0xffffffffu;
    }
    block_rank<kTileThreads, kTileItems>(key, shift, p.bits, count, rank);
    for (int b = threadIdx.x; b < kBins; b += kTileThreads)
        goes_to[b] = mine[int64_t(b) * p.tiles + tile] - count[(kTileThreads / 64) * kBins + b];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kTileItems; ++i) {
        const int64_t at = base + i * 64;
        if (at >= p.T) continue;
        const int64_t to = row + (goes_to[(key[i] >> shift) & ((1u << p.bits) - 1)] + rank[i]);
        keys_out[to] = key[i];
        places_out[to] = keys ? places[row + at] : static_cast<int32_t>(at);
    }
}

// ---- sums --------------------------------------------------------------------

constexpr int kSnap = 63;                // a row of at most this many places is not cut
constexpr int kShare = 32;               // places of a share
constexpr int kWave = 64, kBlock = 256, kWaves = kBlock / kWave, kBatch = 8, kJoinShares = 16;

// The cut before a share: its first place (in the window of the wave that made it); inside (bit 31): the row of that place has places before it too.
struct Cut {
    uint32_t row, place_inside;
    __device__ __forceinline__ uint32_t place() const { return place_inside & 0x7fffffffu; }
    __device__ __forceinline__ bool inside() const { return place_inside >> 31; }
};

struct ShareGeom {
    int64_t shares;                      // of a peer; it has shares + 1 cuts
    uint32_t slices;                     // column slices of a share
    uint32_t blocks;                     // of a peer, in the kernel at hand
};

// VE elements of a row as they lie in memory, so that loads in flight take few registers.
template <int DT, int VE> struct Raw {
    static constexpr int WORDS = DT == 0 ? VE : (VE + 1) / 2;
    uint32_t w[WORDS];
    __device__ __forceinline__ void load(const char *p)
    {
        if constexpr (DT == 1 && VE == 1) w[0] = *reinterpret_cast<const uint16_t *>(p);
        else if constexpr (WORDS == 1) w[0] = load_vec<true, uint32_t>(p);
        else if constexpr (WORDS == 2) put(load_vec<true, u32x2>(p));
        else put(load_vec<true, u32x4>(p));
        if constexpr (WORDS == 8) {
            const u32x4 v = load_vec<true, u32x4>(p + 16);
#pragma unroll
            for (int k = 0; k < 4; ++k) w[4 + k] = v[k];
        }
    }
    template <typename V> __device__ __forceinline__ void put(const V &v)
    {
#pragma unroll
        for (int k = 0; k < static_cast<int>(sizeof(V) / 4); ++k) w[k] = v[k];
    }
    __device__ __forceinline__ float operator[](int k) const
    {
        if constexpr (DT == 0) return __uint_as_float(w[k]);
        else return __uint_as_float(k & 1 ? w[k / 2] & 0xffff0000u : w[k / 2] << 16);
    }
};
template <int DT, int VE> __device__ __forceinline__ void load_run(const char *p, float (&f)[VE])
{
    Raw<DT, VE> raw;
    raw.load(p);
#pragma unroll
    for (int k = 0; k < VE; ++k) f[k] = raw[k];
}
template <int DT, int VE> __device__ __forceinline__ void store_run(char *p, const float (&f)[VE])
{
    if constexpr (VE >= 4) store_elems<DT, VE, true>(p, f);
    else if constexpr (VE == 2 && DT == 0) store_vec<true, u32x2>(p, u32x2{__float_as_uint(f[0]), __float_as_uint(f[1])});
    else if constexpr (VE == 2) store_vec<false, uint32_t>(p, bf16_pair(f[0], f[1]));
    else store_one<DT>(p, f[0]);
}

// The columns of a table that a wave works on: lane l has VE of them, those of the last lane that has any ending with
// the row (it repeats columns of the lane before).
template <int ST, int YT, int VE, bool ADD> struct Columns {
    static constexpr int ES = ST == 0 ? 4 : 2, EY = YT == 0 ? 4 : 2;
    int32_t width, c, at_c;              // this lane's columns c .. c + VE - 1, read from at_c on
    bool any, whole;                     // it has columns; VE of them
    __device__ __forceinline__ Columns(int64_t w, uint32_t slice)
    {
        width = static_cast<int32_t>(w);
        c = static_cast<int32_t>((slice * kWave + (threadIdx.x & 63)) * VE);
        any = c < width;
        whole = c + VE <= width;
        at_c = whole ? c : width - VE;                                // (width >= VE; a lane without columns reads the last ones, too)
    }
    __device__ __forceinline__ void load(const char *row, Raw<YT, VE> &r) const { r.load(row + at_c * EY); }
    __device__ __forceinline__ void store(char *row, const float (&f)[VE]) const
    {
        if (!any) return;
        if (whole) {
            float v[VE];
            if constexpr (ADD) {
                load_run<ST, VE>(row + c * ES, v);
#pragma unroll
                for (int k = 0; k < VE; ++k) v[k] += f[k];
                store_run<ST, VE>(row + c * ES, v);
            } else store_run<ST, VE>(row + c * ES, f);
        } else {
#pragma unroll
            for (int k = 0; k < VE; ++k) {
                const int32_t e = at_c + k;
                if (e >= c && e < width) store_one<ST>(row + e * ES, ADD ? load_one<ST>(row + e * ES) + f[k] : f[k]);
            }
        }
    }
    __device__ __forceinline__ void store_partial(float *to, const float (&f)[VE]) const
    {
        if (!any) return;
#pragma unroll
        for (int k = 0; k < VE; ++k) {
            const int32_t e = at_c + k;
            if (e >= c && e < width) to[e] = f[k];
        }
    }
};

// A share a wave and column slice.  Rows, places and all branches are the same for the whole wave.
template <int ST, int YT, int VE, bool ADD>
__global__ __launch_bounds__(kBlock) void embed_grad_kernel(const uint32_t *__restrict__ keys, const int32_t *__restrict__ places,
                                                            const char *__restrict__ dy, int64_t dy_stride, char *__restrict__ base, TableGeom g,
                                                            ShareGeom s, float scale, Cut *__restrict__ cuts, float *__restrict__ partials)
{
    constexpr int ES = ST == 0 ? 4 : 2, EY = YT == 0 ? 4 : 2;
    const uint32_t peer = blockIdx.x / s.blocks;
    const uint32_t part = blockIdx.x % s.blocks * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t share = part / s.slices, slice = part % s.slices;  // the slices of a share side by side: whole rows are read and written at a time
    if (share >= s.shares) return;
    const int lane = threadIdx.x & 63;
    const uint32_t vocab = static_cast<uint32_t>(g.vocab);
    const uint32_t *key = keys + peer * g.T;
    // the sorted places from 64 before the share to 128 after its start, a place a lane: all that the cuts and the
    // sums look at, requested at once
    const int64_t first = int64_t(share) * kShare;
    uint32_t k_of[3];
    int32_t p_of[2];
#pragma unroll
    for (int q = 0; q < 3; ++q) {
        const int64_t at = first + (q - 1) * kWave + lane;
        const bool there = at >= 0 && at < g.T;
        k_of[q] = there ? key[at] : vocab;
        if (q < 2) p_of[q] = there ? places[peer * g.T + at] : 0;
    }
    // A cut lies before place kShare * share; where the row there has at most kSnap places on both sides it moves to the row's
    // first.  `at`: place of the cut in the window.
    auto cut_at = [&](int at, uint32_t row) {
        const uint64_t same[3] = {__ballot(k_of[0] == row), __ballot(k_of[1] == row), __ballot(k_of[2] == row)};
        // places of the row among the 64 before the cut and the 64 from it on
        const int shift = at - kWave;                                 // 0 or kShare
        const uint64_t before = shift == 0 ? same[0] : same[0] >> shift | same[1] << (kWave - shift);
        const uint64_t after = shift == 0 ? same[1] : same[1] >> shift | same[2] << (kWave - shift);
        const int b = __popcll(before), a = __popcll(after);
        if (row >= vocab || a == 0 || b == 0) return Cut{row, static_cast<uint32_t>(at)};
        if (a + b <= kSnap) return Cut{row, static_cast<uint32_t>(at - b)};
        return Cut{row, static_cast<uint32_t>(at) | 0x80000000u};
    };
    const uint32_t row0 = __builtin_amdgcn_readfirstlane(k_of[1]);
    const Cut from = cut_at(kWave, row0), to = cut_at(kWave + kShare, __builtin_amdgcn_readlane(k_of[1], kShare));
    if (slice == 0 && lane == 0) {
        Cut *mine = cuts + peer * (s.shares + 1) + share;
        mine[0] = from;
        if (share + 1 == s.shares) mine[1] = Cut{vocab, 0};
    }
    const Columns<ST, YT, VE, ADD> columns(g.width, slice);
    char *table = base + peer * g.peer_stride * ES;
    const char *rows = dy + peer * g.T * dy_stride * EY;
    float *slot = partials + (peer * s.shares + share) * 2 * g.width;

    // its places lie at begin .. end - 1 of the window; those without a token come last and do not count
    const uint32_t begin = from.place();
    const uint32_t tokens_end = __popcll(__ballot(k_of[1] < vocab)) + kWave;
    const uint32_t end = to.place() < tokens_end ? to.place() : tokens_end;
    if (begin >= end) return;
    auto key_at = [&](uint32_t at) -> uint32_t {
        return at < kWave ? __builtin_amdgcn_readlane(k_of[0], at) : __builtin_amdgcn_readlane(k_of[1], at - kWave);
    };
    auto request = [&](uint32_t at, Raw<YT, VE> (&v)[kBatch]) {       // the rows of up to kBatch places; beyond the last one that one again
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            const uint32_t e = at + u < end ? at + u : end - 1;
            const int32_t p = e < kWave ? __builtin_amdgcn_readlane(p_of[0], e) : __builtin_amdgcn_readlane(p_of[1], e - kWave);
            columns.load(rows + int64_t(p) * dy_stride * EY, v[u]);
        }
    };

    float acc[VE] = {};
    uint32_t row = from.row;
    bool head = from.inside();                                        // the row began in a share before
    auto finish = [&]() {                                             // all places of `row` are in
        if (head) columns.store_partial(slot, acc);
        else {
#pragma unroll
            for (int k = 0; k < VE; ++k) acc[k] *= scale;
            columns.store(table + int64_t(row) * g.width * ES, acc);
        }
        head = false;
#pragma unroll
        for (int k = 0; k < VE; ++k) acc[k] = 0.f;
    };
    auto add = [&](uint32_t at, const Raw<YT, VE> (&v)[kBatch]) {
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            if (at + u >= end) break;
            const uint32_t k = key_at(at + u);
            if (row != k) {
                finish();
                row = k;
            }
#pragma unroll
            for (int e = 0; e < VE; ++e) acc[e] += v[u][e];
        }
    };
    // the rows of the next places are requested before those of these are added
    Raw<YT, VE> even[kBatch], odd[kBatch];
    request(begin, even);
    for (uint32_t at = begin; at < end; at += 2 * kBatch) {
        if (at + kBatch < end) request(at + kBatch, odd);
        add(at, even);
        if (at + kBatch >= end) break;
        if (at + 2 * kBatch < end) request(at + 2 * kBatch, even);
        add(at + kBatch, odd);
    }
    if (!to.inside()) finish();
    else columns.store_partial(head ? slot : slot + g.width, acc);         // the row goes on in the next share
}

// Few places and small tables in one launch, without a sort: a wave has a few rows of a table and a column slice, looks at all
// tokens of the peer, up to four a lane, and takes those of each of its rows in ascending order of their places.
constexpr int kScanPlaces = 256;

template <int ST, int YT, int VE, bool ADD>
__global__ __launch_bounds__(kBlock) void embed_grad_scan_kernel(const int32_t *__restrict__ tokens, const char *__restrict__ dy, int64_t dy_stride,
                                                                 char *__restrict__ base, TableGeom g, ShareGeom s, uint32_t run_rows,
                                                                 float scale)
{
    constexpr int ES = ST == 0 ? 4 : 2, EY = YT == 0 ? 4 : 2, CHUNKS = kScanPlaces / kWave;
    const uint32_t peer = blockIdx.x / s.blocks;
    const uint32_t part = blockIdx.x % s.blocks * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t run = part / s.slices, slice = part % s.slices;
    const uint32_t vocab = static_cast<uint32_t>(g.vocab), row0 = run * run_rows;
    if (row0 >= vocab) return;
    const uint32_t rows = vocab - row0 < run_rows ? vocab - row0 : run_rows;
    const int lane = threadIdx.x & 63;
    uint32_t mine[CHUNKS];                                            // a token's row of this wave's, or any number from `rows` on
    uint64_t any = 0;
#pragma unroll
    for (int q = 0; q < CHUNKS; ++q) {
        const int64_t at = q * kWave + lane;
        mine[q] = at < g.T ? static_cast<uint32_t>(tokens[peer * g.T + at]) - row0 : rows;
        any |= __ballot(mine[q] < rows);
    }
    const Columns<ST, YT, VE, ADD> columns(g.width, slice);
    char *table = base + (peer * g.peer_stride + int64_t(row0) * g.width) * ES;
    const char *from = dy + peer * g.T * dy_stride * EY;
    if (any == 0 && ADD) return;
    for (uint32_t r = 0; r < rows; ++r) {
        float acc[VE] = {};
        bool some = false;
        if (any != 0) {
#pragma unroll
            for (int q = 0; q < CHUNKS; ++q) {
                uint64_t places = __ballot(mine[q] == r);
                some |= places != 0;
                while (places != 0) {
                    Raw<YT, VE> v[kBatch];
                    uint64_t rest = places;
#pragma unroll
                    for (int u = 0; u < kBatch; ++u) {                // the lowest kBatch of them; where there are fewer, the last one again
                        columns.load(from + int64_t(q * kWave + __builtin_ctzll(rest)) * dy_stride * EY, v[u]);
                        if ((rest & (rest - 1)) != 0) rest &= rest - 1;
                    }
#pragma unroll
                    for (int u = 0; u < kBatch; ++u) {
                        if (places == 0) break;
#pragma unroll
                        for (int e = 0; e < VE; ++e) acc[e] += v[u][e];
                        places &= places - 1;
                    }
                }
            }
        }
        if (!some && ADD) continue;
#pragma unroll
        for (int e = 0; e < VE; ++e) acc[e] *= scale;
        columns.store(table + int64_t(r) * g.width * ES, acc);
    }
}

// Rows cut by shares: the share in which such a row ends adds its partial sums, in the order of the shares.
template <int ST, bool ADD>
__global__ __launch_bounds__(kBlock) void embed_grad_join_kernel(char *__restrict__ base, TableGeom g, ShareGeom s, float scale,
                                                                 const Cut *__restrict__ cuts, const float *__restrict__ partials)
{
    constexpr int ES = ST == 0 ? 4 : 2;
    __shared__ float wave_sum[kWaves][kWave];
    const uint32_t peer = blockIdx.x / s.blocks;
    const Cut *cut = cuts + peer * (s.shares + 1);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t share0 = int64_t(blockIdx.x % s.blocks) * kJoinShares;
    bool ends = false;                                                // a row that began before this lane's share ends in it
    if (lane < kJoinShares && share0 + lane < s.shares) {
        const Cut in = cut[share0 + lane];
        const Cut out = cut[share0 + lane + 1];
        ends = in.inside() && !(out.inside() && out.row == in.row);
    }
    uint64_t ending = __ballot(ends);                                 // the same in every wave
    for (; ending; ending &= ending - 1) {
        const int64_t last = share0 + __builtin_ctzll(ending);
        const uint32_t row = cut[last].row;
        int64_t first = last - 1;                                         // the share in which the row begins
        while (true) {
            const int64_t at = first - lane;
            const bool middle = at >= 0 && cut[at].inside() && cut[at].row == row;
            const uint64_t stop = ~__ballot(middle);
            if (stop) {
                first -= __builtin_ctzll(stop);
                break;
            }
            first -= 64;
        }
        const float *mine = partials + peer * s.shares * 2 * g.width;
        const int64_t count = last - first + 1, each = (count + kWaves - 1) / kWaves;
        for (int64_t c0 = int64_t(blockIdx.y) * kWave; c0 < g.width; c0 += int64_t(gridDim.y) * kWave) {
            const int64_t c = c0 + lane;
            float acc = 0.f;
            if (c < g.width) {
                const int64_t q_end = (wave + 1) * each < count ? (wave + 1) * each : count;
                for (int64_t q = wave * each; q < q_end; q += 8) {    // eight partial sums requested at a time
                    float v[8];
#pragma unroll
                    for (int u = 0; u < 8; ++u)
                        v[u] = q + u < q_end ? mine[((first + q + u) * 2 + (q + u == 0 ? 1 : 0)) * g.width + c] : 0.f;
                    acc += ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
                }
            }
            wave_sum[wave][lane] = acc;
            __syncthreads();
            if (wave == 0 && c < g.width) {
                float sum = 0.f;
#pragma unroll
                for (int w = 0; w < kWaves; ++w) sum += wave_sum[w][lane];
                char *to = base + (peer * g.peer_stride + int64_t(row) * g.width + c) * ES;
                const float f = scale * sum;
                store_one<ST>(to, ADD ? load_one<ST>(to) + f : f);
            }
            __syncthreads();
        }
    }
}

// ---- launches ----------------------------------------------------------------

constexpr int64_t kOneBlock = 8192;      // places that one block sorts

int64_t padded(int64_t bytes) { return (bytes + 255) / 256 * 256; }

// Elements of a lane: as few as let a wave have all columns, at most 16 bytes of the table.
int lane_elems(const TableGeom &g, int state_dtype)
{
    int ve = 1;
    while (ve < (state_dtype == 0 ? 4 : 8) && kWave * ve < g.width) ve *= 2;
    return ve;
}

ShareGeom shares_of(const TableGeom &g) { return ShareGeom{(g.T + kShare - 1) / kShare, 1, 0}; }

struct Work {
    int64_t keys[2], places[2], bins, cuts, partials, bytes;
};

Work layout(const TableGeom &g)
{
    Work w{};
    int64_t at = 0;
    auto take = [&](int64_t bytes) {
        const int64_t here = at;
        at += padded(bytes);
        return here;
    };
    const int64_t list = 4 * g.N * g.T;
    const bool tiled = g.T > kOneBlock;
    for (int k = 0; k < (tiled ? 2 : 1); ++k) {
        w.keys[k] = take(list);
        w.places[k] = take(list);
    }
    if (tiled) w.bins = take(4 * g.N * kBins * ((g.T + kTile - 1) / kTile));
    const ShareGeom s = shares_of(g);
    w.cuts = take(static_cast<int64_t>(sizeof(Cut)) * g.N * (s.shares + 1));
    w.partials = take(g.T > kSnap ? 4 * g.N * s.shares * 2 * g.width : 0);
    w.bytes = at;
    return w;
}

template <int ST, int YT, int VE, bool ADD>
void launch_sums(void *base, const TableGeom &g, float scale, const void *dy, int64_t dy_stride, const uint32_t *keys, const int32_t *places,
                 Cut *cuts, float *partials, hipStream_t stream)
{
    if (g.T == 0) return;
    ShareGeom s = shares_of(g);
    s.slices = static_cast<uint32_t>((g.width + kWave * VE - 1) / (kWave * VE));
    s.blocks = static_cast<uint32_t>((s.shares * s.slices + kWaves - 1) / kWaves);
    embed_grad_kernel<ST, YT, VE, ADD><<<static_cast<uint32_t>(s.blocks * g.N), kBlock, 0, stream>>>(keys, places, static_cast<const char *>(dy), dy_stride, static_cast<char *>(base), g, s,
                                                                    scale, cuts, partials);
    if (g.T <= kSnap) return;                                         // no row is cut
    const int64_t column_blocks = (g.width + kWave - 1) / kWave;
    s.blocks = static_cast<uint32_t>((s.shares + kJoinShares - 1) / kJoinShares);
    const dim3 joins(static_cast<uint32_t>(s.blocks * g.N), static_cast<uint32_t>(column_blocks < 16 ? column_blocks : 16));
    embed_grad_join_kernel<ST, ADD><<<joins, kBlock, 0, stream>>>(static_cast<char *>(base), g, s, scale, cuts, partials);
}

// Without a sort: few places, and tables that are written in about the time of a launch.
bool scan_does(const TableGeom &g) { return g.T > 0 && g.T <= kScanPlaces && g.N * g.vocab * g.width <= (int64_t(1) << 23); }

template <int ST, int YT, int VE, bool ADD>
void launch_scan(void *base, const TableGeom &g, const int32_t *tokens, float scale, const void *dy, int64_t dy_stride, hipStream_t stream)
{
    // as few rows a wave (2 .. 16) as keep the waves at 16384: rows with places wait for their loads one after the other (27 tables of
    // 1001 x 100: 2 rows 8.2 us, 16 rows 9.6), and a wave's start costs as much as some rows (64 of 3785 x 24: 25.6 and 10.8)
    const int64_t slices = (g.width + kWave * VE - 1) / (kWave * VE);
    uint32_t rows = 2;
    while (rows < 16 && g.N * g.vocab * slices / rows > 16384) rows *= 2;
    ShareGeom s{(g.vocab + rows - 1) / rows, static_cast<uint32_t>(slices), 0};
    s.blocks = static_cast<uint32_t>((s.shares * s.slices + kWaves - 1) / kWaves);
    embed_grad_scan_kernel<ST, YT, VE, ADD><<<static_cast<uint32_t>(s.blocks * g.N), kBlock, 0, stream>>>(
        tokens, static_cast<const char *>(dy), dy_stride, static_cast<char *>(base), g, s, rows, scale);
}

template <int ST, int YT, bool ADD>
void launch(void *base, const TableGeom &g, const int32_t *tokens, float scale, const void *dy, int64_t dy_stride, const uint32_t *keys,
            const int32_t *places, Cut *cuts, float *partials, hipStream_t stream)
{
    if (scan_does(g)) {
        auto scan = [&](auto f) { f(base, g, tokens, scale, dy, dy_stride, stream); };
        switch (lane_elems(g, ST)) {
        case 1: return scan(launch_scan<ST, YT, 1, ADD>);
        case 2: return scan(launch_scan<ST, YT, 2, ADD>);
        case 4: return scan(launch_scan<ST, YT, 4, ADD>);
        default: return scan(launch_scan<ST, YT, ST == 0 ? 4 : 8, ADD>);
        }
    }
    auto go = [&](auto f) { f(base, g, scale, dy, dy_stride, keys, places, cuts, partials, stream); };
    switch (lane_elems(g, ST)) {
    case 1: return go(launch_sums<ST, YT, 1, ADD>);
    case 2: return go(launch_sums<ST, YT, 2, ADD>);
    case 4: return go(launch_sums<ST, YT, 4, ADD>);
    default: return go(launch_sums<ST, YT, ST == 0 ? 4 : 8, ADD>);
    }
}

}  // namespace

bool embed_grad_fits(const TableGeom &g)
{
    // blocks of the sums' kernel (4 shares and slices of 64 columns or more each), threads of the sort and the clearing
    const int64_t sums = shares_of(g).shares * ((g.width + kWave - 1) / kWave) / 4 + 1, clear = g.vocab * g.width / 4 + g.T + 1024;
    return sums <= 0xffffffffLL / kBlock / g.N && clear <= 0xffffffffLL / g.N;
}

int64_t embed_grad_work_bytes(const TableGeom &g) { return layout(g).bytes; }

hipError_t launch_embed_grad(void *base, int state_dtype, const TableGeom &g, const int32_t *tokens, float scale, const void *dy,
                             int dy_dtype, int64_t dy_stride, bool accumulate, void *work, hipStream_t stream)
{
    const Work w = layout(g);
    char *at = static_cast<char *>(work);
    uint32_t *keys[2] = {reinterpret_cast<uint32_t *>(at + w.keys[0]), reinterpret_cast<uint32_t *>(at + w.keys[1])};
    int32_t *places[2] = {reinterpret_cast<int32_t *>(at + w.places[0]), reinterpret_cast<int32_t *>(at + w.places[1])};
    const uint32_t N = static_cast<uint32_t>(g.N);
    SortPlan p{static_cast<int32_t>(g.T), 0, 0, static_cast<uint32_t>(g.vocab), 0, g.T > 0 ? N : 0};
    int key_bits = 0;
    while ((uint64_t(g.vocab) >> key_bits) != 0) ++key_bits;          // keys 0 .. vocab
    p.passes = (key_bits + 7) / 8;
    p.bits = (key_bits + p.passes - 1) / p.passes;
    const int32_t es = state_dtype == 0 ? 4 : 2;
    Fill fill{static_cast<char *>(base), g.peer_stride * es, g.vocab * g.width * es, 0, 0};
    // Threads of the sort's blocks, and so of those that clear.  From 257 to 1024 places 256 (16 tables of 30000 x 128 from 1000: 50.6 us,
    // with 1024 threads 55.3).  Up to 256 places 64 sort as well and leave room for more blocks, but clear slower: 4096 tables of 200 x 16
    // from 50 added to in 41.5 us (with 256 threads 45.3), cleared and written in 37.0 (37.1), 1024 of 200 x 64 from 64 in 25.4 (22.2),
    // 256 of 600 x 64 from 200 in 22.6 (19.3), 16 of 30000 x 128 from 200 in 64 (48).
    const int threads = g.T > kOneBlock ? kTileThreads : g.T > 1024 ? 1024 : g.T > 256 || (!accumulate && fill.table_bytes > (32 << 10)) ? 256 : 64;
    fill.blocks = accumulate ? 0 : static_cast<uint32_t>((fill.table_bytes + 16 * threads - 1) / (16 * threads));
    const uint32_t fill_blocks = fill.blocks * N;
    int sorted = 0;
    if (scan_does(g)) {
    } else if (g.T > kOneBlock) {
        p.tiles = static_cast<uint32_t>((g.T + kTile - 1) / kTile);
        p.sort_blocks = p.tiles * N;
        uint32_t *bins = reinterpret_cast<uint32_t *>(at + w.bins);
        const uint32_t launches = 2 * p.passes, each = (fill_blocks + launches - 1) / launches;
        auto some = [&]() {                                           // how much of the clearing goes with the next launch
            return fill_blocks - fill.first < each ? fill_blocks - fill.first : each;
        };
        for (int pass = 0; pass < p.passes; ++pass) {
            const uint32_t *from = pass ? keys[1 - sorted] : nullptr;
            const int32_t *from_places = pass ? places[1 - sorted] : nullptr;
            sort_count_kernel<<<p.sort_blocks + some(), kTileThreads, 0, stream>>>(tokens, from, p, p.bits * pass, bins, fill);
            fill.first += some();
            sort_scan_kernel<<<N, 1024, 0, stream>>>(bins, int64_t(kBins) * p.tiles);
            sort_move_kernel<<<p.sort_blocks + some(), kTileThreads, 0, stream>>>(tokens, from, from_places, p, p.bits * pass, bins, keys[sorted],
                                                                                  places[sorted], fill);
            fill.first += some();
            sorted = 1 - sorted;
        }
        sorted = 1 - sorted;
    } else if (p.sort_blocks + fill_blocks > 0) {
        auto go = [&](auto kernel) { kernel<<<p.sort_blocks + fill_blocks, threads, 0, stream>>>(tokens, p, keys[0], places[0], fill); };
        if (g.T > 4096) go(sort_block_kernel<1024, 8>);
        else if (g.T > 2048) go(sort_block_kernel<1024, 4>);
        else if (threads == 1024) go(sort_block_kernel<1024, 2>);
        else if (threads == 256) go(sort_block_kernel<256, 4>);
        else go(sort_block_kernel<64, 4>);
    }
    Cut *cuts = reinterpret_cast<Cut *>(at + w.cuts);
    float *partials = reinterpret_cast<float *>(at + w.partials);
    auto go = [&](auto add) {
        constexpr bool ADD = decltype(add)::value;
        auto f = state_dtype == 0 ? (dy_dtype == 0 ? launch<0, 0, ADD> : launch<0, 1, ADD>) : (dy_dtype == 0 ? launch<1, 0, ADD> : launch<1, 1, ADD>);
        f(base, g, tokens, scale, dy, dy_stride, keys[sorted], places[sorted], cuts, partials, stream);
    };
    if (accumulate) go(std::true_type{});
    else go(std::false_type{});
    return hipGetLastError();
}

}  // namespace moshpit
