// The gradient of the peers' embedding tables for gfx950:
//   grad_i[v][:] = scale * sum over t with tokens[i][t] == v of dy[i][t][:]      (binary32 sums, rounded once)
// for every row v of every table (rows without a token: zeros, or untouched where the gradient is added).
//
// Tokens first: each peer's places are sorted by token, stably (a radix sort, 8 bits a pass), so that the
// places of a row lie side by side in ascending order.  Then the sums, in one pass over dy and the tables.
// The sorted places and the ends of the table's rows are merged into one list of T + vocab items
// (a row's end comes after its places) and cut into shares of `share` items, one to a group of lanes: a
// frequent token is as many shares as its places take, a stretch of rows without tokens is shares of zeros,
// and every share moves about as many bytes.  A cut moves to the start of its row where the row has at
// most 63 places.  A row that is still cut leaves a partial sum per share, and a last kernel adds those in
// ascending order.  Which sums are formed and in which order follows from the sizes and tokens alone.
//
// Bound by HBM: dy is read once, the tables' gradient is written once.
#include <hip/hip_runtime.h>

#include "local_ops.h"
#include "row_elems.h"

namespace moshpit {
namespace {

// ---- places sorted by token --------------------------------------------------

constexpr int kBins = 256;

struct SortPlan {
    int32_t T, passes;
    uint32_t vocab;
    uint32_t tiles;                      // of a peer; block b works on tile b % tiles of peer b / tiles
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

// Where each of a block's items goes within the block when they are ordered by the 8 bits of their key from
// `shift` on, stably.  Item i of lane l of wave w is number w * 64 * ITEMS + i * 64 + l of the block.
// count: LDS, (waves + 1) * kBins; afterwards count[waves * kBins + b] is where bin b begins in the block.
template <int THREADS, int ITEMS>
__device__ __forceinline__ void block_rank(const uint32_t (&key)[ITEMS], int shift, uint32_t *count, uint32_t (&rank)[ITEMS])
{
    constexpr int WAVES = THREADS / 64;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int b = threadIdx.x; b < WAVES * kBins; b += THREADS) count[b] = 0;
    __syncthreads();
    uint32_t *mine = count + wave * kBins;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const uint32_t digit = (key[i] >> shift) & (kBins - 1);
        uint64_t same = ~uint64_t(0);
#pragma unroll
        for (int b = 0; b < 8; ++b) {
            const uint64_t has = __ballot((digit >> b) & 1);
            same &= ((digit >> b) & 1) ? has : ~has;
        }
        const uint32_t below = __popcll(same & ((uint64_t(1) << lane) - 1));
        const uint32_t before = mine[digit];
        rank[i] = before + below;
        wave_order();                                            // every lane has read before one adds
        if (below == 0) mine[digit] = before + static_cast<uint32_t>(__popcll(same));
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
        uint32_t upto = sum;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const uint32_t v = __shfl_up(upto, off, 64);
            if (lane >= off) upto += v;
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) start[lane * 4 + k] = upto - sum + c[k];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const uint32_t digit = (key[i] >> shift) & (kBins - 1);
        rank[i] += mine[digit] + start[digit];
    }
}

// All passes of a peer's sort by one block, T <= THREADS * ITEMS.
template <int THREADS, int ITEMS>
__global__ __launch_bounds__(THREADS) void sort_block_kernel(const int32_t *__restrict__ tokens, SortPlan p, uint32_t *__restrict__ keys,
                                                             int32_t *__restrict__ places)
{
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
        block_rank<THREADS, ITEMS>(key, 8 * pass, count, rank);
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
                                                                   SortPlan p, int shift, uint32_t *__restrict__ bins)
{
    __shared__ uint32_t count[kBins];
    const uint32_t peer = blockIdx.x / p.tiles, tile = blockIdx.x % p.tiles;
    const int64_t row = int64_t(peer) * p.T;
    for (int b = threadIdx.x; b < kBins; b += kTileThreads) count[b] = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kTileItems; ++i) {
        const int64_t at = int64_t(tile) * kTile + i * kTileThreads + threadIdx.x;
        if (at < p.T) atomicAdd(&count[(pass_key(tokens, keys, row + at, p.vocab) >> shift) & (kBins - 1)], 1u);
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
        uint32_t upto = sum;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const uint32_t w = __shfl_up(upto, off, 64);
            if (lane >= off) upto += w;
        }
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
                                                                  int32_t *__restrict__ places_out)
{
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
    block_rank<kTileThreads, kTileItems>(key, shift, count, rank);
    for (int b = threadIdx.x; b < kBins; b += kTileThreads)
        goes_to[b] = mine[int64_t(b) * p.tiles + tile] - count[(kTileThreads / 64) * kBins + b];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kTileItems; ++i) {
        const int64_t at = base + i * 64;
        if (at >= p.T) continue;
        const int64_t to = row + (goes_to[(key[i] >> shift) & (kBins - 1)] + rank[i]);
        keys_out[to] = key[i];
        places_out[to] = keys ? places[row + at] : static_cast<int32_t>(at);
    }
}

// ---- sums --------------------------------------------------------------------

constexpr int kSnap = 63;                // a row of at most this many places is not cut
constexpr int kWave = 64, kBlock = 256, kBatch = 8, kJoinShares = 16;

// What a share left behind: its first row, whether that row began in a share before, and its last row + 1
// among those that end in it (row .. end - 1 end here).
struct ShareRecord {
    uint32_t row, end;
    int32_t carried_in;
};

struct ShareGeom {
    int64_t shares;                      // of a peer
    uint32_t blocks;                     // of a peer, in each of the two kernels
    int32_t share, lanes_log2, slices;   // items of a share; lanes of its group; column slices
};

// The cut before item d of the merged list: rows 0..v-1 have ended and j places have been taken.  The merged list
// has key[j] + j ascending, and j is the first place with key[j] + j >= d.  Lanes of a group search together.
__device__ __forceinline__ void find_cut(const uint32_t *__restrict__ key, int64_t T, int64_t vocab, int64_t d, int lane, int lanes, int lanes_log2,
                                         uint64_t group_mask, int64_t &v, int64_t &j, bool &inside)
{
    int64_t lo = d > vocab ? d - vocab : 0, hi = d < T ? d : T;       // (lo <= hi where d <= T + vocab)
    while (lo < hi) {
        const int64_t step = ((hi - lo) >> lanes_log2) + 1;           // probes lo, lo + step, ...
        const int64_t at = lo + lane * step;
        const bool below = at < hi && int64_t(key[at]) + at < d;
        const int n = __popcll(__ballot(below) & group_mask);         // the first n probes are below
        if (n == 0) { hi = lo; break; }
        const int64_t last = lo + (n - 1) * step;
        const int64_t next = lo + n * step;
        lo = last + 1;
        hi = n < lanes && next < hi ? next : hi;
    }
    j = lo;
    v = d - j;
    inside = false;
    if (j == 0 || v >= vocab || key[j - 1] != v) return;
    // places of row v lie on both sides of the cut: count those before it and, if they are few, those after it
    int64_t before = 0, after = 0;
    for (int64_t k = 0; k <= kSnap && before == k; k += lanes) {
        const int64_t at = j - 1 - k - lane;
        before += __popcll(__ballot(at >= 0 && key[at] == v) & group_mask);
    }
    for (int64_t k = 0; k <= kSnap && after == k; k += lanes) {
        const int64_t at = j + k + lane;
        after += __popcll(__ballot(at < T && key[at] == v) & group_mask);
    }
    if (before + after <= kSnap) j -= before;
    else inside = true;
}

template <int ST, int YT, int VE, bool WIDE, bool ADD>
__global__ __launch_bounds__(kBlock) void embed_grad_kernel(const uint32_t *__restrict__ keys, const int32_t *__restrict__ places,
                                                            const char *__restrict__ dy, int64_t dy_stride, char *__restrict__ base, TableGeom g,
                                                            ShareGeom s, float scale, ShareRecord *__restrict__ records,
                                                            float *__restrict__ partials)
{
    constexpr int ES = ST == 0 ? 4 : 2, EY = YT == 0 ? 4 : 2;
    const int lanes = 1 << s.lanes_log2, lane = threadIdx.x & (lanes - 1);
    const uint32_t peer = blockIdx.x / s.blocks;
    const int64_t share = int64_t(blockIdx.x % s.blocks) * (kBlock >> s.lanes_log2) + (threadIdx.x >> s.lanes_log2);
    if (share >= s.shares) return;                                    // (whole groups; the ballots below look at a group's own lanes)
    const uint64_t group_mask = lanes == 64 ? ~uint64_t(0) : ((uint64_t(1) << lanes) - 1) << (threadIdx.x & 63 & ~(lanes - 1));
    const uint32_t *key = keys + peer * g.T;
    const int32_t *place = places + peer * g.T;
    const int64_t items = g.T + g.vocab;
    int64_t row, j, end, j_end;
    bool carried, cut;
    const int64_t d0 = share * s.share, d1 = d0 + s.share < items ? d0 + s.share : items;
    find_cut(key, g.T, g.vocab, d0, lane, lanes, s.lanes_log2, group_mask, row, j, carried);
    find_cut(key, g.T, g.vocab, d1, lane, lanes, s.lanes_log2, group_mask, end, j_end, cut);

    const int64_t c = (int64_t(blockIdx.y) * lanes + lane) * VE;
    const int64_t at_c = WIDE && c + VE > g.width ? g.width - VE : c;  // the last vector of a row ends with the row
    char *table = base + peer * g.peer_stride * ES;
    const char *rows = dy + peer * g.T * dy_stride * EY;
    float *slot = partials + (peer * s.shares + share) * 2 * g.width;
    const uint32_t vocab = static_cast<uint32_t>(g.vocab);
    if (lane == 0 && blockIdx.y == 0) records[peer * s.shares + share] = ShareRecord{static_cast<uint32_t>(row), static_cast<uint32_t>(end), carried};

    float acc[VE] = {};
    auto store_row = [&](int64_t r, const float (&f)[VE]) {
        if (c >= g.width) return;
        char *to = table + r * g.width * ES;
        if (c + VE <= g.width) {
            float v[VE];
            if constexpr (ADD) {
                load_elems<ST, VE>(to + c * ES, v);
#pragma unroll
                for (int k = 0; k < VE; ++k) v[k] += f[k];
                store_elems<ST, VE>(to + c * ES, v);
            } else store_elems<ST, VE>(to + c * ES, f);
        } else {
#pragma unroll
            for (int k = 0; k < VE; ++k) {
                const int64_t e = at_c + k;
                if (e < c || e >= g.width) continue;
                store_one<ST>(to + e * ES, ADD ? load_one<ST>(to + e * ES) + f[k] : f[k]);
            }
        }
    };
    auto store_partial = [&](float *to) {
        if (c >= g.width) return;
#pragma unroll
        for (int k = 0; k < VE; ++k) {
            const int64_t e = at_c + k;
            if (e >= c && e < g.width) to[e] = acc[k];
        }
    };
    bool head = carried, any = carried;                               // any: the row has places in this share or before
    auto finish = [&]() {                                             // the end of `row`
        if (head) store_partial(slot);
        else if (any || !ADD) {
            float f[VE];
#pragma unroll
            for (int k = 0; k < VE; ++k) f[k] = scale * acc[k];
            store_row(row, f);
        }
        head = any = false;
#pragma unroll
        for (int k = 0; k < VE; ++k) acc[k] = 0.f;
        ++row;
    };
    while (j < j_end) {
        const int64_t left = j_end - j;
        const int n = left < kBatch ? static_cast<int>(left) : kBatch;
        uint32_t k_of[kBatch];
        float v[kBatch][VE];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            k_of[u] = u < n ? key[j + u] : vocab;
            if (k_of[u] >= vocab) continue;                           // (no token: after every row's end)
            const char *from = rows + int64_t(place[j + u]) * dy_stride * EY;
            if constexpr (WIDE) {
                if (c < g.width) load_elems<YT, VE>(from + at_c * EY, v[u]);
            } else {
#pragma unroll
                for (int k = 0; k < VE; ++k) v[u][k] = c + k < g.width ? load_one<YT>(from + (c + k) * EY) : 0.f;
            }
        }
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            if (k_of[u] >= vocab) continue;
            while (row < k_of[u]) finish();
            any = true;
#pragma unroll
            for (int k = 0; k < VE; ++k) acc[k] += v[u][k];
        }
        if (k_of[kBatch - 1] >= vocab) break;
        j += n;
    }
    while (row < end) finish();
    if (cut) store_partial(head ? slot : slot + g.width);             // the row goes on in the next share
}

// Rows cut by shares: the share in which such a row ends adds its partial sums, in the order of the shares.
template <int ST, bool ADD>
__global__ __launch_bounds__(kBlock) void embed_grad_join_kernel(char *__restrict__ base, TableGeom g, ShareGeom s, float scale,
                                                                 const ShareRecord *__restrict__ records, const float *__restrict__ partials)
{
    constexpr int ES = ST == 0 ? 4 : 2, kWaves = kBlock / kWave;
    __shared__ float wave_sum[kWaves][kWave];
    const uint32_t peer = blockIdx.x / s.blocks;
    const ShareRecord *record = records + peer * s.shares;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t share0 = int64_t(blockIdx.x % s.blocks) * kJoinShares;
    const ShareRecord candidate = lane < kJoinShares && share0 + lane < s.shares ? record[share0 + lane] : ShareRecord{0, 0, 0};
    uint64_t ending = __ballot(candidate.carried_in && candidate.end != candidate.row);      // the same in every wave
    for (; ending; ending &= ending - 1) {
        const int64_t last = share0 + __builtin_ctzll(ending);
        const ShareRecord here = record[last];
        int64_t first = last - 1;                                         // the share in which the row begins
        while (true) {
            const int64_t at = first - lane;
            const bool middle = at >= 0 && record[at].carried_in && record[at].row == here.row;
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
                int64_t q = wave * each;
                for (; q + 8 <= q_end; q += 8) {
                    float v[8];
    #pragma unroll
                    for (int u = 0; u < 8; ++u) v[u] = mine[((first + q + u) * 2 + (q + u == 0 ? 1 : 0)) * g.width + c];
                    acc += ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
                }
                for (; q < q_end; ++q) acc += mine[((first + q) * 2 + (q == 0 ? 1 : 0)) * g.width + c];
            }
            wave_sum[wave][lane] = acc;
            __syncthreads();
            if (wave == 0 && c < g.width) {
                float sum = 0.f;
    #pragma unroll
                for (int w = 0; w < kWaves; ++w) sum += wave_sum[w][lane];
                char *to = base + (peer * g.peer_stride + int64_t(here.row) * g.width + c) * ES;
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

ShareGeom shares_of(const TableGeom &g)
{
    ShareGeom s;
    s.share = 32;
    s.shares = (g.T + g.vocab + s.share - 1) / s.share;
    s.blocks = 0;
    s.lanes_log2 = 3;
    s.slices = 0;
    return s;
}

struct Work {
    int64_t keys[2], places[2], bins, records, partials, bytes;
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
    w.records = take(static_cast<int64_t>(sizeof(ShareRecord)) * g.N * s.shares);
    w.partials = take(g.T > kSnap ? 4 * g.N * s.shares * 2 * g.width : 0);
    w.bytes = at;
    return w;
}

template <int ST, int YT, bool ADD>
void launch(void *base, const TableGeom &g, float scale, const void *dy, int64_t dy_stride, const uint32_t *keys, const int32_t *places,
            ShareRecord *records, float *partials, hipStream_t stream)
{
    constexpr int VE = ST == 0 ? 4 : 8;                               // 16 bytes of the table a lane
    ShareGeom s = shares_of(g);
    while (s.lanes_log2 < 6 && (int64_t(VE) << s.lanes_log2) < g.width) ++s.lanes_log2;
    s.slices = static_cast<int32_t>((g.width + (int64_t(VE) << s.lanes_log2) - 1) / (int64_t(VE) << s.lanes_log2));
    const int64_t per_block = kBlock >> s.lanes_log2;
    s.blocks = static_cast<uint32_t>((s.shares + per_block - 1) / per_block);
    const dim3 grid(static_cast<uint32_t>(s.blocks * g.N), static_cast<uint32_t>(s.slices));
    auto kernel = g.width >= VE ? embed_grad_kernel<ST, YT, VE, true, ADD> : embed_grad_kernel<ST, YT, VE, false, ADD>;
    kernel<<<grid, kBlock, 0, stream>>>(keys, places, static_cast<const char *>(dy), dy_stride, static_cast<char *>(base), g, s, scale, records,
                                        partials);
    if (g.T <= kSnap) return;                                         // no row is cut
    const int64_t column_blocks = (g.width + kWave - 1) / kWave;
    s.blocks = static_cast<uint32_t>((s.shares + kJoinShares - 1) / kJoinShares);
    const dim3 joins(static_cast<uint32_t>(s.blocks * g.N), static_cast<uint32_t>(column_blocks < 16 ? column_blocks : 16));
    embed_grad_join_kernel<ST, ADD><<<joins, kBlock, 0, stream>>>(static_cast<char *>(base), g, s, scale, records, partials);
}

}  // namespace

bool embed_grad_fits(const TableGeom &g)
{
    // the sums' kernel: 4 shares a block at least; the sort: a tile a block at least
    return shares_of(g).shares / 4 + 1 <= 0xffffffffLL / kBlock / g.N && (g.T / 1024 + 1) <= 0xffffffffLL / 1024 / g.N;
}

int64_t embed_grad_work_bytes(const TableGeom &g) { return layout(g).bytes; }

hipError_t launch_embed_grad(void *base, int state_dtype, const TableGeom &g, const int32_t *tokens, float scale, const void *dy,
                             int dy_dtype, int64_t dy_stride, bool accumulate, void *work, hipStream_t stream)
{
    const Work w = layout(g);
    char *at = static_cast<char *>(work);
    uint32_t *keys[2] = {reinterpret_cast<uint32_t *>(at + w.keys[0]), reinterpret_cast<uint32_t *>(at + w.keys[1])};
    int32_t *places[2] = {reinterpret_cast<int32_t *>(at + w.places[0]), reinterpret_cast<int32_t *>(at + w.places[1])};
    SortPlan p{static_cast<int32_t>(g.T), 0, static_cast<uint32_t>(g.vocab), 0};
    while ((uint64_t(g.vocab) >> (8 * p.passes)) != 0) ++p.passes;    // keys 0 .. vocab
    int sorted = 0;
    const uint32_t N = static_cast<uint32_t>(g.N);
    if (g.T > kOneBlock) {
        const int64_t tiles = (g.T + kTile - 1) / kTile;
        p.tiles = static_cast<uint32_t>(tiles);
        const uint32_t grid = p.tiles * N;
        uint32_t *bins = reinterpret_cast<uint32_t *>(at + w.bins);
        for (int pass = 0; pass < p.passes; ++pass) {
            const uint32_t *from = pass ? keys[1 - sorted] : nullptr;
            const int32_t *from_places = pass ? places[1 - sorted] : nullptr;
            sort_count_kernel<<<grid, kTileThreads, 0, stream>>>(tokens, from, p, 8 * pass, bins);
            sort_scan_kernel<<<N, 1024, 0, stream>>>(bins, kBins * tiles);
            sort_move_kernel<<<grid, kTileThreads, 0, stream>>>(tokens, from, from_places, p, 8 * pass, bins, keys[sorted], places[sorted]);
            sorted = 1 - sorted;
        }
        sorted = 1 - sorted;
    } else if (g.T > 1024) {
        sort_block_kernel<1024, 8><<<N, 1024, 0, stream>>>(tokens, p, keys[0], places[0]);
    } else if (g.T > 256) {
        sort_block_kernel<256, 4><<<N, 256, 0, stream>>>(tokens, p, keys[0], places[0]);
    } else if (g.T > 0) {
        sort_block_kernel<64, 4><<<N, 64, 0, stream>>>(tokens, p, keys[0], places[0]);
    }
    ShareRecord *records = reinterpret_cast<ShareRecord *>(at + w.records);
    float *partials = reinterpret_cast<float *>(at + w.partials);
    auto go = [&](auto add) {
        constexpr bool ADD = decltype(add)::value;
        auto f = state_dtype == 0 ? (dy_dtype == 0 ? launch<0, 0, ADD> : launch<0, 1, ADD>) : (dy_dtype == 0 ? launch<1, 0, ADD> : launch<1, 1, ADD>);
        f(base, g, scale, dy, dy_stride, keys[sorted], places[sorted], records, partials, stream);
    };
    if (accumulate) go(std::true_type{});
    else go(std::false_type{});
    return hipGetLastError();
}

}  // namespace moshpit
