// Token embeddings of every peer for gfx950: row `token` of the table that lies in the peer's row of the
// state, times a scale.  out[i][t][:] = round(scale * table_i[tokens[i][t]][:]), the product in binary32.
//
// Bound by HBM: every distinct table row is read once, every output row written once.  A group of lanes
// (a power of two, up to a wave) moves a row, or a wave 64 vectors of a longer one, 16 bytes of output a lane, and
// takes kRows places, whose tokens and then whose rows are requested together: one dependent pair of
// latencies for all of them.  Stores are streaming ones: 16 x 8192 rows of 1024 out of binary32 tables into bfloat16
// in 68 us, with plain ones in 87; 4 x 15274 rows of 1200 binary32 in 57 us (76).  These are calls on the same inputs one after the
// other; with other tables every time, which no cache holds yet, the first takes 82.
#include <hip/hip_runtime.h>

#include "local_ops.h"
#include "row_elems.h"

namespace moshpit {
namespace {

constexpr int kBlock = 256, kRows = 4;

template <int ST, int OT, bool WIDE>
__global__ __launch_bounds__(kBlock) void embed_kernel(const char *__restrict__ base, TableGeom g, const int32_t *__restrict__ tokens,
                                                        float scale, char *__restrict__ out, int64_t out_stride, int32_t lanes_log2, uint32_t chunks)
{
    constexpr int ES = ST == 0 ? 4 : 2, EO = OT == 0 ? 4 : 2, kVec = 16 / EO;
    const int32_t lanes = 1 << lanes_log2;
    const int64_t places = g.N * g.T;
    // this group's part of the block, its column chunk and its first place
    const uint32_t groups = kBlock >> lanes_log2, part = blockIdx.x * groups + (threadIdx.x >> lanes_log2);
    const uint32_t set = part / chunks;
    const int64_t c = (int64_t(part - set * chunks) * lanes + (threadIdx.x & (lanes - 1))) * kVec;
    const int64_t first = int64_t(set) * kRows;
    if (c >= g.width) return;
    const char *row[kRows];
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
        const int64_t at = first + u;
        row[u] = nullptr;
        if (at >= places) continue;
        const int64_t tok = tokens[at];
        if (tok >= 0 && tok < g.vocab) row[u] = base + ((at / g.T) * g.peer_stride + tok * g.width) * ES;
    }
    if constexpr (WIDE) {
        // the last vector of a row ends with the row: it repeats elements of the one before it
        const int64_t at_c = c + kVec <= g.width ? c : g.width - kVec;
        float v[kRows][kVec];
#pragma unroll
        for (int u = 0; u < kRows; ++u)
            if (row[u]) load_elems<ST, kVec>(row[u] + at_c * ES, v[u]);
#pragma unroll
        for (int u = 0; u < kRows; ++u) {
            const int64_t at = first + u;
            if (at >= places) continue;
            float r[kVec];
#pragma unroll
            for (int k = 0; k < kVec; ++k) r[k] = row[u] ? scale * v[u][k] : 0.f;
            store_elems<OT, kVec, true>(out + (at * out_stride + at_c) * EO, r);
        }
    } else {
        for (int u = 0; u < kRows; ++u) {
            const int64_t at = first + u;
            for (int64_t k = c; at < places && k < g.width && k < c + kVec; ++k)
                store_one<OT>(out + (at * out_stride + k) * EO, row[u] ? scale * load_one<ST>(row[u] + k * ES) : 0.f);
        }
    }
}

template <int ST, int OT>
hipError_t launch(const void *base, const TableGeom &g, const int32_t *tokens, float scale, void *out, int64_t out_stride, hipStream_t stream)
{
    constexpr int kVec = OT == 0 ? 4 : 8;
    int32_t lanes_log2 = 0;
    while (lanes_log2 < 6 && (int64_t(kVec) << lanes_log2) < g.width) ++lanes_log2;
    const int64_t chunks = (g.width + (int64_t(kVec) << lanes_log2) - 1) / (int64_t(kVec) << lanes_log2);
    const int64_t parts = (g.N * g.T + kRows - 1) / kRows * chunks, blocks = (parts + (kBlock >> lanes_log2) - 1) / (kBlock >> lanes_log2);
    if (!launchable(blocks, kBlock) || !launchable(parts, 1)) return hipErrorInvalidConfiguration;
    auto kernel = g.width >= kVec ? embed_kernel<ST, OT, true> : embed_kernel<ST, OT, false>;
    kernel<<<static_cast<uint32_t>(blocks), kBlock, 0, stream>>>(static_cast<const char *>(base), g, tokens, scale, static_cast<char *>(out), out_stride,
                                                                 lanes_log2, static_cast<uint32_t>(chunks));
    return hipGetLastError();
}

}  // namespace

hipError_t launch_embed(const void *base, int state_dtype, const TableGeom &g, const int32_t *tokens, float scale, void *out,
                        int out_dtype, int64_t out_stride, hipStream_t stream)
{
    if (g.N * g.T == 0) return hipSuccess;
    auto go = state_dtype == 0 ? (out_dtype == 0 ? launch<0, 0> : launch<0, 1>) : (out_dtype == 0 ? launch<1, 0> : launch<1, 1>);
    return go(base, g, tokens, scale, out, out_stride, stream);
}

}  // namespace moshpit
