// Launch interface of the operators of a peer's local step (token embeddings, 8-bit checkpoints,
// weight gradients, the policy loss, norms, dropout, attention) between api.hip and their kernels.  Types: 0 = binary32,
// 1 = bfloat16.  Strides in elements.  All pointers are device pointers; argument checks are api.hip's.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace moshpit {

// A launch's threads are counted in 32 bits.
inline bool launchable(int64_t blocks, int64_t threads) { return blocks * threads <= 0xffffffffLL; }

// N tables of [vocab][width] elements, table i at `base` + i * peer_stride elements.
struct TableGeom {
    int64_t N, peer_stride, vocab, width;
    int64_t T;                       // tokens of a peer, [N][T] int32; outside [0, vocab): a place without a token
};

// out[i * T + t][:] = scale * table_i[token][:], zeros where there is no token.
hipError_t launch_embed(const void *base, int state_dtype, const TableGeom &g, const int32_t *tokens, float scale, void *out,
                        int out_dtype, int64_t out_stride, hipStream_t stream);

// grad_i[v][:] = [grad_i[v][:] +] scale * sum over t with tokens[i][t] == v of dy[i * T + t][:].
// work: embed_grad_work_bytes(g) bytes, 256-byte aligned, no contents kept from call to call.
// embed_grad_fits: whether a launch of this size is possible (blocks are counted in 31 bits).
bool embed_grad_fits(const TableGeom &g);
int64_t embed_grad_work_bytes(const TableGeom &g);
hipError_t launch_embed_grad(void *base, int state_dtype, const TableGeom &g, const int32_t *tokens, float scale, const void *dy,
                             int dy_dtype, int64_t dy_stride, bool accumulate, void *work, hipStream_t stream);

constexpr int64_t kCheckpointGroup = 32;     // consecutive elements of a row that share a scale byte
__host__ __device__ inline int64_t checkpoint_groups(int64_t width) { return (width + kCheckpointGroup - 1) / kCheckpointGroup; }

hipError_t launch_checkpoint(const void *x, int dtype, int64_t rows, int64_t width, int64_t stride, int8_t *codes, uint8_t *scales,
                             hipStream_t stream);
hipError_t launch_checkpoint_restore(const int8_t *codes, const uint8_t *scales, int64_t rows, int64_t width, void *out, int dtype,
                                     int64_t stride, hipStream_t stream);

// grad_i[o][c] = [grad_i[o][c] +] sum_t dy[i * T + t][o] * value(codes, scales)[i * T + t][c], grad_i at base + i * peer_stride.
struct WeightGradGeom {
    int64_t N, T, outs, ins, dy_stride, peer_stride;
};
bool weight_grad_fits(const WeightGradGeom &g);
int64_t weight_grad_work_bytes(const WeightGradGeom &g, int dy_dtype, int compute_units);
hipError_t launch_weight_grad(const void *dy, int dy_dtype, const int8_t *codes, const uint8_t *scales, const WeightGradGeom &g, void *base,
                              int state_dtype, bool accumulate, void *work, int compute_units, hipStream_t stream);

struct PolicyTerms {
    const float *old_logp, *ref_logp, *advantage, *weight;       // [N][T]; ref_logp may be nullptr (no KL term)
    float clip_low, clip_high, kl_coef;
};
// Row terms of the loss wait in `work` (policy_work_bytes) until they are summed per peer.
int64_t policy_work_bytes(int64_t N, int64_t T, int64_t vocab, int dtype, int compute_units);
hipError_t launch_policy_loss(const void *logits, int dtype, int64_t N, int64_t T, int64_t vocab, int64_t stride, const int32_t *tokens,
                              const PolicyTerms &p, void *grad, int64_t grad_stride, float *logp, float *stats, void *work,
                              int compute_units, hipStream_t stream);
hipError_t launch_token_logp(const void *logits, int dtype, int64_t rows, int64_t vocab, int64_t stride, const int32_t *tokens, float *logp,
                             void *work, int compute_units, hipStream_t stream);

// Root-mean-square norms: rows of `width` elements, row i * T + t for token t of peer i, gain i at `gain` + i * gain_stride elements.
struct NormArgs {
    const char *x, *residual;            // residual, total, codes and scales may be nullptr
    char *total, *out;
    int8_t *codes;
    uint8_t *scales;
    const char *gain;
    int64_t N, T, width, x_stride, residual_stride, total_stride, out_stride, gain_stride;
    float eps;
};
struct NormGradArgs {
    const char *dy, *x, *dtotal;         // dtotal may be nullptr
    char *dx;
    const char *gain;
    int64_t N, T, width, dy_stride, x_stride, dtotal_stride, dx_stride, gain_stride;
    float eps;
};
bool norm_fits(int64_t N, int64_t T, int64_t width);
hipError_t launch_norm(const NormArgs &a, int dtype, int state_dtype, int compute_units, hipStream_t stream);
int64_t norm_grad_work_bytes(int64_t N, int64_t T, int64_t width, int compute_units);
hipError_t launch_norm_grad(const NormGradArgs &a, int dtype, int state_dtype, bool accumulate, char *grad, int64_t grad_stride, void *work,
                            int compute_units, hipStream_t stream);

struct DropoutArgs {
    const char *x, *residual;            // residual and step may be nullptr
    char *out;
    const uint64_t *step;
    int64_t rows, width, x_stride, residual_stride, out_stride;
    uint64_t seed;
    uint32_t cut;                        // of 2^16: elements with fewer are dropped
    float factor;
};
bool dropout_fits(const DropoutArgs &a);
hipError_t launch_dropout(const DropoutArgs &a, int dtype, hipStream_t stream);

// Causal attention: query rows of heads * depth elements, key and value rows of kv_heads * depth, row i * T + t for token t of peer i.
// first: [N][T], the first token that a token sees (a token outside 0 .. its own number: no token).
struct AttentionArgs {
    const char *q, *k, *v;
    char *out;
    float *lse;                          // [N][heads][T]; may be nullptr
    const int32_t *first;
    int64_t N, T, q_stride, k_stride, v_stride, out_stride;
    int32_t heads, kv_heads, depth;
    float scale;
    uint32_t tiles;                      // (launch's own)
};
bool attention_fits(const AttentionArgs &a);
hipError_t launch_attention(AttentionArgs a, int dtype, int compute_units, hipStream_t stream);

// Its backward pass, into dq, dk and dv.
struct AttentionGradArgs {
    const char *q, *k, *v, *out, *dout;
    char *dq, *dk, *dv;
    const float *lse;
    const int32_t *first;
    int64_t N, T, q_stride, k_stride, v_stride, out_stride, dout_stride, dq_stride, dk_stride, dv_stride;
    int32_t heads, kv_heads, depth;
    float scale;
};
bool attention_grad_fits(const AttentionGradArgs &a, int dtype);
int64_t attention_grad_work_bytes(const AttentionGradArgs &a, int dtype, int compute_units);
hipError_t launch_attention_grad(const AttentionGradArgs &a, int dtype, void *work, int compute_units, hipStream_t stream);

// `fresh` new tokens of each of `seqs` sequences a peer against rows spans[..][0] .. spans[..][1] - 1 of its n_keys keys and values.
struct CachedArgs {
    const char *q, *k, *v;
    char *out;
    const int32_t *spans;                // [N][seqs][2]
    int64_t N, n_keys, q_stride, k_stride, v_stride, out_stride;
    int32_t seqs, fresh, heads, kv_heads, depth;
    float scale;
    int32_t col_tiles, splits;           // (launch's own)
};
struct CachedPlan {
    int32_t col_tiles, splits;
    int64_t work_bytes;
    bool fits;
};
CachedPlan cached_plan(const CachedArgs &a, int dtype, int compute_units);
hipError_t launch_cached(CachedArgs a, int dtype, const CachedPlan &p, void *work, hipStream_t stream);

}  // namespace moshpit
