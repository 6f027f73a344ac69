// Launch interface of the operators of a peer's local step (token embeddings, 8-bit checkpoints,
// weight gradients, the policy loss) between api.hip and their kernels.  Types: 0 = binary32,
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

}  // namespace moshpit
