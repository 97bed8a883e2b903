// Shared declarations of the calls of clsa_layer.h: launch plans and launchers.
#pragma once
#include "cache8.cuh"
#include "clsa_layer.h"

namespace clsa {

// Launch shape of the dense attention (dense_attn.cu).
struct DensePlan {
  int fold, tiles, col_warps;  // query columns of a block: 4 (held twice), or col_warps * tiles * 8
  int columns;                 // .. their number
  int col_tiles;               // blocks that share one stretch of the cache, each with its own query columns
  int heads, lanes;            // KV heads of a block; warps that take 16-token granules of one head (and column share) in turn
  int head_groups;             // Hkv / heads
  int slots, slot_bytes;       // the ring: one granule's K and V rows of the block's heads in each slot
  int spans;                   // stretches that the list of granules is cut into, at most
  size_t smem_bytes;
};
DensePlan make_dense_plan(const clsa_params& p, bool eight, const DeviceInfo& dev);
size_t dense_partial_bytes(const DensePlan& plan);
// c: an 8-bit cache, or nullptr (p's own caches). part: dense_partial_bytes of scratch.
cudaError_t launch_dense_attn(const clsa_params& p, const clsa_cache8* c, int window, const DensePlan& plan, const void* q, void* out,
                              float* lse, uint32_t* status, float* part, cudaStream_t stream);

cudaError_t launch_norm_rope_axes(const clsa_norm_rope_spec& spec, const clsa_rope_axes& axes, int num_tokens, const int32_t* positions,
                                  int64_t axis_stride, const clsa_heads* q, const clsa_heads* q_out, const clsa_heads* k,
                                  const clsa_heads* k_out, const DeviceInfo& dev, cudaStream_t stream);
cudaError_t launch_add_norm(const clsa_add_norm_spec& spec, int num_rows, const clsa_rows* x, const clsa_rows* residual,
                            const clsa_rows* sum_out, const clsa_rows* y_out, const clsa_rows* codes_out, const clsa_rows* scales_out,
                            const DeviceInfo& dev, cudaStream_t stream);

}  // namespace clsa
