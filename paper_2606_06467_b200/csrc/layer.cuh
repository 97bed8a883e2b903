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
  int heads, lanes;            // KV heads of a block; warps that take granules of one head (and column share) in turn
  int head_groups;             // Hkv / heads
  int slots, lane_slots, slot_bytes;  // the rings, one per lane: a granule's K and V rows of the block's heads in each slot
  int sub;                     // a granule is so many parts of 16 positions
  int spans;                   // stretches that the list of granules is cut into, at most
  int whole_units;             // 1: a stretch has the units that begin in it, whole (nothing to join)
  int cluster;                 // > 0: each cluster of so many blocks has one unit instead (joined in shared memory)
  int pad;                     // .. else: granules that a unit counts for beyond its own, where the list is cut
  int inbox_bytes;             // a cluster's block: records that it joins
  size_t smem_bytes;
  size_t unit_bytes, scratch_bytes;  // scratch: where each unit lies, then records of partial results (the same for every window)
};
DensePlan make_dense_plan(const clsa_params& p, bool eight, int window, const DeviceInfo& dev);
// c: an 8-bit cache, or nullptr (p's own caches). scratch: 256-byte aligned.
cudaError_t launch_dense_attn(const clsa_params& p, const clsa_cache8* c, int window, const DensePlan& plan, const void* q, void* out,
                              float* lse, uint32_t* status, unsigned char* scratch, cudaStream_t stream);

cudaError_t launch_norm_rope_axes(const clsa_norm_rope_spec& spec, const clsa_rope_axes& axes, int num_tokens, const int32_t* positions,
                                  int64_t axis_stride, const clsa_heads* q, const clsa_heads* q_out, const clsa_heads* k,
                                  const clsa_heads* k_out, const DeviceInfo& dev, cudaStream_t stream);
cudaError_t launch_add_norm(const clsa_add_norm_spec& spec, int num_rows, const clsa_rows* x, const clsa_rows* residual,
                            const clsa_rows* sum_out, const clsa_rows* y_out, const clsa_rows* codes_out, const clsa_rows* scales_out,
                            const DeviceInfo& dev, cudaStream_t stream);

}  // namespace clsa
