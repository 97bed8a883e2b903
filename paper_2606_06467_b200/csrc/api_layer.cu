// C-ABI entry points of clsa_layer.h: argument validation, workspace carving, launches. Every check that can refuse a call runs here on
// the host before anything is enqueued.
#include <math.h>

#include "checks.cuh"
#include "layer.cuh"

namespace clsa {
namespace {

constexpr int kDenseMaxT = 32;

// The params fields that the dense attention uses, and its window (0 where only sizes are asked for).
clsa_status check_dense(const clsa_params* p, int32_t window) {
  if (p == nullptr) return CLSA_ERR_INVALID_ARG;
  if (p->num_seqs < 1 || p->q_per_seq < 1 || p->num_q_heads < 1 || p->num_kv_heads < 1 || p->head_dim < 1 || window < 0)
    return CLSA_ERR_INVALID_ARG;
  if (p->num_q_heads % p->num_kv_heads != 0 || p->num_kv_heads > 1024) return CLSA_ERR_INVALID_ARG;
  if (p->causal != 0 && p->causal != 1) return CLSA_ERR_INVALID_ARG;
  if (p->max_seq_len < 1 || (p->max_seq_len < p->q_per_seq && (p->causal || window > 0))) return CLSA_ERR_INVALID_ARG;
  if (!isfinite(p->sm_scale) || !(p->sm_scale > 0.f)) return CLSA_ERR_INVALID_ARG;
  if (p->num_cache_rows < 1 || p->num_cache_rows > 0x7fffffffLL) return CLSA_ERR_INVALID_ARG;
  if (p->head_dim != 128 || p->q_per_seq > kDenseMaxT || p->num_q_heads / p->num_kv_heads > 16) return CLSA_ERR_UNSUPPORTED;
  // positions, granules of all units and output rows are numbered with 32 bits
  if (p->max_seq_len > 0x7fff0000) return CLSA_ERR_UNSUPPORTED;
  if ((double)p->num_seqs * p->num_kv_heads * ((double)p->max_seq_len / 16 + 2) >= 1073741824.0) return CLSA_ERR_UNSUPPORTED;
  if ((double)p->num_seqs * p->q_per_seq * p->num_q_heads >= 2147483648.0) return CLSA_ERR_UNSUPPORTED;
  return CLSA_OK;
}

clsa_status check_kv16(const clsa_params* p) {
  if (p->k_cache == nullptr || p->v_cache == nullptr || !aligned(p->k_cache, 16) || !aligned(p->v_cache, 16)) return CLSA_ERR_INVALID_ARG;
  if (p->kv_token_stride < p->head_dim || p->kv_token_stride % 8 != 0) return CLSA_ERR_INVALID_ARG;
  if (p->num_kv_heads > 1 && (p->kv_head_stride < p->head_dim || p->kv_head_stride % 8 != 0)) return CLSA_ERR_INVALID_ARG;
  // strides of tiled bulk copies stay below 2^40 bytes
  if (p->kv_token_stride >= (int64_t)1 << 38 || p->kv_head_stride >= (int64_t)1 << 38) return CLSA_ERR_UNSUPPORTED;
  return CLSA_OK;
}

size_t dense_scratch_offset(const DeviceInfo& dev) { return kStatusBytes + attn8_counter_bytes(dev); }  // behind the 8-bit calls' counters

clsa_status dense(const clsa_params* p, const clsa_cache8* c, int32_t window, const void* q, void* out, float* lse, void* workspace,
                  size_t workspace_bytes, clsa_stream stream) {
  CLSA_TRY(check_rows(p));
  if (q == nullptr || out == nullptr || !aligned(q, 16) || !aligned(out, 16) || !aligned(lse, 4)) return CLSA_ERR_INVALID_ARG;
  if (workspace == nullptr || !aligned(workspace, 256)) return CLSA_ERR_WORKSPACE;
  DeviceInfo dev;
  if (!device_info(&dev)) return CLSA_ERR_CUDA;
  const DensePlan plan = make_dense_plan(*p, c != nullptr, window, dev);
  const size_t at = dense_scratch_offset(dev);
  if (workspace_bytes < at + plan.scratch_bytes) return CLSA_ERR_WORKSPACE;
  auto base = static_cast<unsigned char*>(workspace);
  return from_cuda(launch_dense_attn(*p, c, window, plan, q, out, lse, reinterpret_cast<uint32_t*>(base), base + at,
                                     static_cast<cudaStream_t>(stream)));
}

// A matrix of rows of `elements` elements, 16 bytes being `per16` of them (1: bytes without an alignment).
clsa_status check_matrix(const clsa_rows* m, int64_t elements, int per16, int num_rows, bool output) {
  if (m->data == nullptr || (per16 > 1 && !aligned(m->data, 16))) return CLSA_ERR_INVALID_ARG;
  if (m->stride % per16 != 0 || m->stride < 0) return CLSA_ERR_INVALID_ARG;
  if (m->stride < elements && num_rows > 1 && (output || m->stride != 0)) return CLSA_ERR_INVALID_ARG;
  return CLSA_OK;
}
// The bytes of a matrix' rows: runs of `length`, `step` apart.
struct Runs {
  __int128 at, length, step, rows;
  __int128 end() const { return at + (rows - 1) * step + length; }
};
Runs runs_of(const clsa_rows* m, int64_t elements, int size, int num_rows) {
  if (m == nullptr || m->data == nullptr) return {0, 0, 0, 0};
  return {(__int128)reinterpret_cast<uintptr_t>(m->data), (__int128)elements * size, (__int128)m->stride * size, m->stride == 0 ? 1 : num_rows};
}
// Whether two matrices share a byte. Rows of different distances count by the memory from the first to the last of them.
bool overlap(const Runs& a, const Runs& b) {
  if (a.rows == 0 || b.rows == 0 || a.at >= b.end() || b.at >= a.end()) return false;
  if (a.rows == 1 && b.rows == 1) return true;
  if (a.rows > 1 && b.rows > 1 && a.step != b.step) return true;
  const __int128 step = a.rows > 1 ? a.step : b.step, behind = ((b.at - a.at) % step + step) % step;  // of a's next row in front of it
  return behind < a.length || behind + b.length > step;
}

}  // namespace
}  // namespace clsa

using namespace clsa;

extern "C" {

clsa_status clsa_dense_workspace_bytes(const clsa_params* p, size_t* bytes) {
  if (bytes == nullptr) return CLSA_ERR_INVALID_ARG;
  CLSA_TRY(check_dense(p, 0));
  DeviceInfo dev;
  if (!device_info(&dev)) return CLSA_ERR_CUDA;
  const size_t a = make_dense_plan(*p, false, 0, dev).scratch_bytes, b = make_dense_plan(*p, true, 0, dev).scratch_bytes;
  *bytes = (dense_scratch_offset(dev) + (a > b ? a : b) + 255) / 256 * 256;
  return CLSA_OK;
}

clsa_status clsa_dense_attn(const clsa_params* p, int32_t window, const void* q, void* out, float* lse, void* workspace,
                            size_t workspace_bytes, clsa_stream stream) {
  CLSA_TRY(check_dense(p, window));
  CLSA_TRY(check_kv16(p));
  return dense(p, nullptr, window, q, out, lse, workspace, workspace_bytes, stream);
}

clsa_status clsa_dense_attn8(const clsa_params* p, const clsa_cache8* c, int32_t window, const void* q, void* out, float* lse,
                             void* workspace, size_t workspace_bytes, clsa_stream stream) {
  CLSA_TRY(check_dense(p, window));
  CLSA_TRY(check_scale_block(p, c));
  CLSA_TRY(check_kv8(p, c));
  if (c->kv_head_stride >= (int64_t)1 << 39) return CLSA_ERR_UNSUPPORTED;
  return dense(p, c, window, q, out, lse, workspace, workspace_bytes, stream);
}

clsa_status clsa_add_norm(const clsa_add_norm_spec* spec, int32_t num_rows, const clsa_rows* x, const clsa_rows* residual,
                          const clsa_rows* sum_out, const clsa_rows* y_out, const clsa_rows* codes_out, const clsa_rows* scales_out,
                          clsa_stream stream) {
  if (spec == nullptr || x == nullptr || num_rows < 0 || num_rows > 1 << 30) return CLSA_ERR_INVALID_ARG;
  if (spec->dim < 1 || !isfinite(spec->eps) || spec->eps < 0.f || spec->scale_group < 0 || !aligned(spec->weight, 16))
    return CLSA_ERR_INVALID_ARG;
  if ((codes_out == nullptr) != (scales_out == nullptr) || (y_out == nullptr && codes_out == nullptr)) return CLSA_ERR_INVALID_ARG;
  if (codes_out != nullptr && spec->scale_group == 0) return CLSA_ERR_INVALID_ARG;
  const int g = spec->scale_group;
  if (spec->dim % 16 != 0 || spec->dim > 16384) return CLSA_ERR_UNSUPPORTED;
  if (g != 0 && g != spec->dim && (g != 32 && g != 64 && g != 128)) return CLSA_ERR_UNSUPPORTED;
  if (g != 0 && spec->dim % g != 0) return CLSA_ERR_INVALID_ARG;
  if (num_rows == 0) return CLSA_OK;
  CLSA_TRY(check_matrix(x, spec->dim, 8, num_rows, false));
  if (residual != nullptr) CLSA_TRY(check_matrix(residual, spec->dim, 8, num_rows, false));
  if (sum_out != nullptr) CLSA_TRY(check_matrix(sum_out, spec->dim, 8, num_rows, true));
  if (y_out != nullptr) CLSA_TRY(check_matrix(y_out, spec->dim, 8, num_rows, true));
  if (codes_out != nullptr) {
    CLSA_TRY(check_matrix(codes_out, spec->dim, 16, num_rows, true));
    CLSA_TRY(check_matrix(scales_out, spec->dim / g, 1, num_rows, true));
  }
  // Blocks write some rows while others read theirs: an output shares no byte with another argument, but for sum_out and y_out, which may be an
  // input's own rows (whose elements the thread that writes them has read).
  const clsa_rows weight = {const_cast<void*>(spec->weight), 0};
  const Runs outs[4] = {runs_of(sum_out, spec->dim, 2, num_rows), runs_of(y_out, spec->dim, 2, num_rows), runs_of(codes_out, spec->dim, 1, num_rows),
                        runs_of(scales_out, g > 0 ? spec->dim / g : 0, 1, num_rows)};
  const Runs ins[3] = {runs_of(x, spec->dim, 2, num_rows), runs_of(residual, spec->dim, 2, num_rows), runs_of(&weight, spec->dim, 2, 1)};
  for (int o = 0; o < 4; ++o) {
    for (int i = 0; i < o; ++i)
      if (overlap(outs[o], outs[i])) return CLSA_ERR_INVALID_ARG;
    for (int i = 0; i < 3; ++i) {
      const bool own = o < 2 && i < 2 && outs[o].at == ins[i].at && outs[o].rows == ins[i].rows && (num_rows == 1 || outs[o].step == ins[i].step);
      if (!own && overlap(outs[o], ins[i])) return CLSA_ERR_INVALID_ARG;
    }
  }
  DeviceInfo dev;
  if (!device_info(&dev)) return CLSA_ERR_CUDA;
  return from_cuda(launch_add_norm(*spec, num_rows, x, residual, sum_out, y_out, codes_out, scales_out, dev, static_cast<cudaStream_t>(stream)));
}

clsa_status clsa_norm_rope_axes(const clsa_norm_rope_spec* spec, const clsa_rope_axes* axes, int32_t num_tokens, const int32_t* positions,
                                int64_t axis_stride, const clsa_heads* q, const clsa_heads* q_out, const clsa_heads* k,
                                const clsa_heads* k_out, clsa_stream stream) {
  CLSA_TRY(check_norm_rope(spec, num_tokens, q, q_out, k, k_out));
  if (axes == nullptr || axes->num_axes < 1 || axes->num_axes > CLSA_MAX_AXES || spec->rot_dim == 0) return CLSA_ERR_INVALID_ARG;
  for (int i = 0; i < spec->rot_dim / 2; ++i)
    if (axes->axis_of_pair[i] >= axes->num_axes) return CLSA_ERR_INVALID_ARG;
  if (axis_stride != 0 && axis_stride < num_tokens) return CLSA_ERR_INVALID_ARG;
  if (num_tokens == 0) return CLSA_OK;
  if (positions == nullptr || !aligned(positions, 4)) return CLSA_ERR_INVALID_ARG;
  DeviceInfo dev;
  if (!device_info(&dev)) return CLSA_ERR_CUDA;
  return from_cuda(launch_norm_rope_axes(*spec, *axes, num_tokens, positions, axis_stride, q, q_out, k, k_out, dev, static_cast<cudaStream_t>(stream)));
}

}  // extern "C"
