// C-ABI entry points of the 8-bit cache calls: argument validation, workspace carving, launches. Every check that can refuse
// a call runs here on the host before anything is enqueued.
#include <math.h>

#include "cache8.cuh"

namespace clsa {
namespace {

bool aligned(const void* ptr, size_t a) { return (reinterpret_cast<uintptr_t>(ptr) % a) == 0; }

#define CLSA_TRY(expr)                     \
  do {                                     \
    const clsa_status st__ = (expr);       \
    if (st__ != CLSA_OK) return st__;      \
  } while (0)

clsa_status from_cuda(cudaError_t e) { return e == cudaSuccess ? CLSA_OK : CLSA_ERR_CUDA; }

clsa_status check_heads(const clsa_heads* h, int dim, bool output) {
  if (h->data == nullptr || !aligned(h->data, 16)) return CLSA_ERR_INVALID_ARG;
  if (h->num_heads < 1 || h->num_heads > 1024) return CLSA_ERR_INVALID_ARG;
  if (h->token_stride % 8 != 0 || h->head_stride % 8 != 0) return CLSA_ERR_INVALID_ARG;
  if (h->num_heads > 1 && h->head_stride < dim) return CLSA_ERR_INVALID_ARG;
  if (h->token_stride < (output ? dim : 0)) return CLSA_ERR_INVALID_ARG;
  return CLSA_OK;
}

clsa_status check_spec(const clsa_norm_rope_spec* s) {
  if (s == nullptr) return CLSA_ERR_INVALID_ARG;
  if ((s->norm != 0 && s->norm != 1) || (s->interleaved != 0 && s->interleaved != 1)) return CLSA_ERR_INVALID_ARG;
  if (s->head_dim < 1 || s->rot_dim < 0 || s->rot_dim > s->head_dim) return CLSA_ERR_INVALID_ARG;
  if (s->norm && (!isfinite(s->eps) || s->eps < 0.f)) return CLSA_ERR_INVALID_ARG;
  if (s->rot_dim > 0 && (s->inv_freq == nullptr || !aligned(s->inv_freq, 4) || !isfinite(s->rot_scale))) return CLSA_ERR_INVALID_ARG;
  if (!aligned(s->q_weight, 16) || !aligned(s->k_weight, 16)) return CLSA_ERR_INVALID_ARG;
  if (s->head_dim != 64 && s->head_dim != 128 && s->head_dim != 256) return CLSA_ERR_UNSUPPORTED;
  if (s->rot_dim % 16 != 0) return CLSA_ERR_UNSUPPORTED;
  return CLSA_OK;
}

// The params fields that these calls use.
clsa_status check_params(const clsa_params* p) {
  if (p == nullptr) return CLSA_ERR_INVALID_ARG;
  if (p->num_seqs < 1 || p->q_per_seq < 1 || p->num_q_heads < 1 || p->num_kv_heads < 1 || p->head_dim < 1 || p->idx_dim < 1 ||
      p->top_k < 1)
    return CLSA_ERR_INVALID_ARG;
  if (p->num_q_heads % p->num_kv_heads != 0 || p->num_kv_heads > 1024) return CLSA_ERR_INVALID_ARG;
  if (p->causal != 0 && p->causal != 1) return CLSA_ERR_INVALID_ARG;
  if (p->max_seq_len < p->q_per_seq) return CLSA_ERR_INVALID_ARG;
  if (!isfinite(p->sm_scale) || !(p->sm_scale > 0.f)) return CLSA_ERR_INVALID_ARG;
  if ((int64_t)p->num_seqs * p->q_per_seq > (int64_t)1 << 30) return CLSA_ERR_INVALID_ARG;
  if (p->num_cache_rows < 1 || p->num_cache_rows > 0x7fffffffLL) return CLSA_ERR_INVALID_ARG;
  // kernels number positions, 32-token stages, score tiles and appended rows with 32 bits
  if (p->max_seq_len > 0x7fff0000) return CLSA_ERR_UNSUPPORTED;
  if ((double)p->num_seqs * p->q_per_seq * p->num_kv_heads * ((p->top_k + 31) / 32) >= 2147483648.0) return CLSA_ERR_UNSUPPORTED;
  if ((double)p->num_seqs * ((p->max_seq_len + 31) / 32) >= 2147483648.0) return CLSA_ERR_UNSUPPORTED;
  if ((double)p->num_seqs * (2 * p->num_kv_heads + 1) >= 2147483648.0) return CLSA_ERR_UNSUPPORTED;
  if (p->head_dim != 128) return CLSA_ERR_UNSUPPORTED;
  if (p->idx_dim != 64 && p->idx_dim != 128) return CLSA_ERR_UNSUPPORTED;
  if (p->num_q_heads / p->num_kv_heads > 16) return CLSA_ERR_UNSUPPORTED;
  return CLSA_OK;
}

clsa_status check_scale_block(const clsa_params* p, const clsa_cache8* c) {
  if (c == nullptr) return CLSA_ERR_INVALID_ARG;
  const int sb = c->scale_block;
  if (sb != 16 && sb != 32 && sb != 64 && sb != 128) return CLSA_ERR_INVALID_ARG;
  if (p->block_table != nullptr && p->block_size % sb != 0) return CLSA_ERR_INVALID_ARG;
  return CLSA_OK;
}

clsa_status check_rows(const clsa_params* p) {
  if (p->seq_len == nullptr || !aligned(p->seq_len, 4)) return CLSA_ERR_INVALID_ARG;
  if (p->block_table == nullptr) {
    if (p->seq_start == nullptr || !aligned(p->seq_start, 8)) return CLSA_ERR_INVALID_ARG;
  } else {
    if (!aligned(p->block_table, 4)) return CLSA_ERR_INVALID_ARG;
    const int bs = p->block_size;
    if (bs < 16 || bs > 4096 || (bs & (bs - 1)) != 0) return CLSA_ERR_INVALID_ARG;
    if ((int64_t)p->max_blocks_per_seq * bs < p->max_seq_len) return CLSA_ERR_INVALID_ARG;
  }
  return CLSA_OK;
}

clsa_status check_kv8(const clsa_params* p, const clsa_cache8* c) {
  if (c->k == nullptr || c->v == nullptr || c->k_scale == nullptr || c->v_scale == nullptr) return CLSA_ERR_INVALID_ARG;
  if (!aligned(c->k, 16) || !aligned(c->v, 16)) return CLSA_ERR_INVALID_ARG;
  if (c->kv_token_stride < p->head_dim || c->kv_token_stride % 16 != 0) return CLSA_ERR_INVALID_ARG;
  if (c->kv_head_stride < p->head_dim || c->kv_head_stride % 16 != 0) return CLSA_ERR_INVALID_ARG;
  if (c->scale_head_stride < (p->num_cache_rows + c->scale_block - 1) / c->scale_block) return CLSA_ERR_INVALID_ARG;
  // row offsets are 32-bit counts of 16 bytes
  if ((double)p->num_cache_rows * (double)(c->kv_token_stride / 16) >= 4294967296.0) return CLSA_ERR_UNSUPPORTED;
  return CLSA_OK;
}

clsa_status check_idx8(const clsa_params* p, const clsa_cache8* c) {
  if (c->idx_k == nullptr || c->idx_k_scale == nullptr || !aligned(c->idx_k, 16)) return CLSA_ERR_INVALID_ARG;
  if (c->idx_token_stride < p->idx_dim || c->idx_token_stride % 16 != 0) return CLSA_ERR_INVALID_ARG;
  return CLSA_OK;
}

clsa_status check_workspace(const void* ws, size_t ws_bytes, size_t need) {
  if (ws == nullptr || !aligned(ws, 256) || ws_bytes < need) return CLSA_ERR_WORKSPACE;
  return CLSA_OK;
}

Cache8Layout make_layout(const clsa_params& p, const DeviceInfo& dev) {
  Cache8Layout w;
  auto align = [](size_t x) { return (x + 255) / 256 * 256; };
  w.counter_off = kStatusBytes;
  w.counter_bytes = attn8_counter_bytes(dev);
  w.scratch_off = w.counter_off + w.counter_bytes;
  w.attn_bytes = attn8_partial_bytes(p, make_attn8_plan(p, dev));
  w.expand_rows = ((int64_t)p.max_seq_len + 63) / 64 * 64;
  w.expand_bytes = p.q_per_seq > kScoresMaxT
                       ? align((size_t)p.num_seqs * w.expand_rows * p.idx_dim * 2) + align((size_t)p.num_seqs * sizeof(int64_t))
                       : 0;
  w.total = w.scratch_off + (w.attn_bytes > w.expand_bytes ? w.attn_bytes : w.expand_bytes);
  return w;
}

}  // namespace
}  // namespace clsa

using namespace clsa;

extern "C" {

clsa_status clsa_norm_rope(const clsa_norm_rope_spec* spec, int32_t num_tokens, const int32_t* positions, const clsa_heads* q,
                           const clsa_heads* q_out, const clsa_heads* k, const clsa_heads* k_out, clsa_stream stream) {
  CLSA_TRY(check_spec(spec));
  if (num_tokens < 0 || num_tokens > 1 << 30) return CLSA_ERR_INVALID_ARG;
  if ((q == nullptr) != (q_out == nullptr) || (k == nullptr) != (k_out == nullptr) || (q == nullptr && k == nullptr))
    return CLSA_ERR_INVALID_ARG;
  const clsa_heads* pairs[2][2] = {{q, q_out}, {k, k_out}};
  for (auto& pr : pairs) {
    if (pr[0] == nullptr) continue;
    if (pr[0]->num_heads != pr[1]->num_heads) return CLSA_ERR_INVALID_ARG;
    if (num_tokens == 0) continue;  // nothing has an address, and no stride means anything
    CLSA_TRY(check_heads(pr[0], spec->head_dim, false));
    CLSA_TRY(check_heads(pr[1], spec->head_dim, num_tokens > 1));
    if (pr[0]->data == pr[1]->data && (pr[0]->token_stride != pr[1]->token_stride ||
                                       (pr[0]->num_heads > 1 && pr[0]->head_stride != pr[1]->head_stride)))
      return CLSA_ERR_INVALID_ARG;
  }
  if (num_tokens == 0) return CLSA_OK;
  if (!aligned(positions, 4) || (positions == nullptr && spec->rot_dim > 0)) return CLSA_ERR_INVALID_ARG;
  DeviceInfo dev;
  if (!device_info(&dev)) return CLSA_ERR_CUDA;
  return from_cuda(launch_norm_rope(*spec, num_tokens, positions, q, q_out, k, k_out, dev, static_cast<cudaStream_t>(stream)));
}

clsa_status clsa_cache8_workspace_bytes(const clsa_params* p, const clsa_cache8* c, size_t* bytes) {
  if (bytes == nullptr) return CLSA_ERR_INVALID_ARG;
  CLSA_TRY(check_params(p));
  CLSA_TRY(check_scale_block(p, c));
  DeviceInfo dev;
  if (!device_info(&dev)) return CLSA_ERR_CUDA;
  *bytes = make_layout(*p, dev).total;
  return CLSA_OK;
}

clsa_status clsa_cache8_append(const clsa_params* p, const clsa_cache8* c, const clsa_norm_rope_spec* spec,
                               const clsa_heads* k_new, const clsa_heads* v_new, const clsa_heads* idx_k_new, void* workspace,
                               size_t workspace_bytes, clsa_stream stream) {
  CLSA_TRY(check_params(p));
  CLSA_TRY(check_rows(p));
  CLSA_TRY(check_scale_block(p, c));
  if ((k_new == nullptr) != (v_new == nullptr) || (k_new == nullptr && idx_k_new == nullptr)) return CLSA_ERR_INVALID_ARG;
  if (k_new != nullptr) {
    CLSA_TRY(check_kv8(p, c));
    CLSA_TRY(check_heads(k_new, p->head_dim, false));
    CLSA_TRY(check_heads(v_new, p->head_dim, false));
    if (k_new->num_heads != p->num_kv_heads || v_new->num_heads != p->num_kv_heads) return CLSA_ERR_INVALID_ARG;
  }
  if (idx_k_new != nullptr) {
    CLSA_TRY(check_idx8(p, c));
    CLSA_TRY(check_heads(idx_k_new, p->idx_dim, false));
    if (idx_k_new->num_heads != 1) return CLSA_ERR_INVALID_ARG;
  }
  if (spec != nullptr) {
    CLSA_TRY(check_spec(spec));
    if (spec->head_dim != p->head_dim) return CLSA_ERR_INVALID_ARG;
  }
  CLSA_TRY(check_workspace(workspace, workspace_bytes, kStatusBytes));
  DeviceInfo dev;
  if (!device_info(&dev)) return CLSA_ERR_CUDA;
  return from_cuda(launch_cache8_append(*p, *c, spec, k_new, v_new, idx_k_new, static_cast<uint32_t*>(workspace), dev,
                                        static_cast<cudaStream_t>(stream)));
}

clsa_status clsa_index_scores8(const clsa_params* p, const clsa_cache8* c, const void* q_idx, float* scores,
                               int64_t score_stride, void* workspace, size_t workspace_bytes, clsa_stream stream) {
  CLSA_TRY(check_params(p));
  CLSA_TRY(check_rows(p));
  CLSA_TRY(check_scale_block(p, c));
  CLSA_TRY(check_idx8(p, c));
  if (q_idx == nullptr || scores == nullptr || !aligned(q_idx, 16) || !aligned(scores, 4)) return CLSA_ERR_INVALID_ARG;
  if (score_stride < p->max_seq_len) return CLSA_ERR_INVALID_ARG;
  const bool expand = p->q_per_seq > kScoresMaxT;
  // tiled bulk copies address the expanded keys with 32-bit row coordinates
  if (expand && (int64_t)p->num_seqs * (((int64_t)p->max_seq_len + 63) / 64 * 64) > 0x7fffffffLL) return CLSA_ERR_UNSUPPORTED;
  CLSA_TRY(check_workspace(workspace, workspace_bytes, kStatusBytes));
  DeviceInfo dev;
  if (!device_info(&dev)) return CLSA_ERR_CUDA;
  auto status = static_cast<uint32_t*>(workspace);
  auto s = static_cast<cudaStream_t>(stream);
  if (!expand) return from_cuda(launch_index_scores8(*p, *c, q_idx, scores, score_stride, status, dev, s));
  const Cache8Layout w = make_layout(*p, dev);
  CLSA_TRY(check_workspace(workspace, workspace_bytes, w.total));
  unsigned char* keys = static_cast<unsigned char*>(workspace) + w.scratch_off;
  const size_t key_bytes = ((size_t)p->num_seqs * w.expand_rows * p->idx_dim * 2 + 255) / 256 * 256;
  auto starts = reinterpret_cast<int64_t*>(keys + key_bytes);
  if (launch_index_expand8(*p, *c, keys, starts, w.expand_rows, status, dev, s) != cudaSuccess) return CLSA_ERR_CUDA;
  clsa_params e = *p;
  e.idx_k_cache = keys;
  e.idx_token_stride = p->idx_dim;
  e.seq_start = starts;
  e.block_table = nullptr;
  e.num_cache_rows = (int64_t)p->num_seqs * w.expand_rows;
  return from_cuda(launch_index_scores_gemm(e, q_idx, scores, score_stride, true, status, dev, s));
}

clsa_status clsa_sparse_attn8(const clsa_params* p, const clsa_cache8* c, const void* q, const int32_t* idx,
                              const int32_t* count, void* out, float* lse, const clsa_attn_hints* hints, void* workspace,
                              size_t workspace_bytes, clsa_stream stream) {
  CLSA_TRY(check_params(p));
  CLSA_TRY(check_rows(p));
  CLSA_TRY(check_scale_block(p, c));
  CLSA_TRY(check_kv8(p, c));
  if (q == nullptr || idx == nullptr || count == nullptr || out == nullptr) return CLSA_ERR_INVALID_ARG;
  if (!aligned(q, 16) || !aligned(out, 16) || !aligned(idx, 4) || !aligned(count, 4) || !aligned(lse, 4))
    return CLSA_ERR_INVALID_ARG;
  const clsa_attn_hints h = hints != nullptr ? *hints : clsa_attn_hints{0, 0, 0, 0};
  for (int32_t v : {h.reverse, h.keep_rows, h.only_q_pending})
    if (v != 0 && v != 1) return CLSA_ERR_INVALID_ARG;
  if (h.shared_gpu < 0 || h.shared_gpu > 4) return CLSA_ERR_INVALID_ARG;
  if (h.shared_gpu != 0) return CLSA_ERR_UNSUPPORTED;
  if (workspace == nullptr || !aligned(workspace, 256)) return CLSA_ERR_WORKSPACE;
  DeviceInfo dev;
  if (!device_info(&dev)) return CLSA_ERR_CUDA;
  const Attn8Plan plan = make_attn8_plan(*p, dev);
  const Cache8Layout w = make_layout(*p, dev);
  CLSA_TRY(check_workspace(workspace, workspace_bytes, w.scratch_off + w.attn_bytes));
  auto base = static_cast<unsigned char*>(workspace);
  return from_cuda(launch_sparse_attn8(*p, *c, plan, q, idx, count, out, lse, h, reinterpret_cast<uint32_t*>(base),
                                       reinterpret_cast<uint32_t*>(base + w.counter_off),
                                       reinterpret_cast<float*>(base + w.scratch_off), dev, static_cast<cudaStream_t>(stream)));
}

}  // extern "C"
