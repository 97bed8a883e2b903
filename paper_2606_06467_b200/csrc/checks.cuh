// Checks of arguments that the entry points of several headers make.
#pragma once
#include "clsa_cache8.h"
#include "common.cuh"

namespace clsa {

inline bool aligned(const void* ptr, size_t a) { return (reinterpret_cast<uintptr_t>(ptr) % a) == 0; }
inline clsa_status from_cuda(cudaError_t e) { return e == cudaSuccess ? CLSA_OK : CLSA_ERR_CUDA; }

#define CLSA_TRY(expr)                     \
  do {                                     \
    const clsa_status st__ = (expr);       \
    if (st__ != CLSA_OK) return st__;      \
  } while (0)

clsa_status check_heads(const clsa_heads* h, int dim, bool output);
clsa_status check_spec(const clsa_norm_rope_spec* s);
// clsa_norm_rope's heads (and their agreement), but not its positions
clsa_status check_norm_rope(const clsa_norm_rope_spec* spec, int32_t num_tokens, const clsa_heads* q, const clsa_heads* q_out,
                            const clsa_heads* k, const clsa_heads* k_out);
clsa_status check_scale_block(const clsa_params* p, const clsa_cache8* c);
clsa_status check_rows(const clsa_params* p);
clsa_status check_kv8(const clsa_params* p, const clsa_cache8* c);

}  // namespace clsa
