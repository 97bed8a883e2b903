// RMS norm of each query and key head and the position rotation, one pass over bf16 heads (a few operations per byte:
// bound by HBM for a prefill chunk, by one launch and one memory round trip for a decode step).
//
// A head of D dimensions is held by D / 8 lanes of a warp, 16 bytes each; the sum of squares is a butterfly over those
// lanes, the partner of a half-split rotation comes by one shuffle per dimension. A block takes one token: its threads
// first issue the loads of all their heads, then compute the token's rot_dim / 2 angles once for all heads (64-bit
// product and reduction, 32-bit functions) into shared memory, so that the angles hide behind the loads.
#include "cache8.cuh"

namespace clsa {
namespace {

constexpr int kThreads = 256;

struct NormRopeArgs {
  HeadSpec spec;
  const uint16_t* weight[2];  // q, k
  const uint16_t* in[2];
  uint16_t* out[2];
  int64_t in_token[2], in_head[2], out_token[2], out_head[2];
  int heads[2];
  const int32_t* positions;
};

// PASSES heads per group of lanes, loaded together.
template <int LANES, int PASSES>
__global__ void __launch_bounds__(kThreads) norm_rope_kernel(const NormRopeArgs a) {
  constexpr int kGroups = kThreads / LANES;
  __shared__ __align__(16) float tc[LANES * 4], ts[LANES * 4];
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int64_t token = blockIdx.x;
  const int l = threadIdx.x % LANES, group = threadIdx.x / LANES;
  const int pos = a.positions != nullptr ? a.positions[token] : 0;
  if (pos < 0) return;  // padding
  const int head0 = blockIdx.y * (kGroups * PASSES) + group;
  uint4 raw[PASSES];
#pragma unroll
  for (int p = 0; p < PASSES; ++p) {
    const int h = head0 + p * kGroups, side = h >= a.heads[0], hh = side ? h - a.heads[0] : h;
    raw[p] = make_uint4(0, 0, 0, 0);
    if (hh < a.heads[side]) raw[p] = *reinterpret_cast<const uint4*>(a.in[side] + token * a.in_token[side] + hh * a.in_head[side] + 8 * l);
  }
  float c[8], s[8];
  if (a.spec.rot_dim > 0) {
    for (int i = threadIdx.x; i < a.spec.rot_dim / 2; i += kThreads) turn_of(pos, a.spec.inv_freq[i], a.spec.rot_scale, &tc[i], &ts[i]);
    __syncthreads();
    load_turns(c, s, tc, ts, a.spec.rot_dim, a.spec.interleaved, l);
  }
#pragma unroll
  for (int p = 0; p < PASSES; ++p) {
    const int h = head0 + p * kGroups, side = h >= a.heads[0], hh = side ? h - a.heads[0] : h;
    float x[8];
    unpack_bf16x8(x, raw[p]);
    if (a.spec.norm) {
      float w[8];
      load_weight8(w, a.weight[side], 8 * l);
      head_norm<LANES>(x, w, a.spec.eps);
    }
    if (a.spec.rot_dim > 0) head_rotate<LANES>(x, c, s, a.spec.rot_dim, a.spec.interleaved, l);
    if (hh < a.heads[side]) {
      const uint4 r = make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
      *reinterpret_cast<uint4*>(a.out[side] + token * a.out_token[side] + hh * a.out_head[side] + 8 * l) = r;
    }
  }
}

template <int LANES>
void launch(const NormRopeArgs& a, int num_tokens, const DeviceInfo& dev, cudaStream_t stream) {
  constexpr int kGroups = kThreads / LANES;
  const int passes = (a.heads[0] + a.heads[1] + kGroups - 1) / kGroups;
  // few tokens: one pass per block, as many blocks as there are passes (the angles are formed in each of them)
  int per = (int64_t)num_tokens * passes <= 4 * dev.sm_count ? 1 : (passes < 4 ? passes : 4);
  const dim3 grid((unsigned)num_tokens, (unsigned)((passes + per - 1) / per));
  if (per == 1) norm_rope_kernel<LANES, 1><<<grid, kThreads, 0, stream>>>(a);
  else if (per == 2) norm_rope_kernel<LANES, 2><<<grid, kThreads, 0, stream>>>(a);
  else if (per == 3) norm_rope_kernel<LANES, 3><<<grid, kThreads, 0, stream>>>(a);
  else norm_rope_kernel<LANES, 4><<<grid, kThreads, 0, stream>>>(a);
}

}  // namespace

cudaError_t launch_norm_rope(const clsa_norm_rope_spec& spec, int num_tokens, const int32_t* positions, const clsa_heads* q,
                             const clsa_heads* q_out, const clsa_heads* k, const clsa_heads* k_out, const DeviceInfo& dev,
                             cudaStream_t stream) {
  NormRopeArgs a = {};
  a.spec = {spec.norm, spec.rot_dim, spec.interleaved, spec.eps, spec.rot_scale, spec.inv_freq};
  a.weight[0] = static_cast<const uint16_t*>(spec.q_weight);
  a.weight[1] = static_cast<const uint16_t*>(spec.k_weight);
  const clsa_heads* in[2] = {q, k};
  const clsa_heads* out[2] = {q_out, k_out};
  for (int i = 0; i < 2; ++i) {
    if (in[i] == nullptr) continue;
    a.in[i] = static_cast<const uint16_t*>(in[i]->data);
    a.out[i] = static_cast<uint16_t*>(out[i]->data);
    a.in_token[i] = in[i]->token_stride; a.in_head[i] = in[i]->head_stride;
    a.out_token[i] = out[i]->token_stride; a.out_head[i] = out[i]->head_stride;
    a.heads[i] = in[i]->num_heads;
  }
  a.positions = positions;
  if (spec.head_dim == 64) launch<8>(a, num_tokens, dev, stream);
  else if (spec.head_dim == 128) launch<16>(a, num_tokens, dev, stream);
  else launch<32>(a, num_tokens, dev, stream);
  return cudaGetLastError();
}

}  // namespace clsa
