// RMS norm of each query and key head and the position rotation, one pass over bf16 heads (a few operations per byte:
// bound by HBM for a prefill chunk, by one launch and one memory round trip for a decode step).
//
// A head of D dimensions is held by D / 8 lanes of a warp, 16 bytes each; the sum of squares is a butterfly over those
// lanes, the partner of a half-split rotation sits in the same lane (a lane of the turned dimensions has 4 of each half). A warp
// takes heads of one token, 32 / (D / 8) in a pass, four passes' loads and then their work together. The token's rot_dim / 2 angles (64-bit product and reduction, 32-bit
// functions) are formed once per warp and folded with the weights into two factors per dimension, so that a dimension costs a
// product, a multiply-add and a scaling, two dimensions per instruction. Warps are independent of one another. How many of a
// token's heads a warp takes follows from the number of tokens: few tokens are spread over many warps (each forms the angles
// anew), many keep a token together.
// 4096 tokens of 32 + 8 heads of 128: 84 MB in 17.1 us, 4.9 TB/s, 0.76 of a measured copy (10.8 us with the input in L2; 18.1 and
// 14.2 before a lane had its own partners). What is missing is the launch and the ramp of one wave: two to five passes at a time
// measure the same, rings of asynchronous copies took 29 to 35, loading ahead by a batch 19.5. 16 tokens: 2.2 us, one launch.
#include "cache8.cuh"

namespace clsa {
namespace {

constexpr int kThreads = 128;
constexpr int kUnroll = 4;  // passes that are loaded and worked on together

struct NormRopeArgs {
  HeadSpec spec;
  const uint16_t* weight[2];  // q, k
  const uint16_t* in[2];
  uint16_t* out[2];
  int64_t in_token[2], in_head[2], out_token[2], out_head[2];
  int heads[2];
  const int32_t* positions;
  int num_tokens, parts, part_heads;  // warps per token, heads of each
};

// DENSE: heads lie head_dim apart, in and out (strides are immediates then). PAIR: the pairs lie half the turned dimensions apart,
// and a lane of those has 4 dimensions of each half, 8 bytes apiece, and so the partner of each; ALL: every dimension is turned.
// Not PAIR: partners are neighbours, or nothing is turned.
template <int LANES, bool DENSE, bool PAIR, bool ALL>
__global__ void __launch_bounds__(kThreads, 7) norm_rope_kernel(const __grid_constant__ NormRopeArgs a) {
  constexpr int kGroups = 32 / LANES;  // heads of a pass
  __shared__ __align__(16) float turns[kThreads / 32][2][LANES * 4];
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, l = lane % LANES, group = lane / LANES;
  const uint32_t item = blockIdx.x * (kThreads / 32) + warp;
  const int rot = a.spec.rot_dim;
  const bool turned = ALL || 8 * l < rot;
  const int at0 = PAIR && turned ? 4 * l : 8 * l;                                // this lane's first quad of a head
  const int apart = !PAIR || !turned ? 4 : ALL ? 4 * LANES : rot >> 1;           // and its second, behind it
  const uint32_t token = item / (uint32_t)a.parts;
  if (token >= (uint32_t)a.num_tokens) return;
  const int part0 = (int)(item - token * a.parts) * a.part_heads;
  const int pos = a.positions != nullptr ? a.positions[token] : 0;
  // the heads of one side (0: queries, 1: keys) that this warp has, and its lanes' shares of the first pass
  uint4 raw[kUnroll];
  const uint16_t* in;
  uint16_t* out;
  int64_t in_step, out_step;
  int left;  // heads from this batch's first one on
  auto begin = [&](int side) {
    const int before = side ? a.heads[0] : 0;
    const int lo = max(part0 - before, 0);
    left = min(part0 + a.part_heads - before, a.heads[side]) - lo;
    in = a.in[side] + token * a.in_token[side] + (lo + group) * a.in_head[side] + at0;
    out = a.out[side] + token * a.out_token[side] + (lo + group) * a.out_head[side] + at0;
    in_step = DENSE ? 256 : kGroups * a.in_head[side];
    out_step = DENSE ? 256 : kGroups * a.out_head[side];
  };
  auto load8 = [&](const uint16_t* at) -> uint4 {
    if (!PAIR) return *reinterpret_cast<const uint4*>(at);
    const uint2 lo = *reinterpret_cast<const uint2*>(at), hi = *reinterpret_cast<const uint2*>(at + apart);
    return make_uint4(lo.x, lo.y, hi.x, hi.y);
  };
  auto load = [&]() {
#pragma unroll
    for (int k = 0; k < kUnroll; ++k) {
      raw[k] = make_uint4(0, 0, 0, 0);
      if (group + k * kGroups < left) raw[k] = load8(in + k * in_step);
    }
  };
  int side = 0;
  begin(0);
  if (left <= 0) begin(side = 1);
  load();  // under way while the angles are formed
  if (pos < 0) return;  // padding
  float* tc = turns[warp][0];
  float* ts = turns[warp][1];
  if (rot > 0) {
    for (int i = lane; i < rot / 2; i += 32) turn_of(pos, a.spec.inv_freq[i], a.spec.rot_scale, &tc[i], &ts[i]);
    __syncwarp();
  }
  const bool norm = a.spec.norm;
  const float eps = a.spec.eps;
  while (true) {
    // z_i = r (x_i A_i + x_partner B_i) with A = w cos, B = -+ w_partner sin and r the root of the mean square's inverse
    uint64_t A[4], B[4];
    {
      uint4 wr = make_uint4(0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u);  // ones
      if (norm && a.weight[side] != nullptr) wr = load8(a.weight[side] + at0);
      const uint32_t w4[4] = {wr.x, wr.y, wr.z, wr.w};
      if (PAIR) {
        float4 c = make_float4(1.f, 1.f, 1.f, 1.f), s = make_float4(0.f, 0.f, 0.f, 0.f);
        if (turned) {
          c = *reinterpret_cast<const float4*>(tc + 4 * l);
          s = *reinterpret_cast<const float4*>(ts + 4 * l);
        }
        const uint64_t c2[2] = {pack2(c.x, c.y), pack2(c.z, c.w)}, s2[2] = {pack2(s.x, s.y), pack2(s.z, s.w)};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          A[k] = mul2(bf16x2_to_f32x2(w4[k]), c2[k & 1]);
          B[k] = mul2(bf16x2_to_f32x2(w4[k ^ 2]), s2[k & 1]) ^ (k < 2 ? 0x8000000080000000ull : 0ull);
        }
      }
      float c[8], s[8];
      if (!PAIR && rot > 0) load_turns(c, s, tc, ts, rot, true, l);
#pragma unroll
      for (int k = 0; k < 4 && !PAIR; ++k) {
        const uint64_t w = bf16x2_to_f32x2(w4[k]);
        const uint32_t p = __byte_perm(w4[k], 0u, 0x1032);  // partners are neighbours
        A[k] = turned ? mul2(w, pack2(c[2 * k], c[2 * k + 1])) : w;
        B[k] = turned ? mul2(bf16x2_to_f32x2(p), pack2(-s[2 * k], s[2 * k + 1])) : 0ull;
      }
    }
    auto one = [&](const uint4& raw) -> uint4 {
      const uint32_t in4[4] = {raw.x, raw.y, raw.z, raw.w};
      uint64_t x[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) x[k] = bf16x2_to_f32x2(in4[k]);
      float r = 1.f;
      if (norm) {
        const float2 s2 = unpack2(fma2(x[3], x[3], fma2(x[2], x[2], fma2(x[1], x[1], mul2(x[0], x[0])))));
        float ss = s2.x + s2.y;
#pragma unroll
        for (int m = LANES / 2; m >= 1; m >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, m);
        r = rsqrtf(fmaf(ss, 1.f / (8 * LANES), eps));
      }
      const uint64_t r2 = pack2(r, r);
      uint32_t o[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        uint64_t other = PAIR ? x[k ^ 2] : bf16x2_to_f32x2(__byte_perm(in4[k], 0u, 0x1032));
        if (!turned) other = 0ull;  // (an infinity times a zero sine is none)
        const float2 z = unpack2(mul2(fma2(x[k], A[k], mul2(other, B[k])), r2));
        o[k] = pack_bf16x2(z.x, z.y);
      }
      return make_uint4(o[0], o[1], o[2], o[3]);
    };
#pragma unroll 1
    while (true) {
#pragma unroll
      for (int k = 0; k < kUnroll; ++k) {
        if (k * kGroups >= left) break;  // the same for the whole warp
        const uint4 z = one(raw[k]);
        if (group + k * kGroups < left) {
          if (PAIR) {
            *reinterpret_cast<uint2*>(out + k * out_step) = make_uint2(z.x, z.y);
            *reinterpret_cast<uint2*>(out + k * out_step + apart) = make_uint2(z.z, z.w);
          } else {
            *reinterpret_cast<uint4*>(out + k * out_step) = z;
          }
        }
      }
      left -= kUnroll * kGroups;
      if (left <= 0) break;
      in += kUnroll * in_step;
      out += kUnroll * out_step;
      load();
    }
    if (side == 1) break;
    begin(side = 1);
    if (left <= 0) break;
    load();
  }
}

template <int LANES>
void launch(NormRopeArgs& a, const DeviceInfo& dev, cudaStream_t stream) {
  constexpr int kGroups = 32 / LANES;
  const int heads = a.heads[0] + a.heads[1];
  // parts of a token: as many as give every SM about 16 warps, each a whole number of the heads that a warp holds at a time (us with 8, 16
  // and 32 warps: 777 tokens of 32 + 8 heads 4.8, 4.5, 5.4, 2048 tokens 11.7, 10.0, 11.2, up to 256 tokens the same)
  int64_t parts = (16 * (int64_t)dev.sm_count + a.num_tokens - 1) / a.num_tokens;
  const int most = (heads + kGroups - 1) / kGroups;
  if (parts > most) parts = most;
  a.part_heads = (int)((most + parts - 1) / parts) * kGroups;
  a.parts = (heads + a.part_heads - 1) / a.part_heads;
  const int64_t warps = (int64_t)a.num_tokens * a.parts;
  const unsigned blocks = (unsigned)((warps + kThreads / 32 - 1) / (kThreads / 32));
  bool dense = true;
  for (int i = 0; i < 2; ++i) dense = dense && (a.heads[i] <= 1 || (a.in_head[i] == 8 * LANES && a.out_head[i] == 8 * LANES));
  const bool pair = a.spec.rot_dim > 0 && !a.spec.interleaved, all = pair && a.spec.rot_dim == 8 * LANES;
  void (*kernel)(const NormRopeArgs) =
      dense ? (all ? norm_rope_kernel<LANES, true, true, true> : pair ? norm_rope_kernel<LANES, true, true, false> : norm_rope_kernel<LANES, true, false, false>)
            : (all ? norm_rope_kernel<LANES, false, true, true> : pair ? norm_rope_kernel<LANES, false, true, false> : norm_rope_kernel<LANES, false, false, false>);
  kernel<<<blocks, kThreads, 0, stream>>>(a);
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
  a.num_tokens = num_tokens;
  if (spec.head_dim == 64) launch<8>(a, dev, stream);
  else if (spec.head_dim == 128) launch<16>(a, dev, stream);
  else launch<32>(a, dev, stream);
  return cudaGetLastError();
}

}  // namespace clsa
