// The newest tokens' K, V and K_idx rows into the 8-bit caches: per block of SB cache rows and head, the largest magnitude of
// the new rows gives the block's power-of-two scale, and each element is rounded once to e4m3.
//
// A block of threads takes one scale block of one sequence and one or more heads of the list K heads, V heads, K_idx: 16 (or,
// for 64-wide indexer keys, 8) lanes per row with 16 bytes each, all rows of a head in registers between the pass that finds
// the maximum and the pass that writes the codes, so every element is read once. Bound by HBM for long prompts (2 bytes in,
// 1 out), by one launch and two dependent round trips for a decode step. K's norm and rotation happen on the way in fp32.
// A scale block that holds older rows is re-coded by the same threads when its exponent grows.
#include "cache8.cuh"

namespace clsa {
namespace {

struct AppendArgs {
  HeadSpec spec;
  const uint16_t* k_weight;
  int has_spec;
  const uint16_t* src[3];  // K, V, K_idx
  int64_t src_token[3], src_head[3];
  uint8_t* code[3];
  uint8_t* scale[3];
  int64_t code_token[3], code_head[3], scale_head;
  int heads[3];
  int idx_dim;
  const int64_t* seq_start;
  const int32_t* seq_len;
  const int32_t* block_table;
  int block_shift, max_blocks;
  int64_t num_rows;
  int T, max_seq_len, spans, heads_per_block, items;
  uint32_t* status;
};

// Smallest exponent e with amax <= 448 * 2^e = 1.75 * 2^(e + 8), within the allowed range.
__device__ __forceinline__ int need_exponent(float amax) {
  const uint32_t bits = __float_as_uint(amax);
  const int e = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);
  return min(max(e, kScaleExpMin), kScaleExpMax);
}

// One head of one scale block: rows `lo` .. `hi` - 1 of the block are new, rows below `lo` older ones of the sequence.
template <int SB, int THREADS, int LANES>
__device__ __forceinline__ void append_head(const uint16_t* src, int64_t src_token, uint8_t* code, int64_t code_token,
                                            uint8_t* scale, int lo, int hi, bool norm, bool rotate, const AppendArgs& a,
                                            const float* tc, const float* ts, float* red) {
  constexpr int kRowsPerPass = THREADS / LANES;
  constexpr int R = SB / kRowsPerPass;
  const int l = threadIdx.x % LANES, sub = threadIdx.x / LANES;
  float x[R][8];
  {
    uint4 raw[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int row = r * kRowsPerPass + sub;
      raw[r] = make_uint4(0, 0, 0, 0);
      if (row >= lo && row < hi) raw[r] = *reinterpret_cast<const uint4*>(src + (int64_t)(row - lo) * src_token + 8 * l);
    }
#pragma unroll
    for (int r = 0; r < R; ++r) unpack_bf16x8(x[r], raw[r]);
  }
  const int e_old = lo > 0 ? scale_exponent(*scale) : kScaleExpMin;  // every thread reads it before the barrier below
  if (norm) {
    float w[8];
    load_weight8(w, a.k_weight, 8 * l);
#pragma unroll
    for (int r = 0; r < R; ++r) head_norm<LANES>(x[r], w, a.spec.eps);
  }
  if (rotate) {
    const int half = a.spec.rot_dim >> 1;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int row = r * kRowsPerPass + sub;
      float c[8], s[8];
      load_turns(c, s, tc + row * half, ts + row * half, a.spec.rot_dim, a.spec.interleaved, l);
      head_rotate<LANES>(x[r], c, s, a.spec.rot_dim, a.spec.interleaved, l);
    }
  }
  float amax = 0.f;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int row = r * kRowsPerPass + sub;
    if (row >= lo && row < hi) {  // (table entries of other rows are not set)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float m = fabsf(x[r][i]);
        if (m <= 3.4028234663852886e38f) amax = fmaxf(amax, m);  // finite
      }
    }
  }
#pragma unroll
  for (int m = 16; m >= 1; m >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, m));
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = amax;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < THREADS / 32; ++w) amax = fmaxf(amax, red[w]);
  const int e = max(need_exponent(amax), e_old);
  const float inv = exp2_int(-e);
  if (threadIdx.x == 0) *scale = (uint8_t)(e + 127);
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int row = r * kRowsPerPass + sub;
    uint2* dst = reinterpret_cast<uint2*>(code + (int64_t)row * code_token + 8 * l);
    if (row >= lo && row < hi) {
      uint2 v;
      v.x = f32x2_to_e4m3x2(x[r][0] * inv, x[r][1] * inv) | f32x2_to_e4m3x2(x[r][2] * inv, x[r][3] * inv) << 16;
      v.y = f32x2_to_e4m3x2(x[r][4] * inv, x[r][5] * inv) | f32x2_to_e4m3x2(x[r][6] * inv, x[r][7] * inv) << 16;
      *dst = v;
    } else if (row < lo && e > e_old) {  // an older row: its codes move down by e - e_old exponents
      const float f = exp2_int(max(e_old - e, -60));
      const uint2 v = *dst;
      const uint32_t in[4] = {e4m3x2_to_f16x2(v.x), e4m3x2_hi_to_f16x2(v.x), e4m3x2_to_f16x2(v.y), e4m3x2_hi_to_f16x2(v.y)};
      uint32_t o[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] = f32x2_to_e4m3x2(f16_lo(in[i]) * f, f16_hi(in[i]) * f);
      *dst = make_uint2(o[0] | o[1] << 16, o[2] | o[3] << 16);
    }
  }
}

template <int SB, int THREADS>
__global__ void __launch_bounds__(THREADS) cache8_append_kernel(const AppendArgs a) {
  extern __shared__ __align__(16) float turns[];  // cosines, then sines: [SB][rot_dim / 2] each
  __shared__ float red[2][THREADS / 32];
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int b = blockIdx.x / a.spans, span = blockIdx.x % a.spans;
  const int n = a.seq_len[b];
  const bool reports = span == 0 && blockIdx.y == 0 && threadIdx.x == 0;
  if (n < a.T || n > a.max_seq_len) {
    if (reports) flag_status(a.status, CLSA_DEV_BAD_SEQLEN);
    return;
  }
  const int first = n - a.T;                      // position of the first new token
  const int begin = (first / SB + span) * SB;     // first position of this scale block
  if (begin >= n) return;
  const int lo = max(first - begin, 0), hi = min(n - begin, SB);
  if (a.block_table == nullptr && a.seq_start[b] % SB != 0) {
    if (reports) flag_status(a.status, CLSA_DEV_BAD_SCALE_BLOCK);
    return;
  }
  // a multiple of SB: sequences start on one, and pages are whole scale blocks
  const int64_t row0 = cache_row(a.block_table, a.block_shift, a.max_blocks, a.seq_start, a.num_rows, b, begin);
  if (row0 < 0 || row0 + hi > a.num_rows) {
    if (threadIdx.x == 0 && blockIdx.y == 0) flag_status(a.status, CLSA_DEV_BAD_INDEX);
    return;
  }
  const int item0 = blockIdx.y * a.heads_per_block, item1 = min(item0 + a.heads_per_block, a.items);
  const int half = a.spec.rot_dim >> 1;
  float* tc = turns;
  float* ts = turns + SB * half;
  const bool rotate = a.has_spec && a.spec.rot_dim > 0;
  if (rotate && item0 < a.heads[0]) {
    for (int i = threadIdx.x; i < (hi - lo) * half; i += THREADS) {
      const int row = lo + i / half, j = i % half;
      turn_of(begin + row, a.spec.inv_freq[j], a.spec.rot_scale, &tc[row * half + j], &ts[row * half + j]);
    }
    __syncthreads();
  }
  const int64_t tok0 = (int64_t)b * a.T + (begin + lo - first);  // the first new token of this block
  for (int item = item0; item < item1; ++item) {
    const int kind = item < a.heads[0] ? 0 : (item < a.heads[0] + a.heads[1] ? 1 : 2);
    const int h = item - (kind > 0 ? a.heads[0] : 0) - (kind > 1 ? a.heads[1] : 0);
    const uint16_t* src = a.src[kind] + tok0 * a.src_token[kind] + h * a.src_head[kind];
    uint8_t* code = a.code[kind] + row0 * a.code_token[kind] + h * a.code_head[kind];
    uint8_t* scale = a.scale[kind] + h * a.scale_head + row0 / SB;
    float* r = red[item & 1];
    if (kind == 2 && a.idx_dim == 64)
      append_head<SB, THREADS, 8>(src, a.src_token[kind], code, a.code_token[kind], scale, lo, hi, false, false, a, tc, ts, r);
    else
      append_head<SB, THREADS, 16>(src, a.src_token[kind], code, a.code_token[kind], scale, lo, hi,
                                   kind == 0 && a.has_spec && a.spec.norm, kind == 0 && rotate, a, tc, ts, r);
  }
}

template <int SB, int THREADS>
cudaError_t launch(const AppendArgs& a, unsigned blocks_x, unsigned blocks_y, cudaStream_t stream) {
  const size_t smem = a.has_spec ? (size_t)SB * a.spec.rot_dim * sizeof(float) : 0;
  if (smem > 48 * 1024) {
    const cudaError_t err = cudaFuncSetAttribute(cache8_append_kernel<SB, THREADS>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (err != cudaSuccess) return err;
  }
  cache8_append_kernel<SB, THREADS><<<dim3(blocks_x, blocks_y), THREADS, smem, stream>>>(a);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_cache8_append(const clsa_params& p, const clsa_cache8& c, const clsa_norm_rope_spec* spec,
                                 const clsa_heads* k_new, const clsa_heads* v_new, const clsa_heads* idx_new, uint32_t* status,
                                 const DeviceInfo& dev, cudaStream_t stream) {
  AppendArgs a = {};
  if (spec != nullptr && k_new != nullptr) {
    a.has_spec = 1;
    a.spec = {spec->norm, spec->rot_dim, spec->interleaved, spec->eps, spec->rot_scale, spec->inv_freq};
    a.k_weight = static_cast<const uint16_t*>(spec->k_weight);
  }
  const clsa_heads* in[3] = {k_new, v_new, idx_new};
  void* code[3] = {c.k, c.v, c.idx_k};
  void* scale[3] = {c.k_scale, c.v_scale, c.idx_k_scale};
  for (int i = 0; i < 3; ++i) {
    if (in[i] == nullptr) continue;
    a.src[i] = static_cast<const uint16_t*>(in[i]->data);
    a.src_token[i] = in[i]->token_stride;
    a.src_head[i] = in[i]->head_stride;
    a.code[i] = static_cast<uint8_t*>(code[i]);
    a.scale[i] = static_cast<uint8_t*>(scale[i]);
    a.code_token[i] = i < 2 ? c.kv_token_stride : c.idx_token_stride;
    a.code_head[i] = i < 2 ? c.kv_head_stride : 0;
    a.heads[i] = in[i]->num_heads;
    a.items += a.heads[i];
  }
  a.scale_head = c.scale_head_stride;
  a.idx_dim = p.idx_dim;
  a.seq_start = p.seq_start;
  a.seq_len = p.seq_len;
  a.block_table = p.block_table;
  while (p.block_table != nullptr && (1 << a.block_shift) < p.block_size) ++a.block_shift;
  a.max_blocks = p.max_blocks_per_seq;
  a.num_rows = p.num_cache_rows;
  a.T = p.q_per_seq;
  a.max_seq_len = p.max_seq_len;
  a.status = status;
  a.spans = (p.q_per_seq - 1 + c.scale_block - 1) / c.scale_block + 1;  // scale blocks that T consecutive positions can touch
  const int64_t bx = (int64_t)p.num_seqs * a.spans;
  // Heads per block: a block that takes several K heads forms its rows' angles once for all of them.
  a.heads_per_block = 1;
  while (a.heads_per_block < 8 && bx * ((a.items + 2 * a.heads_per_block - 1) / (2 * a.heads_per_block)) >= 4 * dev.sm_count)
    a.heads_per_block *= 2;
  const unsigned by = (unsigned)((a.items + a.heads_per_block - 1) / a.heads_per_block);
  switch (c.scale_block) {
    case 16: return launch<16, 128>(a, (unsigned)bx, by, stream);
    case 32: return launch<32, 128>(a, (unsigned)bx, by, stream);
    case 64: return launch<64, 256>(a, (unsigned)bx, by, stream);
    default: return launch<128, 256>(a, (unsigned)bx, by, stream);
  }
}

}  // namespace clsa
