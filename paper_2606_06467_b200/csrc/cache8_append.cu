// The newest tokens' K, V and K_idx rows into the 8-bit caches: per block of SB cache rows and head, the largest magnitude of
// the new rows gives the block's power-of-two scale, and each element is rounded once to e4m3.
//
// Chunks (T > 1): a block of threads takes one scale block of one sequence and K and V of one to four heads (or K_idx), the rows of
// the next on their way while it works on one: 16 (or, for 64-wide indexer keys, 8) lanes per row with 16 bytes each, all rows of a
// head in registers between the pass that finds the maximum and the pass that writes the codes, so every element is read once.
// K's norm and rotation happen on the way in fp32. The angles of the rows are built by the addition theorem: a row's position is
// begin + 8 u + v, and cosines and sines of SB / 8 + 8 positions, formed once for all the block's K heads, give those of all SB
// rows; the part of v is folded with the weights once per head, which leaves seven packed operations per pair of dimensions.
// A scale block that holds older rows is re-coded by the same threads when its exponent grows.
// 4096 tokens of 8 heads, indexer keys, norm and rotation over all dimensions, 64-row blocks that straddle the tokens' ends:
// 26.7 MB in 11.6 us (the bytes alone would take 4.1; on a GPU where it took 11.3: aligned 10.8, without rotation 9.0, without norm 7.2): a launch, the chain
// length - page - rows, a barrier per head, and instruction issue at 16 warps per SM, which the rows in registers allow
// (80 registers and half as many warps again measured the same). A rotation that turns the whole head, half apart, has both
// partners in one lane (PAIR: 13.4 -> 11.4; other rotations exchange raw words, 13.0).
// Single tokens (T = 1): half a warp per row, no block barrier; what does not depend on the sequence's length (the row, the
// weight, the frequencies) is fetched together with it. Bound by a launch and two dependent round trips: 16 sequences of 8 heads 3.0 us.
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
  int num_seqs, T, max_seq_len, spans, items;
  int heads_per_block, head_groups;  // chunks: heads of a block of threads, such groups (K_idx is a group behind them)
  uint32_t* status;
};

// Smallest exponent e with amax <= 448 * 2^e = 1.75 * 2^(e + 8), within the allowed range.
__device__ __forceinline__ int need_exponent(float amax) {
  const uint32_t bits = __float_as_uint(amax);
  const int e = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);
  return min(max(e, kScaleExpMin), kScaleExpMax);
}

// Eight codes times a power of two, rounded again.
__device__ __forceinline__ uint2 recode(uint2 v, float f) {
  const uint32_t in[4] = {e4m3x2_to_f16x2(v.x), e4m3x2_hi_to_f16x2(v.x), e4m3x2_to_f16x2(v.y), e4m3x2_hi_to_f16x2(v.y)};
  uint32_t o[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) o[i] = f32x2_to_e4m3x2(f16_lo(in[i]) * f, f16_hi(in[i]) * f);
  return make_uint2(o[0] | o[1] << 16, o[2] | o[3] << 16);
}

// A lane's 8 codes: consecutive, or 4 of each half of the head.
template <bool PAIR, int LANES>
__device__ __forceinline__ uint2 get_codes(const uint8_t* at) {
  if (!PAIR) return *reinterpret_cast<const uint2*>(at);
  return make_uint2(*reinterpret_cast<const uint32_t*>(at), *reinterpret_cast<const uint32_t*>(at + 4 * LANES));
}
template <bool PAIR, int LANES>
__device__ __forceinline__ void put_codes(uint8_t* at, uint2 v) {
  if (!PAIR) {
    *reinterpret_cast<uint2*>(at) = v;
  } else {
    *reinterpret_cast<uint32_t*>(at) = v.x;
    *reinterpret_cast<uint32_t*>(at + 4 * LANES) = v.y;
  }
}

constexpr float kLargest = 3.4028234663852886e38f;  // what is larger is not finite and does not count for a scale

// A lane's 8 dimensions of a cosine or sine table row, as pairs.
__device__ __forceinline__ void load_pairs(uint64_t (&p)[4], const float* t, bool inter, int i0) {
  const float4 a = *reinterpret_cast<const float4*>(t + i0);
  if (inter) {
    p[0] = pack2(a.x, a.x); p[1] = pack2(a.y, a.y); p[2] = pack2(a.z, a.z); p[3] = pack2(a.w, a.w);
  } else {
    const float4 b = *reinterpret_cast<const float4*>(t + i0 + 4);
    p[0] = pack2(a.x, a.y); p[1] = pack2(a.z, a.w); p[2] = pack2(b.x, b.y); p[3] = pack2(b.z, b.w);
  }
}

__device__ __forceinline__ void load_quad(uint64_t (&p)[2], const float* t) {
  const float4 a = *reinterpret_cast<const float4*>(t);
  p[0] = pack2(a.x, a.y);
  p[1] = pack2(a.z, a.w);
}

// One head of one scale block: rows `lo` .. `hi` - 1 of the block are new, rows below `lo` older ones of the sequence. SPEC: the
// rows go through K's norm and rotation first (LANES 16); bc, bs: cosines and sines of positions begin + 8 u, then of 0 .. 7.
template <int SB, int THREADS, int LANES>
struct Rows {
  static constexpr int kPerPass = THREADS / LANES;  // a multiple of 8: a lane's rows share their place among 8
  static constexpr int R = SB / kPerPass;
  uint4 raw[R];
  // Zeros for rows that are not new. pair: 4 dimensions of each half of the head per lane instead of 8 consecutive ones.
  __device__ __forceinline__ void load(const uint16_t* src, int64_t src_token, int lo, int hi, bool pair) {
    const int l = threadIdx.x % LANES, sub = threadIdx.x / LANES;
    if (pair) {
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const int row = r * kPerPass + sub;
        const uint16_t* at = src + (row - lo) * src_token + 4 * l;
        raw[r] = make_uint4(0, 0, 0, 0);
        if (row >= lo && row < hi) {
          const uint2 f = *reinterpret_cast<const uint2*>(at), b = *reinterpret_cast<const uint2*>(at + 4 * LANES);
          raw[r] = make_uint4(f.x, f.y, b.x, b.y);
        }
      }
    } else {
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const int row = r * kPerPass + sub;
        raw[r] = make_uint4(0, 0, 0, 0);
        if (row >= lo && row < hi) raw[r] = *reinterpret_cast<const uint4*>(src + (row - lo) * src_token + 8 * l);
      }
    }
  }
};
// PAIR: the rotation turns the whole head, half apart, and a lane has 4 dimensions of each half.
template <int SB, int THREADS, int LANES, bool SPEC, bool PAIR = false>
__device__ __forceinline__ void append_head(const Rows<SB, THREADS, LANES>& rows, uint8_t* code, int64_t code_token,
                                            uint8_t* scale, int lo, int hi, const AppendArgs& a, const float* bc, const float* bs,
                                            const float* unit, float* red) {
  constexpr int kRowsPerPass = THREADS / LANES, R = Rows<SB, THREADS, LANES>::R;
  const auto& raw = rows.raw;
  const int l = threadIdx.x % LANES, sub = threadIdx.x / LANES;
  const int e_old = lo > 0 ? scale_exponent(*scale) : kScaleExpMin;  // every thread reads it before the barrier below
  uint64_t x[R][4];
  float amax = 0.f;
  if constexpr (SPEC) {
    const int rot = a.spec.rot_dim, half = rot >> 1, hl = rot >> 4;
    const bool turned = 8 * l < rot, inter = a.spec.interleaved;
    const int partner = l < hl ? l + hl : (l < 2 * hl ? l - hl : l);
    const int i0 = !turned ? 0 : inter ? 4 * l : (l < hl ? 8 * l : 8 * l - half);
    // z_i = r (x_i w_i cos + x_partner w'_i sin), w' the partner's weight with the sign of its term; by the addition theorem, over the
    // row's u and the lane's v: w cos = cu (w cv) - su (w sv), w' sin = su (w' cv) + cu (w' sv). Lanes that are not turned have
    // cu = 1 and su = 0 of `unit`.
    uint64_t w[4], wc[4], ws[4], pc[4], ps[4];
    const float *cu_row = turned ? bc + i0 : unit, *su_row = turned ? bs + i0 : unit + 8;
    const int u_step = turned ? half : 0;
    {
      uint4 wr = make_uint4(0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u);  // ones
      if (a.spec.norm && a.k_weight != nullptr) {
        if (PAIR) {
          const uint2 f = *reinterpret_cast<const uint2*>(a.k_weight + 4 * l), b = *reinterpret_cast<const uint2*>(a.k_weight + 4 * LANES + 4 * l);
          wr = make_uint4(f.x, f.y, b.x, b.y);
        } else {
          wr = *reinterpret_cast<const uint4*>(a.k_weight + 8 * l);
        }
      }
      const uint32_t w4[4] = {wr.x, wr.y, wr.z, wr.w};
      const float sg = l < hl ? -1.f : 1.f;
#pragma unroll
      for (int k = 0; k < 4; ++k) w[k] = bf16x2_to_f32x2(w4[k]);
      if (PAIR) {
        uint64_t cv[2], sv[2];
        load_quad(cv, bc + (SB / 8 + (sub & 7)) * half + 4 * l);
        load_quad(sv, bs + (SB / 8 + (sub & 7)) * half + 4 * l);
#pragma unroll
        for (int k = 0; k < 4; ++k) {  // z = x_k w cos -+ x_(k ^ 2) w' sin, the sign of the front half negative
          const uint64_t flip = k < 2 ? 0x8000000080000000ull : 0ull;
          wc[k] = mul2(w[k], cv[k & 1]);
          ws[k] = mul2(w[k], sv[k & 1]) ^ 0x8000000080000000ull;
          pc[k] = mul2(w[k ^ 2], cv[k & 1]) ^ flip;
          ps[k] = mul2(w[k ^ 2], sv[k & 1]) ^ flip;
        }
      } else if (rot > 0) {
        uint64_t cv[4], sv[4];
        load_pairs(cv, turned ? bc + (SB / 8 + (sub & 7)) * half + i0 : unit, inter, 0);
        load_pairs(sv, turned ? bs + (SB / 8 + (sub & 7)) * half + i0 : unit + 8, inter, 0);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const uint32_t p = inter ? __byte_perm(w4[k], 0u, 0x1032) : __shfl_sync(0xffffffffu, w4[k], partner, LANES);
          const uint64_t wp = turned ? mul2(bf16x2_to_f32x2(p), inter ? pack2(-1.f, 1.f) : pack2(sg, sg)) : 0ull;
          wc[k] = mul2(w[k], cv[k]);
          ws[k] = mul2(w[k], sv[k]) ^ 0x8000000080000000ull;
          pc[k] = mul2(wp, cv[k]);
          ps[k] = mul2(wp, sv[k]);
        }
      }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int row = r * kRowsPerPass + sub;
      const uint32_t in4[4] = {raw[r].x, raw[r].y, raw[r].z, raw[r].w};
#pragma unroll
      for (int k = 0; k < 4; ++k) x[r][k] = bf16x2_to_f32x2(in4[k]);
      float root = 1.f;
      if (a.spec.norm) {
        const float2 s2 = unpack2(fma2(x[r][3], x[r][3], fma2(x[r][2], x[r][2], fma2(x[r][1], x[r][1], mul2(x[r][0], x[r][0])))));
        float ss = s2.x + s2.y;
#pragma unroll
        for (int m = LANES / 2; m >= 1; m >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, m);
        root = rsqrtf(fmaf(ss, 1.f / (8 * LANES), a.spec.eps));
      }
      const uint64_t r2 = pack2(root, root);
      if (PAIR) {
        uint64_t cu[2], su[2], z[4];
        load_quad(cu, bc + (row >> 3) * half + 4 * l);
        load_quad(su, bs + (row >> 3) * half + 4 * l);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const uint64_t f = fma2(cu[k & 1], wc[k], mul2(su[k & 1], ws[k])), fp = fma2(su[k & 1], pc[k], mul2(cu[k & 1], ps[k]));
          z[k] = mul2(fma2(x[r][k], f, mul2(x[r][k ^ 2], fp)), r2);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) x[r][k] = z[k];
      } else if (rot > 0) {
        uint64_t cu[4], su[4];
        load_pairs(cu, cu_row + (row >> 3) * u_step, inter, 0);
        load_pairs(su, su_row + (row >> 3) * u_step, inter, 0);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          uint32_t p = inter ? __byte_perm(in4[k], 0u, 0x1032) : __shfl_sync(0xffffffffu, in4[k], partner, LANES);
          if (!turned) p = 0u;  // (an infinity times a zero sine is none)
          const uint64_t f = fma2(cu[k], wc[k], mul2(su[k], ws[k])), fp = fma2(su[k], pc[k], mul2(cu[k], ps[k]));
          x[r][k] = mul2(fma2(x[r][k], f, mul2(bf16x2_to_f32x2(p), fp)), r2);
        }
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) x[r][k] = mul2(mul2(x[r][k], w[k]), r2);
      }
      if (row >= lo && row < hi) {  // (rows that are not new are zeros under a norm of zeros)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float2 z = unpack2(x[r][k]);
          amax = fmaxf(amax, fmaxf(fabsf(z.x), fabsf(z.y)));  // a NaN does not count
        }
      }
    }
  } else {
    uint32_t top = 0u;  // bf16 magnitudes order as integers (rows that are not new are zeros)
#pragma unroll
    for (int r = 0; r < R; ++r) {
      top = __vmaxu2(__vmaxu2(top, raw[r].x & 0x7fff7fffu), __vmaxu2(raw[r].y & 0x7fff7fffu, __vmaxu2(raw[r].z & 0x7fff7fffu, raw[r].w & 0x7fff7fffu)));
      const uint32_t in4[4] = {raw[r].x, raw[r].y, raw[r].z, raw[r].w};
#pragma unroll
      for (int k = 0; k < 4; ++k) x[r][k] = bf16x2_to_f32x2(in4[k]);
    }
    amax = __uint_as_float(max(top << 16, top & 0xffff0000u));
    if (amax != amax) amax = INFINITY;
  }
  auto block_max = [&](float v) {
#pragma unroll
    for (int m = 16; m >= 1; m >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, m));
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < THREADS / 32; ++w) v = fmaxf(v, red[w]);
    return v;
  };
  amax = block_max(amax);
  if (amax > kLargest) {  // something is not finite (the same for the whole block): the largest of the rest
    amax = 0.f;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int row = r * kRowsPerPass + sub;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float2 z = unpack2(x[r][k]);
        if (row >= lo && row < hi && fabsf(z.x) <= kLargest) amax = fmaxf(amax, fabsf(z.x));
        if (row >= lo && row < hi && fabsf(z.y) <= kLargest) amax = fmaxf(amax, fabsf(z.y));
      }
    }
    __syncthreads();
    amax = block_max(amax);
  }
  const int e = max(need_exponent(amax), e_old);
  const float inv = exp2_int(-e);
  const uint64_t inv2 = pack2(inv, inv);
  if (threadIdx.x == 0) *scale = (uint8_t)(e + 127);
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int row = r * kRowsPerPass + sub;
    uint8_t* dst = code + row * code_token + (PAIR ? 4 : 8) * l;
    if (row >= lo && row < hi) {
      uint32_t o[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float2 z = unpack2(mul2(x[r][k], inv2));
        o[k] = f32x2_to_e4m3x2(z.x, z.y);
      }
      put_codes<PAIR, LANES>(dst, make_uint2(o[0] | o[1] << 16, o[2] | o[3] << 16));
    } else if (row < lo && e > e_old) {  // an older row: its codes move down by e - e_old exponents
      put_codes<PAIR, LANES>(dst, recode(get_codes<PAIR, LANES>(dst), exp2_int(max(e_old - e, -60))));
    }
  }
}

template <int SB, int THREADS>
__global__ void __launch_bounds__(THREADS, 512 / THREADS) cache8_append_kernel(const __grid_constant__ AppendArgs a) {
  extern __shared__ __align__(16) float turns[];  // cosines, then sines: [SB / 8 + 8][rot_dim / 2] each
  __shared__ __align__(16) float unit[16];  // the cosines and sines of no angle
  __shared__ float red[2][THREADS / 32];
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int b = blockIdx.x / a.spans, span = blockIdx.x % a.spans;
  const int n = a.seq_len[b];
  const int64_t start = a.block_table == nullptr ? a.seq_start[b] : 0;
  const bool reports = span == 0 && blockIdx.y == 0 && threadIdx.x == 0;
  if (n < a.T || n > a.max_seq_len) {
    if (reports) flag_status(a.status, CLSA_DEV_BAD_SEQLEN);
    return;
  }
  const int first = n - a.T;                      // position of the first new token
  const int begin = (first / SB + span) * SB;     // first position of this scale block
  if (begin >= n) return;
  const int lo = max(first - begin, 0), hi = min(n - begin, SB);
  const int64_t tok0 = (int64_t)b * a.T + (begin + lo - first);  // the first new token of this block
  const bool idx_block = (int)blockIdx.y >= a.head_groups;       // K_idx; the others K and V of heads h0 .. h1 - 1
  const int h0 = blockIdx.y * a.heads_per_block, h1 = min(h0 + a.heads_per_block, a.heads[0]);
  const int half = a.spec.rot_dim >> 1, lanes = half > 32 ? 64 : 32;  // threads that share a position's angles
  const float freq = !idx_block && (int)threadIdx.x % lanes < half ? a.spec.inv_freq[threadIdx.x % lanes] : 0.f;
  const bool pair = a.spec.rot_dim == 128 && !a.spec.interleaved;  // (K's head size is 128)
  Rows<SB, THREADS, 16> next;
  const int kind0 = idx_block ? 2 : 0;
  if (!idx_block || a.idx_dim == 128)  // the first rows do not depend on where they go
    next.load(a.src[kind0] + tok0 * a.src_token[kind0] + (idx_block ? 0 : h0 * a.src_head[0]), a.src_token[kind0], lo, hi, pair && !idx_block);
  if (start % SB != 0) {
    if (reports) flag_status(a.status, CLSA_DEV_BAD_SCALE_BLOCK);
    return;
  }
  // a multiple of SB: sequences start on one, and pages are whole scale blocks
  const int64_t row0 = cache_row(a.block_table, a.block_shift, a.max_blocks, a.seq_start, a.num_rows, b, begin);
  if (row0 < 0 || row0 + hi > a.num_rows) {
    if (threadIdx.x == 0 && blockIdx.y == 0) flag_status(a.status, CLSA_DEV_BAD_INDEX);
    return;
  }
  const int64_t block = row0 / SB;
  if (idx_block) {
    uint8_t* code = a.code[2] + row0 * a.code_token[2];
    if (a.idx_dim == 64) {
      Rows<SB, THREADS, 8> rows;
      rows.load(a.src[2] + tok0 * a.src_token[2], a.src_token[2], lo, hi, false);
      append_head<SB, THREADS, 8, false>(rows, code, a.code_token[2], a.scale[2] + block, lo, hi, a, nullptr, nullptr, nullptr, red[0]);
    } else {
      append_head<SB, THREADS, 16, false>(next, code, a.code_token[2], a.scale[2] + block, lo, hi, a, nullptr, nullptr, nullptr, red[0]);
    }
    return;
  }
  float* bc = turns;
  float* bs = turns + (SB / 8 + 8) * half;
  if (half > 0) {
    // positions begin + 8 u (with the scale), then 0 .. 7
    const int j = threadIdx.x % lanes;
    if (j < half) {
#pragma unroll 4
      for (int u = threadIdx.x / lanes; u < SB / 8 + 8; u += THREADS / lanes)
        turn_of(u < SB / 8 ? begin + 8 * u : u - SB / 8, freq, u < SB / 8 ? a.spec.rot_scale : 1.f, &bc[u * half + j], &bs[u * half + j]);
    }
    if (threadIdx.x < 16) unit[threadIdx.x] = threadIdx.x < 8 ? 1.f : 0.f;
    __syncthreads();
  }
  const int count = 2 * (h1 - h0);
#pragma unroll 1
  for (int i = 0; i < count; ++i) {  // K of the heads, then V of them
    const int kind = i >= h1 - h0, h = h0 + i - (kind ? h1 - h0 : 0);
    const Rows<SB, THREADS, 16> rows = next;
    if (i + 1 < count) {
      const int k2 = i + 1 >= h1 - h0, h2 = h0 + i + 1 - (k2 ? h1 - h0 : 0);
      next.load(a.src[k2] + tok0 * a.src_token[k2] + h2 * a.src_head[k2], a.src_token[k2], lo, hi, pair && k2 == 0);
    }
    uint8_t* code = a.code[kind] + row0 * a.code_token[kind] + h * a.code_head[kind];
    uint8_t* scale = a.scale[kind] + h * a.scale_head + block;
    if (kind == 0 && pair)
      append_head<SB, THREADS, 16, true, true>(rows, code, a.code_token[kind], scale, lo, hi, a, bc, bs, unit, red[i & 1]);
    else if (kind == 0 && a.has_spec)
      append_head<SB, THREADS, 16, true>(rows, code, a.code_token[kind], scale, lo, hi, a, bc, bs, unit, red[i & 1]);
    else
      append_head<SB, THREADS, 16, false>(rows, code, a.code_token[kind], scale, lo, hi, a, nullptr, nullptr, nullptr, red[i & 1]);
  }
}

// T = 1: a half warp per (sequence, item), two items of one sequence per warp.
constexpr int kTokenThreads = 128;
template <int SB>
__global__ void __launch_bounds__(kTokenThreads) cache8_append_token_kernel(const AppendArgs a) {
  __shared__ __align__(16) float turns[kTokenThreads / 32][2][64];
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, l = lane & 15;
  const int pairs = (a.items + 1) / 2;
  const uint32_t id = blockIdx.x * (kTokenThreads / 32) + warp;
  const int b = (int)(id / (uint32_t)pairs), pair = (int)(id - (uint32_t)b * pairs);
  if (b >= a.num_seqs) return;
  const int item = 2 * pair + (lane >> 4);
  const int kind = item < a.heads[0] ? 0 : (item < a.heads[0] + a.heads[1] ? 1 : 2);
  const int h = item - (kind > 0 ? a.heads[0] : 0) - (kind > 1 ? a.heads[1] : 0);
  const bool mine = item < a.items && (kind < 2 || 8 * l < a.idx_dim);  // this lane holds 8 elements of a row
  const int n = a.seq_len[b];
  const int64_t start = a.block_table == nullptr ? a.seq_start[b] : 0;
  uint4 raw = make_uint4(0, 0, 0, 0);
  if (mine) raw = *reinterpret_cast<const uint4*>(a.src[kind] + b * a.src_token[kind] + h * a.src_head[kind] + 8 * l);
  const bool spec = a.has_spec && 2 * pair < a.heads[0];  // K rows among the warp's two
  const int half = spec ? a.spec.rot_dim >> 1 : 0;
  float w[8], freq[2] = {0.f, 0.f};
  if (spec && a.spec.norm) load_weight8(w, a.k_weight, 8 * l);
#pragma unroll
  for (int i = 0; i < 2; ++i)
    if (lane + 32 * i < half) freq[i] = a.spec.inv_freq[lane + 32 * i];
  if (n < 1 || n > a.max_seq_len) {
    if (pair == 0 && lane == 0) flag_status(a.status, CLSA_DEV_BAD_SEQLEN);
    return;
  }
  const int pos = n - 1, begin = pos / SB * SB, lo = pos - begin;
  if (start % SB != 0) {
    if (pair == 0 && lane == 0) flag_status(a.status, CLSA_DEV_BAD_SCALE_BLOCK);
    return;
  }
  const int64_t row0 = cache_row(a.block_table, a.block_shift, a.max_blocks, a.seq_start, a.num_rows, b, begin);
  if (row0 < 0 || row0 + lo >= a.num_rows) {
    if (pair == 0 && lane == 0) flag_status(a.status, CLSA_DEV_BAD_INDEX);
    return;
  }
  uint8_t* code = a.code[kind] + row0 * a.code_token[kind] + h * a.code_head[kind] + 8 * l;
  uint8_t* scale = a.scale[kind] + h * a.scale_head + row0 / SB;
  const int e_old = mine && lo > 0 ? scale_exponent(*scale) : kScaleExpMin;
  float x[8];
  unpack_bf16x8(x, raw);
  if (spec) {
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = x[i];
    if (a.spec.norm) head_norm<16>(y, w, a.spec.eps);
    if (half > 0) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
        if (lane + 32 * i < half) turn_of(pos, freq[i], a.spec.rot_scale, &turns[warp][0][lane + 32 * i], &turns[warp][1][lane + 32 * i]);
      __syncwarp();
      float c[8], s[8];
      load_turns(c, s, turns[warp][0], turns[warp][1], a.spec.rot_dim, a.spec.interleaved, l);
      head_rotate<16>(y, c, s, a.spec.rot_dim, a.spec.interleaved, l);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = kind == 0 ? y[i] : x[i];
  }
  float amax = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float m = fabsf(x[i]);
    if (m <= 3.4028234663852886e38f) amax = fmaxf(amax, m);  // finite
  }
#pragma unroll
  for (int m = 8; m >= 1; m >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, m));
  if (!mine) return;
  const int e = max(need_exponent(amax), e_old);
  const float inv = exp2_int(-e);
  uint2 v;
  v.x = f32x2_to_e4m3x2(x[0] * inv, x[1] * inv) | f32x2_to_e4m3x2(x[2] * inv, x[3] * inv) << 16;
  v.y = f32x2_to_e4m3x2(x[4] * inv, x[5] * inv) | f32x2_to_e4m3x2(x[6] * inv, x[7] * inv) << 16;
  *reinterpret_cast<uint2*>(code + lo * a.code_token[kind]) = v;
  if (lo > 0 && e > e_old) {  // the block's older rows move down by e - e_old exponents
    const float f = exp2_int(max(e_old - e, -60));
    for (int r0 = 0; r0 < lo; r0 += 8) {
      uint2 old[8];
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (r0 + i < lo) old[i] = *reinterpret_cast<const uint2*>(code + (r0 + i) * a.code_token[kind]);
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (r0 + i < lo) *reinterpret_cast<uint2*>(code + (r0 + i) * a.code_token[kind]) = recode(old[i], f);
    }
  }
  if (l == 0) *scale = (uint8_t)(e + 127);
}

template <int SB, int THREADS>
cudaError_t launch(const AppendArgs& a, unsigned blocks_x, unsigned blocks_y, cudaStream_t stream) {
  const size_t smem = a.has_spec ? (size_t)(SB / 8 + 8) * a.spec.rot_dim * sizeof(float) : 0;
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
  a.num_seqs = p.num_seqs;
  a.T = p.q_per_seq;
  a.max_seq_len = p.max_seq_len;
  a.status = status;
  if (p.q_per_seq == 1) {
    const int64_t warps = (int64_t)p.num_seqs * ((a.items + 1) / 2);
    const unsigned blocks = (unsigned)((warps + kTokenThreads / 32 - 1) / (kTokenThreads / 32));
    switch (c.scale_block) {
      case 16: cache8_append_token_kernel<16><<<blocks, kTokenThreads, 0, stream>>>(a); break;
      case 32: cache8_append_token_kernel<32><<<blocks, kTokenThreads, 0, stream>>>(a); break;
      case 64: cache8_append_token_kernel<64><<<blocks, kTokenThreads, 0, stream>>>(a); break;
      default: cache8_append_token_kernel<128><<<blocks, kTokenThreads, 0, stream>>>(a); break;
    }
    return cudaGetLastError();
  }
  a.spans = (p.q_per_seq - 1 + c.scale_block - 1) / c.scale_block + 1;  // scale blocks that T consecutive positions can touch
  const int64_t bx = (int64_t)p.num_seqs * a.spans;
  // Two or four heads per block where that still leaves about 400 threads per SM: they share the angles, and the later ones' loads
  // are hidden. In us with one, two and four heads (* the rule's choice): 4096 tokens of 8 heads, normed and turned, 16-row blocks
  // 15.3, 12.9, 12.0*; 32-row 12.2, 10.7*, 15.4; 64-row 12.3, 11.7*, 16.7; 128-row 14.0, 12.4*, 20.3; 1024 tokens, 64-row 5.9*, 8.4,
  // 13.8; 7 x 333 tokens of 4 heads, 16-row, as they are 5.0*, 5.1, 7.5, normed and turned 7.4*, 6.8, 9.9; 16 x 256 of 8 heads, 64-row
  // 15.7, 17.3*, 19.1. (The count includes spans that hold no tokens, so many short sequences get four: 64 x 4, 64-row 12.8, 11.3, 17.3*.)
  // Threads: four rows each (32-row blocks with two rows each took 12.8 us instead of 10.5, 128-row blocks with eight 21.2 instead of 11.5).
  const int threads = c.scale_block <= 32 ? 128 : c.scale_block == 64 ? 256 : 512;
  a.heads_per_block = 1;
  while (a.heads_per_block < 4 && bx * ((a.heads[0] + 2 * a.heads_per_block - 1) / (2 * a.heads_per_block)) * threads >= (int64_t)400 * dev.sm_count)
    a.heads_per_block *= 2;
  a.head_groups = (a.heads[0] + a.heads_per_block - 1) / a.heads_per_block;
  const unsigned by = (unsigned)(a.head_groups + a.heads[2]);
  switch (c.scale_block) {
    case 16: return launch<16, 128>(a, (unsigned)bx, by, stream);
    case 32: return launch<32, 128>(a, (unsigned)bx, by, stream);
    case 64: return launch<64, 256>(a, (unsigned)bx, by, stream);
    default: return launch<128, 512>(a, (unsigned)bx, by, stream);
  }
}

}  // namespace clsa
