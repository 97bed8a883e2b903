// Shared declarations of the 8-bit cache calls: launchers, the e4m3 / e8m0 conversions, the norm and rotation of a head.
#pragma once
#include "clsa_cache8.h"
#include "common.cuh"

namespace clsa {

constexpr int kScaleExpMin = -100, kScaleExpMax = 120;  // exponents that a scale byte may stand for

// Workspace of the 8-bit calls: header | arrival counters of the attention | partial records of the attention, or the bf16
// keys of a chunk's scores. The counters' place and size depend on the device only, so that launches of different shapes
// can follow one another on one workspace.
struct Cache8Layout {
  size_t counter_off, counter_bytes;
  size_t scratch_off;
  size_t attn_bytes;    // partial records
  size_t expand_bytes;  // bf16 keys and their sequence starts (T > kScoresMaxT)
  int64_t expand_rows;  // rows per sequence of the expanded keys
  size_t total;
};
// Query tokens per sequence that the streaming score kernel takes (a fifth tile of eight would not fit its registers). In us, streamed and
// expanded, 32 tokens over 16 x 32 K keys: 64-wide 30.0 and 52.5, 128-wide 64.2 and 74.1; over 33 K keys 5.8 and 10.0, 9.1 and 11.9.
constexpr int kScoresMaxT = 32;

cudaError_t launch_norm_rope(const clsa_norm_rope_spec& spec, int num_tokens, const int32_t* positions, const clsa_heads* q,
                             const clsa_heads* q_out, const clsa_heads* k, const clsa_heads* k_out, const DeviceInfo& dev,
                             cudaStream_t stream);
cudaError_t launch_cache8_append(const clsa_params& p, const clsa_cache8& c, const clsa_norm_rope_spec* spec,
                                 const clsa_heads* k_new, const clsa_heads* v_new, const clsa_heads* idx_new, uint32_t* status,
                                 const DeviceInfo& dev, cudaStream_t stream);
cudaError_t launch_index_scores8(const clsa_params& p, const clsa_cache8& c, const void* q_idx, float* scores,
                                 int64_t score_stride, uint32_t* status, const DeviceInfo& dev, cudaStream_t stream);
// Half of the sequences' 8-bit keys as bf16 rows, sequence b from row b * rows_per_seq, and those starts
cudaError_t launch_index_expand8(const clsa_params& p, const clsa_cache8& c, void* keys, int64_t* starts, int64_t rows_per_seq,
                                 uint32_t* status, const DeviceInfo& dev, cudaStream_t stream);

// Launch shape of the 8-bit attention kernel.
// How the stages are dealt to the workers: one flat list cut evenly; workers of its own for every unit; or whole units per block,
// of which its warps take some whole and share the last ones.
enum : int { kAttn8Flat = 0, kAttn8Units = 1, kAttn8Blocks = 2 };
struct Attn8Plan {
  int warps;            // warps per block
  int blocks, wpb;      // grid, workers per block
  int workers;          // warps that get a span of the stage list
  int mode;             // kAttn8Flat, kAttn8Units or kAttn8Blocks
  int unit_stages;      // 32-token stages per (query row, KV head) unit
  int64_t units, total_stages;
  size_t smem_bytes;
};
Attn8Plan make_attn8_plan(const clsa_params& p, const DeviceInfo& dev);
size_t attn8_counter_bytes(const DeviceInfo& dev);
size_t attn8_partial_bytes(const clsa_params& p, const Attn8Plan& plan);
cudaError_t launch_sparse_attn8(const clsa_params& p, const clsa_cache8& c, const Attn8Plan& plan, const void* q,
                                const int32_t* idx, const int32_t* count, void* out, float* lse, const clsa_attn_hints& hints,
                                uint32_t* status, uint32_t* arrive, float* part, const DeviceInfo& dev, cudaStream_t stream);

#ifdef __CUDACC__
// Scale byte -> its exponent, brought into the range that the format allows.
__device__ __forceinline__ int scale_exponent(int byte) { return min(max(byte, kScaleExpMin + 127), kScaleExpMax + 127) - 127; }
// 2^e for -126 <= e <= 127.
__device__ __forceinline__ float exp2_int(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// Two e4m3 codes (low 16 bits) -> two f16 values (exact), low byte in the low half.
__device__ __forceinline__ uint32_t e4m3x2_to_f16x2(uint32_t codes) {
  uint32_t r;
  asm("{\n\t.reg .b16 t;\n\tcvt.u16.u32 t, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, t;\n\t}" : "=r"(r) : "r"(codes));
  return r;
}
__device__ __forceinline__ uint32_t e4m3x2_hi_to_f16x2(uint32_t codes) {
  uint32_t r;
  asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, h;\n\t}" : "=r"(r) : "r"(codes));
  return r;
}
// Two fp32 values -> two e4m3 codes, nearest even, saturating; `lo` in the low byte.
__device__ __forceinline__ uint32_t f32x2_to_e4m3x2(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ float f16_lo(uint32_t w) {
  float r;
  asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %1;\n\tcvt.f32.f16 %0, l;\n\t}" : "=f"(r) : "r"(w));
  return r;
}
__device__ __forceinline__ float f16_hi(uint32_t w) {
  float r;
  asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %1;\n\tcvt.f32.f16 %0, h;\n\t}" : "=f"(r) : "r"(w));
  return r;
}
__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                        uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Cache row of position s of sequence b, or -1 where it lies outside the row space. (Positions are in range: s < seq_len.)
__device__ __forceinline__ int64_t cache_row(const int32_t* block_table, int block_shift, int max_blocks,
                                             const int64_t* seq_start, int64_t num_rows, int b, int s) {
  int64_t row;
  if (block_table != nullptr)
    row = ((int64_t)block_table[(int64_t)b * max_blocks + (s >> block_shift)] << block_shift) + (s & ((1 << block_shift) - 1));
  else
    row = seq_start[b] + s;
  return row >= 0 && row < num_rows ? row : -1;
}

// Norm and rotation of one head held by a group of D / 8 lanes of a warp, 8 consecutive dimensions each.
struct HeadSpec {
  int norm, rot_dim, interleaved;
  float eps, rot_scale;
  const float* inv_freq;
};
// cos and sin of pos * inv_freq[i]: the product and its reduction to one turn in 64 bits, the functions in 32.
__device__ __forceinline__ void turn_of(int pos, float freq, float scale, float* c, float* s) {
  const double turns = (double)pos * (double)freq * 0.15915494309189533577;  // 1 / (2 pi)
  const float t = (float)(turns - rint(turns));                                // -1/2 .. 1/2
  sincospif(2.f * t, s, c);
  *c *= scale;
  *s *= scale;
}
template <int LANES>
__device__ __forceinline__ void head_norm(float (&x)[8], const float (&w)[8], float eps) {  // the lanes' shares of 32 / LANES heads
  float ss = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) ss = fmaf(x[i], x[i], ss);
#pragma unroll
  for (int m = LANES / 2; m >= 1; m >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, m);
  const float r = rsqrtf(fmaf(ss, 1.f / (8 * LANES), eps));
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = x[i] * r * w[i];
}
// c, s: cosine and sine of each of the lane's 8 dimensions (1 and 0 outside the rotated ones). `l` is the lane's place in
// its group; all lanes of the warp take part.
template <int LANES>
__device__ __forceinline__ void head_rotate(float (&x)[8], const float (&c)[8], const float (&s)[8], int rot_dim,
                                            int interleaved, int l) {
  const bool turned = 8 * l < rot_dim;  // the other lanes keep their values (an infinity times a zero sine is none)
  if (interleaved) {
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      const float a = x[i], b = x[i + 1];
      if (turned) {
        x[i] = fmaf(a, c[i], -b * s[i]);
        x[i + 1] = fmaf(b, c[i + 1], a * s[i + 1]);
      }
    }
  } else {
    const int hl = rot_dim >> 4;  // lanes that hold the first halves of the pairs
    const int src = l < hl ? l + hl : (l < 2 * hl ? l - hl : l);
    const float sign = l < hl ? -1.f : 1.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float o = __shfl_sync(0xffffffffu, x[i], src, LANES);
      if (turned) x[i] = fmaf(x[i], c[i], sign * o * s[i]);
    }
  }
}
// Two fp32 numbers in a register pair: one instruction works on both.
__device__ __forceinline__ uint64_t pack2(float lo, float hi) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ float2 unpack2(uint64_t v) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
  return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t bf16x2_to_f32x2(uint32_t w) { return pack2(bf16_lo(w), bf16_hi(w)); }

__device__ __forceinline__ void unpack_bf16x8(float (&x)[8], const uint4& w) {
  x[0] = bf16_lo(w.x); x[1] = bf16_hi(w.x); x[2] = bf16_lo(w.y); x[3] = bf16_hi(w.y);
  x[4] = bf16_lo(w.z); x[5] = bf16_hi(w.z); x[6] = bf16_lo(w.w); x[7] = bf16_hi(w.w);
}
__device__ __forceinline__ void load_weight8(float (&w)[8], const uint16_t* weight, int at) {
  if (weight != nullptr) unpack_bf16x8(w, *reinterpret_cast<const uint4*>(weight + at));
  else {
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = 1.f;
  }
}
// A lane's 8 cosines and sines from the tables of rot_dim / 2 entries (shared memory).
__device__ __forceinline__ void load_turns(float (&c)[8], float (&s)[8], const float* tc, const float* ts, int rot_dim,
                                           int interleaved, int l) {
  if (8 * l >= rot_dim) {
#pragma unroll
    for (int i = 0; i < 8; ++i) { c[i] = 1.f; s[i] = 0.f; }
  } else if (interleaved) {
    const float4 a = *reinterpret_cast<const float4*>(tc + 4 * l), b = *reinterpret_cast<const float4*>(ts + 4 * l);
    c[0] = c[1] = a.x; c[2] = c[3] = a.y; c[4] = c[5] = a.z; c[6] = c[7] = a.w;
    s[0] = s[1] = b.x; s[2] = s[3] = b.y; s[4] = s[5] = b.z; s[6] = s[7] = b.w;
  } else {
    const int half = rot_dim >> 1, i0 = 8 * l < half ? 8 * l : 8 * l - half;
#pragma unroll
    for (int i = 0; i < 8; i += 4) {
      const float4 a = *reinterpret_cast<const float4*>(tc + i0 + i), b = *reinterpret_cast<const float4*>(ts + i0 + i);
      c[i] = a.x; c[i + 1] = a.y; c[i + 2] = a.z; c[i + 3] = a.w;
      s[i] = b.x; s[i + 1] = b.y; s[i + 2] = b.z; s[i + 3] = b.w;
    }
  }
}
#endif

}  // namespace clsa
