// The residual's addition and an RMS norm of the sum, in bf16 and/or in 8 bits with a power-of-two scale per group of elements.
//
//   s = x + residual,   y = s (mean s^2 + eps)^(-1/2) weight,   code = e4m3(y 2^-e)
//
// A few operations per byte: bound by HBM for a prefill chunk, by a launch and two memory round trips for a decode step. A block has a
// row at a time, each thread VECS times 8 consecutive elements (16 bytes of x and of the residual), which stay in registers between the sum
// of squares and the outputs, so that everything is read once and written once; two elements per fp32 instruction. Groups of 32, 64 or 128
// elements are 4, 8 or 16 neighbouring lanes: their largest magnitude is a butterfly; a scale for the whole row takes a second sum over the
// block's warps. With many rows the blocks stay, keep the weights and fetch AHEAD rows ahead.
// 8192 rows of 5120 with 8-bit output: 294 MB in 50.6 us, 5.8 TB/s, 0.89 of a measured copy (60.1 with a block per row, 61.6 staying but
// at one element per instruction: 284 instructions per 8 elements; 52.2 two rows ahead with two vectors per thread). 4096 rows of 2560: 14.5 (15.7
// with one vector per thread and three rows ahead); 16 rows: 1.8, one launch.
#include "layer.cuh"

namespace clsa {
namespace {

constexpr int kLoopRows = 4;  // rows per SM from which on blocks stay

struct AddNormArgs {
  const uint16_t* x;
  const uint16_t* residual;
  uint16_t* sum_out;
  uint16_t* y_out;
  uint8_t* codes;
  uint8_t* scales;
  const uint16_t* weight;
  int64_t x_stride, residual_stride, sum_stride, y_stride, codes_stride, scales_stride;
  int dim, group, group_shift, num_rows;  // group_shift: of groups of 32, 64, 128
  float eps, inv_dim;
};

__device__ __forceinline__ void unpack4x2(uint64_t (&v)[4], const uint4& w) {
  v[0] = bf16x2_to_f32x2(w.x); v[1] = bf16x2_to_f32x2(w.y); v[2] = bf16x2_to_f32x2(w.z); v[3] = bf16x2_to_f32x2(w.w);
}
__device__ __forceinline__ uint32_t pack_pair(uint64_t v) {
  const float2 f = unpack2(v);
  return pack_bf16x2(f.x, f.y);
}
__device__ __forceinline__ uint4 pack4x2(const uint64_t (&v)[4]) { return make_uint4(pack_pair(v[0]), pack_pair(v[1]), pack_pair(v[2]), pack_pair(v[3])); }
// Largest magnitude among the finite ones of 8 numbers (a NaN loses every maximum).
__device__ __forceinline__ float largest8(const uint64_t (&v)[4]) {
  float top = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = unpack2(v[i]);
    top = fmaxf(top, fmaxf(fabsf(f.x), fabsf(f.y)));
  }
  if (top == INFINITY) {
    top = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = unpack2(v[i]);
      if (fabsf(f.x) < INFINITY) top = fmaxf(top, fabsf(f.x));
      if (fabsf(f.y) < INFINITY) top = fmaxf(top, fabsf(f.y));
    }
  }
  return top;
}

// AHEAD > 0: a block takes rows blockIdx.x, + gridDim.x, ..; the next AHEAD ones' elements are under way while it works on one.
template <int VECS, int AHEAD>
__global__ void __launch_bounds__(AHEAD > 0 ? 512 : 1024) add_norm_kernel(const __grid_constant__ AddNormArgs a) {
  __shared__ float sums[2][32], tops[32];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, warps = blockDim.x >> 5;
  const int step = 8 * blockDim.x;
  constexpr int kHeld = AHEAD > 0 ? AHEAD : 1;
  uint4 u[kHeld][VECS], v[kHeld][VECS];  // x and the residual as they come
  uint64_t w[VECS][4];     // the weights
  bool in[VECS];
  int64_t row = blockIdx.x;
  const uint16_t* x = a.x + row * a.x_stride + 8 * tid;
  const uint16_t* residual = a.residual + row * a.residual_stride + 8 * tid;
  auto load = [&](int64_t of, uint4 (&u)[VECS], uint4 (&v)[VECS]) {  // the rows one after another
    if (of >= a.num_rows) return;
#pragma unroll
    for (int k = 0; k < VECS; ++k) {
      u[k] = v[k] = make_uint4(0, 0, 0, 0);
      if (in[k]) u[k] = __ldcs(reinterpret_cast<const uint4*>(x + k * step));
      if (in[k] && a.residual != nullptr) v[k] = __ldcs(reinterpret_cast<const uint4*>(residual + k * step));
    }
    x += gridDim.x * a.x_stride;
    residual += gridDim.x * a.residual_stride;
  };
#pragma unroll
  for (int k = 0; k < VECS; ++k) in[k] = 8 * tid + k * step < a.dim;
#pragma unroll
  for (int h = 0; h < kHeld; ++h) load(row + h * (int64_t)gridDim.x, u[h], v[h]);
#pragma unroll
  for (int k = 0; k < VECS; ++k) {
    uint4 raw = make_uint4(0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u);  // ones
    if (in[k] && a.weight != nullptr) raw = *reinterpret_cast<const uint4*>(a.weight + 8 * tid + k * step);
    unpack4x2(w[k], raw);
  }
  const bool by_row = a.group == a.dim;
  int turn = 0;
  auto work = [&](uint4 (&u)[VECS], uint4 (&v)[VECS]) {
    uint64_t s[VECS][4];
    uint64_t ss2 = 0ull;
#pragma unroll
    for (int k = 0; k < VECS; ++k) {
      unpack4x2(s[k], u[k]);
      if (a.residual != nullptr) {  // (x alone keeps the sign of its zeros)
        uint64_t r[4];
        unpack4x2(r, v[k]);
#pragma unroll
        for (int i = 0; i < 4; ++i) s[k][i] = add2(s[k][i], r[i]);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) ss2 = fma2(s[k][i], s[k][i], ss2);
    }
    if (AHEAD > 0) load(row + AHEAD * (int64_t)gridDim.x, u, v);
    float ss = unpack2(ss2).x + unpack2(ss2).y;
#pragma unroll
    for (int d = 16; d >= 1; d >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, d);
    if (warps > 1) {
      if (lane == 0) sums[turn][warp] = ss;
      __syncthreads();
      ss = lane < warps ? sums[turn][lane] : 0.f;
#pragma unroll
      for (int d = 16; d >= 1; d >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, d);
    }
    const float r = rsqrtf(fmaf(ss, a.inv_dim, a.eps));
    const uint64_t r2 = pack2(r, r);
    float top_row = 0.f;
    uint16_t* const sum_out = a.sum_out + row * a.sum_stride + 8 * tid;
    uint16_t* const y_out = a.y_out + row * a.y_stride + 8 * tid;
#pragma unroll
    for (int k = 0; k < VECS; ++k) {
      if (in[k] && a.sum_out != nullptr) *reinterpret_cast<uint4*>(sum_out + k * step) = pack4x2(s[k]);
#pragma unroll
      for (int i = 0; i < 4; ++i) s[k][i] = mul2(mul2(s[k][i], r2), w[k][i]);
      if (in[k] && a.y_out != nullptr) *reinterpret_cast<uint4*>(y_out + k * step) = pack4x2(s[k]);
      if (by_row && in[k]) top_row = fmaxf(top_row, largest8(s[k]));
    }
    turn ^= 1;
    if (a.group == 0) return;
    uint8_t* const scales = a.scales + row * a.scales_stride;
    uint8_t* const codes = a.codes + row * a.codes_stride + 8 * tid;
    if (by_row) {
#pragma unroll
      for (int d = 16; d >= 1; d >>= 1) top_row = fmaxf(top_row, __shfl_xor_sync(0xffffffffu, top_row, d));
      if (warps > 1) {
        if (lane == 0) tops[warp] = top_row;
        __syncthreads();  // (the next row's tops come behind its own sums' barrier)
        top_row = lane < warps ? tops[lane] : 0.f;
#pragma unroll
        for (int d = 16; d >= 1; d >>= 1) top_row = fmaxf(top_row, __shfl_xor_sync(0xffffffffu, top_row, d));
      }
      if (tid == 0) *scales = (uint8_t)(need_exponent(top_row) + 127);
    }
#pragma unroll
    for (int k = 0; k < VECS; ++k) {
      float top = top_row;
      if (!by_row) {  // 4, 8 or 16 neighbouring lanes are a group
        top = in[k] ? largest8(s[k]) : 0.f;
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
        if (a.group_shift > 5) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 4));
        if (a.group_shift > 6) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 8));
      }
      if (!in[k]) continue;
      const int at = 8 * tid + k * step, e = need_exponent(top);
      if (!by_row && (at & ((1 << a.group_shift) - 1)) == 0) scales[at >> a.group_shift] = (uint8_t)(e + 127);
      const float f = exp2_int(-e);
      const uint64_t f2 = pack2(f, f);
      uint32_t c[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 z = unpack2(mul2(s[k][i], f2));
        c[i] = f32x2_to_e4m3x2(z.x, z.y);
      }
      *reinterpret_cast<uint2*>(codes + k * step) = make_uint2(__byte_perm(c[0], c[1], 0x5410), __byte_perm(c[2], c[3], 0x5410));
    }
  };
  if (AHEAD == 0) {
    work(u[0], v[0]);
    return;
  }
#pragma unroll 1
  while (true) {
#pragma unroll
    for (int h = 0; h < kHeld; ++h) {
      if (row >= a.num_rows) return;
      work(u[h], v[h]);
      row += gridDim.x;
    }
  }
}

}  // namespace

cudaError_t launch_add_norm(const clsa_add_norm_spec& spec, int num_rows, const clsa_rows* x, const clsa_rows* residual,
                            const clsa_rows* sum_out, const clsa_rows* y_out, const clsa_rows* codes_out, const clsa_rows* scales_out,
                            const DeviceInfo& dev, cudaStream_t stream) {
  AddNormArgs a = {};
  a.x = static_cast<const uint16_t*>(x->data);
  a.x_stride = x->stride;
  if (residual != nullptr) { a.residual = static_cast<const uint16_t*>(residual->data); a.residual_stride = residual->stride; }
  if (sum_out != nullptr) { a.sum_out = static_cast<uint16_t*>(sum_out->data); a.sum_stride = sum_out->stride; }
  if (y_out != nullptr) { a.y_out = static_cast<uint16_t*>(y_out->data); a.y_stride = y_out->stride; }
  if (codes_out != nullptr) {
    a.codes = static_cast<uint8_t*>(codes_out->data);
    a.codes_stride = codes_out->stride;
    a.scales = static_cast<uint8_t*>(scales_out->data);
    a.scales_stride = scales_out->stride;
    a.group = spec.scale_group;
    while (a.group_shift < 7 && (1 << a.group_shift) < a.group) ++a.group_shift;
  }
  a.weight = static_cast<const uint16_t*>(spec.weight);
  a.dim = spec.dim;
  a.eps = spec.eps;
  a.inv_dim = 1.f / (float)spec.dim;
  a.num_rows = num_rows;
  const int vecs = spec.dim / 8;
  // Many rows: blocks that stay and fetch ahead, as many as the registers allow; else a block, of as many threads as fit, for each row.
  // Up to 256 vectors a row: two per thread where that leaves no more lanes idle (8192 rows of 512, 896, 1536, 8-bit output: 6.8, 12.4, 17.9 us with
  // one, 5.9, 11.0, 16.8 with two; of 768, where a quarter would be: 10.0 and 10.4). Beyond: two where two such blocks fit on an SM, else
  // four (4096 rows of 8192, a scale per row: 47 us and 39.6; of 7168, where they fit: 34.9 and 35.8).
  const bool loop = num_rows > kLoopRows * dev.sm_count;
  auto lanes = [&](int per) { return ((vecs + per - 1) / per + 31) / 32 * 32; };
  const int per = loop ? (vecs <= 256 && 2 * lanes(2) > lanes(1) ? 1 : vecs <= 896 ? 2 : 4) : vecs <= 1024 ? 1 : 2;
  const int threads = lanes(per);
  void (*kernel)(const AddNormArgs) = loop ? (per == 1 ? add_norm_kernel<1, 3> : per == 2 ? add_norm_kernel<2, 1> : add_norm_kernel<4, 1>)
                                           : (per == 1 ? add_norm_kernel<1, 0> : add_norm_kernel<2, 0>);
  int64_t blocks = num_rows;
  if (loop) {
    const int regs = per == 1 ? 64 : per == 2 ? 72 : 128;
    int64_t fit = 65536 / ((int64_t)threads * regs);
    if (fit > 32) fit = 32;
    if (fit < 1) fit = 1;
    if (blocks > fit * dev.sm_count) blocks = fit * dev.sm_count;
  }
  kernel<<<(unsigned)blocks, threads, 0, stream>>>(a);
  return cudaGetLastError();
}

}  // namespace clsa
