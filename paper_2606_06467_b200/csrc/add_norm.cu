// The residual's addition and an RMS norm of the sum, in bf16 and/or in 8 bits with a power-of-two scale per group of elements.
//
//   s = x + residual,   y = s (mean s^2 + eps)^(-1/2) weight,   code = e4m3(y 2^-e)
//
// A few operations per byte: bound by HBM for a prefill chunk, by a launch and two memory round trips for a decode step. A block has one
// row, each thread VECS times 8 consecutive elements (16 bytes of x and of the residual), which stay in registers between
// the sum of squares and the outputs, so that everything is read once and written once. Groups of 32, 64 or 128 elements are 4, 8 or 16
// neighbouring lanes: their largest magnitude is a butterfly; a scale for the whole row takes a second sum over the block's warps.
#include "layer.cuh"

namespace clsa {
namespace {

struct AddNormArgs {
  const uint16_t* x;
  const uint16_t* residual;
  uint16_t* sum_out;
  uint16_t* y_out;
  uint8_t* codes;
  uint8_t* scales;
  const uint16_t* weight;
  int64_t x_stride, residual_stride, sum_stride, y_stride, codes_stride, scales_stride;
  int dim, group;
  float eps, inv_dim;
};

__device__ __forceinline__ uint4 pack8(const float (&v)[8]) {
  return make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
}
// Largest magnitude among the finite ones of 8 numbers.
__device__ __forceinline__ float largest8(const float (&v)[8]) {
  float top = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float a = fabsf(v[i]);
    if (a <= 3.4028234663852886e38f) top = fmaxf(top, a);
  }
  return top;
}

template <int VECS>
__global__ void __launch_bounds__(1024) add_norm_kernel(const __grid_constant__ AddNormArgs a) {
  __shared__ float sums[32], tops[32];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, threads = blockDim.x, warps = threads >> 5;
  const int64_t row = blockIdx.x;
  float s[VECS][8];
  float ss = 0.f;
#pragma unroll
  for (int k = 0; k < VECS; ++k) {
    const int at = 8 * (tid + k * threads);
    uint4 u = make_uint4(0, 0, 0, 0), v = u;
    if (at < a.dim) {
      u = *reinterpret_cast<const uint4*>(a.x + row * a.x_stride + at);
      if (a.residual != nullptr) v = *reinterpret_cast<const uint4*>(a.residual + row * a.residual_stride + at);
    }
    float r[8];
    unpack_bf16x8(s[k], u);
    unpack_bf16x8(r, v);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (a.residual != nullptr) s[k][i] += r[i];
      ss = fmaf(s[k][i], s[k][i], ss);
    }
  }
#pragma unroll
  for (int d = 16; d >= 1; d >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, d);
  if (warps > 1) {
    if (lane == 0) sums[warp] = ss;
    __syncthreads();
    ss = lane < warps ? sums[lane] : 0.f;
#pragma unroll
    for (int d = 16; d >= 1; d >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, d);
  }
  const float r = rsqrtf(fmaf(ss, a.inv_dim, a.eps));
  const bool by_row = a.group == a.dim;
  float top_row = 0.f;
#pragma unroll
  for (int k = 0; k < VECS; ++k) {
    const int at = 8 * (tid + k * threads);
    if (at < a.dim && a.sum_out != nullptr) *reinterpret_cast<uint4*>(a.sum_out + row * a.sum_stride + at) = pack8(s[k]);
    float w[8] = {1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f};
    if (at < a.dim && a.weight != nullptr) unpack_bf16x8(w, *reinterpret_cast<const uint4*>(a.weight + at));
#pragma unroll
    for (int i = 0; i < 8; ++i) s[k][i] = s[k][i] * r * w[i];
    if (at < a.dim && a.y_out != nullptr) *reinterpret_cast<uint4*>(a.y_out + row * a.y_stride + at) = pack8(s[k]);
    if (a.group > 0 && at < a.dim) top_row = fmaxf(top_row, largest8(s[k]));
  }
  if (a.group == 0) return;
  if (by_row) {
#pragma unroll
    for (int d = 16; d >= 1; d >>= 1) top_row = fmaxf(top_row, __shfl_xor_sync(0xffffffffu, top_row, d));
    if (warps > 1) {
      if (lane == 0) tops[warp] = top_row;
      __syncthreads();
      top_row = lane < warps ? tops[lane] : 0.f;
#pragma unroll
      for (int d = 16; d >= 1; d >>= 1) top_row = fmaxf(top_row, __shfl_xor_sync(0xffffffffu, top_row, d));
    }
    if (tid == 0) a.scales[row * a.scales_stride] = (uint8_t)(need_exponent(top_row) + 127);
  }
#pragma unroll
  for (int k = 0; k < VECS; ++k) {
    const int at = 8 * (tid + k * threads);
    float top = top_row;
    if (!by_row) {
      top = at < a.dim ? largest8(s[k]) : 0.f;
      for (int d = a.group / 16; d >= 1; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
    }
    if (at >= a.dim) continue;
    const int e = need_exponent(top);
    if (!by_row && at % a.group == 0) a.scales[row * a.scales_stride + at / a.group] = (uint8_t)(e + 127);
    const float f = exp2_int(-e);
    const uint32_t lo = f32x2_to_e4m3x2(s[k][0] * f, s[k][1] * f) | f32x2_to_e4m3x2(s[k][2] * f, s[k][3] * f) << 16;
    const uint32_t hi = f32x2_to_e4m3x2(s[k][4] * f, s[k][5] * f) | f32x2_to_e4m3x2(s[k][6] * f, s[k][7] * f) << 16;
    *reinterpret_cast<uint2*>(a.codes + row * a.codes_stride + at) = make_uint2(lo, hi);
  }
}

}  // namespace

cudaError_t launch_add_norm(const clsa_add_norm_spec& spec, int num_rows, const clsa_rows* x, const clsa_rows* residual,
                            const clsa_rows* sum_out, const clsa_rows* y_out, const clsa_rows* codes_out, const clsa_rows* scales_out,
                            const DeviceInfo& dev, cudaStream_t stream) {
  (void)dev;
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
  }
  a.weight = static_cast<const uint16_t*>(spec.weight);
  a.dim = spec.dim;
  a.eps = spec.eps;
  a.inv_dim = 1.f / (float)spec.dim;
  const int vecs = (spec.dim + 7) / 8;
  const int per = vecs <= 512 ? 1 : vecs <= 1024 ? 2 : 4;
  const int threads = ((vecs + per - 1) / per + 31) / 32 * 32;
  void (*kernel)(const AddNormArgs) = per == 1 ? add_norm_kernel<1> : per == 2 ? add_norm_kernel<2> : add_norm_kernel<4>;
  kernel<<<(unsigned)num_rows, threads, 0, stream>>>(a);
  return cudaGetLastError();
}

}  // namespace clsa
