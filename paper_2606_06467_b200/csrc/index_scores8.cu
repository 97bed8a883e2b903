// Index scores over 8-bit keys (Eq. 3, first half, for a cache of e4m3 codes with a power-of-two scale per block), for up to
// 32 query tokens per sequence: one stream over the keys, bound by HBM (1 byte per element in, 2 T operations on it).
//
// The products run on warp-level f16 matrix instructions: 16 keys x 16 dimensions against up to 8 query tokens. e4m3 codes
// convert to f16 exactly (one conversion instruction per two codes -- the arithmetic that is left beside the loads), and a
// bf16 query row, scaled by a power of two so that its largest magnitude lies in [2^13, 2^14), is exact in f16 down to 2^-31 of it.
// Sums are fp32; the row's and the key's powers of two are applied to the finished sum, which does not round.
// The contraction index inside an instruction is a dummy, so the fragments are taken as the bytes lie: a lane loads 32 (16 for
// 64-wide keys) consecutive bytes of one key row with one load, four lanes cover the row, a warp-wide load covers 8 whole rows,
// and word w of the lane's bytes is its share of the instruction's w-th step. No shared memory, no shuffles.
// A key's sum does not depend on where the key sits, so equal keys get bit-identical scores (the top-k's tie-break).
#include "cache8.cuh"

namespace clsa {
namespace {

constexpr int kThreads = 256;
constexpr int kWarpKeys = 32;                           // keys a warp takes at a time: two 16-row tiles
constexpr int kTile = kWarpKeys * (kThreads / 32);      // keys of a block's tile

struct Scores8Args {
  const uint8_t* keys;
  const uint8_t* scale;
  int64_t tok_stride;
  const uint16_t* q;
  const int64_t* seq_start;
  const int32_t* seq_len;
  const int32_t* block_table;
  int block_shift, max_blocks, scale_shift;
  int64_t num_rows;
  float* scores;
  int64_t score_stride;
  int T, causal, max_seq_len, tiles_per_seq;
  int64_t total_tiles;
  uint32_t* status;
};

template <int WORDS>
__device__ __forceinline__ void load_key(uint32_t (&w)[WORDS], const uint8_t* p, bool ok) {
#pragma unroll
  for (int i = 0; i < WORDS; ++i) w[i] = 0u;
  if (!ok) return;
  if constexpr (WORDS == 8) {
    asm volatile("ld.global.L1::no_allocate.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
                 : "l"(p));
  } else {
    asm volatile("ld.global.L1::no_allocate.v4.b32 {%0,%1,%2,%3}, [%4];"
                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "l"(p));
  }
}

// NT: n-tiles of 8 query tokens.
template <int DIDX, int NT, int MIN_BLOCKS>
__global__ void __launch_bounds__(kThreads, MIN_BLOCKS) index_scores8_kernel(const Scores8Args a) {
  constexpr int W = DIDX / 16;  // instruction steps = 32-bit words of a lane's share of a key row
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int g = lane >> 2, j = lane & 3;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  int cur_b = -1;
  uint32_t qb[NT][W][2];
  float qf[NT][2];  // power of two of query tokens 2j and 2j + 1 of each n-tile
  for (int64_t tile = blockIdx.x; tile < a.total_tiles; tile += gridDim.x) {
    const int b = (int)(tile / a.tiles_per_seq);
    const int s0 = (int)(tile % a.tiles_per_seq) * kTile + warp * kWarpKeys;
    const int n = a.seq_len[b];
    if (n < a.T || n > a.max_seq_len) {
      if (threadIdx.x == 0 && s0 == 0) flag_status(a.status, CLSA_DEV_BAD_SEQLEN);
      continue;
    }
    if (s0 >= n) continue;
    // ---- the keys' bytes and scale bytes: everything in flight at once ---------------------------------------------
    uint32_t kw[2][2][W];
    int sb[2][2];
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      const int s = s0 + m * 16;  // 16 positions from here lie in one page
      int64_t row = -1;
      if (s < n) {
        if (a.block_table != nullptr)
          row = ((int64_t)__ldg(a.block_table + (int64_t)b * a.max_blocks + (s >> a.block_shift)) << a.block_shift) +
                (s & ((1 << a.block_shift) - 1));
        else
          row = a.seq_start[b] + s;
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int i = g + 8 * h;
        const int64_t r = row + i;
        const bool live = s + i < n;
        const bool ok = live && row >= 0 && r < a.num_rows;
        if (live && !ok) flag_status(a.status, CLSA_DEV_BAD_INDEX);
        load_key<W>(kw[m][h], a.keys + (ok ? r : 0) * a.tok_stride + j * (4 * W), ok);
        sb[m][h] = ok ? a.scale[r >> a.scale_shift] : 127;
      }
    }
    if (b != cur_b) {
      cur_b = b;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const int t = nt * 8 + g;
        const uint16_t* q = a.q + ((int64_t)b * a.T + t) * DIDX + j * (4 * W);
        uint32_t raw[W][2];
        float amax = 0.f;
#pragma unroll
        for (int w = 0; w < W; ++w) {
          const uint2 v = t < a.T ? *reinterpret_cast<const uint2*>(q + 4 * w) : make_uint2(0u, 0u);
          raw[w][0] = v.x; raw[w][1] = v.y;
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const float lo = fabsf(bf16_lo(raw[w][i])), hi = fabsf(bf16_hi(raw[w][i]));
            if (lo <= 3.4028234663852886e38f) amax = fmaxf(amax, lo);  // finite
            if (hi <= 3.4028234663852886e38f) amax = fmaxf(amax, hi);
          }
        }
        amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
        amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
        const int shift = min(13 + 127 - (int)(__float_as_uint(amax) >> 23), 120);
        const float up = exp2_int(shift), down = exp2_int(-shift);
#pragma unroll
        for (int w = 0; w < W; ++w)
#pragma unroll
          for (int i = 0; i < 2; ++i) qb[nt][w][i] = pack_f16x2(bf16_lo(raw[w][i]) * up, bf16_hi(raw[w][i]) * up);
        qf[nt][0] = __shfl_sync(0xffffffffu, down, 8 * j);      // lane (2j, 0) has query token 2j of the tile
        qf[nt][1] = __shfl_sync(0xffffffffu, down, 8 * j + 4);
      }
    }
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      float acc[NT][4];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) { acc[nt][0] = 0.f; acc[nt][1] = 0.f; acc[nt][2] = 0.f; acc[nt][3] = 0.f; }
#pragma unroll
      for (int w = 0; w < W; ++w) {
        const uint32_t a0 = e4m3x2_to_f16x2(kw[m][0][w]), a2 = e4m3x2_hi_to_f16x2(kw[m][0][w]);
        const uint32_t a1 = e4m3x2_to_f16x2(kw[m][1][w]), a3 = e4m3x2_hi_to_f16x2(kw[m][1][w]);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) mma_f16(acc[nt], a0, a1, a2, a3, qb[nt][w][0], qb[nt][w][1]);
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int s = s0 + m * 16 + g + 8 * h;
        const float kf = exp2_int(scale_exponent(sb[m][h]));
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const int t = nt * 8 + 2 * j + i;
            const int visible = a.causal ? n - a.T + t + 1 : n;
            if (t < a.T && s < visible) a.scores[((int64_t)b * a.T + t) * a.score_stride + s] = acc[nt][2 * h + i] * qf[nt][i] * kf;
          }
      }
    }
  }
}

// ---- more than 32 query tokens: the keys as bf16 rows (exact) for the tensor-core GEMM ---------------------------------
__global__ void __launch_bounds__(256) index_expand8_kernel(const Scores8Args a, int idx_dim, uint4* out, int64_t* starts,
                                                            int64_t rows_per_seq, int blocks_per_seq) {
  const int per_row = idx_dim / 16;  // 16 codes per thread
  const int b = blockIdx.x / blocks_per_seq, blk = blockIdx.x % blocks_per_seq;
  const int n = a.seq_len[b];
  if (blk == 0 && threadIdx.x == 0) starts[b] = b * rows_per_seq;
  if (n < a.T || n > a.max_seq_len) {
    if (blk == 0 && threadIdx.x == 0) flag_status(a.status, CLSA_DEV_BAD_SEQLEN);
    return;
  }
  const int s = (int)(((int64_t)blk * 256 + threadIdx.x) / per_row), part = threadIdx.x % per_row;
  if (s >= n) return;
  const int64_t row = cache_row(a.block_table, a.block_shift, a.max_blocks, a.seq_start, a.num_rows, b, s);
  uint4 w = make_uint4(0, 0, 0, 0);
  int e = 0;
  if (row >= 0) {
    w = *reinterpret_cast<const uint4*>(a.keys + row * a.tok_stride + part * 16);
    e = scale_exponent(a.scale[row >> a.scale_shift]);
  } else if (part == 0) {
    flag_status(a.status, CLSA_DEV_BAD_INDEX);
  }
  const float f = exp2_int(e);
  const uint32_t in[4] = {w.x, w.y, w.z, w.w};
  uint32_t o[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t lo = e4m3x2_to_f16x2(in[i]), hi = e4m3x2_hi_to_f16x2(in[i]);
    o[2 * i] = pack_bf16x2(f16_lo(lo) * f, f16_hi(lo) * f);
    o[2 * i + 1] = pack_bf16x2(f16_lo(hi) * f, f16_hi(hi) * f);
  }
  uint4* dst = out + ((int64_t)b * rows_per_seq + s) * (per_row * 2) + part * 2;
  dst[0] = make_uint4(o[0], o[1], o[2], o[3]);
  dst[1] = make_uint4(o[4], o[5], o[6], o[7]);
}

Scores8Args make_args(const clsa_params& p, const clsa_cache8& c, uint32_t* status) {
  Scores8Args a = {};
  a.keys = static_cast<const uint8_t*>(c.idx_k);
  a.scale = static_cast<const uint8_t*>(c.idx_k_scale);
  a.tok_stride = c.idx_token_stride;
  a.seq_start = p.seq_start;
  a.seq_len = p.seq_len;
  a.block_table = p.block_table;
  while (p.block_table != nullptr && (1 << a.block_shift) < p.block_size) ++a.block_shift;
  a.max_blocks = p.max_blocks_per_seq;
  while ((1 << a.scale_shift) < c.scale_block) ++a.scale_shift;
  a.num_rows = p.num_cache_rows;
  a.T = p.q_per_seq;
  a.causal = p.causal;
  a.max_seq_len = p.max_seq_len;
  a.status = status;
  return a;
}

template <int DIDX>
void launch(const Scores8Args& a, int sm_count, cudaStream_t stream) {
  auto grid = [&](int per_sm) {
    const int64_t g = (int64_t)sm_count * per_sm;
    return (unsigned)(g < a.total_tiles ? g : a.total_tiles);
  };
  if (a.T <= 8) index_scores8_kernel<DIDX, 1, 3><<<grid(3), kThreads, 0, stream>>>(a);
  else if (a.T <= 16) index_scores8_kernel<DIDX, 2, 2><<<grid(2), kThreads, 0, stream>>>(a);
  else index_scores8_kernel<DIDX, 4, 2><<<grid(2), kThreads, 0, stream>>>(a);
}

}  // namespace

cudaError_t launch_index_scores8(const clsa_params& p, const clsa_cache8& c, const void* q_idx, float* scores,
                                 int64_t score_stride, uint32_t* status, const DeviceInfo& dev, cudaStream_t stream) {
  Scores8Args a = make_args(p, c, status);
  a.q = static_cast<const uint16_t*>(q_idx);
  a.scores = scores;
  a.score_stride = score_stride;
  a.tiles_per_seq = (p.max_seq_len + kTile - 1) / kTile;
  a.total_tiles = (int64_t)p.num_seqs * a.tiles_per_seq;
  if (p.idx_dim == 128) launch<128>(a, dev.sm_count, stream);
  else launch<64>(a, dev.sm_count, stream);
  return cudaGetLastError();
}

cudaError_t launch_index_expand8(const clsa_params& p, const clsa_cache8& c, void* keys, int64_t* starts, int64_t rows_per_seq,
                                 uint32_t* status, const DeviceInfo& dev, cudaStream_t stream) {
  (void)dev;
  const Scores8Args a = make_args(p, c, status);
  const int64_t threads = (int64_t)p.max_seq_len * (p.idx_dim / 16);
  const int per_seq = (int)((threads + 255) / 256);
  index_expand8_kernel<<<(unsigned)((int64_t)p.num_seqs * per_seq), 256, 0, stream>>>(a, p.idx_dim, static_cast<uint4*>(keys), starts,
                                                                                      rows_per_seq, per_seq);
  return cudaGetLastError();
}

}  // namespace clsa
