// Index scores over 8-bit keys (Eq. 3, first half, for a cache of e4m3 codes with a power-of-two scale per block), for up to
// 32 query tokens per sequence: one stream over the keys, bound by HBM (1 byte per element in, 2 T operations on it).
//
// The products run on warp-level f16 matrix instructions: 16 keys x 16 dimensions against up to 8 query tokens. e4m3 codes
// convert to f16 exactly (one conversion instruction per two codes -- the arithmetic that is left beside the loads), and a
// bf16 query row, scaled by a power of two so that its largest magnitude lies in [2^13, 2^14), is exact in f16 down to 2^-31 of it.
// Sums are fp32; the row's and the key's powers of two are applied to the finished sum, which does not round.
// The contraction index inside an instruction is a dummy, so the fragments are taken as the bytes lie: four lanes share a key
// row, a lane takes the row's 16-byte chunks j and j + 4 (the one chunk j of 64-wide keys), and word w of a chunk is its share of
// one step. Every warp streams tiles of 4 KB through a ring of its own: asynchronous 16-byte copies three tiles ahead (192 KB in
// flight per SM), each lane reading back exactly what it copied, so there is no barrier and no shuffle. 16 keys share a page and a
// scale (pages and scale blocks are multiples of 16 rows), so addresses, bounds and scales cost once per 16 keys. Warps take
// chunks of up to four tiles round-robin: all of them read one moving window of the cache, and a sequence's query is converted
// once per chunk. The sequences' lengths wait in shared memory, and a tile's page numbers are fetched one tile before its keys.
// A key's sum does not depend on where the key sits, so equal keys get bit-identical scores (the top-k's tie-break).
// 16 sequences of 128 K keys, one token each: 277 MB in 48.2 us, 5.75 TB/s, 0.89 of a measured copy. 24 ragged sequences of up to
// 32 K 64-wide keys, four tokens each: 11.6 us for 32 MB, the uneven ends and the ramp of the rings. 16 sequences of 32 K keys with
// 8, 16 and 32 tokens: 13.9, 18.7, 30.0 us of 64-wide keys, 21.7, 30.0, 64.2 of 128-wide ones (with 32 tokens some accumulators spill).
#include "attn_common.cuh"
#include "cache8.cuh"

namespace clsa {
namespace {

constexpr int kWarps = 16;
constexpr int kTileBytes = 4096;               // keys of a tile: 32 of 128 dimensions, 64 of 64
constexpr int kStages = 3;
constexpr int kLengths = 2048;                 // sequences whose lengths are kept in shared memory

struct Scores8Args {
  const uint8_t* keys;
  const uint8_t* scale;
  int64_t tok_stride;
  const uint16_t* q;
  const int64_t* seq_start;
  const int32_t* seq_len;
  const int32_t* block_table;
  int block_shift, max_blocks, scale_shift;
  int num_rows;
  uint32_t page_limit;  // pages of the row space (the last one may be cut short)
  float* scores;
  int64_t score_stride;
  int num_seqs, T, causal, max_seq_len;
  int chunk_keys;  // keys a warp takes from one sequence at a time
  uint32_t chunks_per_seq, num_chunks;
  uint32_t* status;
};

// NT: n-tiles of 8 query tokens.
template <int DIDX, int NT>
__global__ void __launch_bounds__(kWarps * 32, 1) index_scores8_kernel(const __grid_constant__ Scores8Args a) {
  constexpr int C = DIDX / 64;                 // 16-byte chunks of a key row that a lane holds
  constexpr int kTileKeys = kTileBytes / DIDX;
  constexpr int M = kTileKeys / 16;            // 16-key groups of a tile
  extern __shared__ __align__(16) unsigned char smem[];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int g = lane >> 2, j = lane & 3;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const unsigned char* mine = smem + warp * (kStages * kTileBytes) + lane * 16;
  const uint32_t mine_u32 = smem_u32(mine);
  // (sequence, position, length) of the tiles in the ring, and the cache rows of their groups (-1: none)
  int4* tiles = reinterpret_cast<int4*>(smem + kWarps * kStages * kTileBytes) + warp * kStages * 2;

  int* lengths = reinterpret_cast<int*>(smem + kWarps * kStages * (kTileBytes + 2 * (int)sizeof(int4)));
  // A sequence's length, 0 if it is refused (flagged by the warp that has its first chunk).
  auto length_of = [&](int b, bool report) -> int {
    const int n = a.seq_len[b];
    const bool bad_len = n < a.T || n > a.max_seq_len;
    if (bad_len || (a.block_table == nullptr && (a.seq_start[b] & ((1 << a.scale_shift) - 1)) != 0)) {
      if (report) flag_status(a.status, bad_len ? CLSA_DEV_BAD_SEQLEN : CLSA_DEV_BAD_SCALE_BLOCK);
      return 0;
    }
    return n;
  };
  for (int i = threadIdx.x; i < min(a.num_seqs, kLengths); i += kWarps * 32) lengths[i] = length_of(i, blockIdx.x == 0);
  __syncthreads();

  // The tiles of this warp in order: chunks `chunk`, + gridDim.x * kWarps, ..; empty ones are passed over. The next tile is known
  // one ahead of its copies, its page numbers on their way.
  uint32_t chunk = blockIdx.x + warp * gridDim.x;
  const uint32_t step = gridDim.x * kWarps;
  int b = -1, s = 0, n = 0, s_end = 0;
  const int32_t* table = nullptr;
  int64_t start = 0;  // (start + position may pass 32 bits where max_seq_len is a loose bound)
  int page[M];
  const bool one_run = a.block_table == nullptr || (1 << a.block_shift) >= kTileKeys;  // a tile's rows follow one another
  auto next_tile = [&]() {  // b = -1 behind the last one
    s += kTileKeys;
    while (s >= s_end) {
      if (chunk >= a.num_chunks) {
        b = -1;
        return;
      }
      b = (int)(chunk / a.chunks_per_seq);
      s = (int)(chunk - (uint32_t)b * a.chunks_per_seq) * a.chunk_keys;
      chunk += step;
      n = b < kLengths ? lengths[b] : length_of(b, s == 0 && lane == 0);
      s_end = min(n, s + a.chunk_keys);
      if (s < s_end) {
        if (a.block_table != nullptr) table = a.block_table + (int64_t)b * a.max_blocks;
        else start = a.seq_start[b];
      }
    }
    if (table != nullptr) {
      page[0] = __ldg(table + (s >> a.block_shift));
      if (!one_run) {
#pragma unroll
        for (int m = 1; m < M; ++m) page[m] = s + 16 * m < n ? __ldg(table + ((s + 16 * m) >> a.block_shift)) : 0;
      }
    }
  };
  const uint8_t* lane_keys = a.keys + g * a.tok_stride + 16 * j;
  const int64_t stride8 = 8 * a.tok_stride;
  auto issue = [&](int slot) {  // the copies of the tile found last, into the ring
    if (b >= 0) {
      int rows[4] = {-1, -1, -1, -1};
      const uint32_t to = mine_u32 + slot * kTileBytes;
      // row of position pos, and how many of `want` rows from it on lie in the row space
      auto locate = [&](int pg, int pos, int want, int& row) -> int {
        row = -1;
        if (table != nullptr) {
          if ((uint32_t)pg < a.page_limit) row = (pg << a.block_shift) + (pos & ((1 << a.block_shift) - 1));
        } else {
          const int64_t r = start + pos;
          if (r >= 0 && r < a.num_rows) row = (int)r;
        }
        const int have = row >= 0 && row < a.num_rows ? min(want, a.num_rows - row) : 0;
        if (have < want && lane == 0) flag_status(a.status, CLSA_DEV_BAD_INDEX);
        return have;
      };
      int row, have = 0;
      if (one_run) have = locate(page[0], s, min(n - s, kTileKeys), row);
      if (have == kTileKeys) {  // the usual tile
        const uint8_t* src = lane_keys + row * a.tok_stride;
#pragma unroll
        for (int r = 0; r < 2 * M; ++r, src += stride8)
#pragma unroll
          for (int c = 0; c < C; ++c)
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;\n" ::"r"(to + (r * C + c) * 512), "l"(src + 64 * c) : "memory");
#pragma unroll
        for (int m = 0; m < M; ++m) rows[m] = row + 16 * m;
      } else {
        const bool whole = one_run && (table != nullptr || row >= 0);  // (a tile that begins before row 0 may end behind it)
#pragma unroll
        for (int m = 0; m < M; ++m) {
          const int pos = s + 16 * m, want = max(min(n - pos, 16), 0);
          const int in = whole ? max(min(have - 16 * m, want), 0) : locate(page[m], pos, want, row);
          const int row_m = whole ? row + 16 * m : row;
          if (in > 0) rows[m] = row_m;
          const uint8_t* src = lane_keys + (in > 0 ? row_m : 0) * a.tok_stride;
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int c = 0; c < C; ++c)  // rows that are none become zeros
              asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;\n" ::"r"(to + ((m * 2 + h) * C + c) * 512),
                           "l"(g + 8 * h < in ? src + h * stride8 + 64 * c : a.keys), "r"(g + 8 * h < in ? 16 : 0) : "memory");
        }
      }
      if (lane == 0) {
        tiles[2 * slot] = make_int4(b, s, n, 0);
        tiles[2 * slot + 1] = make_int4(rows[0], rows[1], rows[2], rows[3]);
      }
      next_tile();
    } else if (lane == 0) {
      tiles[2 * slot] = make_int4(-1, 0, 0, 0);
    }
    cp_async_commit();
  };
  next_tile();
#pragma unroll
  for (int i = 0; i < kStages; ++i) issue(i);
  __syncwarp();

  int cur_b = -1;
  uint32_t qb[NT][C * 4][2];
  float qf[NT][2];  // power of two of query tokens 2j and 2j + 1 of each n-tile
  bool far = false;  // one of them lies outside 2^-60 .. 2^60
  for (int slot = 0;; slot = slot + 1 == kStages ? 0 : slot + 1) {
    const int4 t = tiles[2 * slot];
    if (t.x < 0) break;
    const int4 r4 = tiles[2 * slot + 1];
    const int rows[4] = {r4.x, r4.y, r4.z, r4.w};
    int sb[M];  // the groups' scale bytes, on their way while the copies land
#pragma unroll
    for (int m = 0; m < M; ++m) sb[m] = rows[m] >= 0 ? a.scale[rows[m] >> a.scale_shift] : 127;
    if (t.x != cur_b) {
      cur_b = t.x;
      far = false;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const int tok = nt * 8 + g;
        const uint16_t* q = a.q + ((int64_t)cur_b * a.T + tok) * DIDX + j * 16;
        uint32_t top = 0u;  // bf16 magnitudes order as integers
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
          for (int w = 0; w < 4; w += 2) {
            const uint4 v = tok < a.T ? *reinterpret_cast<const uint4*>(q + 64 * c + 4 * w) : make_uint4(0u, 0u, 0u, 0u);
            qb[nt][c * 4 + w][0] = v.x;
            qb[nt][c * 4 + w][1] = v.y;
            qb[nt][c * 4 + w + 1][0] = v.z;
            qb[nt][c * 4 + w + 1][1] = v.w;
            top = __vmaxu2(__vmaxu2(top, v.x & 0x7fff7fffu), __vmaxu2(v.y & 0x7fff7fffu, __vmaxu2(v.z & 0x7fff7fffu, v.w & 0x7fff7fffu)));
          }
        top = __vmaxu2(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = __vmaxu2(top, __shfl_xor_sync(0xffffffffu, top, 2));
        // (255 - 127: something is not finite, and neither are the scores)
        const int shift = top == 0u ? 0 : min(13 + 127 - (int)(max(top & 0xffffu, top >> 16) >> 7), 120);
        far = far || shift > 60 || shift < -60;
        const float up = exp2_int(shift), down = exp2_int(-shift);
#pragma unroll
        for (int w = 0; w < C * 4; ++w)
#pragma unroll
          for (int i = 0; i < 2; ++i) qb[nt][w][i] = pack_f16x2(bf16_lo(qb[nt][w][i]) * up, bf16_hi(qb[nt][w][i]) * up);
        qf[nt][0] = __shfl_sync(0xffffffffu, down, 8 * j);  // lane (2j, 0) has query token 2j of the tile
        qf[nt][1] = __shfl_sync(0xffffffffu, down, 8 * j + 4);
      }
      far = __any_sync(0xffffffffu, far);
    }
    cp_async_wait<kStages - 1>();
    const unsigned char* data = mine + slot * kTileBytes;
    float acc[M][NT][4];
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) { acc[m][nt][0] = 0.f; acc[m][nt][1] = 0.f; acc[m][nt][2] = 0.f; acc[m][nt][3] = 0.f; }
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const uint4 lo = *reinterpret_cast<const uint4*>(data + ((m * 2) * C + c) * 512), hi = *reinterpret_cast<const uint4*>(data + ((m * 2 + 1) * C + c) * 512);
        const uint32_t wl[4] = {lo.x, lo.y, lo.z, lo.w}, wh[4] = {hi.x, hi.y, hi.z, hi.w};
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const uint32_t a0 = e4m3x2_to_f16x2(wl[w]), a2 = e4m3x2_hi_to_f16x2(wl[w]);
          const uint32_t a1 = e4m3x2_to_f16x2(wh[w]), a3 = e4m3x2_hi_to_f16x2(wh[w]);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) mma_f16(acc[m][nt], a0, a1, a2, a3, qb[nt][c * 4 + w][0], qb[nt][c * 4 + w][1]);
        }
      }
    __syncwarp();  // every lane has read this tile's entry
    issue(slot);
    __syncwarp();
    float kf[M];
#pragma unroll
    for (int m = 0; m < M; ++m) kf[m] = exp2_int(scale_exponent(sb[m]));
    auto put = [&](auto score) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int tok = nt * 8 + 2 * j + i;
          if (tok < a.T) {
            const int left = (a.causal ? t.z - a.T + tok + 1 : t.z) - t.y - g;  // keys that it sees from this lane's first one on
            float* dst = a.scores + ((int64_t)t.x * a.T + tok) * a.score_stride + t.y + g;
#pragma unroll
            for (int m = 0; m < M; ++m)
#pragma unroll
              for (int h = 0; h < 2; ++h)
                if (16 * m + 8 * h < left) dst[16 * m + 8 * h] = score(acc[m][nt][2 * h + i], qf[nt][i], kf[m]);
          }
        }
    };
    // Sums (2^-27 .. 2^30) stay floats under the query's power while that is ordinary. Else the two powers' product (2^-220 .. 2^235) is
    // applied in two halves, so that what lies between is a float wherever the score is. (Halves for every query: 11.1 -> 11.4 us for
    // 24 ragged sequences of four tokens.)
    if (!far) {
      put([](float sum, float q, float k) { return sum * q * k; });
    } else {
      put([](float sum, float q, float k) {
        const int e = (int)(__float_as_uint(q) >> 23) + (int)(__float_as_uint(k) >> 23) - 254;
        return sum * exp2_int(e >> 1) * exp2_int(e - (e >> 1));
      });
    }
  }
  cp_async_wait<0>();
}

// ---- more than 32 query tokens: half of the keys' values as bf16 rows (exact: 2^-110 .. 1.75 * 2^127) for the tensor-core GEMM ----
__global__ void __launch_bounds__(256) index_expand8_kernel(const Scores8Args a, int idx_dim, uint4* out, int64_t* starts,
                                                            int64_t rows_per_seq, int blocks_per_seq) {
  const int per_row = idx_dim / 16;  // 16 codes per thread
  const int b = blockIdx.x / blocks_per_seq, blk = blockIdx.x % blocks_per_seq;
  const int n = a.seq_len[b];
  if (blk == 0 && threadIdx.x == 0) starts[b] = b * rows_per_seq;
  const bool off_block = a.block_table == nullptr && (a.seq_start[b] & ((1 << a.scale_shift) - 1)) != 0;
  const bool bad_len = n < a.T || n > a.max_seq_len;
  if ((bad_len || off_block) && blk == 0 && threadIdx.x == 0) flag_status(a.status, bad_len ? CLSA_DEV_BAD_SEQLEN : CLSA_DEV_BAD_SCALE_BLOCK);
  if (bad_len) return;
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
  const float f = exp2_int(e - 1);
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
  a.num_rows = (int)p.num_cache_rows;
  a.page_limit = (uint32_t)((p.num_cache_rows + (1 << a.block_shift) - 1) >> a.block_shift);
  a.num_seqs = p.num_seqs;
  a.T = p.q_per_seq;
  a.causal = p.causal;
  a.max_seq_len = p.max_seq_len;
  a.status = status;
  return a;
}

template <int DIDX>
cudaError_t launch(const Scores8Args& a, const DeviceInfo& dev, cudaStream_t stream) {
  void (*kernel)(const Scores8Args) = a.T <= 8 ? index_scores8_kernel<DIDX, 1> : a.T <= 16 ? index_scores8_kernel<DIDX, 2> : index_scores8_kernel<DIDX, 4>;
  constexpr int kSmem = kWarps * kStages * (kTileBytes + 2 * (int)sizeof(int4)) + kLengths * (int)sizeof(int);
  const cudaError_t err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
  if (err != cudaSuccess) return err;
  const uint32_t blocks = a.num_chunks < (uint32_t)dev.sm_count ? a.num_chunks : (uint32_t)dev.sm_count;
  kernel<<<blocks, kWarps * 32, kSmem, stream>>>(a);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_index_scores8(const clsa_params& p, const clsa_cache8& c, const void* q_idx, float* scores,
                                 int64_t score_stride, uint32_t* status, const DeviceInfo& dev, cudaStream_t stream) {
  Scores8Args a = make_args(p, c, status);
  a.q = static_cast<const uint16_t*>(q_idx);
  a.scores = scores;
  a.score_stride = score_stride;
  // Four tiles per chunk, fewer where that would leave a warp less than four chunks (us with one, two, four tiles: one sequence of 4 K keys
  // 3.3, 3.8, 5.1, four of 8 K 3.8, 4.2, 5.5, 24 ragged ones of up to 32 K 10.7, 10.6, 11.9; 64 ragged ones of up to 32 K 32.2, 29.1, 30.8).
  const int tile = kTileBytes / p.idx_dim;
  a.chunk_keys = 4 * tile;
  while (a.chunk_keys > tile && (int64_t)p.num_seqs * p.max_seq_len < (int64_t)4 * kWarps * dev.sm_count * a.chunk_keys) a.chunk_keys /= 2;
  a.chunks_per_seq = (uint32_t)((p.max_seq_len + (int64_t)a.chunk_keys - 1) / a.chunk_keys);
  a.num_chunks = (uint32_t)p.num_seqs * a.chunks_per_seq;
  return p.idx_dim == 128 ? launch<128>(a, dev, stream) : launch<64>(a, dev, stream);
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
