// Attention of the newest T tokens of every sequence over all of its cached rows, or those of a window.
//
//   x_s = sm_scale q . K_s,   O = sum_s exp(x_s) V_s / sum_s exp(x_s)   over the positions that a query sees
//
// The T queries of a sequence and the query heads of a KV head's group are columns of one product, so that a row of the cache
// is read once for all of them: with up to about 16 columns the launch is bound by HBM.
//
// Work. A granule is 16 or 32 consecutive positions, starting on a multiple of that, of `heads` KV heads; its 16-row parts lie in one
// page and one scale block each. The granules of all (sequence, head group) units form one list, sequence after sequence; its length is
// known on the device only, where every block adds up the lengths and takes an even stretch of the list (to which a unit's beginning and end
// count, too), whatever the sequences' lengths are (or a unit's even share, with the cluster that has the unit, or whole units: make_dense_plan). Four warps fetch granules into rings by tiled bulk
// copies (one for K, one for V: the rows of every head, 128-byte swizzle); eight warps consume them, each with one head's rows: `lanes`
// warps take a head's granules in turn, `col_warps` share a head's query columns. A block that holds several heads reads whole token rows,
// 16 or 32 at a time: what DRAM likes best. Every consuming lane has a ring of its own, so that a slot's rounds are waited for by the same
// warps; a fetching warp's lane has one slot, and waits for it, looks up its next page and issues its copies beside the others.
// Products are formed transposed, tokens along M of warp-level instructions:
//   S^T[16 tokens x 8 columns] = K Q^T,   O^T[128 x 8 columns] += V^T P^T
// Up to 16 columns that is enough to keep up with HBM. Beyond, a block's warps divide the columns, and the instruction rate decides: 64 columns run
// at 0.24 to 0.27 PFLOP/s over bf16 rows, 0.21 over codes, which every column share converts for itself.
//
// Softmax. One pass, in the log2 domain, relative to a reference per column that moves only when a weight would exceed 2^8 (one
// vote per granule, no reduction over its tokens otherwise). Weights are rounded to what the matrix instruction takes beside V. bf16: two
// parts of 8 bits each (p and what its rounding left) where that costs nothing, with up to 32 columns: the error of a single part is as
// large as the output's own rounding (beyond, one: 16 sequences of 8192 tokens, 64 columns, 127 us with it and 157 with two); up to 4 columns are held twice and the second copy takes the second parts. 8-bit caches: f16,
// 2^-11 of each weight, and 2^-36 of the largest one with its V's scale. Denominators are sums of the unrounded weights in fp32.
// Granules that some query sees in part only run a second instance of the step: positions out of sight get logits of -inf, and V rows that nobody sees
// are taken as zeros (a weight of 0 times a NaN is none). Blocks in which a sequence ends pay for it, and for an epilogue and
// queries in the middle of their stretch, with code that comes from memory: about 10 us, which the cut of the list makes up for.
//
// 8-bit caches. Codes convert to f16 exactly; the scale exponents ek, ev are the same for all of a 16-row part, so that they are one number
// per warp: x = (d 2^(ek - 22)) qf with qf = 2^22 sm_scale / (the power of two that q was scaled by). As in the sparse attention,
// numerators have a reference of their own, m near the largest x - mx + ev, and 2^m meets the finished quotient. Scale bytes come with their rows:
// the fetching warp copies the words that they lie in, and the slot's barrier counts those copies (fetched by the consumers, 32 granules at a
// time, they held up whoever began a sequence: 24 ragged sequences of up to 32768 tokens, 15 columns, 103 us, 85 with the words).
//
// Joining. A unit that lies in one stretch is finished by its block. Of the others every block leaves one record per column (128
// unnormalised outputs, reference, sum, in fp32), and a second kernel, whose launch overlaps the first one's end, joins a row's records in
// the order of the stretches. A cluster's blocks send each column's record to the block that finishes it, which joins them in the order of
// their ranks. Results do not depend on timing.
//
// Measured (HBM's measured rate 6.55 TB/s). 16 sequences of 32768 tokens, 32 / 8 heads: bf16 315 us, 6.8 TB/s; 8-bit 168 us, 6.4 TB/s. 24 ragged ones up to
// 32768 tokens in pages of 16 rows: 4 tokens of 32 / 8 heads, bf16, 260 us, 6.4 TB/s; 3 tokens of 20 / 4, 8-bit, 79 us, 5.3 TB/s. The last 512 tokens of
// 64 sequences, 20 / 4 heads: 15.8 us, 4.2 TB/s (a launch's start, one-off code and the joining do not overlap the reading). One sequence
// of 777 tokens and one KV head: 4.9 us, of 8192 tokens and 8 heads 11.4 us, of 131072 tokens 88 us, 6.1 TB/s.
// Slower: granules of 16 rows fetched as 16-byte copies by the fetching warps (one KV head, 64 x 4096 tokens, 8-bit: 43 us for 25 at that time; bf16 45 for
// 41); sixteen consuming warps of one column tile each instead of eight of two (8-bit draft 151 us for 110 at that time).
#include <cuda.h>

#include <atomic>
#include <type_traits>

#include "attn_common.cuh"
#include "dense_units.h"
#include "layer.cuh"

namespace clsa {
namespace {

constexpr int kConsumers = 8;             // consuming warps
constexpr int kProducers = 4;             // .. and fetching ones
constexpr int kThreads = (kConsumers + kProducers) * 32;
constexpr int kConsumerRegs = 224, kProducerRegs = 56;  // 8 x 32 x 224 + 4 x 32 x 56 = 64512 = kThreads x 168, what a launch gets
constexpr int kJoinThreads = 256;
constexpr int kPerLane = 4;                       // sequences to a lane where every warp adds up the lengths by itself
constexpr int kMaxSlots = 24;                     // 24 granules of one head are what shared memory holds
constexpr int kMergeBytes = kConsumers * 8 * kPartialStride * 4;  // a column tile of every consuming warp
constexpr int kCtrlBytes = 1024;
constexpr uint32_t kSpinLimit = 1u << 22;  // polls of a barrier: seconds
constexpr float kLazy = 8.f;
// 8-bit: the numerators' reference lies 2^11 below the largest weight that it was set by and moves when one would exceed 2^15 (f16 ends at 2^16), so that
// f16's smallest steps are 2^-35 of the largest weight and not 2^-24: weights of a long flat tail behind one large weight would be rounded to such steps or to
// nothing, while the denominators count them.
constexpr float kAbove8 = 11.f, kLazy8 = 15.f;
constexpr float kNone = -3.4028234663852886e38f;  // a reference before the first token
constexpr int kHeldBack = 22;                     // of K's exponent, kept for the query's factor: d 2^(ek - 22) is finite and keeps its last bits

struct DenseArgs {
  const uint16_t* q;
  uint16_t* out;
  float* lse;
  uint32_t* status;
  float* part;
  int2* units;  // per (sequence, head group): 2 x the first stretch it lies in + whether another unit is in front of it there, the last one
  const int64_t* seq_start;
  const int32_t* seq_len;
  const int32_t* block_table;
  const uint8_t* ks;
  const uint8_t* vs;
  int64_t scale_head, scale_bytes, num_rows;  // scale_bytes: from the first head's first scale byte to behind the last one's last
  int head_shift;                             // of the heads of a block
  int scale_shift, block_shift, max_blocks, pages;
  int num_seqs, T, num_q_heads, group, columns_used;  // columns_used: T * group
  int window, causal, max_seq_len;
  int gran_shift;   // a granule is 16 or 32 positions
  int two_boxes;    // 1: its two halves are fetched apart (pages of 16 rows)
  int columns, col_tiles, heads, lanes, col_warps, head_groups, slots, lane_slots, spans, min_shift;
  int whole_units;  // 1: a stretch has the units that begin in it, whole
  int cluster;      // > 0: each cluster of so many blocks (2^cluster_shift) has one unit, cut evenly; 0: stretches of the list
  int cluster_shift;
  int pad;          // granules that a unit's beginning and end count for, where the list is cut
  uint32_t ring_inv;   // ceil(2^16 / lane_slots): slot / lane_slots = slot * ring_inv >> 16 for slots below 128
  uint32_t group_inv;  // ceil(2^16 / group): c / group = c * group_inv >> 16 for the columns, of which there are at most 512
  float scale_log2;
};

// ---- barriers and copies --------------------------------------------------------------------------------------------
__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_expect_tx(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ bool mbar_try_wait(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}"
               : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
  return ok != 0;
}
// Bounded wait; false once the limit ran out here or in another role (nothing waits any more then, and the results mean nothing).
__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity, volatile uint32_t* abort_flag) {
  if (mbar_try_wait(bar, parity)) return true;
  for (uint32_t it = 0; it < kSpinLimit; ++it) {
    if (mbar_try_wait(bar, parity)) return true;
    if ((it & 63u) == 63u) {
      if (*abort_flag != 0u) return false;
      __nanosleep(64);
    }
  }
  *abort_flag = 1u;
  return false;
}
__device__ __forceinline__ bool mbar_test(uint32_t bar, uint32_t parity) {  // without waiting
  uint32_t ok;
  asm volatile("{\n.reg .pred p;\nmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}"
               : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
  return ok != 0;
}
// Bounded wait for the records that other blocks of the cluster send, which the barrier counts; false once the limit ran out.
__device__ __forceinline__ bool records_wait(uint32_t bar) {
  for (uint32_t it = 0; it < 4 * kSpinLimit; ++it) {
    uint32_t ok;
    asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], 0;\nselp.u32 %0, 1, 0, p;\n}"
                 : "=r"(ok) : "r"(bar) : "memory");
    if (ok != 0) return true;
    if ((it & 63u) == 63u) __nanosleep(64);
  }
  return false;
}
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
               ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}
__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, int w, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
               ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(w), "r"(bar) : "memory");
}
__device__ __forceinline__ void ldmatrix_b8_x2_trans(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m16n16.x2.trans.shared.b8 {%0,%1,%2,%3}, [%4];\n"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
__device__ __forceinline__ void named_barrier(int id, int threads) { asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory"); }

constexpr int kMaxCluster = 8;
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }
__device__ __forceinline__ uint32_t peer_address(uint32_t at, int block) {  // of a place in the shared memory of a block of the cluster
  uint32_t there;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(at), "r"(block));
  return there;
}
__device__ __forceinline__ void peer_store(uint32_t at, float4 v, uint32_t bar) {  // 16 bytes that a barrier there counts
  asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v4.f32 [%0], {%1, %2, %3, %4}, [%5];"
               ::"r"(at), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w), "r"(bar) : "memory");
}

// ---- which positions and granules a sequence has ----------------------------------------------------------------------
struct Seq {
  int n;      // its length, 0 if it counts as empty
  int first;  // first position that some query sees
  int base;   // .. rounded down to a granule
  int gran;   // granules (one for an empty sequence, whose outputs have to be written too)
  bool bad;
};
__device__ __forceinline__ Seq look_at(const DenseArgs& a, int len) {
  Seq s;
  s.bad = len < (a.causal || a.window ? a.T : 0) || len > a.max_seq_len;
  s.n = s.bad ? 0 : len;
  s.first = a.window ? max(0, s.n - a.T + 1 - a.window) : 0;
  s.base = s.first >> a.gran_shift << a.gran_shift;
  s.gran = max(1, (s.n - s.base + (1 << a.gran_shift) - 1) >> a.gran_shift);
  return s;
}
// How the list of `total` granules is cut: the first total % spans stretches have one more than total / spans.
struct Cut {
  int spans, each, more;
  __device__ __forceinline__ Cut(const DenseArgs& a, int total) {
    spans = min(a.spans, max(1, (total + (1 << a.min_shift) - 1) >> a.min_shift));
    each = (int)((uint32_t)total / (uint32_t)spans);
    more = total - each * spans;
  }
  __device__ __forceinline__ int begin(int s) const { return s * each + min(s, more); }
  __device__ __forceinline__ int owner(int g) const {
    const int big = more * (each + 1);
    return g < big ? (int)((uint32_t)g / (uint32_t)(each + 1)) : more + (int)((uint32_t)(g - big) / (uint32_t)each);
  }
};
// Sum over the block, and of the threads before this one. `sums`: a word for each warp and one more.
template <int THREADS>
__device__ __forceinline__ int block_scan(int v, int* sums, int& before) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int incl = v;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int o = __shfl_up_sync(0xffffffffu, incl, d);
    if (lane >= d) incl += o;
  }
  if (lane == 31) sums[warp] = incl;
  __syncthreads();
  int total = 0;
  before = incl - v;
#pragma unroll
  for (int w = 0; w < THREADS / 32; ++w) {
    const int x = sums[w];
    if (w < warp) before += x;
    total += x;
  }
  __syncthreads();
  return total;
}

// Row r of K's 16 as the first product sees them holds token r for bf16. For codes it is k_token(r), chosen so that a lane's word of the
// transposing 8-bit loads, four consecutive V rows (v_token), holds the tokens whose weights the transposed first product gives
// it, and so that the eight rows that either load reads together lie in different banks of the 128-byte swizzle.
__device__ __forceinline__ int k_token(int r) { return r < 4 ? r : r < 8 ? r + 8 : r - 4; }
__device__ __forceinline__ int v_token(int i) { return k_token(2 * (i >> 2) + (i & 1) + ((i & 2) << 2)); }

__device__ __forceinline__ int token_of(const DenseArgs& a, int col) { return (int)((uint32_t)col * a.group_inv >> 16); }

// Records of partial results (kPartialStride floats: 128 outputs, then mx, l, m) folded into a running one; a lane has four outputs.
struct Folded {
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  float mx = kNone, l = 0.f, m = kNone;
  __device__ __forceinline__ void scale(float f) { acc.x *= f; acc.y *= f; acc.z *= f; acc.w *= f; }
  __device__ __forceinline__ void add(float f, float4 v) {
    acc.x = fmaf(f, v.x, acc.x); acc.y = fmaf(f, v.y, acc.y); acc.z = fmaf(f, v.z, acc.z); acc.w = fmaf(f, v.w, acc.w);
  }
  // One record more, this one's outputs shared with another that has the same head.
  __device__ __forceinline__ void fold_pair(float4 head, float4 v0, float4 v1, Folded& other) {
    const float xn = fmaxf(mx, head.x), mold = (mx - xn) + m, mnew = (head.x - xn) + head.z, mn = fmaxf(mold, mnew);
    const float so = fast_exp2(mold - mn), sn = fast_exp2(mnew - mn);
    l = fmaf(fast_exp2(head.x - xn), head.y, l * fast_exp2(mx - xn));
    mx = xn;
    m = mn;
    scale(so);
    other.scale(so);
    add(sn, v0);
    other.add(sn, v1);
  }
  // Up to 8 records, lane i (mod 8) having the i-th one's head (no_head where there is none) and fetch(i) its outputs.
  template <class F>
  __device__ __forceinline__ void fold8(float4 head, int count, F fetch) {
    float4 v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      v[i] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (i < count) v[i] = fetch(i);
    }
    mx = head.x;
#pragma unroll
    for (int d = 4; d >= 1; d >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
    const float own = (head.x - mx) + head.z;
    m = own;
#pragma unroll
    for (int d = 4; d >= 1; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
    l = fast_exp2(head.x - mx) * head.y;
#pragma unroll
    for (int d = 4; d >= 1; d >>= 1) l += __shfl_xor_sync(0xffffffffu, l, d);
    const float share = fast_exp2(own - m);
#pragma unroll
    for (int i = 0; i < 8; ++i) add(__shfl_sync(0xffffffffu, share, i), v[i]);
  }
  // A few records whose heads every lane of the warp has.
  template <int N>
  __device__ __forceinline__ void fold_few(const float4 (&head)[N], const float4 (&v)[N]) {
    float xn = mx;
#pragma unroll
    for (int i = 0; i < N; ++i) xn = fmaxf(xn, head[i].x);
    const float mold = (mx - xn) + m;
    float mn = mold;
#pragma unroll
    for (int i = 0; i < N; ++i) mn = fmaxf(mn, (head[i].x - xn) + head[i].z);
    l *= fast_exp2(mx - xn);
    scale(fast_exp2(mold - mn));
#pragma unroll
    for (int i = 0; i < N; ++i) {
      l = fmaf(fast_exp2(head[i].x - xn), head[i].y, l);
      add(fast_exp2(((head[i].x - xn) + head[i].z) - mn), v[i]);
    }
    mx = xn;
    m = mn;
  }
  __device__ __forceinline__ void write(const DenseArgs& a, int64_t item, int quad) const {
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    if (l != 0.f) {  // 2^m in two halves: it may not be a float
      const float inv = __fdividef(1.f, l), half = fast_exp2(0.5f * m);
      v = make_float4(acc.x * inv * half * half, acc.y * inv * half * half, acc.z * inv * half * half, acc.w * inv * half * half);
    }
    *reinterpret_cast<uint2*>(a.out + item * 128 + quad * 4) = make_uint2(pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w));
    if (a.lse != nullptr && quad == 0) a.lse[item] = l != 0.f ? (mx + log2f(l)) * kLn2 : -INFINITY;
  }
};
// `count` records that lie `step` apart, outputs 4 quad .. + 7 of each: two running ones that have the same head.
__device__ __forceinline__ void fold_parts(const float4* part, int step, int count, int quad, Folded& f0, Folded& f1) {
  float4 head = part[32], v0 = part[quad], v1 = part[quad + 1];
  f0.acc = v0;
  f1.acc = v1;
  f0.mx = head.x; f0.l = head.y; f0.m = head.z;
  if (count > 1) {
    part += step;
    head = part[32]; v0 = part[quad]; v1 = part[quad + 1];
  }
#pragma unroll 1
  for (int i = count - 1; i > 0; --i) {  // (one ahead)
    const float4 of = head, w0 = v0, w1 = v1;
    if (i > 1) {
      part += step;
      head = part[32]; v0 = part[quad]; v1 = part[quad + 1];
    }
    f0.fold_pair(of, w0, w1, f1);
  }
  f1.mx = f0.mx; f1.l = f0.l; f1.m = f0.m;
}
__device__ __forceinline__ float4 no_head() { return make_float4(kNone, 0.f, kNone, 0.f); }

// The record of column cc of head hh that block `block` leaves of the unit that its stretch begins (which = 0) or ends in (1).
__device__ __forceinline__ float4* record_at(const DenseArgs& a, int block, int which, int hh, int cc) {
  return reinterpret_cast<float4*>(a.part) + ((((int64_t)block * 2 + which) * a.heads + hh) * a.columns + cc) * (kPartialStride / 4);
}

// ---- the kernel --------------------------------------------------------------------------------------------------------
// EIGHT: an 8-bit cache. NT: column tiles per warp (two where there are more than 8 columns: a fragment of the cache feeds both).
// PARTS (bf16): 1, the weights' rounding is all there is; 2, a second product takes what it left; 3 (NT = 1, up to 4 columns), columns 4 .. 7
// repeat the first four and take it. SUB: 16-row parts of a granule. PIPED (SUB = 1): a granule's first product is formed while the one before it is
// finished.
template <bool EIGHT, int NT, int PARTS, int SUB, bool PIPED>
__global__ void __launch_bounds__(kThreads, 1)
dense_attn_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const __grid_constant__ DenseArgs a) {
  extern __shared__ unsigned char smem_dyn[];
  const uint32_t raw = smem_u32(smem_dyn), base = (raw + 1023u) & ~1023u;
  unsigned char* base_ptr = smem_dyn + (base - raw);
  constexpr int kSub = SUB, kGran = 16 * SUB;
  const int row_bytes = EIGHT ? 128 : 256;
  const uint32_t half_bytes = (uint32_t)(a.heads * kGran * row_bytes);  // a slot's K rows, then its V rows
  const uint32_t ring_bytes = (uint32_t)a.slots * 2u * half_bytes;
  float* merge = reinterpret_cast<float*>(base_ptr + ring_bytes);
  unsigned char* ctrl = base_ptr + ring_bytes + kMergeBytes;
  const uint32_t bars = base + ring_bytes + kMergeBytes;
  // Of a cluster: the records of the columns that this block finishes, [column tile][column][block], and barriers that count their bytes. The
  // columns of a tile, of every head and column share, are dealt to the cluster's blocks: column k to block k mod cluster.
  auto inbox_at = [&](int nt, int k) {
    return reinterpret_cast<float*>(ctrl + kCtrlBytes) + (nt * a.heads * a.col_warps * 8 + (k >> a.cluster_shift << a.cluster_shift)) * kPartialStride;
  };
  auto inbox_bar = [&](int nt) { return bars + (uint32_t)kCtrlBytes - 16u + 8u * nt; };
  auto full_bar = [&](int s) { return bars + 16u * s; };
  auto empty_bar = [&](int s) { return bars + 16u * s + 8u; };
  uint32_t* slot_mask = reinterpret_cast<uint32_t*>(ctrl + 16 * kMaxSlots);   // rows of the slot that exist
  uint32_t* slot_blocks = reinterpret_cast<uint32_t*>(ctrl + 20 * kMaxSlots);  // 8-bit: the low two bits of its parts' scale blocks
  volatile uint32_t* abort_flag = reinterpret_cast<volatile uint32_t*>(ctrl + 24 * kMaxSlots);
  // 8-bit: the words that the parts' scale bytes lie in, [slot][part][K, V][head]: 24 x 16 bytes in all. Before that, of use while the
  // block looks for its work:
  uint32_t* slot_scales = reinterpret_cast<uint32_t*>(ctrl + 24 * kMaxSlots + 16);
  int* found = reinterpret_cast<int*>(ctrl + 24 * kMaxSlots + 16);  // first sequence of this block's stretch, granules before it, its length
  int64_t* found_start = reinterpret_cast<int64_t*>(found + 6);  // .. and its first row
  int* sums = found + 8;

  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (tid < a.slots) {
    mbar_init(full_bar(tid), EIGHT ? 1 + 4 * a.heads : 1);  // the rows; lanes' copies of scale bytes
    mbar_init(empty_bar(tid), a.heads * a.col_warps);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  } else if (tid == kMaxSlots) {
    *abort_flag = 0u;
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_k) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_v) : "memory");
  }
  // (Blocks of clusters are (rank, head group, sequence and column tile), of stretches (stretch and column tile).)
  const int HG = a.head_groups;
  const int rank = (int)blockIdx.x, tiled = a.cluster > 0 ? (int)blockIdx.z : (int)blockIdx.x;
  const int span = a.col_tiles > 1 ? tiled / a.col_tiles : tiled, ct = tiled - span * a.col_tiles;
  auto column_of = [&](int k, int nt) {  // the query column; -1 if there is none
    const int col = ct * a.columns + ((k >> 3) & (a.col_warps - 1)) * NT * 8 + nt * 8 + (k & 7);
    return col < a.columns_used && !(PARTS == 3 && (k & 4)) ? col : -1;
  };
  if (a.cluster > 1 && warp > 0 && warp <= NT) {
    const uint32_t bar = inbox_bar(warp - 1);
    int mine = 0;
    for (int k = rank + a.cluster * lane; k < a.heads * a.col_warps * 8; k += a.cluster * 32) mine += column_of(k, warp - 1) >= 0;
    mine = __reduce_add_sync(0xffffffffu, mine);
    if (lane == 0) {
      mbar_init(bar, 1);
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
      mbar_expect_tx(bar, (uint32_t)(mine * a.cluster * kPartialStride * 4));
    }
  }
  __syncthreads();
  if (a.cluster > 1) cluster_arrive();  // (whoever has seen all of the cluster arrive may write to its inboxes)
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");  // behind this grid's own wait, as in every kernel of the library

  // This block's stretch of the list: the first sequence that it reaches into (its number, the granules before it, length and first row), and
  // its granules, span_lo .. span_hi - 1. The list is cut with a.pad places more behind every unit; `place_of` takes a place of that list to the
  // granule there, or the next one.
  auto place_of = [&](int at, int list_base, int granule_base, int gran) {
    const int off = at - list_base, unit = (int)((uint32_t)off / (uint32_t)(gran + a.pad));
    return granule_base + unit * gran + min(off - unit * (gran + a.pad), gran);
  };
  const bool paged = a.block_table != nullptr;
  int total = 0, b_first, base_first, len_first;
  int64_t start_first;
  int span_lo, span_hi, hg_first = 0;
  if (a.cluster > 0) {  // no list: the unit's granules count from 0, those of its sequence's head groups before it below
    b_first = span;
    hg_first = (int)blockIdx.y;
    len_first = a.seq_len[b_first];
    start_first = paged ? 0 : a.seq_start[b_first];
  } else {
    if (a.num_seqs > 32 * kPerLane) {
      int len = 0, gran = 0, before = 0;
      int64_t begin = 0;
      auto read = [&](int i) {
        gran = 0;
        if (i >= a.num_seqs) return;
        len = a.seq_len[i];
        if (!paged) begin = a.seq_start[i];
        gran = look_at(a, len).gran;
      };
      for (int b0 = 0; b0 < a.num_seqs; b0 += kThreads) {
        read(b0 + tid);
        total += block_scan<kThreads>(gran, sums, before);
      }
      total = total * HG + (a.num_seqs * HG - 1) * a.pad;  // (nothing behind the last one)
      const Cut cut(a, total);
      const int from = cut.begin(span), to = cut.begin(span + 1), pad = a.pad * HG;
      if (tid == 0) { found[3] = total; found[5] = total; }
      for (int b0 = 0, run = 0; b0 < a.num_seqs; b0 += kThreads) {
        read(b0 + tid);
        const int sum = block_scan<kThreads>(gran, sums, before);
        const int lo = (run + before) * HG, list = lo + (b0 + tid) * pad, list_end = list + gran * HG + pad;
        if (gran > 0 && list <= from && from < list_end) {
          found[0] = b0 + tid;
          found[1] = lo;
          found[2] = len;
          found[4] = place_of(from, list, lo, gran);
          *found_start = begin;
        }
        if (gran > 0 && list <= to && to < list_end) found[3] = place_of(to, list, lo, gran);
        run += sum;
        if (run * HG + min(a.num_seqs, b0 + kThreads) * pad > to) break;
      }
    } else if (warp == 0) {  // kPerLane sequences to a lane
      int len[kPerLane], gran[kPerLane], mine = 0;
      int64_t begin[kPerLane];
#pragma unroll
      for (int k = 0; k < kPerLane; ++k) {
        const int i = lane * kPerLane + k;
        len[k] = i < a.num_seqs ? a.seq_len[i] : 0;
        begin[k] = i < a.num_seqs && !paged ? a.seq_start[i] : 0;
      }
#pragma unroll
      for (int k = 0; k < kPerLane; ++k) {
        gran[k] = lane * kPerLane + k < a.num_seqs ? look_at(a, len[k]).gran : 0;
        mine += gran[k];
      }
      int incl = mine;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const int o = __shfl_up_sync(0xffffffffu, incl, d);
        if (lane >= d) incl += o;
      }
      const int all = __shfl_sync(0xffffffffu, incl, 31) * HG + (a.num_seqs * HG - 1) * a.pad;  // (nothing behind the last one)
      const Cut cut(a, all);
      const int from = cut.begin(span), to = cut.begin(span + 1), pad = a.pad * HG;
      if (lane == 0) { found[3] = all; found[5] = all; }
      __syncwarp();
      int lo = (incl - mine) * HG, list = lo + lane * kPerLane * pad;
#pragma unroll
      for (int k = 0; k < kPerLane; ++k) {
        const int list_end = list + gran[k] * HG + pad;
        if (gran[k] > 0 && list <= from && from < list_end) {
          found[0] = lane * kPerLane + k;
          found[1] = lo;
          found[2] = len[k];
          found[4] = place_of(from, list, lo, gran[k]);
          *found_start = begin[k];
        }
        if (gran[k] > 0 && list <= to && to < list_end) found[3] = place_of(to, list, lo, gran[k]);
        lo += gran[k] * HG;
        list = list_end;
      }
    }
    __syncthreads();
    total = found[5];
    b_first = found[0];
    base_first = found[1];
    len_first = found[2];
    span_hi = found[3];  // (all of it, unless another stretch begins somewhere)
    span_lo = found[4];
    start_first = *found_start;
    __syncthreads();  // (the place is free now)
  }
  if (a.cluster > 0) {
    const int g = look_at(a, len_first).gran;
    base_first = -hg_first * g;
    span_lo = g * rank >> a.cluster_shift;
    span_hi = g * (rank + 1) >> a.cluster_shift;
  } else if (span >= Cut(a, total).spans) {
    return;
  }
  if (a.whole_units) {  // the units that begin in the stretch, whole
    const int g = look_at(a, len_first).gran;
    span_lo = base_first + (span_lo - base_first + g - 1) / g * g;  // (within the sequence, or the next one's beginning)
  }

  if (warp >= kConsumers) {
    // ---------------- producers: lane i of warp w has slot w + 4 i ----------------
    // (Copies are issued lane by lane: with all slots' in one warp 64 sequences of 4096 tokens of one 8-bit KV head took 34 us.)
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kProducerRegs));
    const int slot = warp - kConsumers + kProducers * lane;
    int b = b_first, seq_base = base_first;
    Seq s = look_at(a, len_first);
    int64_t start = start_first;
    // The ring is one of lane_slots slots for each consuming lane, so that a slot's granules are waited for by the same warps in every round
    // (a warp that waited for a round while the one before had not landed yet would take the parity of the one before that). Granules
    // go to the lanes in turn: slot s holds granules number k = s % lane_slots, + lane_slots, .. of its lane.
    const int ring = (int)((uint32_t)slot * a.ring_inv >> 16);
    int k = slot - ring * a.lane_slots;
    auto list_at = [&]() { return span_lo + k * a.lanes + ring; };
    int at = list_at();  // the place of this lane's next granule in the list
    // its place: position, head group, page table entry
    bool valid, fresh = false;  // fresh: the first granule of its unit
    int pos, hg, entry, entry2 = -1;
    auto place = [&]() {
      valid = slot < a.slots && at < span_hi;
      if (!valid && !(a.whole_units && slot < a.slots)) return;
      while (b < a.num_seqs && at >= seq_base + s.gran * HG) {
        seq_base += s.gran * HG;
        if (++b == a.num_seqs) break;
        s = look_at(a, a.seq_len[b]);
        start = paged ? 0 : a.seq_start[b];
      }
      if (b == a.num_seqs) { valid = false; return; }
      hg = a.cluster > 0 ? hg_first : (int)((uint32_t)(at - seq_base) / (uint32_t)s.gran);
      const int unit = seq_base + hg * s.gran, i = at - unit;
      if (a.whole_units) {
        valid = unit < span_hi;
      } else if (a.cluster == 0 && i == 0 && ct == 0) {
        a.units[(int64_t)b * HG + hg] = make_int2(2 * span + (unit == span_lo ? 0 : 1), Cut(a, total).owner(unit + s.gran - 1 + (b * HG + hg) * a.pad));
      }
      fresh = i == 0;
      pos = s.base + kGran * i;
      entry = entry2 = -1;
      if (paged && valid) {
        const int32_t* row_of_table = a.block_table + (int64_t)b * a.max_blocks;
        if (pos < s.n) entry = row_of_table[pos >> a.block_shift];
        if (kSub == 2 && a.two_boxes && pos + 16 < s.n) entry2 = row_of_table[(pos >> a.block_shift) + 1];
      }
    };
    uint32_t parity = 0;                      // of the round that is waited for
    int row32 = 0, row32b = 0, z = 0;         // row (of its second half, where that is apart) and head of the granule that waits for its slot
    int rounds = -1;                          // .. and the number of this lane's last round
    uint32_t mask = 0u;                       // .. and what of it exists
    bool pending = false, alive = true;
    while (true) {
      // Issue what waits for its slot, and find the next granules' places once that has been tried: their lookups are under way meanwhile.
#pragma unroll 1
      for (uint32_t it = 0;; ++it) {
        const bool ready = pending && mbar_test(empty_bar(slot), parity);
        if (ready) {
          slot_mask[slot] = mask;
          if (EIGHT) slot_blocks[slot] = (uint32_t)(row32 >> a.scale_shift & 3) | (uint32_t)((a.two_boxes ? row32b : row32 + 16) >> a.scale_shift & 3) << 2;
          const uint32_t bar = full_bar(slot), dst = base + (uint32_t)slot * 2u * half_bytes;
          mbar_expect_tx(bar, 2u * half_bytes);
          if (EIGHT) {
            tma_load_3d(dst, &map_k, 0, row32, z, bar);
            tma_load_3d(dst + half_bytes, &map_v, 0, row32, z, bar);
            if (a.two_boxes) {
              tma_load_3d(dst + half_bytes / 2, &map_k, 0, row32b, z, bar);
              tma_load_3d(dst + half_bytes + half_bytes / 2, &map_v, 0, row32b, z, bar);
            }
          } else {
            tma_load_4d(dst, &map_k, 0, row32, z, 0, bar);
            tma_load_4d(dst + half_bytes, &map_v, 0, row32, z, 0, bar);
            if (kSub == 2 && a.two_boxes) {
              tma_load_4d(dst + half_bytes / 2, &map_k, 0, row32b, z, 0, bar);
              tma_load_4d(dst + half_bytes + half_bytes / 2, &map_v, 0, row32b, z, 0, bar);
            }
          }
          pending = false;
          ++rounds;
        }
        if (EIGHT) {  // the scale bytes of the granules just issued: 4 lanes each and head, (part, K or V, head)
          __syncwarp();
          uint32_t todo = __ballot_sync(0xffffffffu, ready);
          while (todo != 0u) {
            uint32_t mine = todo;
#pragma unroll
            for (int k = 1; k < 8; ++k) {
              if (k << (a.head_shift + 2) >= 32) break;
              todo &= todo - 1u;
              if (lane >> (a.head_shift + 2) >= k) mine = todo;
            }
            todo &= todo - 1u;
            const int j = max(__ffs(mine) - 1, 0), its = warp - kConsumers + kProducers * j;
            const int part = lane >> (a.head_shift + 1) & 1, side = lane >> a.head_shift & 1, head = lane & (a.heads - 1);
            const uint32_t there = __shfl_sync(0xffffffffu, mask, j) >> (16 * part) & 0xffffu;
            const int first_row = __shfl_sync(0xffffffffu, row32, j), second_row = __shfl_sync(0xffffffffu, row32b, j);
            const int first_head = __shfl_sync(0xffffffffu, z, j);
            if (mine != 0u) {
              if (there != 0u) {
                const int row = part == 0 ? first_row : a.two_boxes ? second_row : first_row + 16;
                const int64_t at_byte = (int64_t)(first_head + head) * a.scale_head + (row >> a.scale_shift);
                const uint8_t* from = side ? a.vs : a.ks;
                const uint32_t skip = (uint32_t)(reinterpret_cast<uintptr_t>(from + at_byte) & 3u);  // words are copied; not beyond the last byte
                const int64_t left = a.scale_bytes - at_byte + skip;
                const uint32_t dst = smem_u32(slot_scales + (its << (a.head_shift + 2)) + (lane & (4 * a.heads - 1)));
                asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;\n" ::"r"(dst), "l"(from + at_byte - skip), "r"(left < 4 ? (int)left : 4) : "memory");
              }
              asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(full_bar(its)) : "memory");
            }
          }
        }
        if (it == 0) {
          place();
          k += a.lane_slots;
          at = list_at();
          // A unit comes up: its queries on their way to L2 (behind all the rows that are asked for they would take as long as those).
          for (uint32_t todo = __ballot_sync(0xffffffffu, valid && fresh && rounds >= 0); todo != 0u; todo &= todo - 1u) {
            const int j = __ffs(todo) - 1;
            const uint16_t* src = a.q + ((int64_t)__shfl_sync(0xffffffffu, b, j) * a.T * a.num_q_heads + __shfl_sync(0xffffffffu, hg, j) * a.heads * a.group) * 128;
            for (int t = 0; t < a.T; ++t, src += (int64_t)a.num_q_heads * 128)
              for (int k64 = lane; k64 < a.heads * a.group * 2; k64 += 32) asm volatile("prefetch.global.L2 [%0];" ::"l"(src + k64 * 64));
          }
        }
        if (!__any_sync(0xffffffffu, pending)) break;
        if (it > 0) __nanosleep(64);  // (the consumers want the issue slots)
        if (it >= kSpinLimit) *abort_flag = 1u;
        if ((it & 63u) == 63u) {
          if (__any_sync(0xffffffffu, *abort_flag != 0u)) {
            alive = false;
            break;
          }
        }
      }
      if (!alive || !__any_sync(0xffffffffu, valid)) break;
      // the next granule's row, and what of it exists
      pending = valid;
      parity ^= 1u;
      if (valid) {
        bool bad = s.bad;
        uint32_t bad_bit = CLSA_DEV_BAD_SEQLEN;
        if (EIGHT && !paged && (start & 15) != 0) { bad = true; bad_bit = CLSA_DEV_BAD_SCALE_BLOCK; }
        // a box of `rows` rows from cache row `row` on: where to fetch it from (somewhere outside for one of zeros), its rows that exist
        auto box = [&](int64_t row, int rows, int& from) {
          from = -kGran;
          if (row <= -rows || row >= a.num_rows) return 0u;
          from = (int)row;
          uint32_t m = 0xffffffffu >> (32 - rows);
          if (row < 0) m &= 0xffffffffu << (int)-row;
          if (row + rows > a.num_rows) m &= 0xffffffffu >> (int)(32 - (a.num_rows - row));
          return m;
        };
        auto row_of = [&](int of_entry) {
          if (!paged) return start + pos;
          return of_entry >= 0 && of_entry < a.pages ? ((int64_t)of_entry << a.block_shift) + (pos & ((1 << a.block_shift) - 1)) : (int64_t)-kGran;
        };
        if (kSub == 2 && a.two_boxes) {  // (16-row pages: both halves are whole pages)
          mask = box(row_of(entry), 16, row32);
          mask |= box(entry2 >= 0 && entry2 < a.pages ? (int64_t)entry2 << 4 : (int64_t)-kGran, 16, row32b) << 16;
        } else {
          mask = box(row_of(entry), kGran, row32);
        }
        if (bad) {
          flag_status(a.status, bad_bit);
          mask = 0u;
        } else if (mask != 0xffffffffu >> (32 - kGran)) {
          const int from = max(0, s.first - pos), to = min(kGran, s.n - pos);
          const uint32_t wanted = to > from ? (0xffffffffu >> (32 - to)) & (0xffffffffu << from) : 0u;
          if ((wanted & ~mask) != 0u) flag_status(a.status, CLSA_DEV_BAD_INDEX);
        }
        z = hg * a.heads;
      }
    }
    if (!alive) {  // given up: the copies under way still land in this block's memory
      if (lane == 0) flag_status(a.status, CLSA_DEV_TIMEOUT);
      if (rounds >= 0)
        for (uint32_t it = 0; it < kSpinLimit && !mbar_test(full_bar(slot), (uint32_t)rounds & 1u); ++it) __nanosleep(64);
      if (EIGHT) asm volatile("cp.async.wait_all;" ::: "memory");
    }
    return;
  }

  // ---------------- consumers ----------------
  asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kConsumerRegs));
  const int my_cw = warp % a.col_warps, my_head = (warp / a.col_warps) % a.heads, my_lane = warp / (a.col_warps * a.heads);
  const int rowq = lane >> 2, hcol = (lane & 3) * 2, t7 = lane & 7;
  const bool second = PARTS == 3 && (lane & 2) != 0;  // this lane's columns take what the rounding left
  const int G = a.group, T = a.T;
  const int col0 = ct * a.columns + my_cw * NT * 8;
  // the query token of this lane's two columns of each tile (columns past the last one count as the last token's)
  auto tok_of = [&](int nt, int h) { return min(T - 1, token_of(a, col0 + nt * 8 + (PARTS == 3 ? (hcol + h) & 3 : hcol + h))); };
  // this lane's places in a slot's K and V rows (its 16-row parts lie part_step apart)
  const uint32_t part_step = a.two_boxes ? half_bytes / 2 : 2048u, head_at = (uint32_t)my_head * (kSub == 2 && !a.two_boxes ? 4096u : 2048u);
  uint32_t k_at, v_at;
  int row_lo, row_hi;  // tokens of rows rowq and rowq + 8 of the first product
  if (EIGHT) {
    const int kt = k_token(t7 + 8 * ((lane >> 3) & 1)), vt = v_token(lane & 15);
    k_at = base + head_at + (uint32_t)(kt * 128 + (((lane >> 4) ^ (kt & 7)) << 4));
    v_at = base + head_at + (uint32_t)(vt * 128 + (((lane >> 4) ^ (vt & 7)) << 4)) + half_bytes;
    row_lo = k_token(rowq);
    row_hi = k_token(rowq + 8);
  } else {
    const int kt = t7 + 8 * ((lane >> 3) & 1), vt = t7 + 8 * (lane >> 4);
    k_at = base + head_at + (uint32_t)(kt * 128 + (((lane >> 4) ^ t7) << 4));
    v_at = base + head_at + (uint32_t)(vt * 128 + ((((lane >> 3) & 1) ^ t7) << 4)) + half_bytes;
    row_lo = rowq;
    row_hi = rowq + 8;
  }
  const uint32_t upper = half_bytes / (kSub == 2 && a.two_boxes ? 4 : 2);  // from dimensions 0 .. 63 of the bf16 rows to 64 .. 127
  int b = b_first, seq_base = base_first, cur = span_lo, len_b = len_first;
  int seq = 0;                           // granules of this block before the segment
  const int ring0 = my_lane * a.lane_slots;
  int slot = 0;                          // of this lane's ring: its next granule's, and the parity of that round
  uint32_t round = 0;

  bool more = a.cluster > 0 || cur < span_hi;  // (a cluster's block without granules takes part in the joining)
  while (more && b < a.num_seqs) {
    const Seq s = look_at(a, len_b);
    int len_next = 0;  // asked for here and not where it is used
    if (b + 1 < a.num_seqs) asm volatile("ld.global.b32 %0, [%1];" : "=r"(len_next) : "l"(a.seq_len + b + 1));
    for (int hg = a.cluster > 0 ? hg_first : (int)((uint32_t)(cur - seq_base) / (uint32_t)s.gran); hg < HG && more; ++hg) {
      const int unit = seq_base + hg * s.gran;
      const int lo = cur - unit, hi = a.whole_units ? s.gran : min(span_hi - unit, s.gran);
      const int g = hg * a.heads + my_head;  // KV head
      // queries, as B operands: column rowq of a tile
      uint32_t qb[NT][8][2];
      float qf[NT][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const int col = col0 + nt * 8 + (PARTS == 3 ? rowq & 3 : rowq);
        const bool used = col < a.columns_used;
        const int t = token_of(a, col), j = col - t * G;
        const uint16_t* src = a.q + (((int64_t)b * T + t) * a.num_q_heads + g * G + j) * 128;
        if (EIGHT) {
          float amax = 0.f;
#pragma unroll
          for (int st = 0; st < 8; ++st) {  // dimensions 16 st + 4 (lane & 3) .. + 3
            const uint2 v = used ? *reinterpret_cast<const uint2*>(src + 16 * st + 2 * hcol) : make_uint2(0u, 0u);
            qb[nt][st][0] = v.x;
            qb[nt][st][1] = v.y;
          }
#pragma unroll
          for (int st = 0; st < 8; ++st)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              const float x = fabsf(bf16_lo(qb[nt][st][k])), y = fabsf(bf16_hi(qb[nt][st][k]));
              if (x <= 3.4028234663852886e38f) amax = fmaxf(amax, x);  // finite
              if (y <= 3.4028234663852886e38f) amax = fmaxf(amax, y);
            }
          amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
          amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
          const int shift = min(13 + 127 - (int)(__float_as_uint(amax) >> 23), 120);  // largest magnitude into [2^13, 2^14)
          const float up = exp2_int(shift);
#pragma unroll
          for (int st = 0; st < 8; ++st)
#pragma unroll
            for (int k = 0; k < 2; ++k) qb[nt][st][k] = pack_f16x2(bf16_lo(qb[nt][st][k]) * up, bf16_hi(qb[nt][st][k]) * up);
#pragma unroll
          for (int h = 0; h < 2; ++h) {  // scale_log2 2^(kHeldBack - shift), in halves; never 0, so that it leaves a logit of -inf one
            const int e = kHeldBack - __shfl_sync(0xffffffffu, shift, 4 * (hcol + h));
            qf[nt][h] = fminf(fmaxf(a.scale_log2 * exp2_int(e >> 1) * exp2_int(e - (e >> 1)), 1.4012984643e-45f), 3.4028234663852886e38f);
          }
        } else {
#pragma unroll
          for (int ks = 0; ks < 8; ++ks) {  // dimensions 16 ks + hcol, + 1, and those + 8
            qb[nt][ks][0] = used ? *reinterpret_cast<const uint32_t*>(src + ks * 16 + hcol) : 0u;
            qb[nt][ks][1] = used ? *reinterpret_cast<const uint32_t*>(src + ks * 16 + hcol + 8) : 0u;
          }
        }
      }
      float o[NT][8][4], mx[NT][2], m[NT][2], l[NT][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
        for (int h = 0; h < 2; ++h) { mx[nt][h] = kNone; m[nt][h] = EIGHT ? kNone : 0.f; l[nt][h] = 0.f; }
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i) o[nt][j][i] = 0.f;
      }
      // every query sees [all_from, all_to)
      const int all_from = a.window ? max(0, s.n - a.window) : 0, all_to = a.causal ? s.n - T + 1 : s.n;

      // U parts of 16 rows, whose K and V rows are at kb[] and vb[], in two steps. The first product: x, rows rowq (columns hcol, hcol + 1) and
      // rowq + 8.
      auto first_product = [&](auto u_const, const uint32_t* kb, float (*x)[NT][4]) {
        constexpr int U = decltype(u_const)::value;
        constexpr bool kOdd = U * NT == 1;  // two chains of dependent products where there would be one
        float odd[NT][4];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            odd[nt][k] = 0.f;
#pragma unroll
            for (int u = 0; u < U; ++u) x[u][nt][k] = 0.f;
          }
        if (EIGHT) {
#pragma unroll
          for (int st = 0; st < 4; ++st)
#pragma unroll
            for (int u = 0; u < U; ++u) {
              uint32_t kf[4];
              ldmatrix_x4(kf, kb[u] ^ (uint32_t)(st << 5));
#pragma unroll
              for (int k = 0; k < 2; ++k) {
                const uint32_t a0 = e4m3x2_to_f16x2(kf[2 * k]), a2 = e4m3x2_hi_to_f16x2(kf[2 * k]);
                const uint32_t a1 = e4m3x2_to_f16x2(kf[2 * k + 1]), a3 = e4m3x2_hi_to_f16x2(kf[2 * k + 1]);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) mma_f16(kOdd && k ? odd[nt] : x[u][nt], a0, a1, a2, a3, qb[nt][2 * st + k][0], qb[nt][2 * st + k][1]);
              }
            }
        } else {
#pragma unroll
          for (int ks = 0; ks < 8; ++ks)
#pragma unroll
            for (int u = 0; u < U; ++u) {
              uint32_t kf[4];
              ldmatrix_x4(kf, (kb[u] ^ (uint32_t)((ks & 3) << 5)) + (ks & 4 ? upper : 0u));
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) mma_bf16(kOdd && (ks & 1) ? odd[nt] : x[u][nt], kf, qb[nt][ks][0], qb[nt][ks][1]);
            }
        }
        if (kOdd) {
#pragma unroll
          for (int k = 0; k < 4; ++k) x[0][0][k] += odd[0][k];
        }
      };
      // Everything behind it. pos0: the (first) part's first position. MASKED (U = 1): some query does not see all of it, rows_ok has its rows
      // that exist. codes: the scale bytes (8-bit caches): K's, V's.
      auto finish = [&](auto u_const, auto masked_const, int pos0, float (*x)[NT][4], const uint32_t* vb, uint32_t rows_ok, const uint32_t* codes) {
        constexpr int U = decltype(u_const)::value;
        constexpr bool MASKED = decltype(masked_const)::value;
        if constexpr (MASKED) {
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int h = 0; h < 2; ++h) {  // the column's query token sees `seen` positions from `from` on
              const int here = s.n - T + tok_of(nt, h), from = a.window ? max(0, here - a.window + 1) : 0;
              const unsigned seen = (unsigned)max(0, (a.causal ? here + 1 : s.n) - from);
              if ((unsigned)(pos0 + row_lo - from) >= seen || !(rows_ok >> row_lo & 1u)) x[0][nt][h] = -INFINITY;
              if ((unsigned)(pos0 + row_hi - from) >= seen || !(rows_ok >> row_hi & 1u)) x[0][nt][2 + h] = -INFINITY;
            }
        }
        // y: logits in the log2 domain (two columns to a register pair) less their columns' references
        uint64_t y[U][NT][2], kf2[U];
        float ev[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const float kf = EIGHT ? exp2_int(scale_exponent(codes[u] & 255u) - kHeldBack) : a.scale_log2;
          kf2[u] = pack2(kf, kf);
          ev[u] = EIGHT ? (float)scale_exponent(codes[u] >> 8) : 0.f;
        }
        auto relate = [&](int nt) {
          const uint64_t less = pack2(-mx[nt][0], -mx[nt][1]);
#pragma unroll
          for (int u = 0; u < U; ++u)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
              const uint64_t d = pack2(x[u][nt][2 * r], x[u][nt][2 * r + 1]);
              y[u][nt][r] = EIGHT ? add2(mul2(mul2(d, kf2[u]), pack2(qf[nt][0], qf[nt][1])), less) : fma2(d, kf2[u], less);
            }
        };
        // references: moved only where a weight would leave its range
        bool move = false;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          relate(nt);
          float top[2] = {-INFINITY, -INFINITY}, top_e[2] = {-INFINITY, -INFINITY};
#pragma unroll
          for (int u = 0; u < U; ++u) {
            const float2 lo2 = unpack2(y[u][nt][0]), hi2 = unpack2(y[u][nt][1]);
            const float most[2] = {fmaxf(lo2.x, hi2.x), fmaxf(lo2.y, hi2.y)};
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              top[h] = fmaxf(top[h], most[h]);
              if (EIGHT) top_e[h] = fmaxf(top_e[h], most[h] + ev[u]);
            }
          }
          move = move || fmaxf(top[0], top[1]) > kLazy || (EIGHT && (top_e[0] > m[nt][0] + kLazy8 || top_e[1] > m[nt][1] + kLazy8));
        }
        if (__any_sync(0xffffffffu, move)) {
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              float tops[U], top = -INFINITY;
#pragma unroll
              for (int u = 0; u < U; ++u) {
                const float kf = unpack2(kf2[u]).x, d = fmaxf(x[u][nt][h], x[u][nt][h + 2]);  // (the factors are positive)
                tops[u] = EIGHT ? d * kf * qf[nt][h] : d * kf;
#pragma unroll
                for (int d = 4; d <= 16; d <<= 1) tops[u] = fmaxf(tops[u], __shfl_xor_sync(0xffffffffu, tops[u], d));
                top = fmaxf(top, tops[u]);
              }
              const float mxn = fmaxf(mx[nt][h], top), drop = mx[nt][h] - mxn;
              float alpha = fast_exp2(drop);
              l[nt][h] *= alpha;
              mx[nt][h] = mxn;
              if (EIGHT) {
                const float mo = m[nt][h] + drop;
                float mn = mo;
#pragma unroll
                for (int u = 0; u < U; ++u) mn = fmaxf(mn, (tops[u] - mxn) + ev[u] - kAbove8);
                alpha = fast_exp2(mo - mn);
                m[nt][h] = mn;
              }
#pragma unroll
              for (int c = 0; c < 8; ++c) { o[nt][c][h] *= alpha; o[nt][c][h + 2] *= alpha; }
            }
            relate(nt);
          }
        }
        // weights, as the second product's B operand: column rowq of a tile
        uint32_t pb[U][NT][2], pc[U][NT][2];  // (pc: what the rounding of pb left)
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
              const float2 e = unpack2(y[u][nt][r]);
              const float p0 = fast_exp2(e.x), p1 = fast_exp2(e.y);
              const float2 sum = unpack2(add2(pack2(l[nt][0], l[nt][1]), pack2(p0, p1)));
              l[nt][0] = sum.x;
              l[nt][1] = sum.y;
              if (EIGHT) {
                const float2 w = unpack2(add2(y[u][nt][r], pack2(ev[u] - m[nt][0], ev[u] - m[nt][1])));
                pb[u][nt][r] = movmatrix_trans(pack_f16x2(fast_exp2(w.x), fast_exp2(w.y)));
              } else {
                uint32_t first = pack_bf16x2(p0, p1);
                if (PARTS > 1) {
                  const uint32_t rest = pack_bf16x2(p0 - bf16_lo(first), p1 - bf16_hi(first));
                  if (PARTS == 3) first = second ? rest : first;
                  else pc[u][nt][r] = movmatrix_trans(rest);
                }
                pb[u][nt][r] = movmatrix_trans(first);
              }
            }
        auto add_to = [&](float (&d)[4], int u, int nt, const uint32_t (&v)[4]) {
          if (EIGHT) {
            mma_f16(d, v[0], v[1], v[2], v[3], pb[u][nt][0], pb[u][nt][1]);
          } else {
            mma_bf16(d, v, pb[u][nt][0], pb[u][nt][1]);
            if (PARTS == 2) mma_bf16(d, v, pc[u][nt][0], pc[u][nt][1]);
          }
        };
        // O^T += V^T P^T, with the V rows that keep_lo and keep_hi let through
        auto second_product = [&](uint32_t keep_lo, uint32_t keep_hi, auto multiply) {
          if (EIGHT) {
#pragma unroll
            for (int c = 0; c < 8; c += 2)
#pragma unroll
              for (int u = 0; u < U; ++u) {
                uint32_t v[4];
                ldmatrix_b8_x2_trans(v, vb[u] ^ (uint32_t)(c << 4));
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                  const uint32_t v0 = MASKED ? v[2 * j] & keep_lo : v[2 * j], v1 = MASKED ? v[2 * j + 1] & keep_lo : v[2 * j + 1];
                  const uint32_t a4[4] = {e4m3x2_to_f16x2(v0), e4m3x2_to_f16x2(v1), e4m3x2_hi_to_f16x2(v0), e4m3x2_hi_to_f16x2(v1)};
                  multiply(u, c + j, a4);
                }
              }
          } else {
#pragma unroll
            for (int c = 0; c < 8; ++c)
#pragma unroll
              for (int u = 0; u < U; ++u) {
                uint32_t v[4];
                ldmatrix_x4_trans(v, (vb[u] ^ (uint32_t)((c & 3) << 5)) + (c & 4 ? upper : 0u));
                if (MASKED) { v[0] &= keep_lo; v[1] &= keep_lo; v[2] &= keep_hi; v[3] &= keep_hi; }
                multiply(u, c, v);
              }
          }
        };
        auto all_columns = [&](int u, int c, const uint32_t (&v)[4]) {
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) add_to(o[nt][c], u, nt, v);
        };
        if constexpr (!MASKED) {
          second_product(0u, 0u, all_columns);
        } else {
          // Rows that a query does not see have weight 0 there, and 0 times a NaN or an infinity is none: rows that nobody sees count
          // as zeros. V rows of this lane's words: bf16 tokens hcol, + 1 (low and high half), those + 8; codes v_token(4 (lane & 3)) ..
          auto keep = [&](auto visible, uint32_t& k_lo, uint32_t& k_hi) {
            k_lo = k_hi = 0u;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const int row = EIGHT ? v_token(2 * hcol + k) : hcol + (k & 1) + 8 * (k >> 1);
              if (!visible(row)) continue;
              if (EIGHT) k_lo |= 0xffu << (8 * k);
              else if (k < 2) k_lo |= 0xffffu << (16 * k);
              else k_hi |= 0xffffu << (16 * (k - 2));
            }
          };
          uint32_t any_lo, any_hi, all_lo, all_hi;
          keep([&](int row) { return ((rows_ok >> row) & 1u) && pos0 + row >= s.first && pos0 + row < s.n; }, any_lo, any_hi);
          keep([&](int row) { return ((rows_ok >> row) & 1u) && pos0 + row >= all_from && pos0 + row < all_to; }, all_lo, all_hi);
          bool strange = false;  // a number that is not finite in a row that some queries see and others do not
          if (__any_sync(0xffffffffu, any_lo != all_lo || any_hi != all_hi)) {
            const uint32_t part_lo = any_lo & ~all_lo, part_hi = any_hi & ~all_hi;
            auto look = [&](uint32_t w) {
              if (EIGHT) return ((w & 0x7fu) == 0x7fu) | ((w & 0x7f00u) == 0x7f00u) | ((w & 0x7f0000u) == 0x7f0000u) | ((w & 0x7f000000u) == 0x7f000000u);
              return ((w & 0x7f80u) == 0x7f80u) | ((w & 0x7f800000u) == 0x7f800000u);
            };
#pragma unroll 1
            for (int c = 0; c < 8; c += EIGHT ? 2 : 1) {
              uint32_t v[4];
              if (EIGHT) ldmatrix_b8_x2_trans(v, vb[0] ^ (uint32_t)(c << 4));
              else ldmatrix_x4_trans(v, (vb[0] ^ (uint32_t)((c & 3) << 5)) + (c & 4 ? upper : 0u));
#pragma unroll
              for (int k = 0; k < 4; ++k) strange = strange || look(v[k] & (EIGHT || k < 2 ? part_lo : part_hi));
            }
          }
          if (!__any_sync(0xffffffffu, strange)) {
            second_product(any_lo, any_hi, all_columns);
          } else {  // one query token at a time, with the rows that it sees; the other columns' sums are dropped
#pragma unroll 1
            for (int t = 0; t < T; ++t) {
              uint32_t one_lo, one_hi;
              const int here = s.n - T + t, to = a.causal ? here + 1 : s.n;
              keep([&](int row) { return ((rows_ok >> row) & 1u) && pos0 + row < to && (a.window == 0 || pos0 + row > here - a.window); }, one_lo, one_hi);
              second_product(one_lo, one_hi, [&](int u, int c, const uint32_t (&v)[4]) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                  float d[4] = {o[nt][c][0], o[nt][c][1], o[nt][c][2], o[nt][c][3]};
                  add_to(d, u, nt, v);
#pragma unroll
                  for (int k = 0; k < 4; ++k) o[nt][c][k] = tok_of(nt, k & 1) == t ? d[k] : o[nt][c][k];
                }
              });
            }
          }
        }
      };

      // This lane's granules of the block are those with number my_lane mod lanes.
      const int end = seq + hi - lo;
      int n = seq + ((my_lane - seq) & (a.lanes - 1));  // (a power of two)
      const auto all_parts = std::integral_constant<int, kSub>();
      const int pos_step = kGran * a.lanes;
      int pos = s.base + kGran * (lo + n - seq);
      const int last_whole = all_to - kGran;  // every query sees all of a granule from all_from to here
      // 8-bit: where in their words this head's scale bytes lie, but for the block's number
      const uint32_t skip_k = EIGHT ? (uint32_t)(reinterpret_cast<uintptr_t>(a.ks) + g * a.scale_head) & 3u : 0u;
      const uint32_t skip_v = EIGHT ? (uint32_t)(reinterpret_cast<uintptr_t>(a.vs) + g * a.scale_head) & 3u : 0u;
      // With PIPED a granule that every query sees whole has its first product formed while the one before it is finished: `held_x` is that
      // product of the granule whose V rows are at held_vb, in slot held_slot.
      float held_x[kSub][NT][4];
      uint32_t held_vb = 0u;
      int held_slot = -1;
      auto release = [&](int which) {
        __syncwarp();
        if (lane == 0) mbar_arrive(empty_bar(which));
      };
      for (; PIPED || n < end; n += a.lanes, pos += pos_step) {
        const bool any = !PIPED || n < end;
        uint32_t codes[kSub] = {};
        const int here = ring0 + slot;
        const uint32_t off = (uint32_t)here * 2u * half_bytes;
        uint32_t kb[kSub], vb[kSub];
#pragma unroll
        for (int u = 0; u < kSub; ++u) {
          kb[u] = k_at + off + (uint32_t)u * part_step;
          vb[u] = v_at + off + (uint32_t)u * part_step;
        }
        uint32_t rows_ok = 0u;
        if (any) {
          if (!mbar_wait(full_bar(here), round, abort_flag) && lane == 0) flag_status(a.status, CLSA_DEV_TIMEOUT);
          rows_ok = slot_mask[here];
          if (++slot == a.lane_slots) { slot = 0; round ^= 1u; }
          if (EIGHT) {
            const uint32_t blocks = slot_blocks[here];
            const uint32_t* words = slot_scales + (here << (a.head_shift + 2)) + my_head;
#pragma unroll
            for (int u = 0; u < kSub; ++u) {
              const uint32_t block = blocks >> (2 * u);
              const uint32_t k_byte = words[2 * u * a.heads] >> (((skip_k + block) & 3u) * 8u) & 255u;
              const uint32_t v_byte = words[(2 * u + 1) * a.heads] >> (((skip_v + block) & 3u) * 8u) & 255u;
              codes[u] = k_byte | v_byte << 8;
            }
          }
        }
        const bool whole = rows_ok == 0xffffffffu >> (32 - kGran) && pos >= all_from && pos <= last_whole;
        if constexpr (PIPED) {
          static_assert(!PIPED || kSub == 1, "one part");
          if (whole && held_slot >= 0) {
            float x[kSub][NT][4];
            first_product(all_parts, kb, x);
            finish(all_parts, std::false_type(), 0, held_x, &held_vb, 0xffffu, codes);
            release(held_slot);
            held_slot = here;
            held_vb = vb[0];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int k = 0; k < 4; ++k) held_x[0][nt][k] = x[0][nt][k];
            continue;
          }
          if (held_slot >= 0) {
            finish(all_parts, std::false_type(), 0, held_x, &held_vb, 0xffffu, codes);
            release(held_slot);
            held_slot = -1;
          }
          if (!any) break;
          if (whole) {
            first_product(all_parts, kb, held_x);
            held_slot = here;
            held_vb = vb[0];
            continue;
          }
        } else if (whole) {
          first_product(all_parts, kb, held_x);
          finish(all_parts, std::false_type(), 0, held_x, vb, 0xffffu, codes);
          release(here);
          continue;
        }
        // (8-bit: unrolled, because the compiler spills around the loop: the 8-bit draft case 81.5 us and 79. bf16: not, 64 columns 135 and 126.)
#pragma unroll (EIGHT ? kSub : 1)
        for (int u = 0; u < kSub; ++u) {
          const uint32_t kb1 = kb[0] + (uint32_t)u * part_step, vb1 = vb[0] + (uint32_t)u * part_step;
          const uint32_t code1 = u == 0 ? codes[0] : codes[kSub - 1];
          float x[1][NT][4];
          first_product(std::integral_constant<int, 1>(), &kb1, x);
          finish(std::integral_constant<int, 1>(), std::true_type(), pos + 16 * u, x, &vb1, rows_ok >> (16 * u), &code1);
        }
        release(here);
      }
      seq = end;
      cur = unit + hi;
      more = cur < span_hi;

      // ---- what becomes of the segment: the lanes' parts meet in shared memory, a column tile at a time ----------------
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
          for (int d = 4; d <= 16; d <<= 1) l[nt][h] += __shfl_xor_sync(0xffffffffu, l[nt][h], d);
        }
      if (PARTS == 3) {
#pragma unroll
        for (int c = 0; c < 8; ++c)
#pragma unroll
          for (int k = 0; k < 4; ++k) o[0][c][k] += __shfl_xor_sync(0xffffffffu, o[0][c][k], 2);
      }
      const bool whole_unit = lo == 0 && hi == s.gran;
      const int which = lo > 0 || unit == span_lo ? 0 : 1;
      auto together = [&]() {
        if (a.lanes > 1) named_barrier(1 + my_head * a.col_warps + my_cw, a.lanes * 32);
        else __syncwarp();
      };
      // (What follows is formed anew for every segment: the compiler would rather form it ahead, and spill over the work.)
      int this_lane = lane, this_warp = warp;
      asm volatile("" : "+r"(this_lane), "+r"(this_warp));
      const int share = this_warp & (a.heads * a.col_warps - 1), half = this_lane >> 4, quad = 2 * (this_lane & 15);  // (head, column share)
      float* mine = merge + this_warp * 8 * kPartialStride + (this_lane & 3) * 2 * kPartialStride;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          if (PARTS == 3 && second) continue;
          float* dst = mine + h * kPartialStride + (this_lane >> 2);
#pragma unroll
          for (int c = 0; c < 8; ++c) { dst[16 * c] = o[nt][c][h]; dst[16 * c + 8] = o[nt][c][h + 2]; }
          if (this_lane < 4) *reinterpret_cast<float4*>(mine + h * kPartialStride + 128) = make_float4(mx[nt][h], l[nt][h], m[nt][h], 0.f);
        }
        together();
        if (nt == 0 && a.cluster > 1) cluster_wait();  // the inboxes are there
        // the lanes' parts of a column become one: a half warp per column, 8 outputs a lane
        const int cols = min(PARTS == 3 ? 4 : 8, a.columns_used - col0 - nt * 8);
        const int lane_step = a.heads * a.col_warps * 8 * (kPartialStride / 4);
#pragma unroll 1
        for (int c = 2 * my_lane + half; c - half < cols; c += 2 * a.lanes) {
          if (c >= cols) continue;
          const float4* part = reinterpret_cast<const float4*>(merge + (share * 8 + c) * kPartialStride);
          Folded f0, f1;
          fold_parts(part, lane_step, a.lanes, quad, f0, f1);
          const int col = col0 + nt * 8 + c, t = token_of(a, col);
          if (a.cluster > 1) {  // to the block that finishes the column
            const int k = share * 8 + c, owner = k & (a.cluster - 1);
            const uint32_t rec = peer_address(smem_u32(inbox_at(nt, k) + rank * kPartialStride), owner), bar = peer_address(inbox_bar(nt), owner);
            peer_store(rec + 16u * quad, f0.acc, bar);
            peer_store(rec + 16u * quad + 16u, f1.acc, bar);
            if (quad == 0) peer_store(rec + 512u, make_float4(f0.mx, f0.l, f0.m, 0.f), bar);
          } else if (!whole_unit) {  // left for the second kernel to join
            float4* rec = record_at(a, (int)blockIdx.x, which, share / a.col_warps, (share & (a.col_warps - 1)) * NT * 8 + nt * 8 + c);
            rec[quad] = f0.acc;
            rec[quad + 1] = f1.acc;
            if (quad == 0) rec[32] = make_float4(f0.mx, f0.l, f0.m, 0.f);
          } else {
            const int64_t item = ((int64_t)b * T + t) * a.num_q_heads + g * G + (col - t * G);
            f0.write(a, item, quad);
            f1.write(a, item, quad + 1);
          }
        }
        together();
      }
    }
    seq_base += s.gran * HG;
    ++b;
    len_b = len_next;
  }
  if (a.cluster > 1) {  // the columns that this block finishes, once every block's records of them are there
    asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory");  // (its records are on their way; waited for below only)
    bool all_sent = false;
#pragma unroll 1
    for (int nt = 0; nt < NT; ++nt) {
      if (!__all_sync(0xffffffffu, records_wait(inbox_bar(nt)))) {
        // Given up. Records that are still to come would be written to memory that this block has left: it stays until every thread has sent its
        // own (each wait in front of that is bounded, and a block that gave up sends as well), and those on their way have landed.
        if (lane == 0) flag_status(a.status, CLSA_DEV_TIMEOUT);
        if (!all_sent) cluster_wait();
        all_sent = true;
        records_wait(inbox_bar(nt));
      }
#pragma unroll 1
      for (int k = rank + a.cluster * warp; k < a.heads * a.col_warps * 8; k += a.cluster * kConsumers) {
        const int col = column_of(k, nt), head_of = (k >> 3) / a.col_warps, who = lane & 7;
        if (col < 0) continue;
        const float4* rec = reinterpret_cast<const float4*>(inbox_at(nt, k));
        Folded f;
        f.fold8(who < a.cluster ? rec[who * (kPartialStride / 4) + 32] : no_head(), a.cluster, [&](int i) { return rec[i * (kPartialStride / 4) + lane]; });
        const int t = token_of(a, col);
        f.write(a, ((int64_t)b_first * T + t) * a.num_q_heads + (hg_first * a.heads + head_of) * G + (col - t * G), lane);
      }
    }
  }
}

// Joins the records of the rows whose unit several stretches share. A row's part (all 128 outputs, or SPLIT of them 32 each, with a block
// of its own then) has SHARE warps, a warp's lanes 4 outputs each of SPLIT records at a time; a lane has BATCH records in flight.
template <int SHARE, int SPLIT, int BATCH>
__global__ void __launch_bounds__(kJoinThreads) dense_join_kernel(const __grid_constant__ DenseArgs a) {
  constexpr int kWarps = kJoinThreads / 32, kParts = kWarps / SHARE, kWide = 32 / SPLIT;  // lanes of a record
  __shared__ float4 heads[SHARE * SPLIT > 1 ? kWarps * SPLIT : 1], sums[SHARE * SPLIT > 1 ? kWarps * 32 : 1];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, sub = lane / kWide;
  const int64_t part = (int64_t)blockIdx.x * kParts + warp / SHARE, row = part / SPLIT;  // (sequence, token, head)
  const int quad = (int)(part % SPLIT) * kWide + lane % kWide;                              // of the row's outputs
  const int own = warp % SHARE * SPLIT + sub;
  const int h = (int)(row % a.num_q_heads), t = (int)(row / a.num_q_heads % a.T), b = (int)(row / a.num_q_heads / a.T);
  const int g = h / a.group, hg = g / a.heads, hh = g - hg * a.heads, col = t * a.group + (h - g * a.group), ct = col / a.columns, cc = col - ct * a.columns;
  // a stretch's records lie `step` apart, the first one's perhaps among those of the units that it ends in
  const float4* from = record_at(a, ct, 0, hh, cc);
  const int64_t step = (int64_t)a.col_tiles * 2 * a.heads * a.columns * (kPartialStride / 4);
  asm volatile("griddepcontrol.wait;" ::: "memory");
  int2 unit = make_int2(0, 0);
  if (b < a.num_seqs) unit = __ldcg(&a.units[(int64_t)b * a.head_groups + hg]);
  const int first = unit.x >> 1, last = unit.y;
  const Noted noted = noted_unit(unit.x, unit.y, a.spans);
  const bool joined = noted == Noted::kCut;
  if (noted == Noted::kNever && lane == 0) flag_status(a.status, CLSA_DEV_TIMEOUT);  // (a fetching warp gave up before this unit)
  if (SHARE == 1 ? !joined : !__syncthreads_or(joined)) return;
  const int aside = unit.x & 1 ? a.heads * a.columns * (kPartialStride / 4) : 0;
  Folded f;
  if (joined) {
    for (int s0 = first + own; s0 <= last; s0 += BATCH * SHARE * SPLIT) {
      float4 head[BATCH], v[BATCH];
      const float4* at = from + s0 * step;
#pragma unroll
      for (int i = 0; i < BATCH; ++i) {
        head[i] = no_head();
        v[i] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (s0 + i * SHARE * SPLIT <= last) {
          const float4* rec = at + (i == 0 && s0 == first ? aside : 0);
          head[i] = __ldcg(rec + 32);
          v[i] = __ldcg(rec + quad);
        }
        at += SHARE * SPLIT * step;
      }
      f.fold_few(head, v);
    }
  }
  if (SHARE * SPLIT > 1) {
    sums[warp * 32 + lane] = f.acc;
    if (lane % kWide == 0) heads[warp * SPLIT + sub] = make_float4(f.mx, f.l, f.m, 0.f);
    __syncthreads();
    if (warp % SHARE != 0 || sub != 0 || !joined) return;
    f = Folded();
#pragma unroll
    for (int w = 0; w < SHARE; w += 4 / SPLIT) {  // four partial sums at a time
      float4 head[4], v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int from_warp = warp + w + i / SPLIT, k = i % SPLIT;
        head[i] = no_head();
        v[i] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (w + i / SPLIT < SHARE) {
          head[i] = heads[from_warp * SPLIT + k];
          v[i] = sums[from_warp * 32 + k * kWide + lane];
        }
      }
      f.fold_few(head, v);
    }
  }
  f.write(a, row, quad);
}

// ---- host side ---------------------------------------------------------------------------------------------------------
using EncodeTiledFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                   const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                   CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiledFn encode_tiled_fn() {
  static EncodeTiledFn fn = nullptr;
  if (fn == nullptr) {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult qres;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &qres) != cudaSuccess || qres != cudaDriverEntryPointSuccess)
      return nullptr;
    fn = reinterpret_cast<EncodeTiledFn>(p);
  }
  return fn;
}

// K or V rows as boxes of `rows` rows of `heads` heads. bf16: [half][head][row][64 elements], codes: [head][row][128].
bool make_map(CUtensorMap* map, const void* ptr, bool eight, const clsa_params& p, int64_t token_stride, int64_t head_stride, int heads, int rows) {
  EncodeTiledFn fn = encode_tiled_fn();
  if (fn == nullptr) return false;
  const cuuint64_t size = eight ? 1 : 2;
  if (p.num_kv_heads == 1) head_stride = 128;  // of one head it means nothing
  const cuuint64_t dims[4] = {eight ? 128u : 64u, (cuuint64_t)p.num_cache_rows, (cuuint64_t)p.num_kv_heads, 2};
  const cuuint64_t strides[3] = {(cuuint64_t)token_stride * size, (cuuint64_t)head_stride * size, 128};
  const cuuint32_t box[4] = {eight ? 128u : 64u, (cuuint32_t)rows, (cuuint32_t)heads, 2};
  const cuuint32_t estr[4] = {1, 1, 1, 1};
  return fn(map, eight ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, eight ? 3 : 4, const_cast<void*>(ptr), dims,
            strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace

// Three ways of dealing the work. Stretches of the list, cut anywhere: even whatever the lengths are, but a second kernel joins them.
// A cluster of blocks per unit, where all fit on the GPU at once: joined in shared memory, but the longest sequence decides. Whole units:
// nothing to join, the longest stretch of them decides. Chosen by an estimate from the longest sequence that the call allows: a block gets its
// share of HBM, but no more than kBlockRate (or what its products keep up with); a cluster's joining costs 0.8 us. Stretches count as 14 us and 0.7 of
// the bytes, between even lengths (measured as 9 us and all of them) and ragged ones. 32 / 8 heads, bf16, us, stretches and clusters (of one block where
// units are enough): 1 x 8192 tokens 19.3 and 11.6, 4 x 4096 21.2 and 15.6 (lengths from 205 to 4096: 16.7 and 12.0), 16 x 4096 50.4 and 44.3 (32.6 and
// 29.4), 4 x 16384 49.9 and 43.2 (33.2 and 33.0); 20 x 8192 107.7 and 103 (54.5 and 64.4), which goes to stretches. 8-bit: 17.7 and 11.1 (14.1 and
// 9.5), 33.1 and 27.0 (24.3 and 22.8), 33.0 and 28.1 (25.5 and 25.3); 62.5 and 65.1 (35.5 and 51.7).
// Fourteen clusters of 8 find place at once, 34 of 4: sixteen of 8 take 24.4 us for 4 x 4096, 32 of 4 take 15.6.
constexpr double kRate = 6500e3, kBlockRate = 85e3, kBlockRate8 = 65e3;  // bytes per us
// Where the list is cut, a unit's beginning and end count for what they take a block (other queries, a granule that some queries see in part, an
// epilogue: kUnitCost), in granules at the rate of HBM or of the products. Nothing for them, 10 us for them: the 8-bit draft case 85 and 79 us, 8 drafted
// tokens over bf16 103 and 100, 16 sequences of 16 heads' one 38.6 and 37.
constexpr double kUnitCost = 10.0;

DensePlan make_dense_plan(const clsa_params& p, bool eight, int window, const DeviceInfo& dev) {
  DensePlan d = {};
  const int cols = p.q_per_seq * (p.num_q_heads / p.num_kv_heads);
  d.fold = !eight && cols <= 4;
  d.tiles = cols <= 8 ? 1 : 2;
  d.col_warps = cols <= 16 ? 1 : cols <= 32 ? 2 : 4;
  d.columns = d.fold ? 4 : d.tiles * d.col_warps * 8;
  d.col_tiles = (cols + d.columns - 1) / d.columns;
  d.spans = dev.sm_count / d.col_tiles;
  // Granules of 32 positions where the step's instructions bound it: half the votes, waits and barriers (bf16, 16 sequences of 8192 tokens, 32 and 64
  // columns: 122 and 178 us with 16, 103 and 146 with 32; the 8-bit draft case 110 and 105). With fewer columns bf16 rows keep to 16, in half the time
  // from the first row to the last one's end; 9 to 16 columns form a granule's first product beside the one before it instead (284 us, now 260).
  d.sub = eight || d.col_warps > 1 ? 2 : 1;
  const int records = d.tiles * d.col_warps * 8 * kPartialStride * 4;  // of a head in a cluster
  const int gran = 16 * d.sub, head_bytes = gran * (eight ? 256 : 512);  // positions of a granule, bytes of a head's part of it
  int room = dev.max_smem_optin - kMergeBytes - kCtrlBytes - 1024;
  int most = kConsumers / d.col_warps;
  while (p.num_kv_heads % most != 0 || room / (most * head_bytes) < 3) most /= 2;
  d.heads = most;
  const int64_t reach = window > 0 && window < p.max_seq_len - p.q_per_seq ? window + p.q_per_seq + gran : p.max_seq_len;
  const double granules = (double)((reach + gran - 1) / gran);
  double best = 0.7 * granules * head_bytes * p.num_seqs * p.num_kv_heads / kRate + 14.0;
  const double products = (eight ? 100e6 : 265e6) / d.columns;  // bytes per us that the GPU's products keep up with (measured: 64 columns over bf16 241 to 271e6 / columns, 32 and 64 over codes 94e6 and 106e6)
  double block_rate = eight ? kBlockRate8 : kBlockRate;
  if (products / dev.sm_count < block_rate) block_rate = products / dev.sm_count;
  for (int h = most; h >= 1; h /= 2) {
    const int64_t units = (int64_t)p.num_seqs * (p.num_kv_heads / h) * d.col_tiles;
    for (int c = kMaxCluster; c >= 1; c /= 2) {
      if (units * c > (c == 8 ? 112 : c == 4 ? 136 : dev.sm_count) || (c > 1 && c * 2 > granules)) continue;
      if (c > 1 && (room - h * records) / (h * head_bytes) < 2 * kConsumers / (d.col_warps * h)) continue;  // (two slots per lane, as below)
      const double rate = kRate / (double)(units * c) < block_rate ? kRate / (double)(units * c) : block_rate;
      const double cost = granules * h * head_bytes / c / rate + (c > 1 ? 0.8 : 0.0);
      if (cost < best) { best = cost; d.heads = h; d.cluster = c; d.whole_units = 0; }
    }
    const double cost = (double)((units + dev.sm_count - 1) / dev.sm_count) * granules * h * head_bytes * dev.sm_count / kRate;
    if (units > dev.sm_count && cost < best) { best = cost; d.heads = h; d.cluster = 0; d.whole_units = 1; }
  }
  d.lanes = kConsumers / (d.col_warps * d.heads);
  if (d.cluster == 0 && !d.whole_units) {
    d.pad = (int)(kUnitCost * (kRate < products ? kRate : products) / dev.sm_count / (d.heads * head_bytes));
    const int64_t units = (int64_t)p.num_seqs * (p.num_kv_heads / d.heads);
    while (units * d.pad > 1 << 28) d.pad /= 2;  // (places are numbered with 32 bits)
  }
  d.head_groups = p.num_kv_heads / d.heads;
  d.slot_bytes = d.heads * head_bytes;
  if (d.cluster > 1) room -= d.inbox_bytes = d.heads * records;
  d.lane_slots = room / d.slot_bytes;
  if (d.lane_slots > kMaxSlots / d.heads) d.lane_slots = kMaxSlots / d.heads;
  d.lane_slots /= d.lanes;  // (two at least)
  d.slots = d.lane_slots * d.lanes;
  d.smem_bytes = (size_t)d.slots * d.slot_bytes + kMergeBytes + kCtrlBytes + d.inbox_bytes + 1024;
  auto align = [](size_t x) { return (x + 255) / 256 * 256; };
  d.unit_bytes = align((size_t)p.num_seqs * p.num_kv_heads * sizeof(int2));
  // (of the heads that a block has at most: the size does not go by the window)
  d.scratch_bytes = d.unit_bytes + align((size_t)d.spans * d.col_tiles * 2 * most * d.columns * kPartialStride * sizeof(float));
  return d;
}

template <bool EIGHT, int NT, int PARTS, int SUB, bool PIPED>
cudaError_t launch_kernel(const cudaLaunchConfig_t& cfg, const CUtensorMap& map_k, const CUtensorMap& map_v, const DenseArgs& a) {
  auto kernel = dense_attn_kernel<EIGHT, NT, PARTS, SUB, PIPED>;
  // The kernel's warpgroups redistribute the registers that it was launched with: it may not have been built with fewer.
  static std::atomic<uint64_t> known{0};  // devices on which it has been looked at, and allowed its shared memory
  int dev = 0;
  cudaError_t err = cudaGetDevice(&dev);
  if (err != cudaSuccess) return err;
  if (dev >= 64 || !(known.load(std::memory_order_relaxed) >> dev & 1)) {
    cudaFuncAttributes f;
    int room = 0;
    if ((err = cudaFuncGetAttributes(&f, kernel)) != cudaSuccess) return err;
    if (f.numRegs * kThreads < kConsumers * 32 * kConsumerRegs + (kThreads - kConsumers * 32) * kProducerRegs) return cudaErrorInvalidConfiguration;
    if ((err = cudaDeviceGetAttribute(&room, cudaDevAttrMaxSharedMemoryPerBlockOptin, dev)) != cudaSuccess) return err;
    if ((err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, room)) != cudaSuccess) return err;
    if (dev < 64) known.fetch_or(1ull << dev, std::memory_order_relaxed);
  }
  return cudaLaunchKernelEx(&cfg, kernel, map_k, map_v, a);
}

cudaError_t launch_dense_attn(const clsa_params& p, const clsa_cache8* c, int window, const DensePlan& plan, const void* q, void* out,
                              float* lse, uint32_t* status, unsigned char* scratch, cudaStream_t stream) {
  CUtensorMap map_k, map_v;
  const bool eight = c != nullptr;
  const bool two_boxes = plan.sub == 2 && p.block_table != nullptr && p.block_size == 16;
  const int box_rows = two_boxes ? 16 : 16 * plan.sub;
  const int64_t token = eight ? c->kv_token_stride : p.kv_token_stride, head = eight ? c->kv_head_stride : p.kv_head_stride;
  if (!make_map(&map_k, eight ? c->k : p.k_cache, eight, p, token, head, plan.heads, box_rows) ||
      !make_map(&map_v, eight ? c->v : p.v_cache, eight, p, token, head, plan.heads, box_rows))
    return cudaErrorInvalidValue;
  DenseArgs a = {};
  a.q = static_cast<const uint16_t*>(q);
  a.out = static_cast<uint16_t*>(out);
  a.lse = lse;
  a.status = status;
  a.units = reinterpret_cast<int2*>(scratch);
  a.part = reinterpret_cast<float*>(scratch + plan.unit_bytes);
  a.seq_start = p.seq_start;
  a.seq_len = p.seq_len;
  a.block_table = p.block_table;
  if (eight) {
    a.ks = static_cast<const uint8_t*>(c->k_scale);
    a.vs = static_cast<const uint8_t*>(c->v_scale);
    a.scale_head = c->scale_head_stride;
    while ((1 << a.scale_shift) < c->scale_block) ++a.scale_shift;
    a.scale_bytes = (p.num_kv_heads - 1) * c->scale_head_stride + ((p.num_cache_rows - 1) >> a.scale_shift) + 1;
  }
  a.num_rows = p.num_cache_rows;
  while (p.block_table != nullptr && (1 << a.block_shift) < p.block_size) ++a.block_shift;
  a.max_blocks = p.max_blocks_per_seq;
  a.pages = (int)((p.num_cache_rows + (1 << a.block_shift) - 1) >> a.block_shift);
  a.num_seqs = p.num_seqs;
  a.T = p.q_per_seq;
  a.num_q_heads = p.num_q_heads;
  a.group = p.num_q_heads / p.num_kv_heads;
  a.columns_used = a.T * a.group;
  a.window = window < p.max_seq_len ? window : p.max_seq_len;  // (as far as a window reaches)
  a.causal = p.causal;
  a.max_seq_len = p.max_seq_len;
  a.columns = plan.columns;
  a.col_tiles = plan.col_tiles;
  a.heads = plan.heads;
  while ((1 << a.head_shift) < plan.heads) ++a.head_shift;
  a.lanes = plan.lanes;
  a.col_warps = plan.col_warps;
  a.head_groups = plan.head_groups;
  a.slots = plan.slots;
  a.lane_slots = plan.lane_slots;
  a.ring_inv = (65536u + (uint32_t)plan.lane_slots - 1u) / (uint32_t)plan.lane_slots;
  a.spans = plan.spans;
  while ((1 << a.min_shift) < plan.lanes) ++a.min_shift;
  a.gran_shift = plan.sub == 2 ? 5 : 4;
  a.two_boxes = two_boxes;
  a.whole_units = plan.whole_units;
  a.cluster = plan.cluster;
  a.pad = plan.pad;
  while ((1 << a.cluster_shift) < plan.cluster) ++a.cluster_shift;
  a.group_inv = (65536u + (uint32_t)a.group - 1u) / (uint32_t)a.group;
  a.scale_log2 = p.sm_scale * kLog2e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = plan.cluster > 0 ? dim3((unsigned)plan.cluster, (unsigned)plan.head_groups, (unsigned)(p.num_seqs * plan.col_tiles))
                                 : dim3((unsigned)(plan.spans * plan.col_tiles), 1, 1);
  cfg.blockDim = dim3(kThreads, 1, 1);
  cfg.dynamicSmemBytes = plan.smem_bytes;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = plan.cluster;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = plan.cluster > 1 ? 2 : 1;
  const cudaError_t err = eight ? (plan.tiles == 1 ? launch_kernel<true, 1, 1, 2, false>(cfg, map_k, map_v, a) : launch_kernel<true, 2, 1, 2, false>(cfg, map_k, map_v, a))
                          : plan.fold           ? launch_kernel<false, 1, 3, 1, false>(cfg, map_k, map_v, a)
                          : plan.tiles == 1     ? launch_kernel<false, 1, 2, 1, false>(cfg, map_k, map_v, a)
                          : plan.col_warps == 1 ? launch_kernel<false, 2, 2, 1, true>(cfg, map_k, map_v, a)
                          : plan.col_warps == 2 ? launch_kernel<false, 2, 2, 2, false>(cfg, map_k, map_v, a)
                                                : launch_kernel<false, 2, 1, 2, false>(cfg, map_k, map_v, a);
  if (err != cudaSuccess || plan.whole_units || plan.cluster > 0) return err;
  const int64_t rows = (int64_t)a.num_seqs * a.T * a.num_q_heads;
  // Few rows are cut into parts of 32 outputs, so that all SMs take part and everything is in flight at once (148 stretches are 5 per lane).
  const bool few = rows <= 64;
  const int share = rows <= 1024 ? 8 : 2;
  cfg.gridDim = dim3((unsigned)(few ? rows * 4 : (rows * share + 7) / 8), 1, 1);
  cfg.blockDim = dim3(kJoinThreads, 1, 1);
  cfg.dynamicSmemBytes = 0;
  return cudaLaunchKernelEx(&cfg, few ? dense_join_kernel<8, 4, 5> : share == 8 ? dense_join_kernel<8, 1, 5> : dense_join_kernel<2, 1, 5>, a);
}

}  // namespace clsa
