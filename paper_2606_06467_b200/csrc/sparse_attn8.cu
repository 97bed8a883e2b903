// GQA sparse attention over the selected rows of an 8-bit K and V cache (Eq. 4), one launch per layer, T >= 1.
//
//   x_s = sm_scale * (q . code_K[s]) * 2^ek,   O = sum_s exp(x_s) 2^ev code_V[s] / sum_s exp(x_s)
// with ek, ev the exponents of the scale blocks that row s lies in.
//
// e4m3 codes convert to f16 exactly, a query row scaled by a power of two so that its largest magnitude lies in [2^13, 2^14) is
// exact in f16 down to 2^-31 of it, sums are fp32. Weights are rounded to f16, what the matrix instruction takes: 2^-11 of each, which a
// sum over tokens averages out below the outputs' own bf16 rounding of 2^-8 (against 64 bits both this and a form with fp32 weights are
// off by 0.0017 in the norm); the denominators are sums of the unrounded ones. (There is no faster 8-bit form to be had: the
// warp-level e4m3 instruction is carried out as these conversions and f16 products anyway.) A warp-level instruction has up to 8
// query heads of the GQA group in its columns (NT tiles cover the group) and 16 tokens or 16 dimensions along M:
//   S^T[16 tokens x 8 heads] = K[16 x 128] Q^T,   O^T[128 x 8 heads] += V^T[128 x 32 tokens] P^T
// K's fragments are plain matrix loads: a lane's word holds 4 dimensions of a token, its halves are the lane's two shares of a
// step (the contraction index is a dummy, q is laid out to match). V's are the transposing 8-bit loads: a word holds 4
// consecutive tokens of one dimension. K's rows are addressed in the order in which the weights, transposed in registers, then
// meet those tokens. Groups of up to 4 query heads (FOLD) fill the columns twice: columns 4 .. 7 repeat the heads, their lanes take
// the weights of the second 16 tokens where the others take those of the first, and the second product keeps the two halves of
// the sum in the two column halves until the end -- half the logits and weights per lane for a few selects.
//
// In the log2 domain a query head keeps two running references: mx near the largest x_s for the denominators 2^(x_s - mx), and m
// near the largest x_s - mx + ev for the numerators' weights 2^(x_s - mx + ev - m), so that neither underflows however far apart
// the blocks' scales lie; 2^m is applied to the finished quotient. ev meets the difference x_s - mx, which is small where it counts,
// never x_s itself, whose fp32 rounding would swallow it (logits of 1e7: V rows off by whole powers of two). References move only
// when a weight would leave its range (one vote per stage): a stage that moves none needs no reduction over its tokens.
//
// The work is a flat list of 32-token stages, unit = (KV head, query row), heads outermost, so that a prefill chunk's launch
// goes over one head's part of the cache (which fits in L2) before the next. Warp w of W takes a contiguous span of the list
// (unit-aligned where that splits evenly); a warp streams its span through a private ring of cp.async stages, 128 bytes of K
// and of V per token. Units that several warps share are merged by log-sum-exp: partial results meet in shared memory, those of
// units that straddle blocks in global slots (two per block) with an arrival counter; the block that arrives last reads them in
// block order, so results do not depend on timing, and puts the counter back to zero.
//
// 512-token chunk (32 query heads over 8 KV heads, 2048 rows each of 33 K tokens): 185 us. The caches come from DRAM once (98 MB) and
// 2.17 GB cross from L2 to the SMs, 11.8 TB/s; copies alone take 135 us, the arithmetic alone about 160, and what is left is
// their overlap on 12 warps per SM (168 registers each): 59 % of issue slots and of the ALU, which converts the codes at half
// rate, 32 % of the tensor pipe. 16 warps with 128 registers and three half-stage buffers (239 us: a third more instructions),
// 8-row half stages, rows padded instead of permuted (218: a row then lies in two lines), fewer lanes per row (281 with four),
// tcgen05 with two e4m3 pieces per operand (345) all lost. Decode, 16 sequences of 128 K tokens: 67 MB of gathered rows in
// 19.1 us (3.5 TB/s; 15.6 with the rows in L2), a chain of index, page, row and merge round trips on 128 SMs.
#include "attn_common.cuh"
#include "cache8.cuh"

namespace clsa {
namespace {

constexpr int kTok = 32;                  // tokens per stage
constexpr int kStage8Bytes = kTok * 256;  // K rows, then V rows, 128 bytes each
constexpr int kMaxGroup = 16;
constexpr float kLazy = 8.f;              // a weight may exceed its reference by 2^8 before the reference moves
constexpr float kNone = -3.4028234663852886e38f;  // a reference before the first token, below every logit: 2^(x - kNone) of a masked x = -inf is 0, not NaN
// A finished product d of codes and query is at most 128 * 448 * 2^14 < 2^30 in magnitude and meets 2^ek first: of that factor 2^22
// is held back for the query's, so that d 2^(ek - 22) is finite for every ek (120 at most) and d's last bits stay above the smallest
// float (ek -100, d 2^-27: 2^-149). The query's factor is a float up to |q| sm_scale < 2^118.
constexpr int kHeldBack = 22;

struct Attn8Args {
  const uint16_t* q;
  const uint8_t* kc;
  const uint8_t* vc;
  const uint8_t* ks;
  const uint8_t* vs;
  int64_t head_stride, scale_head;
  uint32_t unit;  // 16
  uint32_t stride16;  // token stride in units
  int scale_shift;
  int64_t num_rows;
  const int64_t* seq_start;
  const int32_t* seq_len;
  const int32_t* idx;
  const int32_t* count;
  const int32_t* block_table;
  int block_shift, max_blocks;
  uint32_t page_limit;  // pages of the row space (the last one may be cut short)
  uint16_t* out;
  float* lse;
  uint32_t* status;
  int rows, q_per_seq, num_q_heads, num_kv_heads, group, top_k, max_seq_len;
  int reverse, early, keep, pin;
  int unit_stages, total_stages;
  int mode, span_q, span_rem, workers, wpb;  // Attn8Plan::mode
  float* part;       // records of [group][kPartialStride] floats: W of the workers, then 2 per block
  uint32_t* arrive;  // [blocks][group] arrival counters of the unit that leaves block b to the right, zero between launches
  float scale_log2;
};

// First stage of worker w's span (kAttn8Units: unit u has span_q workers, the first span_rem units one more, its stages cut evenly
// over them; kAttn8Flat: the first span_rem workers take span_q + 1 consecutive stages, the others span_q).
__device__ __forceinline__ int span_begin(int w, const Attn8Args& a) {
  if (a.mode == kAttn8Flat) return w * a.span_q + min(w, a.span_rem);
  const int big = a.span_rem * (a.span_q + 1);
  int u, j, n;
  if (w < big) { n = a.span_q + 1; u = w / n; j = w - u * n; }
  else { n = a.span_q; const int w2 = w - big; u = w2 / n; j = w2 - u * n; u += a.span_rem; }
  return u * a.unit_stages + (int)((int64_t)j * a.unit_stages / n);
}
__device__ __forceinline__ void unit_workers(int u, const Attn8Args& a, int& first, int& last) {
  if (a.mode == kAttn8Units) {
    first = u * a.span_q + min(u, a.span_rem);
    last = first + a.span_q + (u < a.span_rem ? 1 : 0) - 1;
  } else {
    const int big = a.span_rem * (a.span_q + 1);
    auto owner = [&](int s) { return s < big ? s / (a.span_q + 1) : a.span_rem + (s - big) / a.span_q; };
    first = owner(u * a.unit_stages);
    last = owner(u * a.unit_stages + a.unit_stages - 1);
  }
}

// Token of row r of a 16-token tile of the first product: after the transpose of the weights a lane has rows 2 j and 2 j + 1 of
// the tile's first eight and of its last eight, which have to be tokens 4 j .. 4 j + 3.
__device__ __forceinline__ int k_token(int r) { return 4 * ((r >> 1) & 3) + (r & 1) + ((r >> 2) & 2); }
// Where chunk c (16 bytes) of token t of a stage lies: the eight rows that a matrix load reads together (k_token of eight
// consecutive r; eight consecutive tokens for V) fall into different banks.
__device__ __forceinline__ uint32_t k_chunk(int t, int c) { return (uint32_t)(t * 128 + ((c ^ ((t & 1) | ((t >> 1) & 6))) << 4)); }
__device__ __forceinline__ uint32_t v_chunk(int t, int c) { return (uint32_t)(t * 128 + ((c ^ (t & 7)) << 4)); }

// base + units * unit, the unit an argument of the launch: of a known power of two the compiler makes a shift and a high product.
__device__ __forceinline__ const uint8_t* at_unit(const uint8_t* base, uint32_t units, uint32_t unit) {
  const uint8_t* p;
  asm("mad.wide.u32 %0, %1, %2, %3;" : "=l"(p) : "r"(units), "r"(unit), "l"(base));
  return p;
}
__device__ __forceinline__ void cp_async16_plain(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;\n" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void ldmatrix_b8_x2_trans(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m16n16.x2.trans.shared.b8 {%0,%1,%2,%3}, [%4];\n"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}

template <int WARPS, int STAGES>
struct Shape {
  static constexpr int kRing = STAGES * kStage8Bytes;
  static constexpr int kScale = STAGES * kTok * 8;  // per token: 2^(ek - kHeldBack), ev
  static constexpr size_t kSmem = (size_t)WARPS * (kRing + kScale + STAGES * 4) + WARPS * (sizeof(int2) + sizeof(int2));
};

template <int NT, bool FOLD, int WARPS, int STAGES, bool PAGED>
__global__ void __launch_bounds__(WARPS * 32, 1) sparse_attn8_kernel(const __grid_constant__ Attn8Args a) {
  using S = Shape<WARPS, STAGES>;
  extern __shared__ __align__(128) unsigned char smem[];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int rowq = lane >> 2, hcol = FOLD ? 2 * (lane & 1) : 2 * (lane & 3);  // this lane's heads (of each tile): hcol, hcol + 1
  constexpr int NX = FOLD ? 2 : 4;              // tokens of a stage whose logits this lane has
  const bool upper = FOLD && (lane & 2) != 0;   // .. in the stage's second half
  const int G = a.group, NS = a.unit_stages, W = a.workers;
  const int w = (int)blockIdx.x * a.wpb + warp;
  const bool has_work = warp < a.wpb && w < W;
  // This worker's stages: whole units [own_lo, own_hi) (kAttn8Blocks), then the span [s_begin, s_end).
  int own_lo = 0, own_hi = 0, s_begin = 0, s_end = 0;
  if (a.mode == kAttn8Blocks) {
    const int b = (int)blockIdx.x, n = a.span_q + (b < a.span_rem ? 1 : 0), each = n / a.wpb;
    const int shared = (n - each * a.wpb) * NS, parts = min(a.wpb, shared);  // stages that the first `parts` warps share
    const int u0 = b * a.span_q + min(b, a.span_rem), base = (u0 + each * a.wpb) * NS;
    if (has_work) {
      own_lo = (u0 + warp * each) * NS;
      own_hi = own_lo + each * NS;
    }
    s_begin = s_end = base + shared;
    if (warp < parts) {
      s_begin = base + (int)((int64_t)warp * shared / parts);
      s_end = base + (int)((int64_t)(warp + 1) * shared / parts);
    }
  } else if (has_work) {
    s_begin = span_begin(w, a);
    s_end = w + 1 < W ? span_begin(w + 1, a) : a.total_stages;
  }
  unsigned char* ring = smem + warp * S::kRing;
  const uint32_t ring_u32 = smem_u32(ring);
  float2* scales = reinterpret_cast<float2*>(smem + WARPS * S::kRing + warp * S::kScale);
  uint32_t* stage_mask = reinterpret_cast<uint32_t*>(smem + WARPS * (S::kRing + S::kScale)) + warp * STAGES;
  int2* span_tab = reinterpret_cast<int2*>(smem + WARPS * (S::kRing + S::kScale + STAGES * 4));
  int2* split_tab = span_tab + WARPS;
  if (lane == 0) {
    // For the merge: the units that this warp does not have whole and that no earlier warp of the block reaches into -- the
    // one its span starts in, the one it ends in -- or -1.
    const bool any = s_begin < s_end;
    const int uf = s_begin / NS, ul = any ? (s_end - 1) / NS : 0;
    span_tab[warp] = make_int2(s_begin, s_end);
    split_tab[warp] = make_int2(any && (s_begin > uf * NS || s_end < (uf + 1) * NS) && (warp == 0 || s_begin == uf * NS) ? uf : -1,
                                any && ul != uf && s_end < (ul + 1) * NS ? ul : -1);
  }

  // Programmatic dependent launch, as in the bf16 kernels: dependents are released only behind this grid's own wait.
  bool waited = false;
  auto wait_now = [&]() {
    if (!waited) {
      asm volatile("griddepcontrol.wait;" ::: "memory");
      asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
      waited = true;
    }
  };
  if (!a.early) wait_now();

  // Places inside a stage, from the ring's start. This lane copies chunk lane & 7 of tokens 4 it + lane / 8: k_copy[it & 3] and
  // v_copy[it & 1] plus 512 it; it addresses row k_frag of K's fragment loads (plus 2048 for tokens 16 ..), where the chunk
  // pair 2 st is reached by an exclusive or with st << 5, and row v_frag of V's, where chunk c is with c << 4.
  uint32_t k_copy[4], v_copy[2];
#pragma unroll
  for (int i = 0; i < 4; ++i) k_copy[i] = ring_u32 + k_chunk(4 * i + (lane >> 3), lane & 7) - 512u * i;
#pragma unroll
  for (int i = 0; i < 2; ++i) v_copy[i] = ring_u32 + kStage8Bytes / 2 + v_chunk(4 * i + (lane >> 3), lane & 7) - 512u * i;
  const uint32_t k_frag = ring_u32 + k_chunk(k_token(lane & 15), lane >> 4);
  const uint32_t v_frag = ring_u32 + kStage8Bytes / 2 + v_chunk(lane, 0);
  const int my_tok = k_token(rowq) + (upper ? 16 : 0);  // this lane's tokens of a stage: my_tok + {0, 2} and, unfolded, {16, 18}

  int left = own_hi - own_lo + s_end - s_begin;  // stages to go
  while (left > 0) {
    // ---- the next segment: stages [seg_lo, seg_hi) of unit u; the whole units first, so that what the block's warps share
    // ---- ends the walk in either direction --------------------------------------------------------------------------
    const bool own = left > s_end - s_begin;
    const int lo = own ? own_lo : s_begin, hi = own ? own_hi : s_end, to_go = own ? left - (s_end - s_begin) : left;
    const int u = (a.reverse ? lo + to_go - 1 : hi - to_go) / NS;
    const int seg_lo = max(lo, u * NS), seg_hi = min(hi, (u + 1) * NS);
    left -= seg_hi - seg_lo;
    const int g = u / a.rows, r = u - g * a.rows;
    const int h0 = g * G, b = r / a.q_per_seq;
    const int slot_lo = (seg_lo - u * NS) * kTok;
    const int slot_hi = min(a.top_k, (seg_hi - u * NS) * kTok);
    const int32_t* row_idx = a.idx + (int64_t)r * a.top_k;
    // the first positions, fetched together with the count (entries past it are not used)
    int spec[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) spec[i] = !a.reverse && slot_lo + i * kTok + lane < slot_hi ? row_idx[slot_lo + i * kTok + lane] : -1;
    int cnt = a.count[r];
    const int n_raw = a.seq_len[b];
    const bool n_ok = n_raw >= a.q_per_seq && n_raw <= a.max_seq_len;
    const int n = n_ok ? n_raw : 0;  // a sequence with a bad length is never read: no position passes the range check
    const int64_t start = PAGED ? 0 : a.seq_start[b];
    const int32_t* table = PAGED ? a.block_table + (int64_t)b * a.max_blocks : nullptr;
    const bool first_of_row = slot_lo == 0 && g == 0;
    if (cnt < 0 || cnt > a.top_k) {
      if (lane == 0 && first_of_row) flag_status(a.status, CLSA_DEV_BAD_COUNT);
      cnt = cnt < 0 ? 0 : a.top_k;
    }
    const int t_lo = min(cnt, slot_lo), t_hi = min(cnt, slot_hi);
    const int nstages = (t_hi - t_lo + kTok - 1) / kTok;

    float o[NT][8][4];                     // O^T: [head tile][16 dimensions]: dimensions rowq, rowq + 8; heads hcol, hcol + 1
    float m[NT][2], mx[NT][2], l[NT][2];   // references and this lane's share of the denominators of the two heads
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      m[nt][0] = m[nt][1] = mx[nt][0] = mx[nt][1] = kNone;
      l[nt][0] = l[nt][1] = 0.f;
#pragma unroll
      for (int c = 0; c < 8; ++c) { o[nt][c][0] = 0.f; o[nt][c][1] = 0.f; o[nt][c][2] = 0.f; o[nt][c][3] = 0.f; }
    }

    if (nstages > 0) {
      const uint8_t* kbase = a.kc + g * a.head_stride + (lane & 7) * 16;
      const uint8_t* vbase = a.vc + g * a.head_stride + (lane & 7) * 16;
      const uint8_t* ksb = a.ks + g * a.scale_head;
      const uint8_t* vsb = a.vs + g * a.scale_head;
      // Stage i begins at entry t_lo + 32 i of the row's index, or, walking from the end, nstages - 1 - i in the place of i.
      const int32_t* my_idx = row_idx + t_lo;
      const int total = t_hi - t_lo, step = a.reverse ? -kTok : kTok;
      int tok = lane + (a.reverse ? (nstages - 1) * kTok : 0);  // entry that this lane reads next
      auto next_raw = [&]() -> int {                            // its position (-1 past the end), one stage further each time
        const int raw = (uint32_t)tok < (uint32_t)total ? my_idx[tok] : -1;
        tok += step;
        return raw;
      };
      // Positions whose rows may be read: inside the sequence and, without pages, inside the row space too.
      const int pos_lo = PAGED || start >= 0 ? 0 : (int)min((int64_t)n, -start);
      const int pos_hi = PAGED ? n : (int)max((int64_t)pos_lo, min((int64_t)n, a.num_rows - start));
      const uint32_t pos_span = (uint32_t)(pos_hi - pos_lo);
      auto load_blk = [&](int raw) -> int { return PAGED && (uint32_t)raw < (uint32_t)n ? __ldg(table + (raw >> a.block_shift)) : -1; };
      auto settle = [&](int buf, int kb, int vb) {  // the scale bytes of stage i into shared memory
        scales[buf * kTok + lane] = make_float2(exp2_int(scale_exponent(kb) - kHeldBack), (float)scale_exponent(vb));
      };
      auto issue = [&](int i, int buf, int raw, int blk, int& kb, int& vb) {  // the copies of stage i; its scale bytes stay in flight
        if (i < nstages) {
          uint32_t row;
          bool ok;
          if (PAGED) {
            ok = (uint32_t)blk < a.page_limit;  // (-1 where the position is out of range)
            row = ((uint32_t)blk << a.block_shift) + ((uint32_t)raw & ((1u << a.block_shift) - 1u));
            ok = ok && row < (uint32_t)a.num_rows;
          } else {
            ok = (uint32_t)(raw - pos_lo) < pos_span;
            row = (uint32_t)start + (uint32_t)raw;
          }
          const bool raw_live = (uint32_t)((a.reverse ? nstages - 1 - i : i) * kTok + lane) < (uint32_t)total;
          const uint32_t okmask = __ballot_sync(0xffffffffu, ok);
          if (lane == 0) stage_mask[buf] = okmask;
          kb = vb = 127;
          if (ok) {
            kb = ksb[row >> a.scale_shift];
            vb = vsb[row >> a.scale_shift];
          }
          const uint32_t my16 = ok ? row * a.stride16 : 0u;  // 16-byte units: the caches span less than 2^32 of them
          const uint32_t at = (uint32_t)(buf * kStage8Bytes);
          if (okmask == 0xffffffffu && !a.keep) {  // the usual stage
#pragma unroll
            for (int it = 0; it < 8; ++it) {
              const uint32_t units = __shfl_sync(0xffffffffu, my16, 4 * it + (lane >> 3));
              cp_async16_plain(k_copy[it & 3] + at + 512 * it, at_unit(kbase, units, a.unit));
              cp_async16_plain(v_copy[it & 1] + at + 512 * it, at_unit(vbase, units, a.unit));
            }
          } else {  // some rows are none and become zeros, or rows have an L2 priority
            if (!ok && n_ok && raw_live) flag_status(a.status, CLSA_DEV_BAD_INDEX);
            const uint64_t pol = !a.keep ? l2_policy_evict_normal()
                                 : a.pin < 0 || pin_rank((t_lo / kTok + (a.reverse ? nstages - 1 - i : i)) & 7) < a.pin ? l2_policy_evict_last()
                                                                                                                  : l2_policy_evict_first();
#pragma unroll
            for (int it = 0; it < 8; ++it) {
              const int t = 4 * it + (lane >> 3);
              const uint64_t off = (uint64_t)__shfl_sync(0xffffffffu, my16, t) * 16u;
              const bool okt = (okmask >> t) & 1u;
              cp_async16(k_copy[it & 3] + at + 512 * it, kbase + off, okt, pol);
              cp_async16(v_copy[it & 1] + at + 512 * it, vbase + off, okt, pol);
            }
          }
        }
        cp_async_commit();
      };

      // Prologue: the ring filled, the positions of the two stages behind it and the page numbers of the first in registers.
      int raw_p[STAGES], blk_p[STAGES];
#pragma unroll
      for (int i = 0; i < STAGES; ++i) {
        if (a.reverse || i >= 2) raw_p[i] = next_raw();
        else { raw_p[i] = tok < total ? spec[i] : -1; tok += step; }
      }
      int rawX = next_raw(), rawY = next_raw();
#pragma unroll
      for (int i = 0; i < STAGES; ++i) blk_p[i] = load_blk(raw_p[i]);
#pragma unroll
      for (int i = 0; i < STAGES; ++i) issue(i, i, raw_p[i], blk_p[i], raw_p[i], blk_p[i]);  // (now the scale bytes)
      int blkX = load_blk(rawX);
      wait_now();  // with only q pending, everything read so far was complete before this launch; q is read behind the wait

      // q as f16: column rowq = head, step st: dimensions 16 st + 4 (lane & 3) .. + 3.
      uint32_t qb[NT][8][2];
      float qf[NT][2];
      const uint16_t* qbase = a.q + ((int64_t)r * a.num_q_heads + h0) * 128;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const int head = nt * 8 + (FOLD ? rowq & 3 : rowq);
        float amax = 0.f;
#pragma unroll
        for (int st = 0; st < 8; ++st) {
          const uint2 v = head < G ? *reinterpret_cast<const uint2*>(qbase + head * 128 + 16 * st + 4 * (lane & 3)) : make_uint2(0u, 0u);
          qb[nt][st][0] = v.x;
          qb[nt][st][1] = v.y;
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const float lo = fabsf(bf16_lo(qb[nt][st][k])), hi = fabsf(bf16_hi(qb[nt][st][k]));
            if (lo <= 3.4028234663852886e38f) amax = fmaxf(amax, lo);  // finite
            if (hi <= 3.4028234663852886e38f) amax = fmaxf(amax, hi);
          }
        }
        amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
        amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
        const int shift = min(13 + 127 - (int)(__float_as_uint(amax) >> 23), 120);
        const float up = exp2_int(shift), down = exp2_int(-shift);
#pragma unroll
        for (int st = 0; st < 8; ++st)
#pragma unroll
          for (int k = 0; k < 2; ++k) qb[nt][st][k] = pack_f16x2(bf16_lo(qb[nt][st][k]) * up, bf16_hi(qb[nt][st][k]) * up);
#pragma unroll
        for (int h = 0; h < 2; ++h)  // lane 4 h holds head h
          qf[nt][h] = fminf(__shfl_sync(0xffffffffu, down, 4 * (hcol + h)) * a.scale_log2 * exp2_int(kHeldBack), 3.4028234663852886e38f);
      }
#pragma unroll
      for (int i = 0; i + 1 < STAGES; ++i) settle(i, raw_p[i], blk_p[i]);
      int pend_k = raw_p[STAGES - 1], pend_v = blk_p[STAGES - 1];  // settled one iteration after their stage was issued
#pragma unroll 1
      for (int i0 = 0; i0 < nstages; i0 += STAGES)
#pragma unroll
      for (int buf = 0; buf < STAGES; ++buf) {  // every place in the ring a constant (512-token chunk: 194 us without, 184.5 with, then)
        const int i = i0 + buf;
        if (i >= nstages) break;
        const int raw_new = next_raw();
        const int blk_new = load_blk(rawY);
        cp_async_wait<STAGES - 1>();
        __syncwarp();
        const uint32_t at = (uint32_t)(buf * kStage8Bytes);
        const uint32_t okmask = stage_mask[buf];
        float2 sc[NX];  // tokens my_tok + 2 (t & 1) + 16 (t / 2)
#pragma unroll
        for (int t = 0; t < NX; ++t) sc[t] = scales[buf * kTok + my_tok + 2 * (t & 1) + 8 * (t & 2)];
        float s[NT][2][4], s2[NT][2][4];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i) s[nt][k][i] = s2[nt][k][i] = 0.f;
#pragma unroll
        for (int st = 0; st < 4; ++st)
#pragma unroll
          for (int mt = 0; mt < 2; ++mt) {
            uint32_t kf[4];  // chunk 2 st of rows 0-7, 8-15, chunk 2 st + 1 of them
            ldmatrix_x4(kf, (k_frag ^ (uint32_t)(st << 5)) + (at + 2048 * mt));
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              const uint32_t a0 = e4m3x2_to_f16x2(kf[2 * k]), a2 = e4m3x2_hi_to_f16x2(kf[2 * k]);
              const uint32_t a1 = e4m3x2_to_f16x2(kf[2 * k + 1]), a3 = e4m3x2_hi_to_f16x2(kf[2 * k + 1]);
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) mma_f16(k ? s2[nt][mt] : s[nt][mt], a0, a1, a2, a3, qb[nt][2 * st + k][0], qb[nt][2 * st + k][1]);
            }
          }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i) s[nt][k][i] += s2[nt][k][i];
        // x of the lane's tokens and two heads per tile: x[..][2 t + head]; y = x - mx, ye = y + V's exponent
        float x[NT][2 * NX], y[NT][2 * NX], ye[NT][2 * NX];
        bool move = false;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int t = 0; t < NX; ++t) {
            float d[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) d[h] = FOLD ? (upper ? s[nt][1][2 * t + h] : s[nt][0][2 * t + h]) : s[nt][t >> 1][2 * (t & 1) + h];
            const float2 z = unpack2(mul2(mul2(pack2(d[0], d[1]), pack2(sc[t].x, sc[t].x)), pack2(qf[nt][0], qf[nt][1])));
            x[nt][2 * t] = z.x;
            x[nt][2 * t + 1] = z.y;
          }
        if (okmask != 0xffffffffu) {
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 2 * NX; ++i) x[nt][i] = (okmask >> (my_tok + (i & 2) + 4 * (i & 4))) & 1u ? x[nt][i] : -INFINITY;
        }
        auto relate = [&](int nt) {
#pragma unroll
          for (int t = 0; t < NX; ++t) {
            const uint64_t d = add2(pack2(x[nt][2 * t], x[nt][2 * t + 1]), pack2(-mx[nt][0], -mx[nt][1]));
            const float2 z = unpack2(d), ze = unpack2(add2(d, pack2(sc[t].y, sc[t].y)));
            y[nt][2 * t] = z.x;
            y[nt][2 * t + 1] = z.y;
            ye[nt][2 * t] = ze.x;
            ye[nt][2 * t + 1] = ze.y;
          }
        };
        auto largest = [&](const float (&v)[2 * NX], int h) {
          float r = v[h];
#pragma unroll
          for (int t = 1; t < NX; ++t) r = fmaxf(r, v[2 * t + h]);
          return r;
        };
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          relate(nt);
#pragma unroll
          for (int h = 0; h < 2; ++h) move = move || largest(y[nt], h) > kLazy || largest(ye[nt], h) > m[nt][h] + kLazy;
        }
        if (__any_sync(0xffffffffu, move)) {  // some head's references have to move: to the largest seen so far
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            float drop[2];  // what every difference from mx loses
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              float top = largest(x[nt], h);
#pragma unroll
              for (int d = FOLD ? 2 : 4; d <= 16; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
              const float mxn = fmaxf(mx[nt][h], top);
              drop[h] = mx[nt][h] - mxn;
              l[nt][h] *= fast_exp2(drop[h]);
              mx[nt][h] = mxn;
            }
            relate(nt);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              float top = largest(ye[nt], h);
#pragma unroll
              for (int d = FOLD ? 2 : 4; d <= 16; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
              const float mo = m[nt][h] + drop[h], mn = fmaxf(mo, top), alpha = fast_exp2(mo - mn);
              m[nt][h] = mn;
#pragma unroll
              for (int c = 0; c < 8; ++c) { o[nt][c][h] *= alpha; o[nt][c][h + 2] *= alpha; }
            }
          }
        }
        uint32_t pb[NT][4];  // weights as the second product's columns: tokens 4 (lane & 3) + {0, 1}, {2, 3}, then those + 16
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
          for (int t = 0; t < NX; ++t) {
            const float2 w = unpack2(add2(pack2(ye[nt][2 * t], ye[nt][2 * t + 1]), pack2(-m[nt][0], -m[nt][1])));
            const float2 z = unpack2(add2(pack2(l[nt][0], l[nt][1]), pack2(fast_exp2(y[nt][2 * t]), fast_exp2(y[nt][2 * t + 1]))));
            l[nt][0] = z.x;
            l[nt][1] = z.y;
            pb[nt][t] = movmatrix_trans(pack_f16x2(fast_exp2(w.x), fast_exp2(w.y)));
          }
          if (FOLD) {  // columns 0 .. 3 have the weights of the stage's first half, 4 .. 7 those of its second
#pragma unroll
            for (int t = 0; t < 2; ++t) {
              pb[nt][2 + t] = rowq >= 4 ? pb[nt][t] : 0u;
              pb[nt][t] = rowq >= 4 ? 0u : pb[nt][t];
            }
          }
        }
#pragma unroll
        for (int c = 0; c < 8; c += 2) {
          uint32_t v[2][4];  // tokens 0-15 of dimensions 16 c + rowq and + 8, then tokens 16-31
#pragma unroll
          for (int j = 0; j < 2; ++j) ldmatrix_b8_x2_trans(v[j], (v_frag ^ (uint32_t)((c + j) << 4)) + at);
#pragma unroll
          for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              const uint32_t a0 = e4m3x2_to_f16x2(v[j][2 * k]), a2 = e4m3x2_hi_to_f16x2(v[j][2 * k]);
              const uint32_t a1 = e4m3x2_to_f16x2(v[j][2 * k + 1]), a3 = e4m3x2_hi_to_f16x2(v[j][2 * k + 1]);
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) mma_f16(o[nt][c + j], a0, a1, a2, a3, pb[nt][2 * k], pb[nt][2 * k + 1]);
            }
        }
        __syncwarp();  // everyone is done with this buffer before it is refilled
        settle((buf + STAGES - 1) % STAGES, pend_k, pend_v);
        issue(i + STAGES, buf, rawX, blkX, pend_k, pend_v);
        rawX = rawY;
        blkX = blk_new;
        rawY = raw_new;
      }
      cp_async_wait<0>();
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int d = FOLD ? 2 : 4; d <= 16; d <<= 1) l[nt][h] += __shfl_xor_sync(0xffffffffu, l[nt][h], d);
      if (FOLD) {  // the two halves of the sums
#pragma unroll
        for (int c = 0; c < 8; ++c)
#pragma unroll
          for (int i = 0; i < 4; ++i) o[0][c][i] += __shfl_xor_sync(0xffffffffu, o[0][c][i], 2);
      }
    }
    wait_now();  // a segment without tokens has read nothing yet; what follows writes global memory
    if (!n_ok && lane == 0 && first_of_row) flag_status(a.status, CLSA_DEV_BAD_SEQLEN);

    // ---- what becomes of this segment's result (staged through the warp's ring, idle between segments) -------------
    float* mypart = reinterpret_cast<float*>(ring);
    const bool whole = seg_lo == u * NS && seg_hi == (u + 1) * NS;
    __syncwarp();
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int head = nt * 8 + hcol + h;
        if (head < G && !upper) {
          // a whole unit is normalised here; 2^m is applied in two halves: it may not be a float
          const float inv = whole ? (l[nt][h] != 0.f ? 1.f / l[nt][h] : 0.f) : 1.f;
          const float half = whole && l[nt][h] != 0.f ? fast_exp2(0.5f * m[nt][h]) : 1.f;
          float* dst = mypart + head * kPartialStride + rowq;
#pragma unroll
          for (int c = 0; c < 8; ++c) {
            dst[16 * c] = o[nt][c][h] * inv * half * half;
            dst[16 * c + 8] = o[nt][c][h + 2] * inv * half * half;
          }
          if (rowq == 0) *reinterpret_cast<float4*>(mypart + head * kPartialStride + 128) = make_float4(mx[nt][h], l[nt][h], m[nt][h], 0.f);
        }
      }
    __syncwarp();
    if (whole) {
      for (int hh = 0; hh < G; ++hh) {
        const float4 v = *reinterpret_cast<const float4*>(mypart + hh * kPartialStride + lane * 4);
        const float2 ml = *reinterpret_cast<const float2*>(mypart + hh * kPartialStride + 128);
        const int64_t item = (int64_t)r * a.num_q_heads + h0 + hh;
        *reinterpret_cast<uint2*>(a.out + item * 128 + lane * 4) = make_uint2(pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w));
        if (a.lse != nullptr && lane == 0) a.lse[item] = ml.y != 0.f ? (ml.x + log2f(ml.y)) * kLn2 : -INFINITY;
      }
      __syncwarp();
    } else if (left > 0) {
      // more segments follow and will reuse the ring: this partial waits in the worker's global slot
      const int rec4 = G * (kPartialStride / 4);
      float4* slot = reinterpret_cast<float4*>(a.part) + (int64_t)w * rec4;
      const float4* src = reinterpret_cast<const float4*>(mypart);
      for (int i = lane; i < rec4; i += 32) __stcg(slot + i, src[i]);
      __syncwarp();
    }
  }
  wait_now();
  __syncthreads();

  // ---- block-level merge: (unit, query head) jobs dealt over the warps ----------------------------------------------
  const int w0 = (int)blockIdx.x * a.wpb;
  if (w0 >= W) return;
  const int nw = min(W - w0, a.wpb);
  const int b_lo = span_tab[0].x, b_hi = span_tab[nw - 1].y;
  const int rec4 = G * (kPartialStride / 4);
  const float4* early = reinterpret_cast<const float4*>(a.part);
  float4* bpart = reinterpret_cast<float4*>(a.part) + (int64_t)W * rec4;  // 2 records per block: its first unit, its last

  // Up to 32 partials at once, lane i holding the references and sum (mx, l, m) of the i-th and fetch(i) its outputs.
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  float L = 0.f, MX = kNone, M = kNone;
  auto fold = [&](float4 ml, int count, auto fetch) {
    float xn = fmaxf(MX, ml.x);
#pragma unroll
    for (int d = 16; d >= 1; d >>= 1) xn = fmaxf(xn, __shfl_xor_sync(0xffffffffu, xn, d));
    const float mnew = (ml.x - xn) + ml.z, mold = (MX - xn) + M;  // references to x - xn + ev
    float mn = fmaxf(mold, mnew);
#pragma unroll
    for (int d = 16; d >= 1; d >>= 1) mn = fmaxf(mn, __shfl_xor_sync(0xffffffffu, mn, d));
    const float sn = fast_exp2(mnew - mn), so = fast_exp2(mold - mn);
    float sum = fast_exp2(ml.x - xn) * ml.y;
#pragma unroll
    for (int d = 16; d >= 1; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    L = L * fast_exp2(MX - xn) + sum;
    acc.x *= so; acc.y *= so; acc.z *= so; acc.w *= so;
#pragma unroll 4
    for (int i = 0; i < count; ++i) {
      const float4 v = fetch(i);
      const float f = __shfl_sync(0xffffffffu, sn, i);
      acc.x = fmaf(f, v.x, acc.x); acc.y = fmaf(f, v.y, acc.y); acc.z = fmaf(f, v.z, acc.z); acc.w = fmaf(f, v.w, acc.w);
    }
    M = mn;
    MX = xn;
  };
  const float4 nothing = make_float4(kNone, 0.f, kNone, 0.f);

  const int2 my_split = lane < 2 * nw ? split_tab[lane >> 1] : make_int2(-1, -1);
  const int my_unit = lane & 1 ? my_split.y : my_split.x;
  const int2 my_span = lane < nw ? span_tab[lane] : make_int2(0, 0);
  int hh = warp;
  for (uint32_t todo = __ballot_sync(0xffffffffu, my_unit >= 0); todo != 0u; todo &= todo - 1u, hh -= G) {
    const int own = (__ffs(todo) - 1) >> 1, u = __shfl_sync(0xffffffffu, my_unit, __ffs(todo) - 1);
    const int us = u * NS, ue = us + NS;
    const int nparts = __popc(__ballot_sync(0xffffffffu, lane >= own && lane < nw && my_span.x < ue));  // warps own .. share it
    for (; hh < G; hh += WARPS) {
      acc = make_float4(0.f, 0.f, 0.f, 0.f);
      L = 0.f;
      MX = M = kNone;
      auto record = [&](int lw) -> const float4* {  // partial of warp lw: in its ring if the unit was the last of its walk
        const int2 sp = span_tab[lw];
        const int last = a.reverse ? sp.x : sp.y - 1;
        return last >= us && last < ue ? reinterpret_cast<const float4*>(smem + lw * S::kRing) + hh * (kPartialStride / 4)
                                       : early + (int64_t)(w0 + lw) * rec4 + hh * (kPartialStride / 4);
      };
      fold(lane < nparts ? record(own + lane)[32] : nothing, nparts, [&](int i) { return record(own + i)[lane]; });
      const int g = u / a.rows, r = u - g * a.rows;
      const int64_t item = (int64_t)r * a.num_q_heads + g * G + hh;
      if (!(b_lo <= us && b_hi >= ue)) {
        // the unit straddles blocks: leave this block's partial, arrive, and finish the pair if this completes it
        float4* slot = bpart + (int64_t)(2 * blockIdx.x + (b_lo < us ? 1 : 0)) * rec4 + hh * (kPartialStride / 4);
        __stcg(slot + lane, acc);
        if (lane == 0) __stcg(slot + 32, make_float4(MX, L, M, 0.f));
        asm volatile("fence.acq_rel.gpu;" ::: "memory");
        __syncwarp();
        int wf, wl;
        unit_workers(u, a, wf, wl);
        const int blk_first = wf / a.wpb, blk_last = wl / a.wpb;
        const int lo_first = span_begin(blk_first * a.wpb, a);
        uint32_t* counter = a.arrive + blk_first * kMaxGroup + hh;  // one unit at most leaves a block to the right
        unsigned prev = 0;
        if (lane == 0) prev = atomicAdd(counter, 1u);
        prev = __shfl_sync(0xffffffffu, prev, 0);
        if (prev + 1u != (unsigned)(blk_last - blk_first + 1)) continue;
        asm volatile("fence.acq_rel.gpu;" ::: "memory");
        if (lane == 0) *counter = 0u;
        acc = make_float4(0.f, 0.f, 0.f, 0.f);
        L = 0.f;
        MX = M = kNone;
        auto block_record = [&](int b2) {
          const int kind = b2 == blk_first && lo_first < us ? 1 : 0;
          return bpart + (int64_t)(2 * b2 + kind) * rec4 + hh * (kPartialStride / 4);
        };
        for (int b0 = blk_first; b0 <= blk_last; b0 += 32)  // in block order: the result does not depend on who arrived last
          fold(b0 + lane <= blk_last ? __ldcg(block_record(b0 + lane) + 32) : nothing, min(32, blk_last - b0 + 1),
               [&](int i) { return __ldcg(block_record(b0 + i) + lane); });
      }
      if (L != 0.f) {
        const float inv = 1.f / L, half = fast_exp2(0.5f * M);
        acc.x = acc.x * inv * half * half; acc.y = acc.y * inv * half * half;
        acc.z = acc.z * inv * half * half; acc.w = acc.w * inv * half * half;
      }
      *reinterpret_cast<uint2*>(a.out + item * 128 + lane * 4) = make_uint2(pack_bf16x2(acc.x, acc.y), pack_bf16x2(acc.z, acc.w));
      if (a.lse != nullptr && lane == 0) a.lse[item] = L != 0.f ? (MX + log2f(L)) * kLn2 : -INFINITY;
    }
  }
}

constexpr int kWarpsNarrow = 12, kStagesNarrow = 2;  // groups of up to 8 query heads
constexpr int kWarpsWide = 8, kStagesWide = 3;       // wider groups: twice the accumulators per thread

}  // namespace

Attn8Plan make_attn8_plan(const clsa_params& p, const DeviceInfo& dev) {
  Attn8Plan plan;
  const bool wide = p.num_q_heads / p.num_kv_heads > 8;
  plan.warps = wide ? kWarpsWide : kWarpsNarrow;
  plan.smem_bytes = wide ? Shape<kWarpsWide, kStagesWide>::kSmem : Shape<kWarpsNarrow, kStagesNarrow>::kSmem;
  plan.units = (int64_t)p.num_seqs * p.q_per_seq * p.num_kv_heads;
  plan.unit_stages = (p.top_k + kTok - 1) / kTok;
  plan.total_stages = plan.units * plan.unit_stages;
  int64_t blocks, workers;
  if (plan.units <= dev.sm_count) {
    // Every unit has blocks of its own, as many as give a warp two stages. (2048 rows of one sequence, 8 units: 10.7 us with two, 10.0 with
    // one, 11.4 with four; 1024 rows of one unit: 9.7, 10.0, 8.8; 256 rows: all 6.0.)
    int64_t per_unit = dev.sm_count / plan.units;
    const int64_t most = (plan.unit_stages + 2 * plan.warps - 1) / (2 * plan.warps);
    if (per_unit > most) per_unit = most;
    plan.wpb = (int)((plan.unit_stages + per_unit - 1) / per_unit);
    if (plan.wpb > plan.warps) plan.wpb = plan.warps;
    while (per_unit * plan.wpb > plan.unit_stages) --per_unit;  // no worker without a stage
    blocks = plan.units * per_unit;
    workers = blocks * plan.wpb;
    plan.mode = kAttn8Units;
  } else {
    blocks = dev.sm_count;
    workers = plan.total_stages < blocks * plan.warps ? plan.total_stages : blocks * plan.warps;
    plan.wpb = (int)((workers + blocks - 1) / blocks);
    blocks = (workers + plan.wpb - 1) / plan.wpb;
    // Whole units per block, where the blocks with one unit more have at most six stages per warp more than the even share: that
    // leaves no unit to two blocks and few to two warps (2048 rows: 192 units 26.5 us against 30.8 otherwise, 256 units 29.8 against 36.9;
    // 152 units 25.2 against 23.7. 8192 rows, past the bound: 152 units 77.8 against 65.0, 192 units 80.3 against 77.8, but 224 units
    // 85.6 against 92.5). Else, where every unit can have workers of its own and the longest span that results stays
    // within 15 % of the even share, those (8192 rows: 152 units 65.0 against 68.3 for the flat list, 192 units 77.8 against 83.6).
    const int64_t most = (plan.units + blocks - 1) / blocks;
    plan.mode = kAttn8Flat;
    if (plan.wpb == plan.warps && (most * blocks - plan.units) * plan.unit_stages <= 6 * blocks * plan.warps) {
      plan.mode = kAttn8Blocks;
      workers = blocks * plan.warps;
    } else if (workers >= plan.units) {
      const int64_t longest = (plan.unit_stages + workers / plan.units - 1) / (workers / plan.units);
      if (longest * workers * 100 <= plan.total_stages * 115) plan.mode = kAttn8Units;
    }
  }
  plan.blocks = (int)blocks;
  plan.workers = (int)workers;
  return plan;
}

size_t attn8_counter_bytes(const DeviceInfo& dev) { return ((size_t)dev.sm_count * kMaxGroup * sizeof(uint32_t) + 255) / 256 * 256; }

size_t attn8_partial_bytes(const clsa_params& p, const Attn8Plan& plan) {
  const size_t group = (size_t)(p.num_q_heads / p.num_kv_heads);
  return (((size_t)plan.workers + 2 * plan.blocks) * group * kPartialStride * sizeof(float) + 255) / 256 * 256;
}

cudaError_t launch_sparse_attn8(const clsa_params& p, const clsa_cache8& c, const Attn8Plan& plan, const void* q,
                                const int32_t* idx, const int32_t* count, void* out, float* lse, const clsa_attn_hints& hints,
                                uint32_t* status, uint32_t* arrive, float* part, const DeviceInfo& dev, cudaStream_t stream) {
  Attn8Args a = {};
  a.q = static_cast<const uint16_t*>(q);
  a.kc = static_cast<const uint8_t*>(c.k);
  a.vc = static_cast<const uint8_t*>(c.v);
  a.ks = static_cast<const uint8_t*>(c.k_scale);
  a.vs = static_cast<const uint8_t*>(c.v_scale);
  a.head_stride = c.kv_head_stride;
  a.scale_head = c.scale_head_stride;
  a.unit = 16;
  a.stride16 = (uint32_t)(c.kv_token_stride / 16);
  while ((1 << a.scale_shift) < c.scale_block) ++a.scale_shift;
  a.num_rows = p.num_cache_rows;
  a.seq_start = p.seq_start;
  a.seq_len = p.seq_len;
  a.idx = idx;
  a.count = count;
  a.block_table = p.block_table;
  while (p.block_table != nullptr && (1 << a.block_shift) < p.block_size) ++a.block_shift;
  a.max_blocks = p.max_blocks_per_seq;
  a.page_limit = (uint32_t)((p.num_cache_rows + (1 << a.block_shift) - 1) >> a.block_shift);
  a.out = static_cast<uint16_t*>(out);
  a.lse = lse;
  a.status = status;
  a.rows = p.num_seqs * p.q_per_seq;
  a.q_per_seq = p.q_per_seq;
  a.num_q_heads = p.num_q_heads;
  a.num_kv_heads = p.num_kv_heads;
  a.group = p.num_q_heads / p.num_kv_heads;
  a.top_k = p.top_k;
  a.max_seq_len = p.max_seq_len;
  a.reverse = hints.reverse;
  a.early = hints.only_q_pending;
  a.keep = hints.keep_rows;
  // keep_rows: all of the selected set evict_last where half of L2 holds it, else the share of every 8 stages that fits
  a.pin = -1;
  if (hints.keep_rows) {
    const double k_eff = (double)(p.top_k < p.max_seq_len ? p.top_k : p.max_seq_len);
    const double gathered = (double)a.rows * k_eff * p.num_kv_heads * p.head_dim * 2.0;
    const int pin = (int)(8.0 * 0.5 * (double)dev.l2_bytes / gathered + 0.5);
    a.pin = pin >= 8 ? -1 : (pin < 1 ? 1 : pin);
  }
  a.unit_stages = plan.unit_stages;
  a.total_stages = (int)plan.total_stages;  // < 2^31, checked by the entry point
  a.mode = plan.mode;
  const int64_t split = plan.mode == kAttn8Flat ? plan.total_stages : plan.units;  // over the workers, or the blocks
  const int64_t over = plan.mode == kAttn8Blocks ? plan.blocks : plan.workers;
  a.span_q = plan.mode == kAttn8Units ? (int)(plan.workers / plan.units) : (int)(split / over);
  a.span_rem = plan.mode == kAttn8Units ? (int)(plan.workers % plan.units) : (int)(split % over);
  a.workers = plan.workers;
  a.wpb = plan.wpb;
  a.arrive = arrive;
  a.part = part;
  a.scale_log2 = p.sm_scale * kLog2e;
  const bool paged = p.block_table != nullptr, wide = a.group > 8;
  void (*kernel)(const Attn8Args) =
      wide ? (paged ? sparse_attn8_kernel<2, false, kWarpsWide, kStagesWide, true> : sparse_attn8_kernel<2, false, kWarpsWide, kStagesWide, false>)
      : a.group > 4 ? (paged ? sparse_attn8_kernel<1, false, kWarpsNarrow, kStagesNarrow, true> : sparse_attn8_kernel<1, false, kWarpsNarrow, kStagesNarrow, false>)
                    : (paged ? sparse_attn8_kernel<1, true, kWarpsNarrow, kStagesNarrow, true> : sparse_attn8_kernel<1, true, kWarpsNarrow, kStagesNarrow, false>);
  cudaError_t err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)plan.smem_bytes);
  if (err != cudaSuccess) return err;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)plan.blocks, 1, 1);
  cfg.blockDim = dim3((unsigned)plan.warps * 32, 1, 1);
  cfg.dynamicSmemBytes = plan.smem_bytes;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, a);
}

}  // namespace clsa
