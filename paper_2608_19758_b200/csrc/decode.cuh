// Attention of the newest few tokens of every sequence over its paged cache (token by token decoding, verification of drafts),
// with an optional sliding window and sinks:
//   x_ij = scale ks_j q_i . K_j,   visible iff j <= p_i and (W == 0 or p_i - j < W or j < S),   p_i = Lk - Lq + i
//   out_i = sum_j 2^(x_ij - m) vs_j V_j / sum_j 2^(x_ij - m)           (x in units of log2, one pass with a running maximum)
//
// Bound by the bytes of the cache: each is wanted once, the arithmetic of a group of query heads on them is small.  So:
//
// Work split.  The (sequence, KV head, tile of packed rows, block of tokens) items are numbered in that order, and every CTA of a
// grid that fills the GPU takes an equal contiguous share, whatever the lengths: a long sequence is cut wherever shares end.  The
// lengths are read on the device (a captured graph stays valid as sequences grow), so the CTAs find their shares themselves.  A
// unit (sequence, head, tile) cut into parts leaves (O, m, l) of each in the workspace; the CTA that arrives last of each group of
// 16 parts joins these, the last of the groups these, both in the order of the shares: the result does not depend on who is
// last.  One launch.
//
// A CTA is four warps, two CTAs to an SM.  Of a block each warp takes a step of kTok tokens (8 KB), which it copies into its own
// part of shared memory (cp.async, kStages steps ahead) and attends to with its own running maximum and sum: no barrier in the
// loop; the four join at the end of a unit, while the first copies of the next one are on their way.  Copies of hidden tokens
// write zeros without reading, so nothing that stands in a hidden place reaches the sums.  192 KB of an SM take part.
// (By TMA, a box per page and operand, lanes in turn: everything 4 to 6 % slower.)
//
// Measured, whole calls: 64 sequences of 4096 tokens, 8 KV heads, 168 us in BF16 (6.4 TB/s, 0.98 of the copy rate), 100 to 105 us in 8 bits
// (by card; 5.4 TB/s, 0.82; 37 sequences of 8192 tokens, a whole unit per CTA, 6.2 TB/s: the rest is the units' ends, 2.5 parts per CTA);
// 131072 tokens of 4 heads 52 us in BF16, of which 41 are the bytes, 5 the start and 5 the joining of 74 parts per head.
//
// S^T = K Q^T and O^T += V^T P^T are m16n8k16 MMAs of a warp with the tokens (then the dims) as the long side and 8 packed
// (token, query head) rows of the KV head as the short one, NR times: a group of eight heads fills it.  What tcgen05
// would add in rate is not what bounds this, and its 64 rows are what such a group has no use for.  K and V are read from shared
// memory 16 bytes a lane; which of a lane's values play which index of the contraction over dims in K Q^T, or which row (a dim) of
// V^T, is free as long as Q is permuted alike and O stored accordingly, so nothing is transposed but P (8 x 8 at a time, one
// instruction) and pairs of tokens of V (byte permutation).
//
// Precision.  BF16 caches: Q and K as they are; P as a BF16 pair hi + lo (2^-17).  e4m3 caches: K, V exact as F16; Q exact as
// F16 after a power of two per row has brought its maximum to 2^13 .. 2^14 (elements 2^-28 below it round); P as F16 against a
// reference 8 binades below the running maximum, where the steps are 2^-11 relative down to 2^-22 of the maximum.  Sums in 32 bits.
// (The warp-level MMA takes e4m3 operands as such, Q as a pair of them; K Q^T then took twice the instructions: it widens them itself.)
// Scales per page: ks multiplies the logits; vs enters P, in the exponent, so that P V needs none: y = x + log2 vs has the running
// maximum of P, p = 2^(y - m).  The sum of the weights has a reference of its own, l = sum 2^(x - e): scales may lie 2^200 and more
// apart (2^-100 is the writer's for a page of zeros), so what y hides can be the whole of l, and 2^-m is no unit for it.
// (64 ragged sequences of 8-bit pages: 95.6 us with l taken back from P, p / vs, which loses weights and leaves fp32; 94.0 so.  On
// another card 97.5 / 102.)
#pragma once
#include <cuda_bf16.h>
#include "common.cuh"
#include "kv_cache.cuh"
#include "ptx.cuh"

namespace fp2 {

constexpr int kDecWarps = 4;
constexpr int kDecThreads = 32 * kDecWarps;
constexpr int kDecCtasPerSm = 2;
// What the split goes by, in blocks, and what whole calls took with other values (us):
// A unit costs this much beside its blocks (0 / 2 / 4 / 8: 64 ragged sequences of 8-bit pages 141 / 107 / 99 / 107).
constexpr int kDecUnitCost = 4;
// Units up to this long, with that, are not cut: they belong to the share that they begin in (12 / 20: the same 102 / 108).
constexpr int kDecWhole = 12;
// Least share of a CTA, with that (5 / 6 / 8: one sequence of 2048 tokens, BF16, 10.8 / 11.6 / 13.2).
constexpr int kDecMinShare = 5;
// Parts of a unit that are joined at a time, and of these in a warp's registers (all parts by one CTA, four warps side by side: 131072
// tokens BF16 58.4; 16, four at a time 55.5; 8, two at a time 53.8, but 8192 tokens 19.6 against 16.9; 16, two at a time 53.1).
constexpr int kDecGroup = 16;
constexpr int kDecJoin = 2;

template <int FMT, int NR>
struct DecodeCfg {
  static constexpr bool kFp8 = FMT != FMT_BF16;
  static constexpr int kEsz = kFp8 ? 1 : 2;
  static constexpr int kTok = kFp8 ? 32 : 16;                     // tokens of a step
  static constexpr int kBlock = kTok * kDecWarps;                 // tokens of a work item
  static constexpr int kHalf = kTok * 128;                        // kTok rows of 128 bytes
  static constexpr int kTile = kHalf * kEsz;                      // K (or V) of a step, of one head: 4 KB
  static constexpr int kStep = 2 * kTile;
  static constexpr int kStages = 3;
  static constexpr int kRing = kStages * kStep;                   // of a warp
  static constexpr int kRows = 8 * NR;
  // stages that may be filled for the next unit while the warps' results of this one are joined in the others
  static constexpr int kEarly = (kRing - kRows * kHeadDim * 4) / kStep;
  static_assert(kEarly >= 1 && kEarly < kStages, "the join needs room, the next unit a start");
  static constexpr int kSmemBytes = 128 + kDecWarps * kRing;      // 96 KB
};

struct DecodeArgs {
  const uint8_t* q;             // BF16
  long long q_stride_bytes;
  const int32_t *cu, *lk, *page_table;
  const uint8_t *k, *v;
  const float *k_scale, *v_scale;
  __nv_bfloat16* out;
  float* lse;
  float* part_o;                // [2 grid][8 NR][128]
  void* part_ml;                // [2 grid][8 NR] RowState
  int32_t* counters;            // [3][grid], zero between calls: parts of a unit's first group, of a later group, groups of a unit
  int* status;
  int32_t total_q, num_q_heads, group, window, sinks;
  uint32_t group_magic;         // 2^32 / group rounded up, 0 for a group of one: see div_group
  float scale_log2;
  CacheGeom g;
};

// What goes with a row's O: its references and its sum, out = O 2^(m - e) / l, lse = e + log2 l.  Without scales per page e is m.
template <bool OWN_E> struct RowState;
template <> struct alignas(8) RowState<false> {
  float m, l;
  static __device__ __forceinline__ RowState none() { return {-INFINITY, 0.f}; }
  __device__ __forceinline__ float e() const { return m; }
  __device__ __forceinline__ void set_e(float) {}
  __device__ __forceinline__ void store_cg(void* p, long long i) const { __stcg((float2*)p + i, make_float2(m, l)); }
  static __device__ __forceinline__ RowState load_cg(const void* p, long long i) { const float2 v = __ldcg((const float2*)p + i); return {v.x, v.y}; }
};
template <> struct alignas(16) RowState<true> {
  float m, l, own, unused;
  static __device__ __forceinline__ RowState none() { return {-INFINITY, 0.f, -INFINITY, 0.f}; }
  __device__ __forceinline__ float e() const { return own; }
  __device__ __forceinline__ void set_e(float x) { own = x; }
  __device__ __forceinline__ void store_cg(void* p, long long i) const { __stcg((float4*)p + i, make_float4(m, l, own, 0.f)); }
  static __device__ __forceinline__ RowState load_cg(const void* p, long long i) { const float4 v = __ldcg((const float4*)p + i); return {v.x, v.y, v.z, 0.f}; }
};
constexpr int kRowStateBytes = sizeof(RowState<true>);

// One sequence's share of the work
struct DecodeSeq {
  int c0, Lq, L;      // first query row, queries, tokens in the cache
  int ntiles;         // tiles of packed rows of a KV head
  int sb, wb0, nblk;  // blocks: 0 .. sb - 1 (sinks), then wb0 .. ; nblk in all
  long long cost;     // blocks of all units, kDecUnitCost more for each
};

template <typename Cfg>
__device__ __forceinline__ DecodeSeq decode_seq(const DecodeArgs& A, int b, bool report) {
  constexpr int B = Cfg::kBlock;
  DecodeSeq s;
  s.c0 = A.cu[b];
  const int c1 = A.cu[b + 1];
  s.L = A.lk[b];
  s.Lq = c1 - s.c0;
  if (s.c0 < 0 || c1 < s.c0 || c1 > A.total_q || s.L < 0 || s.L > ((long long)A.g.max_pages << A.g.page_shift)) {
    if (report) atomicOr(A.status + kCacheStBad, kBadLength);
    s.Lq = 0;
    s.L = 0;
    s.c0 = 0;
  }
  s.ntiles = (int)(((long long)A.group * s.Lq + Cfg::kRows - 1) / Cfg::kRows);
  // tokens some query sees: below the sinks, and from the first query's window on
  const int first = s.L - s.Lq;
  const int lo = A.window > 0 ? max(0, (int)min((long long)s.L, (long long)first - A.window + 1)) : 0;
  s.wb0 = lo / B;
  s.sb = min((int)(((long long)min(A.sinks, s.L) + B - 1) / B), s.wb0);
  s.nblk = max(1, s.sb + (s.L + B - 1) / B - s.wb0);   // (one for rows that see nothing: they are written)
  s.cost = (long long)s.ntiles * A.g.num_kv_heads * (s.nblk + kDecUnitCost);
  return s;
}

__device__ __forceinline__ void mma_16816_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_16816_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// 8 x 8 matrix of 16-bit elements, row i in the lanes 4 i .. 4 i + 3: transposed
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}
// four e4m3 bytes -> two pairs of F16 (exact)
__device__ __forceinline__ void e4m3x4_to_f16x4(uint32_t x, uint32_t& lo, uint32_t& hi) {
  asm("{\n .reg .b16 l, h;\n mov.b32 {l, h}, %2;\n cvt.rn.f16x2.e4m3x2 %0, l;\n cvt.rn.f16x2.e4m3x2 %1, h;\n}" : "=r"(lo), "=r"(hi) : "r"(x));
}
// 16 bytes global -> shared; zeros without reading
__device__ __forceinline__ void cp_async16(uint32_t smem_dst, const void* gsrc) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_dst), "l"(gsrc) : "memory");
}
__device__ __forceinline__ void cp_async16_if(uint32_t smem_dst, const void* gsrc, bool read) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_dst), "l"(gsrc), "r"(read ? 16u : 0u) : "memory");
}
__device__ __forceinline__ void cp_async4_if(uint32_t smem_dst, const void* gsrc, bool read) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(smem_dst), "l"(gsrc), "r"(read ? 4u : 0u) : "memory");
}
__device__ __forceinline__ uint4 lds128(uint32_t a) {
  uint4 r;
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "r"(a) : "memory");
  return r;
}

// a / b for a >= 0, b > 0; the 64-bit division is a long routine, and seldom needed
__device__ __forceinline__ long long div_ll(long long a, long long b) {
  return ((a | b) >> 32) == 0 ? (long long)((uint32_t)a / (uint32_t)b) : a / b;
}

// x / group for x up to group + 32 (exact while x group < 2^32; a group has at most 2^13 heads)
__device__ __forceinline__ int div_group(const DecodeArgs& A, int x) { return A.group_magic ? (int)__umulhi((uint32_t)x, A.group_magic) : x; }

// A unit's part of this CTA: blocks i0 .. i1 - 1 of it
struct DecodeUnit {
  int b, h, nrows;
  int tok0, rem;               // query (of the sequence) of the first row, rows of that query in front of the tile
  int c0, first_pos, L, sb, wb0;
  int pmin, pmax;              // positions of the first and last row
  int i0, i1;
  bool whole;
  int w0, parts;               // CTAs that share the unit: the first one, how many
};

template <int FMT, int NR>
__global__ void __launch_bounds__(kDecThreads, kDecCtasPerSm)
decode_kernel(DecodeArgs A) {
  using Cfg = DecodeCfg<FMT, NR>;
  constexpr bool FP8 = Cfg::kFp8, OWN_E = FMT == FMT_FP8_PAGE;
  using State = RowState<OWN_E>;
  constexpr int RT = Cfg::kRows, ST = Cfg::kStages, TOK = Cfg::kTok;
  constexpr int G = TOK / 8;             // groups of eight tokens of a step: what a page holds at least
  constexpr uint32_t kAllLive = TOK == 32 ? 0xffffffffu : (1u << TOK) - 1u;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 127) & ~uintptr_t(127));
  __shared__ float page_scales[kDecWarps][ST][2 * G];      // PAGE: ks of the groups, then vs
  __shared__ uint32_t live_s[kDecWarps][ST];               // tokens of the step that were copied
  __shared__ State ml_s[kDecWarps][RT];
  __shared__ long long scan_s[kDecWarps];
  __shared__ long long found_base;                         // (the sequence that the share begins in, what is in front of it)
  __shared__ int found_b, last_s;

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int c = lane & 3, l4 = lane >> 2;
  const int heads = A.g.num_kv_heads, shift = A.g.page_shift, grp = A.group;
  pdl_trigger();
  pdl_wait();

  // ------------------------------ this CTA's share ------------------------------
  // Costs of kDecThreads sequences from b0 on: this thread's and those in front of it; returns their sum.
  auto scan = [&](int b0, long long& lo, long long& cost, bool report) -> long long {
    cost = b0 + tid < A.g.num_seqs ? decode_seq<Cfg>(A, b0 + tid, report).cost : 0;
    long long incl = cost, all = 0;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const long long o = __shfl_up_sync(0xffffffffu, incl, d);
      if (lane >= d) incl += o;
    }
    if (lane == 31) scan_s[warp] = incl;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kDecWarps; ++i) {
      if (i < warp) incl += scan_s[i];
      all += scan_s[i];
    }
    lo = incl - cost;
    return all;
  };
  long long lo, cost, all = scan(0, lo, cost, blockIdx.x == 0);
  long long total = all;
  for (int b0 = kDecThreads; b0 < A.g.num_seqs; b0 += kDecThreads) {
    long long x, y;
    __syncthreads();
    total += scan(b0, x, y, blockIdx.x == 0);
  }
  const long long share = max(div_ll(total + gridDim.x - 1, gridDim.x), (long long)kDecMinShare);
  long long pos = share * blockIdx.x;
  const long long pos_end = min(total, pos + share);
  if (pos >= pos_end) return;
  {
    long long base = 0;
    for (int b0 = 0;; b0 += kDecThreads) {   // (the first 128 sequences' numbers are here still)
      if (b0 > 0) {
        __syncthreads();
        all = scan(b0, lo, cost, false);
      }
      if (pos >= base + lo && pos < base + lo + cost) {
        found_b = b0 + tid;
        found_base = base + lo;
      }
      base += all;
      if (base > pos) break;
    }
    __syncthreads();
  }
  // The unit that `pos` is in: sequence, head, tile, first place.  A unit takes kDecUnitCost places in front of its blocks'.
  int b = found_b;
  DecodeSeq sq = decode_seq<Cfg>(A, b, false);
  int uh, ut;
  long long unit0;
  {
    const long long unit = div_ll(pos - found_base, sq.nblk + kDecUnitCost);
    uh = (int)div_ll(unit, sq.ntiles);
    ut = (int)(unit - (long long)uh * sq.ntiles);
    unit0 = found_base + unit * (sq.nblk + kDecUnitCost);
  }
  // Next part of a unit of the share
  auto next_unit = [&](DecodeUnit& u) -> bool {
    while (pos < pos_end) {
      const int ulen = sq.nblk + kDecUnitCost;
      const long long unit_end = unit0 + ulen;
      if (ulen <= kDecWhole) {
        u.i0 = pos > unit0 ? sq.nblk : 0;
        u.i1 = sq.nblk;
        pos = unit_end;
      } else {
        u.i0 = max(0, (int)(pos - unit0) - kDecUnitCost);
        u.i1 = max(0, (int)(min(unit_end, pos_end) - unit0) - kDecUnitCost);
        pos = min(unit_end, pos_end);
      }
      const bool some = u.i0 < u.i1;
      if (some) {
        u.b = b;
        u.h = uh;
        u.c0 = sq.c0;
        u.L = sq.L;
        u.sb = sq.sb;
        u.wb0 = sq.wb0;
        u.first_pos = sq.L - sq.Lq;
        const int r0 = ut * RT;
        u.nrows = min(RT, grp * sq.Lq - r0);
        u.tok0 = ut ? r0 / grp : 0;
        u.rem = r0 - u.tok0 * grp;
        u.pmin = u.first_pos + u.tok0;
        u.pmax = u.pmin + div_group(A, u.rem + u.nrows - 1);
        u.whole = u.i0 == 0 && u.i1 == sq.nblk;
        u.w0 = blockIdx.x;
        u.parts = 1;
        if (!u.whole) {
          u.w0 = (int)div_ll(unit0 + kDecUnitCost, share);
          u.parts = (int)div_ll(unit_end - 1, share) - u.w0 + 1;
        }
      }
      if (pos >= unit_end) {
        unit0 = unit_end;
        if (++ut == sq.ntiles) {
          ut = 0;
          if (++uh == heads && pos < pos_end) {
            uh = 0;
            do sq = decode_seq<Cfg>(A, ++b, false);
            while (sq.cost == 0 && b + 1 < A.g.num_seqs);   // (items are left: there is one)
          }
        }
      }
      if (some) return true;
    }
    return false;
  };
  // Row of the unit's tile -> query of the sequence and query head
  auto row_of = [&](const DecodeUnit& u, int row, int& tok, int& head) {
    const int x = u.rem + row, d = div_group(A, x);
    tok = u.tok0 + d;
    head = u.h * grp + x - d * grp;
  };

  // ------------------------------ copies ------------------------------
  const uint32_t ring = smem_u32(smem) + warp * Cfg::kRing;
  constexpr int kLanes = 8 * Cfg::kEsz;                    // lanes per row, 16 bytes each
  constexpr int kRowsPer = 32 / kLanes;                    // rows per instruction
  constexpr int kPerGroup = 8 / kRowsPer;                  // instructions per group of eight rows
  const uint32_t row_bytes = (uint32_t)heads * (kHeadDim * Cfg::kEsz);
  const int ch = lane % kLanes, rsub = lane / kLanes;
  const uint32_t dst_lane = ring + (ch >> 3) * Cfg::kHalf + rsub * 128 + (((ch & 7) ^ rsub) << 4);
  auto token0 = [&](const DecodeUnit& u, int i) { return Cfg::kBlock * (i < u.sb ? i : u.wb0 + i - u.sb) + warp * TOK; };
  // Page ids of 32 / G steps: lane G k + j holds the one of step k's tokens 8 j .. 8 j + 7
  auto load_pids = [&](const DecodeUnit& u, int i) -> int {
    i += lane / G;
    const int tok = token0(u, i) + (lane % G) * 8;
    return i < u.i1 && tok < u.L ? A.page_table[(size_t)u.b * A.g.max_pages + (tok >> shift)] : -1;
  };
  int pids = -1, pids_next = -1;
  auto issue = [&](const DecodeUnit& u, int k, int slot) {           // step k of the unit's part, into stage `slot`
    const int i = u.i0 + k;
    if (i < u.i1) {
      const int k0 = k % (32 / G) * G;
      if (k0 == 0) {
        pids = pids_next;
        pids_next = load_pids(u, i + 32 / G);
      }
      const int t0 = token0(u, i);
      int pid[G];
      bool there = true;
#pragma unroll
      for (int j = 0; j < G; ++j) {
        pid[j] = __shfl_sync(0xffffffffu, pids, k0 + j);
        there &= (uint32_t)pid[j] < (uint32_t)A.g.num_pages;
      }
      const bool full = there && t0 + TOK - 1 <= u.pmax && (A.window <= 0 || t0 > u.pmin - A.window || t0 + TOK - 1 < A.sinks);
      const uint32_t dst = dst_lane + slot * Cfg::kStep;
      const uint32_t head_off = (uint32_t)u.h * (kHeadDim * Cfg::kEsz) + ch * 16;
      const int mask = (1 << shift) - 1;
      const uint8_t *kp = A.k + head_off, *vp = A.v + head_off;
      uint32_t live = kAllLive;
      if (full) {
#pragma unroll
        for (int j = 0; j < G; ++j) {
          const uint32_t row = ((uint32_t)pid[j] << shift) + ((t0 + 8 * j) & mask) + rsub;   // (slots of the pool: 31 bits)
#pragma unroll
          for (int q = 0; q < kPerGroup; ++q) {
            const uint64_t off = (uint64_t)(row + q * kRowsPer) * row_bytes;
            const uint32_t d = (dst ^ ((q * kRowsPer) << 4)) + (j * 8 + q * kRowsPer) * 128;
            cp_async16(d, kp + off);
            cp_async16(d + Cfg::kTile, vp + off);
          }
        }
      } else {
        const int my = (lane % TOK) / 8, tok = t0 + lane % TOK;
        int p = pid[0];
#pragma unroll
        for (int j = 1; j < G; ++j) p = my == j ? pid[j] : p;
        const bool wanted = tok <= u.pmax && tok < u.L && (A.window <= 0 || tok > u.pmin - A.window || tok < A.sinks);
        const bool ok = (uint32_t)p < (uint32_t)A.g.num_pages;
        if (__any_sync(0xffffffffu, wanted && !ok) && lane == 0) atomicOr(A.status + kCacheStBad, kBadPage);
        live = __ballot_sync(0xffffffffu, wanted && ok) & kAllLive;
        if (live != 0u) {
#pragma unroll 1
          for (int r = rsub; r < TOK; r += kRowsPer) {
            const bool read = (live >> r) & 1u;
            const int pr = __shfl_sync(0xffffffffu, p, r);           // (rows of one group in all lanes: its page)
            const uint64_t off = read ? (uint64_t)(((uint32_t)pr << shift) + ((t0 + r) & mask)) * row_bytes : 0;
            const uint32_t d = ring + slot * Cfg::kStep + (ch >> 3) * Cfg::kHalf + r * 128 + (((ch & 7) ^ (r & 7)) << 4);
            cp_async16_if(d, kp + off, read);
            cp_async16_if(d + Cfg::kTile, vp + off, read);
          }
        }
      }
      if (lane == 0) live_s[warp][slot] = live;
      if constexpr (FMT == FMT_FP8_PAGE) {
        if (lane < 2 * G) {
          int p = pid[0];
#pragma unroll
          for (int j = 1; j < G; ++j) p = lane % G == j ? pid[j] : p;
          const bool ok = ((live >> (lane % G * 8)) & 0xffu) != 0u;
          cp_async4_if(smem_u32(&page_scales[warp][slot][lane]), (lane < G ? A.k_scale : A.v_scale) + (ok ? (size_t)p * heads + u.h : 0), ok);
        }
      }
    }
    cp_async_commit();
  };

  // Queries: lane (l4, c) holds row l4 of each 8-row tile, and of the contraction the dims that its 16-byte pieces of K hold: step s,
  // dims 32 c + 4 s .. + 3 (e4m3) or 64 (s >> 2) + 16 c + 4 (s & 3) .. + 3 (BF16).  Asked for ahead of the unit's copies: behind
  // them, with the memory busy, they took 4000 cycles.
  uint4 qraw[NR][4];
  float k_scale = 1.f, v_scale = 1.f;
  auto load_q = [&](const DecodeUnit& u) {
#pragma unroll
    for (int n = 0; n < NR; ++n) {
      int tok, head;
      row_of(u, min(n * 8 + l4, u.nrows - 1), tok, head);
      const uint8_t* src = A.q + (long long)(u.c0 + tok) * A.q_stride_bytes + head * (kHeadDim * 2);
#pragma unroll
      for (int s = 0; s < 4; ++s)
        qraw[n][s] = *reinterpret_cast<const uint4*>(src + 2 * (FP8 ? 32 * c + 8 * s : 64 * (s >> 1) + 16 * c + 8 * (s & 1)));
    }
    if constexpr (FMT == FMT_FP8_HEAD) {
      k_scale = A.k_scale[u.h];
      v_scale = A.v_scale[u.h];
    }
  };

  DecodeUnit u;
  if (!next_unit(u)) return;
  pids_next = load_pids(u, u.i0);
  load_q(u);
#pragma unroll 1
  for (int k = 0; k < Cfg::kEarly; ++k) issue(u, k, k);
  for (;;) {
#pragma unroll 1
    for (int k = Cfg::kEarly; k < ST - 1; ++k) issue(u, k, k);

    // ------------------------------ queries ------------------------------
    uint32_t qb[NR][8][2];
    float cs[NR][2];                     // multipliers of rows 2 c, 2 c + 1: what a lane's logits belong to
    int prow[NR][2];
#pragma unroll
    for (int n = 0; n < NR; ++n) {
      int tok, head;
      row_of(u, min(n * 8 + l4, u.nrows - 1), tok, head);
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        qb[n][2 * s][0] = qraw[n][s].x;
        qb[n][2 * s][1] = qraw[n][s].y;
        qb[n][2 * s + 1][0] = qraw[n][s].z;
        qb[n][2 * s + 1][1] = qraw[n][s].w;
      }
      float mul = A.scale_log2;
      if constexpr (FP8) {
        uint32_t a = 0;
#pragma unroll
        for (int s = 0; s < 8; ++s)
#pragma unroll
          for (int k = 0; k < 2; ++k) a = max(a, max(qb[n][s][k] & 0x7fffu, (qb[n][s][k] >> 16) & 0x7fffu));
        a = max(a, __shfl_xor_sync(0xffffffffu, a, 1));
        a = max(a, __shfl_xor_sync(0xffffffffu, a, 2));
        // power of two that brings the row's maximum to [2^13, 2^14): 2^(13 + 127 - e)
        int e = 140 - (int)(a >> 7);
        e = a == 0 || a >= 0x7f80u ? 0 : max(-126, min(126, e));
        const float f = __uint_as_float((uint32_t)(e + 127) << 23), back = __uint_as_float((uint32_t)(127 - e) << 23);
        mul *= back;
        if constexpr (FMT == FMT_FP8_HEAD) mul *= k_scale;
        if constexpr (!OWN_E) mul = fmaxf(mul, 1e-37f);   // (a hidden logit of -inf times zero would be NaN; pages' scales come first)
#pragma unroll
        for (int s = 0; s < 8; ++s)
#pragma unroll
          for (int k = 0; k < 2; ++k) qb[n][s][k] = pack_f16x2(bf16_lo(qb[n][s][k]) * f, bf16_hi(qb[n][s][k]) * f);
      }
#pragma unroll
      for (int v = 0; v < 2; ++v) {      // from the lanes of row 2 c + v
        cs[n][v] = __shfl_sync(0xffffffffu, mul, (2 * c + v) * 4);
        prow[n][v] = u.first_pos + __shfl_sync(0xffffffffu, tok, (2 * c + v) * 4);
      }
    }
    DecodeUnit un;                       // the next one: known early, so that its page ids are there when this one ends
    const bool more = next_unit(un);
    const int pids_un = more ? load_pids(un, un.i0) : -1;
    const float out_scale = FMT == FMT_FP8_HEAD ? v_scale : 1.f;

    float o[NR][8][4];                   // tile t: rows 2 c, 2 c + 1 of two dims of this lane's
    float m[NR][2], l[NR][2];
    float e[OWN_E ? NR : 1][2];          // (else m)
    (void)e;
#pragma unroll
    for (int n = 0; n < NR; ++n) {
#pragma unroll
      for (int t = 0; t < 8; ++t) o[n][t][0] = o[n][t][1] = o[n][t][2] = o[n][t][3] = 0.f;
      m[n][0] = m[n][1] = -INFINITY;
      l[n][0] = l[n][1] = 0.f;
      if constexpr (OWN_E) e[n][0] = e[n][1] = -INFINITY;
    }

    // ------------------------------ steps ------------------------------
    int slot = 0, fill = ST - 1;
#pragma unroll 1
    for (int i = u.i0; i < u.i1; ++i) {
      cp_async_wait_group<ST - 2>();
      __syncwarp();        // the step's copies of all lanes have landed, and the stage of the step before is no longer read
      issue(u, i - u.i0 + ST - 1, fill);
      fill = slot;
      const int now = slot;
      slot = slot + 1 == ST ? 0 : slot + 1;
      const uint32_t live = live_s[warp][now];
      if (live == 0u) continue;
      const int t0 = token0(u, i);
      const uint32_t kb = ring + now * Cfg::kStep, vb = kb + Cfg::kTile;
      // S^T = K Q^T: tile g of 16 tokens, this lane's are l4 and l4 + 8 of each
      float x[NR][TOK / 16][4];
#pragma unroll
      for (int g = 0; g < TOK / 16; ++g) {
#pragma unroll
        for (int n = 0; n < NR; ++n) x[n][g][0] = x[n][g][1] = x[n][g][2] = x[n][g][3] = 0.f;
        const uint32_t krow = kb + (g * 16 + l4) * 128;
#pragma unroll
        for (int v = 0; v < 2 * Cfg::kEsz; ++v) {
          const uint32_t at = krow + (v >> 1) * Cfg::kHalf + (((2 * c + (v & 1)) ^ l4) << 4);
          const uint4 wa = lds128(at), wb = lds128(at + 8 * 128);
          if constexpr (FP8) {
            const uint32_t a[4] = {wa.x, wa.y, wa.z, wa.w}, d[4] = {wb.x, wb.y, wb.z, wb.w};
#pragma unroll
            for (int s = 0; s < 4; ++s) {
              uint32_t a0, a1, a2, a3;
              e4m3x4_to_f16x4(a[s], a0, a2);
              e4m3x4_to_f16x4(d[s], a1, a3);
#pragma unroll
              for (int n = 0; n < NR; ++n) mma_16816_f16(x[n][g], a0, a1, a2, a3, qb[n][4 * v + s][0], qb[n][4 * v + s][1]);
            }
          } else {
#pragma unroll
            for (int n = 0; n < NR; ++n) {
              mma_16816_bf16(x[n][g], wa.x, wb.x, wa.y, wb.y, qb[n][2 * v][0], qb[n][2 * v][1]);
              mma_16816_bf16(x[n][g], wa.z, wb.z, wa.w, wb.w, qb[n][2 * v + 1][0], qb[n][2 * v + 1][1]);
            }
          }
        }
      }
      float vlog[G];
      if constexpr (OWN_E) {
#pragma unroll
        for (int j = 0; j < G; ++j) {
          const float ks = page_scales[warp][now][j], vs = page_scales[warp][now][G + j];
          vlog[j] = vs > 0.f ? __log2f(vs) : 0.f;      // (0: nothing of the group was copied)
#pragma unroll
          for (int n = 0; n < NR; ++n)
#pragma unroll
            for (int v = 0; v < 2; ++v) x[n][j / 2][(j & 1) * 2 + v] *= cs[n][v] * ks;
        }
      }
      if (!(live == kAllLive && t0 + TOK - 1 <= u.pmin && (A.window <= 0 || t0 > u.pmax - A.window || t0 + TOK - 1 < A.sinks))) {
#pragma unroll
        for (int g = 0; g < TOK / 16; ++g)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int j = g * 16 + (e >> 1) * 8 + l4, tok = t0 + j;
#pragma unroll
            for (int n = 0; n < NR; ++n) {
              const int p = prow[n][e & 1];
              const bool see = ((live >> j) & 1u) && tok <= p && (A.window <= 0 || tok > p - A.window || tok < A.sinks);
              if (!see) x[n][g][e] = -INFINITY;
            }
          }
      }
      // y = x mul (+ log2 vs).  m is the reference of the exponentials: 8 below the maximum when it was set, moved when a row has
      // outgrown it by 14 (F16 holds 2^15).  Lanes look at their own tokens; only a move needs the row's maximum.
      auto row_max = [](float a) {
        a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, 4));
        a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, 8));
        return fmaxf(a, __shfl_xor_sync(0xffffffffu, a, 16));
      };
      // e moves with it, to the maximum of x, and by itself when a row has outgrown it by 30 (large weights on small values).
      float my[NR][2], mx[OWN_E ? NR : 1][2];      // this lane's maxima
      (void)mx;
      bool outgrown = false;
#pragma unroll
      for (int n = 0; n < NR; ++n)
#pragma unroll
        for (int v = 0; v < 2; ++v) {
          float a = -INFINITY, w = -INFINITY;
#pragma unroll
          for (int j = 0; j < G; ++j) {
            const float y = x[n][j / 2][(j & 1) * 2 + v];
            a = fmaxf(a, OWN_E ? y + vlog[j] : y);
            w = fmaxf(w, y);
          }
          my[n][v] = OWN_E ? a : a * cs[n][v];
          outgrown |= my[n][v] > m[n][v] + 14.f;
          if constexpr (OWN_E) {
            mx[n][v] = w;
            outgrown |= w > e[n][v] + 30.f;
          }
        }
      if (__any_sync(0xffffffffu, outgrown)) {
#pragma unroll
        for (int n = 0; n < NR; ++n)
#pragma unroll
          for (int v = 0; v < 2; ++v) {
            const float mn = fmaxf(m[n][v], row_max(my[n][v]) - 8.f);
            const float f = mn == m[n][v] ? 1.f : ex2(m[n][v] - mn);
            m[n][v] = mn;
            float g = f;
            if constexpr (OWN_E) {
              const float en = fmaxf(e[n][v], row_max(mx[n][v]));
              g = en == e[n][v] ? 1.f : ex2(e[n][v] - en);
              e[n][v] = en;
            }
            l[n][v] *= g;
#pragma unroll
            for (int t = 0; t < 8; ++t) {
              o[n][t][v] *= f;
              o[n][t][2 + v] *= f;
            }
          }
      }
      uint32_t pb[NR][G], pl[FP8 ? 1 : NR][G];     // P^T: rows l4, tokens 8 j + 2 c, + 1
      (void)pl;
#pragma unroll
      for (int n = 0; n < NR; ++n) {
        float ref[2], ref_e[2];
#pragma unroll
        for (int v = 0; v < 2; ++v) {
          ref[v] = m[n][v] == -INFINITY ? 0.f : m[n][v];
          if constexpr (OWN_E) ref_e[v] = e[n][v] == -INFINITY ? 0.f : e[n][v];
        }
        (void)ref_e;
#pragma unroll
        for (int j = 0; j < G; ++j) {
          float p[2];
#pragma unroll
          for (int v = 0; v < 2; ++v) {
            const float xj = x[n][j / 2][(j & 1) * 2 + v];
            if constexpr (OWN_E) {
              p[v] = ex2(xj + (vlog[j] - ref[v]));
              l[n][v] += ex2(xj - ref_e[v]);
            } else {
              p[v] = ex2(fmaf(xj, cs[n][v], -ref[v]));
              l[n][v] += p[v];
            }
          }
          if constexpr (FP8) {
            pb[n][j] = transpose8(pack_f16x2(p[0], p[1]));
          } else {
            const uint32_t hi = pack_bf16x2(p[0], p[1]);
            pb[n][j] = transpose8(hi);
            pl[n][j] = transpose8(pack_bf16x2(p[0] - bf16_lo(hi), p[1] - bf16_hi(hi)));
          }
        }
      }
      // O^T += V^T P^T.  Contraction: tokens 2c, 2c + 1, 2c + 8, 2c + 9 of each 16; rows: dims 16 l4 + 2 t, + 1 (e4m3) or
      // 64 hv + 8 l4 + 2 t, + 1 (BF16) of this lane.
#pragma unroll
      for (int g = 0; g < TOK / 16; ++g)
#pragma unroll
        for (int hv = 0; hv < Cfg::kEsz; ++hv) {
          uint32_t w[4][4];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const int tok = 2 * c + (k & 1) + (k >> 1) * 8;
            const uint4 v = lds128(vb + hv * Cfg::kHalf + (g * 16 + tok) * 128 + ((l4 ^ (tok & 7)) << 4));
            w[k][0] = v.x; w[k][1] = v.y; w[k][2] = v.z; w[k][3] = v.w;
          }
#pragma unroll
          for (int qd = 0; qd < 4; ++qd) {
            if constexpr (FP8) {
              uint32_t f[4], h[4];
              e4m3x4_to_f16x4(__byte_perm(w[0][qd], w[1][qd], 0x5140), f[0], f[1]);
              e4m3x4_to_f16x4(__byte_perm(w[0][qd], w[1][qd], 0x7362), f[2], f[3]);
              e4m3x4_to_f16x4(__byte_perm(w[2][qd], w[3][qd], 0x5140), h[0], h[1]);
              e4m3x4_to_f16x4(__byte_perm(w[2][qd], w[3][qd], 0x7362), h[2], h[3]);
#pragma unroll
              for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int n = 0; n < NR; ++n)
                  mma_16816_f16(o[n][qd * 2 + k], f[2 * k], f[2 * k + 1], h[2 * k], h[2 * k + 1], pb[n][2 * g], pb[n][2 * g + 1]);
            } else {
              const uint32_t f0 = __byte_perm(w[0][qd], w[1][qd], 0x5410), f1 = __byte_perm(w[0][qd], w[1][qd], 0x7632);
              const uint32_t h0 = __byte_perm(w[2][qd], w[3][qd], 0x5410), h1 = __byte_perm(w[2][qd], w[3][qd], 0x7632);
#pragma unroll
              for (int n = 0; n < NR; ++n) {
                mma_16816_bf16(o[n][hv * 4 + qd], f0, f1, h0, h1, pb[n][2 * g], pb[n][2 * g + 1]);
                mma_16816_bf16(o[n][hv * 4 + qd], f0, f1, h0, h1, pl[n][2 * g], pl[n][2 * g + 1]);
              }
            }
          }
        }
    }
    // The next unit's first copies, into stages that the join below leaves alone.  (All copies of this unit that read anything were
    // waited for in its last step.)
    __syncwarp();
    if (more) {
      load_q(un);
      pids_next = pids_un;
#pragma unroll 1
      for (int k = 0; k < Cfg::kEarly; ++k) issue(un, k, k);
    }

    // ------------------------------ the four warps' results ------------------------------
    auto osm = [&](int w) { return reinterpret_cast<float*>(smem + w * Cfg::kRing + Cfg::kEarly * Cfg::kStep); };   // [row][128]
    auto piece = [](int row, int k) { return k ^ ((row >> 1) & 3); };   // place of a row's 16-byte piece k, against bank conflicts
#pragma unroll
    for (int n = 0; n < NR; ++n)
#pragma unroll
      for (int v = 0; v < 2; ++v) {
        float ls = l[n][v];
        ls += __shfl_xor_sync(0xffffffffu, ls, 4);
        ls += __shfl_xor_sync(0xffffffffu, ls, 8);
        ls += __shfl_xor_sync(0xffffffffu, ls, 16);
        const int row = n * 8 + 2 * c + v;
        State sum = State::none();
        sum.m = m[n][v];
        sum.l = ls;
        if constexpr (OWN_E) sum.set_e(e[n][v]);
        if (l4 == 0) ml_s[warp][row] = sum;
        float* const orow = osm(warp) + row * 128;
#pragma unroll
        for (int t = 0; t < 8; t += 2) {
          const int dim = FP8 ? 16 * l4 + 2 * t : 64 * (t >> 2) + 8 * l4 + 2 * (t & 3);
          *reinterpret_cast<float4*>(orow + piece(row, dim >> 2) * 4) = make_float4(o[n][t][v], o[n][t][2 + v], o[n][t + 1][v], o[n][t + 1][2 + v]);
        }
      }
    // Joins what the warps have put into shared memory.  place < 0: to out and lse; else to that row of the partial results.
    auto join = [&](long long place) {
      __syncthreads();
      for (int k = tid; k < u.nrows * 32; k += kDecThreads) {
        const int row = k >> 5, pc = k & 31;
        State sum = State::none();
#pragma unroll
        for (int w = 0; w < kDecWarps; ++w) {
          sum.m = fmaxf(sum.m, ml_s[w][row].m);
          sum.set_e(fmaxf(sum.e(), ml_s[w][row].e()));
        }
        const float ref = sum.m == -INFINITY ? 0.f : sum.m, ref_e = sum.e() == -INFINITY ? 0.f : sum.e();
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < kDecWarps; ++w) {
          const State part = ml_s[w][row];
          const float f = ex2(part.m - ref);
          const float4 v = *reinterpret_cast<const float4*>(osm(w) + row * 128 + piece(row, pc) * 4);
          sum.l = fmaf(OWN_E ? ex2(part.e() - ref_e) : f, part.l, sum.l);
          acc.x = fmaf(f, v.x, acc.x);
          acc.y = fmaf(f, v.y, acc.y);
          acc.z = fmaf(f, v.z, acc.z);
          acc.w = fmaf(f, v.w, acc.w);
        }
        if (place < 0) {
          int tok, head;
          row_of(u, row, tok, head);
          const size_t at = (size_t)(u.c0 + tok);
          const float inv = sum.l > 0.f ? out_scale / sum.l : sum.l == 0.f ? 0.f : NAN;
          acc = make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv);
          if constexpr (OWN_E) {         // times 2^(m - e), in halves: the whole may be out of range where the result is not
            const float h = ex2(0.5f * (ref - ref_e));
            acc = make_float4(acc.x * h * h, acc.y * h * h, acc.z * h * h, acc.w * h * h);
          }
          uint2 w;
          w.x = pack_bf16x2(acc.x, acc.y);
          w.y = pack_bf16x2(acc.z, acc.w);
          *reinterpret_cast<uint2*>(A.out + (at * A.num_q_heads + head) * kHeadDim + pc * 4) = w;
          if (pc == 0 && A.lse != nullptr)
            A.lse[(size_t)head * A.total_q + at] = sum.l == 0.f ? -INFINITY : (sum.e() + log2f(sum.l)) * 0.6931471805599453f;
        } else {
          __stcg(reinterpret_cast<float4*>(A.part_o + (place + row) * 128) + pc, acc);
          if (pc == 0) sum.store_cg(A.part_ml, place + row);
        }
      }
    };
    // Partial results of the unit stand at place_of(w) of the CTA w that made them: place 1 of the CTA that the unit begins in, place
    // 0 of the others.
    auto place_of = [&](int w) { return (long long)(2 * w + (w == u.w0 ? 1 : 0)) * RT; };
    // Whether all n have arrived at the counter, which then starts again
    auto arrive = [&](int32_t* counter, int n) {
      __threadfence();
      __syncthreads();
      if (tid == 0) {
        const bool last = atomicAdd(counter, 1) == n - 1;
        if (last) *counter = 0;
        last_s = last;
      }
      __syncthreads();
      if (last_s) __threadfence();
      return last_s != 0;
    };
    // n partial results, those of the CTAs w, w + step ..., by warp in turn, then over the warps as above.  Eight rows at a time, of
    // kDecJoin of them at once: all loads of that are on their way together.  A lane keeps the state of one of the eight rows.
    auto join_parts = [&](int w, int step, int n, long long place) {
#pragma unroll 1
      for (int r0 = 0; r0 < u.nrows; r0 += 8) {
        State sum = State::none();
        float4 acc[8];
#pragma unroll
        for (int r = 0; r < 8; ++r) acc[r] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
        for (int k0 = warp; k0 < n; k0 += kDecWarps * kDecJoin) {
          float4 v[kDecJoin][8];
          State part[kDecJoin];
#pragma unroll
          for (int j = 0; j < kDecJoin; ++j) {
            const int k = k0 + j * kDecWarps;
            const long long row = place_of(w + k * step) + r0;
            part[j] = k < n && r0 + (lane & 7) < u.nrows ? State::load_cg(A.part_ml, row + (lane & 7)) : State::none();
#pragma unroll
            for (int r = 0; r < 8; ++r)
              v[j][r] = k < n && r0 + r < u.nrows ? __ldcg(reinterpret_cast<const float4*>(A.part_o + (row + r) * 128) + lane)
                                                  : make_float4(0.f, 0.f, 0.f, 0.f);
          }
#pragma unroll
          for (int j = 0; j < kDecJoin; ++j) {
            const float mn = fmaxf(sum.m, part[j].m), ref = mn == -INFINITY ? 0.f : mn;
            const float f0 = ex2(sum.m - ref), f1 = ex2(part[j].m - ref);
            float g0 = f0, g1 = f1;
            if constexpr (OWN_E) {
              const float en = fmaxf(sum.e(), part[j].e()), ref_e = en == -INFINITY ? 0.f : en;
              g0 = ex2(sum.e() - ref_e);
              g1 = ex2(part[j].e() - ref_e);
              sum.set_e(en);
            }
            sum.m = mn;
            sum.l = fmaf(g1, part[j].l, g0 * sum.l);
#pragma unroll
            for (int r = 0; r < 8; ++r) {
              const float a0 = __shfl_sync(0xffffffffu, f0, r), a1 = __shfl_sync(0xffffffffu, f1, r);
              acc[r].x = fmaf(a1, v[j][r].x, a0 * acc[r].x);
              acc[r].y = fmaf(a1, v[j][r].y, a0 * acc[r].y);
              acc[r].z = fmaf(a1, v[j][r].z, a0 * acc[r].z);
              acc[r].w = fmaf(a1, v[j][r].w, a0 * acc[r].w);
            }
          }
        }
        if (lane < 8) ml_s[warp][r0 + lane] = sum;
#pragma unroll
        for (int r = 0; r < 8; ++r)
          *reinterpret_cast<float4*>(osm(warp) + (r0 + r) * 128 + piece(r0 + r, lane) * 4) = acc[r];
      }
      join(place);
    };
    join(u.whole ? -1 : place_of(blockIdx.x));
    if (!u.whole) {
      // The last CTA of a group of kDecGroup joins the group's results, the last of these the groups'.
      const int group0 = ((int)blockIdx.x - u.w0) / kDecGroup * kDecGroup, groups = (u.parts + kDecGroup - 1) / kDecGroup;
      const int n = min(kDecGroup, u.parts - group0);
      // (counters by CTA: at most one unit that goes on behind it begins in a CTA, and at most one goes on into it)
      if (arrive(A.counters + (group0 ? gridDim.x : 0) + u.w0 + group0, n)) {
        join_parts(u.w0 + group0, 1, n, groups == 1 ? -1 : place_of(u.w0 + group0));
        if (groups > 1 && arrive(A.counters + 2 * gridDim.x + u.w0, groups)) join_parts(u.w0, kDecGroup, groups, -1);
      }
    }
    if (!more) return;
    __syncthreads();      // the join's shared memory is free for the next unit's copies
    u = un;
  }
}

}  // namespace fp2
