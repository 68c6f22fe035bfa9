// Attention of the newest few tokens of every sequence over its paged cache (token by token decoding, verification of drafts),
// with an optional sliding window and sinks:
//   x_ij = scale ks_j q_i . K_j,   visible iff j <= p_i and (W == 0 or p_i - j < W or j < S),   p_i = Lk - Lq + i
//   out_i = sum_j 2^(x_ij - m) vs_j V_j / sum_j 2^(x_ij - m)           (x in units of log2, one pass with a running maximum)
//
// Bound by the bytes of the cache: each is wanted once, the arithmetic of a group of query heads on them is small.  So:
//
// Work split.  The (sequence, KV head, tile of packed rows, 64-token block) items are numbered in that order, and every CTA of a
// grid that fills the GPU takes an equal contiguous share, whatever the lengths: a long sequence is cut wherever shares end.  The
// lengths are read on the device (a captured graph stays valid as sequences grow), so the CTAs find their shares themselves.  A
// unit (sequence, head, tile) cut into parts leaves (O, m, l) of each in the workspace, and the CTA that arrives last joins them,
// in the order of the shares: the result does not depend on who is last.  One launch.
//
// A CTA is four warps, two CTAs to an SM.  Of a block each warp takes 16 tokens, which it copies into its own part of shared
// memory (cp.async, kStages steps ahead) and attends to with its own running maximum and sum: no barrier in the loop; the
// four join at the end of a unit.  Copies of hidden tokens write zeros without reading, so nothing that stands in a hidden place
// reaches the sums.  192 KB in flight per SM.
//
// S = Q K^T and O += P V are m16n8k16 MMAs of a warp, rows = 16 packed (token, query head) pairs of the KV head, MT of these: what
// tcgen05 would add in rate is not what bounds this, and its 64 rows and round trips through tensor memory are what a group of
// eight heads has no use for.  K and V are read from shared memory 16 bytes a lane; which of a lane's values play which index of
// the contraction (over dims in Q K^T) or which column (dims in P V) is free, as long as Q is permuted alike and O stored
// accordingly, so that no transposing is needed but pairing two tokens' values by byte permutation.
//
// Precision.  BF16 caches: Q and K as they are; P as a BF16 pair hi + lo (2^-17).  e4m3 caches: K, V exact as F16; Q exact as
// F16 after a power of two per row has brought its maximum to 2^13 .. 2^14 (elements 2^-28 below it round); P as F16 against a
// reference 8 binades below the running maximum, where the steps are 2^-11 relative down to 2^-22 of the maximum.  Sums in 32 bits.
// Scales per page: ks multiplies the logits; vs enters P, in the exponent, so that P V needs none:
// y = x + log2 vs has the running maximum, p = 2^(y - m), and l adds p / vs.
#pragma once
#include <cuda_bf16.h>
#include "common.cuh"
#include "kv_cache.cuh"
#include "ptx.cuh"

namespace fp2 {

constexpr int kDecWarps = 4;
constexpr int kDecThreads = 32 * kDecWarps;
constexpr int kDecCtasPerSm = 2;
constexpr int kDecBlock = 16 * kDecWarps;     // tokens of a work item
constexpr int kDecMinShare = 2;               // blocks per CTA below which more CTAs do not pay

template <int FMT>
struct DecodeCfg {
  static constexpr int kEsz = FMT == FMT_BF16 ? 2 : 1;
  static constexpr int kHalf = 16 * 128;                          // 16 rows of 128 bytes
  static constexpr int kTile = kHalf * kEsz;                      // K (or V) of 16 tokens of a head
  static constexpr int kStages = FMT == FMT_BF16 ? 3 : 6;
  static constexpr int kRing = kDecWarps * kStages * 2 * kTile;   // 96 KB
  static constexpr int kSmemBytes = 128 + kRing;
};

struct DecodeArgs {
  const uint8_t* q;             // BF16
  long long q_stride_bytes;
  const int32_t *cu, *lk, *page_table;
  const uint8_t *k, *v;
  const float *k_scale, *v_scale;
  __nv_bfloat16* out;
  float* lse;
  float* part_o;                // [2 grid][16 MT][128]
  float2* part_ml;              // [2 grid][16 MT]
  int32_t* counters;            // [grid], zero between calls
  int* status;
  int32_t total_q, num_q_heads, group, window, sinks;
  float scale_log2;
  CacheGeom g;
};

// One sequence's share of the work
struct DecodeSeq {
  int c0, Lq, L;      // first query row, queries, tokens in the cache
  int ntiles;         // tiles of packed rows of a KV head
  int sb, wb0, nblk;  // blocks: 0 .. sb - 1 (sinks), then wb0 .. ; nblk in all
  long long cost;     // items
};

template <int RT>
__device__ __forceinline__ DecodeSeq decode_seq(const DecodeArgs& A, int b, bool report) {
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
  s.ntiles = (int)(((long long)A.group * s.Lq + RT - 1) / RT);
  // tokens some query sees: below the sinks, and from the first query's window on
  const int first = s.L - s.Lq;
  const int lo = A.window > 0 ? max(0, (int)min((long long)s.L, (long long)first - A.window + 1)) : 0;
  s.wb0 = lo / kDecBlock;
  s.sb = min((int)(((long long)min(A.sinks, s.L) + kDecBlock - 1) / kDecBlock), s.wb0);
  s.nblk = max(1, s.sb + (s.L + kDecBlock - 1) / kDecBlock - s.wb0);   // (one for rows that see nothing: they are written)
  s.cost = (long long)s.ntiles * A.g.num_kv_heads * s.nblk;
  return s;
}

__device__ __forceinline__ void mma_16816_bf16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_16816_f16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void cp_async4(uint32_t smem_dst, const void* gsrc, uint32_t src_bytes) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(smem_dst), "l"(gsrc), "r"(src_bytes) : "memory");
}
__device__ __forceinline__ uint4 lds128(uint32_t a) {
  uint4 r;
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "r"(a) : "memory");
  return r;
}

template <int FMT, int MT>
__global__ void __launch_bounds__(kDecThreads, kDecCtasPerSm)
decode_kernel(DecodeArgs A) {
  using Cfg = DecodeCfg<FMT>;
  constexpr bool FP8 = FMT != FMT_BF16;
  constexpr int RT = 16 * MT, ST = Cfg::kStages;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 127) & ~uintptr_t(127));
  __shared__ float page_scales[kDecWarps][ST][4];          // PAGE: ks of tokens 0..7, 8..15, then vs
  __shared__ uint32_t live_s[kDecWarps][ST];               // tokens of the step that were copied
  __shared__ float2 ml_s[kDecWarps][RT];
  __shared__ long long scan_s[kDecWarps];
  __shared__ long long found_base;
  __shared__ int found_b, last_s;

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int c = lane & 3, l4 = lane >> 2;
  const int heads = A.g.num_kv_heads, shift = A.g.page_shift, grp = A.group;
  pdl_trigger();
  pdl_wait();

  // ------------------------------ this CTA's share ------------------------------
  long long total = 0;
  for (int b0 = 0; b0 < A.g.num_seqs; b0 += kDecThreads)
    total += b0 + tid < A.g.num_seqs ? decode_seq<RT>(A, b0 + tid, blockIdx.x == 0).cost : 0;
#pragma unroll
  for (int d = 16; d; d >>= 1) total += __shfl_xor_sync(0xffffffffu, total, d);
  if (lane == 0) scan_s[warp] = total;
  if (tid == 0) found_b = -1;
  __syncthreads();
  total = 0;
#pragma unroll
  for (int i = 0; i < kDecWarps; ++i) total += scan_s[i];
  const long long share = max((total + gridDim.x - 1) / gridDim.x, (long long)kDecMinShare);
  long long pos = share * blockIdx.x;
  const long long pos_end = min(total, pos + share);
  if (pos >= pos_end) return;
  {
    long long base = 0;
    for (int b0 = 0; b0 < A.g.num_seqs; b0 += kDecThreads) {
      const long long cost = b0 + tid < A.g.num_seqs ? decode_seq<RT>(A, b0 + tid, false).cost : 0;
      long long incl = cost;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const long long o = __shfl_up_sync(0xffffffffu, incl, d);
        if (lane >= d) incl += o;
      }
      __syncthreads();
      if (lane == 31) scan_s[warp] = incl;
      __syncthreads();
      long long all = 0;
#pragma unroll
      for (int i = 0; i < kDecWarps; ++i) {
        if (i < warp) incl += scan_s[i];
        all += scan_s[i];
      }
      const long long lo = base + incl - cost;
      if (pos >= lo && pos < lo + cost) {
        found_b = b0 + tid;
        found_base = lo;
      }
      base += all;
      if (base > pos) break;
    }
    __syncthreads();
  }
  int b = found_b;
  long long seq_base = found_base;
  DecodeSeq sq = decode_seq<RT>(A, b, false);

  const uint32_t ring = smem_u32(smem) + warp * (ST * 2 * Cfg::kTile);
  const uint32_t my_scales = smem_u32(&page_scales[warp][0][0]);
  const uint64_t stream_pol = l2_policy_evict_first();

  while (pos < pos_end) {
    while (pos >= seq_base + sq.cost) {
      seq_base += sq.cost;
      sq = decode_seq<RT>(A, ++b, false);
    }
    const long long unit = (pos - seq_base) / sq.nblk;
    const long long unit0 = seq_base + unit * sq.nblk;
    const int i0 = (int)(pos - unit0), i1 = (int)min((long long)sq.nblk, pos_end - unit0);
    const int h = (int)(unit / sq.ntiles), t = (int)(unit % sq.ntiles);
    const int r0 = t * RT;
    const int nrows = min(RT, grp * sq.Lq - r0);
    const int first_pos = sq.L - sq.Lq;
    const int pmin = first_pos + r0 / grp, pmax = first_pos + (r0 + nrows - 1) / grp;
    const int32_t* pt = A.page_table + (size_t)b * A.g.max_pages;

    // ------------------------------ queries ------------------------------
    // Lane (l4, c) holds rows l4 and l4 + 8 of each 16-row tile; contraction step s covers, for it, the dims dim_of(s) .. + 3.
    auto dim_of = [&](int s) { return FP8 ? 32 * c + 4 * s : 64 * (s >> 2) + 16 * c + 4 * (s & 3); };
    uint32_t qa[MT][8][4];
    float cs[MT][2];
    int prow[MT][2];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int row = mt * 16 + u * 8 + l4;
        const int r = r0 + min(row, nrows - 1);
        const int tok = r / grp, head = h * grp + r - tok * grp;
        prow[mt][u] = first_pos + tok;
        const uint8_t* src = A.q + (long long)(sq.c0 + tok) * A.q_stride_bytes + head * (kHeadDim * 2);
        uint32_t w[16];
#pragma unroll
        for (int s = 0; s < 8; s += 2) {
          const uint4 v = *reinterpret_cast<const uint4*>(src + dim_of(s) * 2);
          w[2 * s] = v.x; w[2 * s + 1] = v.y; w[2 * s + 2] = v.z; w[2 * s + 3] = v.w;
        }
        cs[mt][u] = A.scale_log2;
        if constexpr (FP8) {
          uint32_t a = 0;
#pragma unroll
          for (int k = 0; k < 16; ++k) a = max(a, max(w[k] & 0x7fffu, (w[k] >> 16) & 0x7fffu));
          a = max(a, __shfl_xor_sync(0xffffffffu, a, 1));
          a = max(a, __shfl_xor_sync(0xffffffffu, a, 2));
          // power of two that brings the row's maximum to [2^13, 2^14): 2^(13 + 127 - e)
          int e = 140 - (int)(a >> 7);
          e = a == 0 || a >= 0x7f80u ? 0 : max(-126, min(126, e));
          const float f = __uint_as_float((uint32_t)(e + 127) << 23), back = __uint_as_float((uint32_t)(127 - e) << 23);
          cs[mt][u] *= back;
          if constexpr (FMT == FMT_FP8_HEAD) cs[mt][u] *= A.k_scale[h];
#pragma unroll
          for (int k = 0; k < 16; ++k) w[k] = pack_f16x2(bf16_lo(w[k]) * f, bf16_hi(w[k]) * f);
        }
#pragma unroll
        for (int s = 0; s < 8; ++s) {
          qa[mt][s][u] = w[2 * s];
          qa[mt][s][u + 2] = w[2 * s + 1];
        }
      }

    // ------------------------------ copies ------------------------------
    auto token0 = [&](int i) { return kDecBlock * (i < sq.sb ? i : sq.wb0 + i - sq.sb) + warp * 16; };
    // pages of the step's tokens 0..7 and 8..15 (the same one unless pages hold eight); -1: none.  Asked for one step ahead.
    int pid0 = -1, pid1 = -1;
    auto fetch_pages = [&](int i) {
      pid0 = pid1 = -1;
      if (i >= i1) return;
      const int t0 = token0(i);
      if (t0 < sq.L) pid0 = pt[t0 >> shift];
      pid1 = shift >= 4 ? pid0 : t0 + 8 < sq.L ? pt[(t0 + 8) >> shift] : -1;
    };
    auto issue = [&](int i) {
      if (i < i1) {
        const int slot = (i - i0) % ST;
        const int t0 = token0(i);
        const int row = lane & 15, tok = t0 + row;
        const int pid = row < 8 ? pid0 : pid1;
        const bool wanted = tok <= pmax && tok < sq.L && (A.window <= 0 || tok > pmin - A.window || tok < A.sinks);
        const bool there = pid >= 0 && pid < A.g.num_pages;
        if (__any_sync(0xffffffffu, wanted && !there) && lane == 0) atomicOr(A.status + kCacheStBad, kBadPage);
        const uint32_t live = __ballot_sync(0xffffffffu, wanted && there) & 0xffffu;
        if (lane == 0) live_s[warp][slot] = live;
        const uint32_t dst = ring + slot * 2 * Cfg::kTile;
        if (live) {
          const int page_row = t0 & ((1 << shift) - 1);
          constexpr int kLanes = 8 * Cfg::kEsz;           // lanes per row, 16 bytes each
          const int ch = lane % kLanes;
#pragma unroll
          for (int k = 0; k < 16 * kLanes / 32; ++k) {
            const int r = k * (32 / kLanes) + lane / kLanes;
            const uint32_t bytes = (live >> r) & 1u ? 16u : 0u;
            const int p = r < 8 ? pid0 : pid1;
            const int prow_ = shift >= 4 ? page_row + r : r & 7;
            const size_t off = bytes ? ((((size_t)p << shift) + prow_) * heads + h) * (kHeadDim * Cfg::kEsz) + ch * 16 : 0;
            const uint32_t d = dst + (ch >> 3) * Cfg::kHalf + r * 128 + (((ch & 7) ^ (r & 7)) << 4);
            cp_async16(d, A.k + off, bytes, stream_pol);
            cp_async16(d + Cfg::kTile, A.v + off, bytes, stream_pol);
          }
          if constexpr (FMT == FMT_FP8_PAGE) {
            if (lane < 4) {
              const int p = lane & 1 ? pid1 : pid0;
              const bool ok = (live & (lane & 1 ? 0xff00u : 0xffu)) != 0u;
              cp_async4(my_scales + (slot * 4 + lane) * 4, (lane < 2 ? A.k_scale : A.v_scale) + (ok ? (size_t)p * heads + h : 0),
                        ok ? 4u : 0u);
            }
          }
        }
        fetch_pages(i + 1);
      }
      cp_async_commit();
    };

    float o[MT][16][4];
    float m[MT][2], l[MT][2];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
      for (int j = 0; j < 16; ++j) o[mt][j][0] = o[mt][j][1] = o[mt][j][2] = o[mt][j][3] = 0.f;
      m[mt][0] = m[mt][1] = -INFINITY;
      l[mt][0] = l[mt][1] = 0.f;
    }
    fetch_pages(i0);
#pragma unroll 1
    for (int k = 0; k < ST - 1; ++k) issue(i0 + k);

    // ------------------------------ steps ------------------------------
#pragma unroll 1
    for (int i = i0; i < i1; ++i) {
      cp_async_wait_group<ST - 2>();
      __syncwarp();        // the step's copies of all lanes have landed, and the slot of the step before is no longer read
      issue(i + ST - 1);
      const int slot = (i - i0) % ST;
      const uint32_t live = live_s[warp][slot];
      if (live == 0u) continue;
      const int t0 = token0(i);
      const uint32_t kb = ring + slot * 2 * Cfg::kTile, vb = kb + Cfg::kTile;
      // S = Q K^T, tokens 0..7 and 8..15
      float x[MT][2][4];
#pragma unroll
      for (int nt = 0; nt < 2; ++nt) {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) x[mt][nt][0] = x[mt][nt][1] = x[mt][nt][2] = x[mt][nt][3] = 0.f;
        const uint32_t krow = kb + (nt * 8 + l4) * 128;
        if constexpr (FP8) {
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const uint4 v = lds128(krow + (((2 * c + u) ^ l4) << 4));
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const uint32_t b0 = e4m3x2_to_f16x2(w[k] & 0xffffu), b1 = e4m3x2_to_f16x2(w[k] >> 16);
#pragma unroll
              for (int mt = 0; mt < MT; ++mt) mma_16816_f16(x[mt][nt], qa[mt][u * 4 + k], b0, b1);
            }
          }
        } else {
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            const uint4 v = lds128(krow + (u >> 1) * Cfg::kHalf + (((2 * c + (u & 1)) ^ l4) << 4));
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
              mma_16816_bf16(x[mt][nt], qa[mt][u * 2], v.x, v.y);
              mma_16816_bf16(x[mt][nt], qa[mt][u * 2 + 1], v.z, v.w);
            }
          }
        }
      }
      // logits: scales, masks
      float kmul[2] = {1.f, 1.f}, vlog[2] = {0.f, 0.f}, vinv[2] = {1.f, 1.f};
      if constexpr (FMT == FMT_FP8_PAGE) {
#pragma unroll
        for (int nt = 0; nt < 2; ++nt) {
          kmul[nt] = page_scales[warp][slot][nt];
          const float vs = page_scales[warp][slot][2 + nt];
          vlog[nt] = vs > 0.f ? __log2f(vs) : 0.f;
          vinv[nt] = vs > 0.f ? 1.0f / vs : 0.f;
        }
      }
      const bool all = live == 0xffffu && t0 + 15 <= pmin && (A.window <= 0 || t0 > pmax - A.window || t0 + 15 < A.sinks);
      uint32_t pa[MT][4], pl[MT][4];
      (void)pl;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
        for (int nt = 0; nt < 2; ++nt)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float y = x[mt][nt][e] * cs[mt][e >> 1];
            if constexpr (FMT == FMT_FP8_PAGE) y = fmaf(y, kmul[nt], vlog[nt]);
            x[mt][nt][e] = y;
          }
        if (!all) {
#pragma unroll
          for (int nt = 0; nt < 2; ++nt)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int j = nt * 8 + 2 * c + (e & 1), tok = t0 + j, p = prow[mt][e >> 1];
              const bool see = ((live >> j) & 1u) && tok <= p && (A.window <= 0 || tok > p - A.window || tok < A.sinks);
              if (!see) x[mt][nt][e] = -INFINITY;
            }
        }
        float mx[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          float a = fmaxf(fmaxf(x[mt][0][2 * u], x[mt][0][2 * u + 1]), fmaxf(x[mt][1][2 * u], x[mt][1][2 * u + 1]));
          a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, 1));
          mx[u] = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, 2));
        }
        // m is the reference of the exponentials, 8 below the maximum when it was set; moved when a row has outgrown it by 14
        // (F16 holds 2^15)
        if (__any_sync(0xffffffffu, mx[0] > m[mt][0] + 14.f || mx[1] > m[mt][1] + 14.f)) {
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const float mn = fmaxf(m[mt][u], mx[u] - 8.f);
            const float f = mn == m[mt][u] ? 1.f : ex2(m[mt][u] - mn);
            m[mt][u] = mn;
            l[mt][u] *= f;
#pragma unroll
            for (int j = 0; j < 16; ++j) {
              o[mt][j][2 * u] *= f;
              o[mt][j][2 * u + 1] *= f;
            }
          }
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const float ref = m[mt][u] == -INFINITY ? 0.f : m[mt][u];
#pragma unroll
          for (int nt = 0; nt < 2; ++nt) {
            const float p0 = ex2(x[mt][nt][2 * u] - ref), p1 = ex2(x[mt][nt][2 * u + 1] - ref);
            l[mt][u] = FMT == FMT_FP8_PAGE ? fmaf(p0 + p1, vinv[nt], l[mt][u]) : l[mt][u] + (p0 + p1);
            if constexpr (FP8) {
              pa[mt][nt * 2 + u] = pack_f16x2(p0, p1);
            } else {
              const uint32_t hi = pack_bf16x2(p0, p1);
              pa[mt][nt * 2 + u] = hi;
              pl[mt][nt * 2 + u] = pack_bf16x2(p0 - bf16_lo(hi), p1 - bf16_hi(hi));
            }
          }
        }
      }
      // O += P V.  Contraction index 2c, 2c + 1, 2c + 8, 2c + 9 of this lane: those tokens; column l4 of tile j: a dim of its own.
#pragma unroll
      for (int hv = 0; hv < Cfg::kEsz; ++hv) {
        uint32_t w[4][4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int tok = 2 * c + (k & 1) + (k >> 1) * 8;
          const uint4 v = lds128(vb + hv * Cfg::kHalf + tok * 128 + ((l4 ^ (tok & 7)) << 4));
          w[k][0] = v.x; w[k][1] = v.y; w[k][2] = v.z; w[k][3] = v.w;
        }
#pragma unroll
        for (int qd = 0; qd < 4; ++qd) {
          if constexpr (FP8) {
            const uint32_t a0 = __byte_perm(w[0][qd], w[1][qd], 0x5140), a1 = __byte_perm(w[0][qd], w[1][qd], 0x7362);
            const uint32_t b0 = __byte_perm(w[2][qd], w[3][qd], 0x5140), b1 = __byte_perm(w[2][qd], w[3][qd], 0x7362);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const uint32_t f0 = e4m3x2_to_f16x2(((k >> 1 ? a1 : a0) >> (16 * (k & 1))) & 0xffffu);
              const uint32_t f1 = e4m3x2_to_f16x2(((k >> 1 ? b1 : b0) >> (16 * (k & 1))) & 0xffffu);
#pragma unroll
              for (int mt = 0; mt < MT; ++mt) mma_16816_f16(o[mt][qd * 4 + k], pa[mt], f0, f1);
            }
          } else {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              const uint32_t f0 = __byte_perm(w[0][qd], w[1][qd], k ? 0x7632 : 0x5410);
              const uint32_t f1 = __byte_perm(w[2][qd], w[3][qd], k ? 0x7632 : 0x5410);
#pragma unroll
              for (int mt = 0; mt < MT; ++mt) {
                mma_16816_bf16(o[mt][hv * 8 + qd * 2 + k], pa[mt], f0, f1);
                mma_16816_bf16(o[mt][hv * 8 + qd * 2 + k], pl[mt], f0, f1);
              }
            }
          }
        }
      }
    }
    cp_async_wait_all();

    // ------------------------------ the four warps' results ------------------------------
    __syncthreads();      // the ring is free (and so is what the unit before left in shared memory)
    float* const osm = reinterpret_cast<float*>(smem);      // [warp][row][128], 16-byte pieces permuted
    auto piece = [](int k) { return k ^ (k >> 3); };        // of 32 pieces of a row
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        float ls = l[mt][u];
        ls += __shfl_xor_sync(0xffffffffu, ls, 1);
        ls += __shfl_xor_sync(0xffffffffu, ls, 2);
        const int row = mt * 16 + u * 8 + l4;
        if (c == 0) ml_s[warp][row] = make_float2(m[mt][u], ls);
        float* const orow = osm + (warp * RT + row) * 128;
        // tile j's column 2c + e is dim 16 (2c + e) + j (e4m3) or 64 (j >> 3) + 8 (2c + e) + (j & 7) (BF16)
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
          for (int j = 0; j < 16; j += 4) {
            const int dim = FP8 ? 16 * (2 * c + e) + j : 64 * (j >> 3) + 8 * (2 * c + e) + (j & 7);
            *reinterpret_cast<float4*>(orow + piece(dim >> 2) * 4) =
                make_float4(o[mt][j][2 * u + e], o[mt][j + 1][2 * u + e], o[mt][j + 2][2 * u + e], o[mt][j + 3][2 * u + e]);
          }
      }
    __syncthreads();
    const bool whole = i0 == 0 && i1 == sq.nblk;
    const size_t slot_row = (size_t)(2 * blockIdx.x + (i0 == 0 ? 1 : 0)) * RT;
    const float out_scale = FMT == FMT_FP8_HEAD ? A.v_scale[h] : 1.f;
    auto write = [&](int row, int pc, float4 acc, float M, float L) {
      const int r = r0 + row, tok = r / grp, head = h * grp + r - tok * grp;
      const size_t at = (size_t)(sq.c0 + tok);
      const float inv = L > 0.f ? out_scale / L : L == 0.f ? 0.f : NAN;
      uint2 w;
      w.x = pack_bf16x2(acc.x * inv, acc.y * inv);
      w.y = pack_bf16x2(acc.z * inv, acc.w * inv);
      *reinterpret_cast<uint2*>(A.out + (at * A.num_q_heads + head) * kHeadDim + pc * 4) = w;
      if (pc == 0 && A.lse != nullptr)
        A.lse[(size_t)head * A.total_q + at] = L == 0.f ? -INFINITY : (M + log2f(L)) * 0.6931471805599453f;
    };
    for (int k = tid; k < nrows * 32; k += kDecThreads) {
      const int row = k >> 5, pc = k & 31;
      float M = -INFINITY, L = 0.f;
#pragma unroll
      for (int w = 0; w < kDecWarps; ++w) M = fmaxf(M, ml_s[w][row].x);
      const float ref = M == -INFINITY ? 0.f : M;
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < kDecWarps; ++w) {
        const float2 ml = ml_s[w][row];
        const float f = ex2(ml.x - ref);
        const float4 v = *reinterpret_cast<const float4*>(osm + (w * RT + row) * 128 + piece(pc) * 4);
        L = fmaf(f, ml.y, L);
        acc.x = fmaf(f, v.x, acc.x);
        acc.y = fmaf(f, v.y, acc.y);
        acc.z = fmaf(f, v.z, acc.z);
        acc.w = fmaf(f, v.w, acc.w);
      }
      if (whole) {
        write(row, pc, acc, M, L);
      } else {
        __stcg(reinterpret_cast<float4*>(A.part_o + (slot_row + row) * 128) + pc, acc);
        if (pc == 0) __stcg(A.part_ml + slot_row + row, make_float2(M, L));
      }
    }
    if (!whole) {
      const int w0 = (int)(unit0 / share), parts = (int)((unit0 + sq.nblk - 1) / share) - w0 + 1;
      __threadfence();
      __syncthreads();
      if (tid == 0) last_s = atomicAdd(A.counters + w0, 1) == parts - 1;
      __syncthreads();
      if (last_s) {
        __threadfence();
        if (tid == 0) A.counters[w0] = 0;
        auto row_of = [&](int u) { return (size_t)(2 * (w0 + u) + (u == 0 ? 1 : 0)) * RT; };
        for (int k = tid; k < nrows * 32; k += kDecThreads) {
          const int row = k >> 5, pc = k & 31;
          float M = -INFINITY, L = 0.f;
#pragma unroll 4
          for (int u = 0; u < parts; ++u) M = fmaxf(M, __ldcg(A.part_ml + row_of(u) + row).x);
          const float ref = M == -INFINITY ? 0.f : M;
          float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
          for (int u = 0; u < parts; ++u) {
            const float2 ml = __ldcg(A.part_ml + row_of(u) + row);
            const float4 v = __ldcg(reinterpret_cast<const float4*>(A.part_o + (row_of(u) + row) * 128) + pc);
            const float f = ex2(ml.x - ref);
            L = fmaf(f, ml.y, L);
            acc.x = fmaf(f, v.x, acc.x);
            acc.y = fmaf(f, v.y, acc.y);
            acc.z = fmaf(f, v.z, acc.z);
            acc.w = fmaf(f, v.w, acc.w);
          }
          write(row, pc, acc, M, L);
        }
      }
    }
    __syncthreads();      // shared memory is free for the next unit's copies
    pos = unit0 + i1;
  }
}

}  // namespace fp2
