// Writing new tokens into the paged KV cache, and reading an 8-bit cache back as BF16 pages.
//
// Cache formats (fp2_cache_format): BF16; e4m3 with one scale per KV head; e4m3 with one scale per (page, KV head).  In the
// last one the writer chooses the scale: the smallest power of two s with max |x| / s <= 448 over the tokens written to the page,
// not below 2^-100, and for a page that holds earlier tokens not below its present scale.  Powers of two, because then x / s is
// exact (the one rounding is the e4m3 one), a page whose scale grows can be requantised without a second rounding except below
// e4m3's normal range, and a page filled token by token ends with the scale and (that range aside) the codes it would have got at
// once.  An e4m3 value has three mantissa bits at any size: a scale up to twice as large as needed costs nothing but the
// smallest binade.
#pragma once
#include <cuda_bf16.h>
#include "common.cuh"
#include "ptx.cuh"

namespace fp2 {

enum { FMT_BF16 = 0, FMT_FP8_HEAD = 1, FMT_FP8_PAGE = 2 };

// Bits of status word 2 (ST_BAD_LIST of the stage calls): 2 page id outside the pool, 4 lengths that do not fit
constexpr int kCacheStBad = 2;
constexpr int kBadPage = 2, kBadLength = 4;

struct CacheGeom {
  int32_t num_kv_heads, page_shift, num_pages, max_pages;   // page_size = 1 << page_shift
  int32_t num_seqs;
};

// two floats -> two e4m3 (nearest even, saturating; NaN stays NaN), a in the low byte
__device__ __forceinline__ uint32_t pack_e4m3x2(float a, float b) {
  uint16_t d;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(d) : "f"(b), "f"(a));
  return d;
}
__device__ __forceinline__ float2 f16x2_to_float2(uint32_t x) {
  float2 r;
  asm("{\n .reg .b16 l, h;\n mov.b32 {l, h}, %2;\n cvt.f32.f16 %0, l;\n cvt.f32.f16 %1, h;\n}" : "=f"(r.x), "=f"(r.y) : "r"(x));
  return r;
}
__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// Smallest power of two s with amax / s <= 448 = 1.75 * 2^8, for the bits of a non-negative finite BF16 value; at least 2^-100.
__device__ __forceinline__ float page_scale_for(uint32_t amax_bits) {
  const int e = (int)(amax_bits >> 7), m = (int)(amax_bits & 0x7f);   // subnormals have e = 0: below 2^-126, like zero
  const int s = e - 8 + (m > 0x60 ? 1 : 0);
  return __uint_as_float((uint32_t)max(s, 127 - 100) << 23);
}

// Number of page slots reserved in front of sequence b's: its n new tokens touch at most n / p + 2 pages.
__device__ __forceinline__ long long append_slot0(int cu, int b, int shift) { return (long long)(cu >> shift) + 2ll * b; }

// One item = the new tokens of one (page, KV head, K | V); rows of a page in groups of 16 to a warp, so that a warp keeps all it
// reads in registers between the maximum and the rounding: the tokens are read once.  16 lanes to a row (16 bytes of BF16 in, 8
// of e4m3 out each), eight rows in flight per lane.  A CTA of eight warps holds 8 / W items, W = warps per page.
// Bound by memory (2 bytes read and 1 written per element) for prompts, by launch and load latency for single tokens.
constexpr int kAppendThreads = 256;

struct AppendArgs {
  const uint8_t *k_new, *v_new;       // BF16 [total_new][stride]
  long long stride_bytes;             // of a token
  const int32_t *cu, *lk, *page_table;
  uint8_t *k_cache, *v_cache;
  float *k_scale, *v_scale;
  int* status;
  int32_t total_new;
  long long slots;                    // page slots of all sequences
  CacheGeom g;
};

template <int FMT>
__global__ void __launch_bounds__(kAppendThreads)
cache_append_kernel(AppendArgs A) {
  constexpr int kRows = 16;           // rows per warp
  __shared__ uint32_t amax_s[kAppendThreads / 32];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  pdl_trigger();
  pdl_wait();
  const int shift = A.g.page_shift, ps = 1 << shift, heads = A.g.num_kv_heads;
  const int wpi = ps > kRows ? ps / kRows : 1;             // warps per item: 1, 2, 4 or 8
  const int part = warp % wpi;
  const long long item = (long long)blockIdx.x * (kAppendThreads / 32 / wpi) + warp / wpi;
  const int h = (int)(item % heads);
  const bool is_v = (item / heads) & 1;
  const long long slot = item / (2 * heads);
  bool active = slot < A.slots;

  // sequence of the slot: the last one whose first slot is not behind it
  int b = -1;
  if (active) {
    for (int base = 0; base < A.g.num_seqs; base += 32) {
      const int i = base + lane;
      const bool le = i < A.g.num_seqs && append_slot0(A.cu[i], i, shift) <= slot;
      const unsigned bal = __ballot_sync(0xffffffffu, le);
      b += __popc(bal);
      if (bal != 0xffffffffu) break;
    }
    active = b >= 0;
  }
  int first = 0, end = 0, c0 = 0, page_tok = 0, pid = 0;
  if (active) {
    c0 = A.cu[b];
    const int c1 = A.cu[b + 1], L = A.lk[b], n = c1 - c0;
    const bool fits = c0 >= 0 && c1 >= c0 && c1 <= A.total_new && L >= n && L <= ((long long)A.g.max_pages << shift);
    if (!fits && lane == 0) atomicOr(A.status + kCacheStBad, kBadLength);
    first = L - n;
    end = L;
    const long long page = (first >> shift) + (slot - append_slot0(c0, b, shift));
    active = fits && n > 0 && page >= (first >> shift) && page <= ((L - 1) >> shift);   // (offsets that fall: any slot)
    if (active) {
      page_tok = (int)page << shift;
      pid = A.page_table[(size_t)b * A.g.max_pages + page];
      if (pid < 0 || pid >= A.g.num_pages) {
        if (lane == 0) atomicOr(A.status + kCacheStBad, kBadPage);
        active = false;
      }
    }
  }
  const uint8_t* src = is_v ? A.v_new : A.k_new;
  uint8_t* cache = is_v ? A.v_cache : A.k_cache;
  constexpr int esz = FMT == FMT_BF16 ? 2 : 1;
  const int col = lane & 15, half = lane >> 4;
  const int row0 = part * kRows + half;                  // this lane's rows of the page: row0 + 2 i
  auto out_at = [&](int row) {
    return cache + (((size_t)pid * ps + row) * heads + h) * (kHeadDim * esz) + col * (8 * esz);
  };
  uint4 x[kRows / 2];
  uint32_t live = 0;
  if (active) {
#pragma unroll
    for (int i = 0; i < kRows / 2; ++i) {
      const int row = row0 + 2 * i, tok = page_tok + row;
      x[i] = make_uint4(0, 0, 0, 0);
      if (row < ps && tok >= first && tok < end) {
        live |= 1u << i;
        x[i] = *reinterpret_cast<const uint4*>(src + (long long)(c0 + tok - first) * A.stride_bytes + h * (kHeadDim * 2) + col * 16);
      }
    }
  }
  if constexpr (FMT == FMT_BF16) {
    if (!active) return;
#pragma unroll
    for (int i = 0; i < kRows / 2; ++i)
      if ((live >> i) & 1u) *reinterpret_cast<uint4*>(out_at(row0 + 2 * i)) = x[i];
    return;
  }
  float scale = 0.f;
  if constexpr (FMT == FMT_FP8_HEAD) {
    if (!active) return;
    scale = (is_v ? A.v_scale : A.k_scale)[h];
  } else {
    float* const where = (is_v ? A.v_scale : A.k_scale) + (size_t)pid * heads + h;
    const bool keeps = active && first > page_tok;        // rows in front of the new ones are live
    const float before = keeps ? *where : 0.f;
    // maximum of the finite magnitudes, as BF16 bits (ordered like integers)
    uint32_t amax = 0;
    if (active) {
#pragma unroll
      for (int i = 0; i < kRows / 2; ++i) {
        const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const uint32_t lo = w[k] & 0x7fffu, hi = (w[k] >> 16) & 0x7fffu;
          amax = max(amax, lo < 0x7f80u ? lo : 0u);
          amax = max(amax, hi < 0x7f80u ? hi : 0u);
        }
      }
    }
    amax = __reduce_max_sync(0xffffffffu, amax);
    if (wpi > 1) {   // (the same for the whole CTA)
      if (lane == 0) amax_s[warp] = amax;
      __syncthreads();
      for (int i = 0; i < wpi; ++i) amax = max(amax, amax_s[warp - part + i]);
    }
    if (!active) return;
    scale = fmaxf(page_scale_for(amax), before);
    if (keeps && scale > before) {   // earlier rows of the page to the larger scale (a power of two then)
      const float inv = 1.0f / scale;
#pragma unroll 1
      for (int i = 0; i < kRows / 2; ++i) {
        const int row = row0 + 2 * i;
        if (row >= ps || page_tok + row >= first) break;
        uint2* const p = reinterpret_cast<uint2*>(out_at(row));
        const uint2 old = *p;
        uint32_t o[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const uint32_t w = k ? old.y : old.x;
          const float2 a = f16x2_to_float2(e4m3x2_to_f16x2(w & 0xffffu)), c = f16x2_to_float2(e4m3x2_to_f16x2(w >> 16));
          o[k] = pack_e4m3x2(a.x * before * inv, a.y * before * inv) | pack_e4m3x2(c.x * before * inv, c.y * before * inv) << 16;
        }
        *p = make_uint2(o[0], o[1]);
      }
    }
    // every warp of the item has read the old scale before the barrier above, or is the only one
    if (part == 0 && lane == 0) *where = scale;
  }
  // (a scale that a caller put there need not be a power of two; a product with the reciprocal would then round twice)
  const bool pow2 = (__float_as_uint(scale) & 0x7fffffu) == 0u && scale >= 0x1p-126f && scale <= 0x1p126f;
  const float inv = 1.0f / scale;
#pragma unroll
  for (int i = 0; i < kRows / 2; ++i) {
    if (!((live >> i) & 1u)) continue;
    const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
    uint32_t o[4];
    if (pow2) {
#pragma unroll
      for (int k = 0; k < 4; ++k) o[k] = pack_e4m3x2(bf16_lo(w[k]) * inv, bf16_hi(w[k]) * inv);
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) o[k] = pack_e4m3x2(__fdiv_rn(bf16_lo(w[k]), scale), __fdiv_rn(bf16_hi(w[k]), scale));
    }
    *reinterpret_cast<uint2*>(out_at(row0 + 2 * i)) = make_uint2(o[0] | o[1] << 16, o[2] | o[3] << 16);
  }
}

// An 8-bit cache as BF16 pages: out = bf16(code * scale), rows of a last page behind the sequence's end zero.  A work item is
// one group of up to 16 rows of a page, all heads, K or V: consecutive 16-byte pieces to consecutive threads.  Bound by memory:
// one byte read and two written per element.
constexpr int kExpandThreads = 256;

struct ExpandArgs {
  const uint8_t *k_cache, *v_cache;
  const int32_t *page_table, *lk, *out_page_table;
  const float *k_scale, *v_scale;
  uint8_t *k_out, *v_out;
  int* status;
  int32_t out_num_pages;
  CacheGeom g;
};

template <int FMT>
__global__ void __launch_bounds__(kExpandThreads)
cache_expand_kernel(ExpandArgs A) {
  const int lane = threadIdx.x & 31;
  pdl_trigger();
  pdl_wait();
  const int shift = A.g.page_shift, heads = A.g.num_kv_heads;
  const int gshift = shift < 4 ? shift : 4;               // rows of a group
  const int groups = 1 << (shift - gshift);               // per page
  const int pieces = (heads * 8) << gshift;               // 16-byte pieces of a group
  // items: (sequence, group of rows), K and V of it next to each other
  long long item = blockIdx.x;
  long long base = 0;                                      // items in front of the 32 sequences looked at
  for (int b0 = 0; b0 < A.g.num_seqs; b0 += 32) {
    int L = b0 + lane < A.g.num_seqs ? A.lk[b0 + lane] : 0;
    if (L < 0 || L > ((long long)A.g.max_pages << shift)) {
      atomicOr(A.status + kCacheStBad, kBadLength);
      L = 0;
    }
    const long long n = 2ll * groups * (((long long)L + (1 << shift) - 1) >> shift);
    long long incl = n;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const long long o = __shfl_up_sync(0xffffffffu, incl, d);
      if (lane >= d) incl += o;
    }
    const long long total = __shfl_sync(0xffffffffu, incl, 31);
    for (; item < base + total; item += gridDim.x) {
      const int who = __popc(__ballot_sync(0xffffffffu, incl <= item - base));   // sequence b0 + who
      const long long rel = item - base - __shfl_sync(0xffffffffu, incl - n, who);
      const int Lb = __shfl_sync(0xffffffffu, L, who);
      const bool is_v = rel & 1;
      const long long grp = rel >> 1;
      const long long page = grp / groups;
      const int row0 = (int)(grp % groups) << gshift;
      const size_t entry = (size_t)(b0 + who) * A.g.max_pages + page;
      const int pid = A.page_table[entry], oid = A.out_page_table[entry];
      if (pid < 0 || pid >= A.g.num_pages || oid < 0 || oid >= A.out_num_pages) {
        if (threadIdx.x == 0) atomicOr(A.status + kCacheStBad, kBadPage);
        continue;
      }
      const uint8_t* src = (is_v ? A.v_cache : A.k_cache) + (((size_t)pid << shift) + row0) * heads * kHeadDim;
      uint8_t* dst = (is_v ? A.v_out : A.k_out) + (((size_t)oid << shift) + row0) * heads * (kHeadDim * 2);
      const float* scale = (is_v ? A.v_scale : A.k_scale) + (FMT == FMT_FP8_PAGE ? (size_t)pid * heads : 0);
      const long long left = (long long)Lb - (page << shift) - row0;   // live rows of the group, all of them if more
      for (int c = threadIdx.x; c < pieces; c += kExpandThreads) {
        const int hr = c >> 3;                            // row * heads + head
        const int row = hr / heads, head = hr - row * heads;
        uint32_t o[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        if (row < left) {
          const uint4 v = *reinterpret_cast<const uint4*>(src + (size_t)c * 16);
          const float s = scale[head];
          const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const float2 a = f16x2_to_float2(e4m3x2_to_f16x2(w[k] & 0xffffu)), d = f16x2_to_float2(e4m3x2_to_f16x2(w[k] >> 16));
            o[2 * k] = pack_bf16x2(a.x * s, a.y * s);
            o[2 * k + 1] = pack_bf16x2(d.x * s, d.y * s);
          }
        }
        uint4* p = reinterpret_cast<uint4*>(dst + (size_t)c * 32);
        p[0] = make_uint4(o[0], o[1], o[2], o[3]);
        p[1] = make_uint4(o[4], o[5], o[6], o[7]);
      }
    }
    base += total;
  }
}

}  // namespace fp2
