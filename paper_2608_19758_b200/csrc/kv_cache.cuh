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

// Maximum of the magnitudes of BF16 pairs, whatever its signs (a NaN loses against a number; NaN against NaN stays)
__device__ __forceinline__ uint32_t max_abs_bf16x2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("max.xorsign.abs.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}

// An item = the new tokens of one (page, KV head, K | V); rows of a page in groups of 16 to a warp, so that a warp keeps all it
// reads in registers between the maximum and the rounding: the tokens are read once.  16 lanes to a row (16 bytes of BF16 in, 8
// of e4m3 out each), eight rows in flight per lane.  A CTA looks its page up once and goes over the page's heads (or, when there
// are few pages, `split` CTAs share them): what a warp does is wait, for the lengths, then for tokens and page id together, so it
// should not wait again for each head.  41392 tokens, 8 heads, 64 a page: 59.6 us with a CTA and its look-ups for every 32 KB,
// 45.7 so (5.6 TB/s, 0.85 of the copy rate); 256 sequences of one token 9.9 / 6.7 us.  Bound by memory for prompts (2 bytes read and 1
// written per element), by launch and load latency for single tokens.
constexpr int kAppendThreads = 256;

struct AppendArgs {
  const uint8_t *k_new, *v_new;       // BF16 [total_new][stride]
  long long stride_bytes;             // of a token
  const int32_t *cu, *lk, *page_table;
  uint8_t *k_cache, *v_cache;
  float *k_scale, *v_scale;
  int* status;
  int32_t total_new;
  int32_t split;                      // CTAs per page slot
  CacheGeom g;
};

// a / s in 32 bits rounded to odd (towards zero, the last bit set where something was cut off): rounded again to fewer bits, to
// nearest, it gives what the quotient itself would.  Where the remainder, exact in 32 bits, could fall below their range both are
// brought up; a NaN or infinity stays.  (A call: seldom needed, and in line it took registers from the common path, 45.0 against 44.5 us
// for 41392 tokens with a scale per head.)
__device__ __noinline__ float div_to_odd(float a, float s) {
  const float up = s < 0x1p-60f ? 0x1p64f : 1.f;
  a *= up;
  s *= up;
  const float q = __fdiv_rz(a, s), rem = fmaf(-q, s, a);
  return __uint_as_float(__float_as_uint(q) | (rem < 0.f || rem > 0.f ? 1u : 0u));
}

// a * s likewise.  up: 2^64 where what was cut off could fall below the range of 32 bits, else 1
__device__ __forceinline__ float mul_to_odd(float a, float s, float up) {
  const float p = __fmul_rz(a, s), cut = fmaf(a, s * up, -(p * up));
  return __uint_as_float(__float_as_uint(p) | (cut < 0.f || cut > 0.f ? 1u : 0u));
}

// New tokens of one sequence: rows c0 .. c1 - 1, the sequence L tokens long with them
struct AppendSeq {
  int b, c0, c1, L;
  __device__ __forceinline__ bool fits(const AppendArgs& A) const {
    return c0 >= 0 && c1 >= c0 && c1 <= A.total_new && L >= c1 - c0 && L <= ((long long)A.g.max_pages << A.g.page_shift);
  }
  __device__ __forceinline__ long long first_page(int shift) const { return (L - (c1 - c0)) >> shift; }
  __device__ __forceinline__ long long last_page(int shift) const { return (L - 1) >> shift; }
};

// Sequence of a slot: the last one whose first slot is not behind it; 32-way search by a warp.  (Offsets that fall: any sequence.)
__device__ __forceinline__ AppendSeq append_find(const AppendArgs& A, long long slot) {
  const int lane = threadIdx.x & 31, shift = A.g.page_shift;
  int b = 0, n = A.g.num_seqs;
  while (n > 32) {
    const int stride = (n + 31) / 32, i = lane * stride;
    const unsigned bal = __ballot_sync(0xffffffffu, i < n && append_slot0(A.cu[b + min(i, n - 1)], b + i, shift) <= slot);
    const int skip = max(0, __popc(bal) - 1) * stride;
    b += skip;
    n = min(stride, n - skip);
  }
  const int i = b + min(lane, n - 1);
  const int x0 = A.cu[i], x1 = A.cu[i + 1], l = A.lk[i];
  const unsigned bal = __ballot_sync(0xffffffffu, lane < n && append_slot0(x0, i, shift) <= slot);
  const int who = max(0, __popc(bal) - 1);
  return {b + who, __shfl_sync(0xffffffffu, x0, who), __shfl_sync(0xffffffffu, x1, who), __shfl_sync(0xffffffffu, l, who)};
}

// A page of a sequence that fits, by CTA `turn0` of `split`
template <int FMT>
__device__ __forceinline__ void append_page(const AppendArgs& A, const AppendSeq& q, long long page, int turn0, int split) {
  constexpr int kRows = 16;           // rows per warp
  constexpr int kWarps = kAppendThreads / 32;
  __shared__ uint32_t amax_s[kWarps];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int shift = A.g.page_shift, ps = 1 << shift, heads = A.g.num_kv_heads;
  const int wpi = ps > kRows ? ps / kRows : 1;             // warps per item: 1, 2, 4 or 8
  const int part = warp % wpi;
  const int c0 = q.c0, L = q.L, first = L - (q.c1 - c0);
  const int page_tok = (int)page << shift;
  const int pid = A.page_table[(size_t)q.b * A.g.max_pages + page];
  constexpr int esz = FMT == FMT_BF16 ? 2 : 1;
  const int col = lane & 15, half = lane >> 4;
  const int row0 = part * kRows + half;                    // this lane's rows of the page: row0 + 2 i
  uint32_t live = 0;
#pragma unroll
  for (int i = 0; i < kRows / 2; ++i) {
    const int row = row0 + 2 * i, tok = page_tok + row;
    live |= (row < ps && tok >= first && tok < L ? 1u : 0u) << i;
  }
  const long long tok_off = (long long)(c0 + page_tok + row0 - first) * A.stride_bytes + col * 16;
  const bool keeps = first > page_tok;                     // rows in front of the new ones are live
  const int items = 2 * heads, per_turn = kWarps / wpi;    // (the same number of turns for all warps: there is a barrier inside)
  for (int item0 = turn0 * per_turn; item0 < items; item0 += split * per_turn) {
    const int item = item0 + warp / wpi;
    const bool active = item < items;
    const bool is_v = item >= heads;
    const int h = is_v ? item - heads : item;
    const uint8_t* src = (is_v ? A.v_new : A.k_new) + tok_off + h * (kHeadDim * 2);
    uint4 x[kRows / 2];
#pragma unroll
    for (int i = 0; i < kRows / 2; ++i) {
      x[i] = make_uint4(0, 0, 0, 0);
      if (active && ((live >> i) & 1u)) x[i] = *reinterpret_cast<const uint4*>(src + 2 * i * A.stride_bytes);
    }
    if (pid < 0 || pid >= A.g.num_pages) {                 // (looked at as late as this: the tokens need not wait for it)
      if (threadIdx.x == 0) atomicOr(A.status + kCacheStBad, kBadPage);
      return;
    }
    uint8_t* const out = (is_v ? A.v_cache : A.k_cache) + (((size_t)pid * ps + row0) * heads + h) * (kHeadDim * esz) + col * (8 * esz);
    const size_t row_step = (size_t)2 * heads * (kHeadDim * esz);
    if constexpr (FMT == FMT_BF16) {
      if (!active) continue;
#pragma unroll
      for (int i = 0; i < kRows / 2; ++i)
        if ((live >> i) & 1u) *reinterpret_cast<uint4*>(out + i * row_step) = x[i];
      continue;
    }
    float scale = 1.f;
    if constexpr (FMT == FMT_FP8_HEAD) {
      if (!active) continue;
      scale = (is_v ? A.v_scale : A.k_scale)[h];
    } else {
      float* const where = (is_v ? A.v_scale : A.k_scale) + (size_t)pid * heads + h;
      const float before = active && keeps ? *where : 0.f;
      uint32_t m = 0;
#pragma unroll
      for (int i = 0; i < kRows / 2; ++i) m = max_abs_bf16x2(max_abs_bf16x2(max_abs_bf16x2(max_abs_bf16x2(m, x[i].x), x[i].y), x[i].z), x[i].w);
      uint32_t amax = max(m & 0x7fffu, (m >> 16) & 0x7fffu);
      if (__any_sync(0xffffffffu, amax >= 0x7f80u)) {      // an infinity: the finite ones count (NaN has lost already)
        amax = 0;
#pragma unroll
        for (int i = 0; i < kRows / 2; ++i) {
          const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const uint32_t lo = w[k] & 0x7fffu, hi = (w[k] >> 16) & 0x7fffu;
            amax = max(amax, max(lo < 0x7f80u ? lo : 0u, hi < 0x7f80u ? hi : 0u));
          }
        }
      }
      amax = __reduce_max_sync(0xffffffffu, amax);
      if (wpi > 1) {   // (the same for the whole CTA)
        __syncthreads();                                   // (the turn before has been read)
        if (lane == 0) amax_s[warp] = amax;
        __syncthreads();
        for (int i = 0; i < wpi; ++i) amax = max(amax, amax_s[warp - part + i]);
      }
      if (!active) continue;
      scale = fmaxf(page_scale_for(amax), before);
      if (keeps && scale > before) {   // earlier rows of the page to the larger scale (a power of two then)
        const float inv = 1.0f / scale, up = before < 0x1p-60f ? 0x1p64f : 1.f;   // (rounded once: by e4m3)
        auto again = [&](float code) { return mul_to_odd(code, before, up) * inv; };
#pragma unroll 1
        for (int i = 0; i < kRows / 2; ++i) {
          const int row = row0 + 2 * i;
          if (row >= ps || page_tok + row >= first) break;
          uint2* const p = reinterpret_cast<uint2*>(out + i * row_step);
          const uint2 old = *p;
          uint32_t o[2];
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const uint32_t w = k ? old.y : old.x;
            const float2 a = f16x2_to_float2(e4m3x2_to_f16x2(w & 0xffffu)), c = f16x2_to_float2(e4m3x2_to_f16x2(w >> 16));
            o[k] = pack_e4m3x2(again(a.x), again(a.y)) | pack_e4m3x2(again(c.x), again(c.y)) << 16;
          }
          *p = make_uint2(o[0], o[1]);
        }
      }
      // every warp of the item has read the old scale before the barrier above, or is the only one
      if (part == 0 && lane == 0) *where = scale;
    }
    // A power of two divides exactly.  Another scale (a caller's): the quotient lies between the products with a reciprocal rounded
    // down and one rounded up, 2^-21 each way; where both round to the same e4m3 value so does it, and else it is divided, once rounded.
    const bool pow2 = (__float_as_uint(scale) & 0x7fffffu) == 0u, usual = scale >= 0x1p-100f && scale <= 0x1p126f;
    const float inv = 1.0f / scale, inv_lo = inv * (1.f - 0x1p-21f), inv_hi = inv * (1.f + 0x1p-21f);
    auto quantise = [&](uint32_t w, float f) { return pack_e4m3x2(bf16_lo(w) * f, bf16_hi(w) * f); };
    // (the product with a power of two is a BF16 number, but for subnormals, which e4m3 rounds to zero)
    const uint32_t inv2 = (__float_as_uint(inv) >> 16) * 0x10001u;
    auto quantise_pow2 = [&](uint32_t w) { const uint32_t s = mul_bf16x2(w, inv2); return pack_e4m3x2(bf16_lo(s), bf16_hi(s)); };
#pragma unroll
    for (int i = 0; i < kRows / 2; ++i) {
      if (!((live >> i) & 1u)) continue;
      const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
      uint32_t o[4];
      if (pow2 && usual) {
#pragma unroll
        for (int k = 0; k < 4; ++k) o[k] = quantise_pow2(w[k]);
      } else {
        uint32_t differ = usual ? 0u : 1u;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          o[k] = quantise(w[k], inv_lo);
          differ |= o[k] ^ quantise(w[k], inv_hi);
        }
        if (differ) {
#pragma unroll
          for (int k = 0; k < 4; ++k) o[k] = pack_e4m3x2(div_to_odd(bf16_lo(w[k]), scale), div_to_odd(bf16_hi(w[k]), scale));
        }
      }
      *reinterpret_cast<uint2*>(out + i * row_step) = make_uint2(o[0] | o[1] << 16, o[2] | o[3] << 16);
    }
  }
}

// Offsets that do not ascend (a sequence that does not fit) shift its neighbours' slots: the pages of sequences that do fit which no
// slot stands for, all by one CTA.  Apart from the others' code, which has no registers for a loop around a page: prompts 48 us, 55
// with it.
template <int FMT>
__device__ __noinline__ void append_rest(const AppendArgs& A, long long slots) {
  const int shift = A.g.page_shift;
  for (int b = 0; b < A.g.num_seqs; ++b) {
    const AppendSeq q = {b, A.cu[b], A.cu[b + 1], A.lk[b]};
    if (!q.fits(A)) {
      if (threadIdx.x == 0) atomicOr(A.status + kCacheStBad, kBadLength);
      continue;
    }
    if (q.c1 == q.c0) continue;
    for (long long page = q.first_page(shift); page <= q.last_page(shift); ++page) {
      const long long slot = append_slot0(q.c0, b, shift) + page - q.first_page(shift);
      if (slot >= slots || append_find(A, slot).b != b) append_page<FMT>(A, q, page, 0, 1);
    }
  }
}

template <int FMT>
__global__ void __launch_bounds__(kAppendThreads, 4)
cache_append_kernel(const __grid_constant__ AppendArgs A) {
  pdl_trigger();
  pdl_wait();
  const long long slots = (gridDim.x - 1) / A.split, slot = blockIdx.x / A.split;
  if (blockIdx.x == gridDim.x - 1) {   // one CTA looks whether the slots are what the others take them for
    bool ascend = true;
    for (int i = threadIdx.x; i < A.g.num_seqs; i += kAppendThreads) {
      const int x0 = A.cu[i], x1 = A.cu[i + 1];
      ascend &= x0 >= 0 && x1 >= x0 && x1 <= A.total_new;
    }
    if (!__syncthreads_and(ascend)) append_rest<FMT>(A, slots);
    return;
  }
  const AppendSeq q = append_find(A, slot);
  if (!q.fits(A)) {
    if (threadIdx.x == 0) atomicOr(A.status + kCacheStBad, kBadLength);
    return;
  }
  const int shift = A.g.page_shift;
  const long long page = q.first_page(shift) + (slot - append_slot0(q.c0, q.b, shift));
  if (q.c1 == q.c0 || page < q.first_page(shift) || page > q.last_page(shift)) return;
  append_page<FMT>(A, q, page, (int)(blockIdx.x % A.split), A.split);
}

// An 8-bit cache as BF16 pages: out = bf16(code * scale), rows of a last page behind the sequence's end zero.  A work item is
// one group of up to 16 rows of a page, all heads, K or V: consecutive 16-byte pieces to consecutive threads.  Bound by memory:
// one byte read and two written per element.  90816 tokens, 8 heads, 16 a page: 94.5 us, 5.9 TB/s, 0.90 of the copy rate (without the
// question of how a product rounds 92.0; stores of 16 bytes, half a sector each, 102; one / two pieces of a thread on their way 107.7 /
// 98.6).  Three CTAs to an SM: two / four 102.1 / 100.5.
constexpr int kExpandThreads = 256;
constexpr int kExpandBatch = 4;       // pieces of a thread on their way at a time

// whole sectors: 32 bytes per thread and instruction
__device__ __forceinline__ void st_global_32(void* p, const uint32_t (&r)[8]) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]),
               "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
               : "memory");
}

// code * scale has up to 28 bits.  Rounded to 32 bits and then to BF16 it may end on the wrong side of the middle between two BF16
// values, where the first rounding brings it there.  Not so with a scale of 20 bits or less (the product is exact; the writer's powers
// of two), and with few others: it takes one of the eight significands of a code next to a middle (looked at where no product leaves
// the range).
__device__ __forceinline__ bool exact_products(float s) { return (__float_as_uint(s) & 15u) == 0u && s >= 0x1p-100f; }
__device__ __forceinline__ bool rounds_twice(float s) {
  bool bad = !(s >= 0x1p-100f);
#pragma unroll
  for (int c = 8; c < 16; ++c) bad |= (__float_as_uint(s * (c * 0x1p-7f)) & 0xffffu) == 0x8000u;
  return bad && !exact_products(s);
}
// Then the product is rounded to odd, which leaves the one rounding to BF16.  Two codes; a call, to leave its registers to the common path.
__device__ __noinline__ uint32_t widen_rounding_once(uint32_t codes, float s) {
  const float2 a = f16x2_to_float2(e4m3x2_to_f16x2(codes & 0xffffu));
  const float up = s < 0x1p-60f ? 0x1p64f : 1.f;
  return pack_bf16x2(mul_to_odd(a.x, s, up), mul_to_odd(a.y, s, up));
}

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
__global__ void __launch_bounds__(kExpandThreads, 3)
cache_expand_kernel(ExpandArgs A) {
  const int lane = threadIdx.x & 31;
  pdl_trigger();
  pdl_wait();
  const int shift = A.g.page_shift, heads = A.g.num_kv_heads;
  const int gshift = shift < 4 ? shift : 4;               // rows of a group
  const int groups = 1 << (shift - gshift);               // per page
  const int pieces = (heads * 8) << gshift;               // 16-byte pieces of a group
  bool careful = false;
  if constexpr (FMT == FMT_FP8_HEAD) {                     // (a scale per page is looked at where it is used)
    for (int h = threadIdx.x; h < 2 * heads; h += kExpandThreads) careful |= rounds_twice(h < heads ? A.k_scale[h] : A.v_scale[h - heads]);
    careful = __syncthreads_or(careful);
  }
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
      for (int c0 = threadIdx.x; c0 < pieces; c0 += kExpandThreads * kExpandBatch) {
        uint4 v[kExpandBatch];
        float s[kExpandBatch];
#pragma unroll
        for (int k = 0; k < kExpandBatch; ++k) {
          const int c = c0 + k * kExpandThreads, hr = c >> 3;     // row * heads + head
          const int row = hr / heads;
          const bool in = c < pieces && row < left;
          v[k] = in ? *reinterpret_cast<const uint4*>(src + (size_t)c * 16) : make_uint4(0, 0, 0, 0);
          s[k] = in ? scale[hr - row * heads] : 1.f;
        }
        bool once = !careful;                              // the product's rounding to 32 bits loses nothing
        if constexpr (FMT == FMT_FP8_PAGE) {
#pragma unroll
          for (int k = 0; k < kExpandBatch; ++k) once &= exact_products(s[k]);
        }
        if (!once) {
#pragma unroll
          for (int k = 0; k < kExpandBatch; ++k)
            if (c0 + k * kExpandThreads < pieces) {
              const uint32_t w[4] = {v[k].x, v[k].y, v[k].z, v[k].w};
              uint32_t o[8];
#pragma unroll
              for (int j = 0; j < 8; ++j) o[j] = widen_rounding_once(w[j / 2] >> (j & 1) * 16, s[k]);
              st_global_32(dst + (size_t)(c0 + k * kExpandThreads) * 32, o);
            }
          continue;
        }
#pragma unroll
        for (int k = 0; k < kExpandBatch; ++k) {
          const int c = c0 + k * kExpandThreads;
          if (c >= pieces) break;
          const uint32_t w[4] = {v[k].x, v[k].y, v[k].z, v[k].w};
          uint32_t o[8];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float2 a = f16x2_to_float2(e4m3x2_to_f16x2(w[j] & 0xffffu)), d = f16x2_to_float2(e4m3x2_to_f16x2(w[j] >> 16));
            o[2 * j] = pack_bf16x2(a.x * s[k], a.y * s[k]);
            o[2 * j + 1] = pack_bf16x2(d.x * s[k], d.y * s[k]);
          }
          st_global_32(dst + (size_t)c * 32, o);
        }
      }
    }
    base += total;
  }
}

}  // namespace fp2
