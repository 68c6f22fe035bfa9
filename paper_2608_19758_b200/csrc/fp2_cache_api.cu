// C ABI of the paged KV cache (declared in include/fp2.h): appending, reading back as BF16 pages, decoding.  The lengths of the
// sequences are read on the device, so a handle is made once for a cache and no call copies, allocates or waits.
#include <cuda_runtime.h>
#include <math.h>
#include <string.h>

#include <algorithm>
#include <new>

#include "../../include/fp2.h"
#include "common.cuh"
#include "decode.cuh"
#include "kv_cache.cuh"

using namespace fp2;

struct fp2_cache {
  fp2_cache_params prm;
  int device;          // -1: made without a usable device
  int workers;         // CTAs of the decode kernel that are resident at a time
  int page_shift;
  float scale_log2;
  int64_t ws_counters, ws_part_ml, ws_part_o, ws_bytes;
};

constexpr int kMaxDecodeTileRows = 16;
constexpr int64_t kMaxCacheTokens = 1ll << 30;   // positions and windows are 32-bit sums of two such

static int64_t up(int64_t x, int64_t a) { return (x + a - 1) / a * a; }
static bool on(const void* p, size_t a) { return p && reinterpret_cast<uintptr_t>(p) % a == 0; }

template <int FMT, int NR>
static bool set_decode_attr() {
  return cudaFuncSetAttribute(decode_kernel<FMT, NR>, cudaFuncAttributeMaxDynamicSharedMemorySize, DecodeCfg<FMT, NR>::kSmemBytes) ==
         cudaSuccess;
}
template <int FMT>
static bool set_decode_attrs() {
  return set_decode_attr<FMT, 1>() && set_decode_attr<FMT, 2>();
}

extern "C" fp2_status fp2_cache_create(const fp2_cache_params* p, fp2_cache** out) {
  if (!p || !out) return FP2_ERR_INVALID_ARG;
  if (p->max_seqs <= 0 || p->num_q_heads <= 0 || p->num_kv_heads <= 0 || p->num_q_heads % p->num_kv_heads != 0)
    return FP2_ERR_INVALID_ARG;
  if (p->num_pages <= 0 || p->max_pages_per_seq <= 0 || !(p->softmax_scale >= 0.f) || isinf(p->softmax_scale))
    return FP2_ERR_INVALID_ARG;
  if (p->head_dim != kHeadDim) return FP2_ERR_UNSUPPORTED;
  int shift = 3;
  while (shift <= 7 && (1 << shift) != p->page_size) ++shift;
  if (shift > 7) return FP2_ERR_UNSUPPORTED;
  if (p->format != FP2_CACHE_BF16 && p->format != FP2_CACHE_FP8_HEAD && p->format != FP2_CACHE_FP8_PAGE)
    return FP2_ERR_UNSUPPORTED;
  if ((int64_t)p->num_pages << shift > 0x7fffffffll) return FP2_ERR_CAPACITY;   // slots are 31-bit
  if ((int64_t)p->max_pages_per_seq << shift > kMaxCacheTokens || (int64_t)p->num_q_heads * kHeadDim > 1 << 20)
    return FP2_ERR_CAPACITY;
  fp2_cache* c = new (std::nothrow) fp2_cache();
  if (!c) return FP2_ERR_CUDA;
  c->prm = *p;
  c->page_shift = shift;
  const double sc = p->softmax_scale > 0.f ? (double)p->softmax_scale : 1.0 / sqrt((double)kHeadDim);
  c->scale_log2 = (float)(sc * 1.4426950408889634);
  c->device = -1;
  int dev = -1, sms = 0, major = 0;
  if (cudaGetDevice(&dev) == cudaSuccess && cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) == cudaSuccess &&
      cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) == cudaSuccess) {
    if (major != 10) { delete c; return FP2_ERR_UNSUPPORTED; }
    if (!set_decode_attrs<FMT_BF16>() || !set_decode_attrs<FMT_FP8_HEAD>() || !set_decode_attrs<FMT_FP8_PAGE>()) {
      (void)cudaGetLastError();
      delete c;
      return FP2_ERR_CUDA;
    }
    c->device = dev;
  } else {
    (void)cudaGetLastError();
    sms = 0;
  }
  c->workers = std::max(sms, 1) * kDecCtasPerSm;
  int64_t o = 1024;                                        // status block
  c->ws_counters = o; o += up(12 * (int64_t)c->workers, 1024);
  c->ws_part_ml = o;  o += up(2ll * c->workers * kMaxDecodeTileRows * kRowStateBytes, 1024);
  c->ws_part_o = o;   o += 2ll * c->workers * kMaxDecodeTileRows * kHeadDim * 4;
  c->ws_bytes = o;
  *out = c;
  return FP2_OK;
}

extern "C" fp2_status fp2_cache_sizes(const fp2_cache* c, int64_t* workspace_bytes) {
  if (!c || !workspace_bytes) return FP2_ERR_INVALID_ARG;
  *workspace_bytes = c->ws_bytes;
  return FP2_OK;
}

extern "C" void fp2_cache_destroy(fp2_cache* c) { delete c; }

static CacheGeom geom(const fp2_cache* c, int num_seqs) {
  return CacheGeom{c->prm.num_kv_heads, c->page_shift, c->prm.num_pages, c->prm.max_pages_per_seq, num_seqs};
}

// What all calls take.  No sequences: nothing is read, and arrays of them (page table, lengths, offsets) may be NULL, as those of
// empty tensors are.
static fp2_status check_cache(const fp2_cache* c, const void* k, const void* v, const void* pt, const void* lk, const float* ks,
                              const float* vs, const void* ws, int32_t num_seqs) {
  if (!c || !on(k, 16) || !on(v, 16) || !on(ws, 1024)) return FP2_ERR_INVALID_ARG;
  if (c->prm.format != FP2_CACHE_BF16 && (!ks || !vs)) return FP2_ERR_INVALID_ARG;
  if (num_seqs != 0 && (!pt || !lk)) return FP2_ERR_INVALID_ARG;
  return num_seqs < 0 || num_seqs > c->prm.max_seqs ? FP2_ERR_INVALID_ARG : FP2_OK;
}

static fp2_status check_device(const fp2_cache* c) {
  if (c->device < 0) return FP2_ERR_CUDA;
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess) return FP2_ERR_CUDA;
  return dev == c->device ? FP2_OK : FP2_ERR_INVALID_ARG;
}

// A launch that may overlap the end of its predecessor on the stream: every kernel here waits for it before it reads or writes
// global memory (pdl_wait).
template <typename Args>
static fp2_status launch(void (*kernel)(Args), int64_t grid, unsigned block, size_t smem, fp2_stream stream, const Args& args) {
  if (grid > 0x7fffffffll) return FP2_ERR_CAPACITY;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)grid);
  cfg.blockDim = dim3(block);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = reinterpret_cast<cudaStream_t>(stream);
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, args) == cudaSuccess ? FP2_OK : FP2_ERR_CUDA;
}

extern "C" fp2_status fp2_cache_append(const fp2_cache* c, const void* k_new, const void* v_new, int64_t new_stride,
                                       const int32_t* page_table, const int32_t* cu, const int32_t* lk, int32_t num_seqs,
                                       int32_t total_new, void* k, void* v, float* ks, float* vs, void* workspace,
                                       fp2_stream stream) {
  fp2_status s = check_cache(c, k, v, page_table, lk, ks, vs, workspace, num_seqs);
  if (s != FP2_OK) return s;
  if ((!cu && num_seqs > 0) || total_new < 0) return FP2_ERR_INVALID_ARG;
  if (num_seqs == 0 || total_new == 0) return FP2_OK;
  if (!on(k_new, 16) || !on(v_new, 16)) return FP2_ERR_INVALID_ARG;
  if (new_stride < (int64_t)c->prm.num_kv_heads * kHeadDim || new_stride % 8 != 0) return FP2_ERR_INVALID_ARG;
  if ((s = check_device(c)) != FP2_OK) return s;
  AppendArgs a;
  a.k_new = (const uint8_t*)k_new; a.v_new = (const uint8_t*)v_new;
  a.stride_bytes = new_stride * 2;
  a.cu = cu; a.lk = lk; a.page_table = page_table;
  a.k_cache = (uint8_t*)k; a.v_cache = (uint8_t*)v;
  a.k_scale = ks; a.v_scale = vs;
  a.status = (int*)workspace;
  a.total_new = total_new;
  a.g = geom(c, num_seqs);
  const int64_t slots = (int64_t)(total_new >> c->page_shift) + 2ll * num_seqs;   // see append_slot0
  // A CTA per page, or up to one per turn of its warps as long as there are no more than 18 CTAs per SM: four are resident, and
  // with few waves of long ones the last wave leaves the chip idle.  41392 tokens, 64 / 128 a page, up to 4 / 9 / 18 / 27 per SM:
  // 55.2 / 48.6 / 46.6 / 49.9 us, 71.2 / 51.3 / 48.8 / 50.0.
  const int64_t turns = (2ll * c->prm.num_kv_heads * std::max(1, c->prm.page_size / 16) + 7) / 8;
  a.split = (int32_t)std::max<int64_t>(1, std::min<int64_t>(turns, 18 * (c->workers / kDecCtasPerSm) / slots));
  const int64_t grid = slots * a.split + 1;   // (one for the pages that no slot stands for)
  auto kernel = c->prm.format == FP2_CACHE_BF16 ? cache_append_kernel<FMT_BF16>
                : c->prm.format == FP2_CACHE_FP8_HEAD ? cache_append_kernel<FMT_FP8_HEAD> : cache_append_kernel<FMT_FP8_PAGE>;
  return launch(kernel, grid, kAppendThreads, 0, stream, a);
}

extern "C" fp2_status fp2_cache_expand(const fp2_cache* c, const void* k, const void* v, const int32_t* page_table,
                                       const int32_t* lk, int32_t num_seqs, const float* ks, const float* vs, void* k_out,
                                       void* v_out, const int32_t* out_page_table, int32_t out_num_pages, void* workspace,
                                       fp2_stream stream) {
  if (c && c->prm.format == FP2_CACHE_BF16) return FP2_ERR_UNSUPPORTED;   // it is BF16 pages already
  fp2_status s = check_cache(c, k, v, page_table, lk, ks, vs, workspace, num_seqs);
  if (s != FP2_OK) return s;
  if (out_num_pages < 0) return FP2_ERR_INVALID_ARG;
  if (num_seqs == 0) return FP2_OK;
  if (!out_page_table) return FP2_ERR_INVALID_ARG;
  if (out_num_pages > 0 && (!on(k_out, 32) || !on(v_out, 32))) return FP2_ERR_INVALID_ARG;
  if ((s = check_device(c)) != FP2_OK) return s;
  ExpandArgs a;
  a.k_cache = (const uint8_t*)k; a.v_cache = (const uint8_t*)v;
  a.page_table = page_table; a.lk = lk; a.out_page_table = out_page_table;
  a.k_scale = ks; a.v_scale = vs;
  a.k_out = (uint8_t*)k_out; a.v_out = (uint8_t*)v_out;
  a.status = (int*)workspace;
  a.out_num_pages = out_num_pages;
  a.g = geom(c, num_seqs);
  const int64_t groups = (int64_t)num_seqs * c->prm.max_pages_per_seq * std::max(1, c->prm.page_size / 16) * 2;
  const int64_t grid = std::min<int64_t>(groups, (int64_t)(c->workers / kDecCtasPerSm) * 8);
  return launch(c->prm.format == FP2_CACHE_FP8_HEAD ? cache_expand_kernel<FMT_FP8_HEAD> : cache_expand_kernel<FMT_FP8_PAGE>, grid,
                kExpandThreads, 0, stream, a);
}

// Packed rows of a tile, 8 or 16, by the rows that a sequence has on average: its pages are copied once for all rows of a tile.
// 32 sequences of 4096 tokens, heads 32 / 8, tiles of 8 / 16 rows, us: 4 rows BF16 86 / 88, head scales 54 / 57, page scales 57 / 69;
// 8 rows 89 / 90, 55 / 58, 57 / 71; 12 rows 165 / 92, 98 / 60, 99 / 73; 20 rows 247 / 168, 147 / 103, 147 / 127.  Tiles of 32 rows, whose
// accumulators do not fit the registers, took 236, 165 and 167 for 20 rows, and were behind for 32, 256 and 1024 rows too.
template <int FMT>
static fp2_status launch_decode(int64_t rows, int64_t grid, fp2_stream stream, const DecodeArgs& a) {
  return rows <= 8 ? launch(decode_kernel<FMT, 1>, grid, kDecThreads, DecodeCfg<FMT, 1>::kSmemBytes, stream, a)
                   : launch(decode_kernel<FMT, 2>, grid, kDecThreads, DecodeCfg<FMT, 2>::kSmemBytes, stream, a);
}

extern "C" fp2_status fp2_decode(const fp2_cache* c, const void* q, int64_t q_stride, const void* k, const void* v,
                                 const int32_t* page_table, const int32_t* cu, const int32_t* lk, int32_t num_seqs,
                                 int32_t total_q, const float* ks, const float* vs, int32_t window_tokens, int32_t sink_tokens,
                                 void* out, float* lse, void* workspace, fp2_stream stream) {
  fp2_status s = check_cache(c, k, v, page_table, lk, ks, vs, workspace, num_seqs);
  if (s != FP2_OK) return s;
  if ((!cu && num_seqs > 0) || total_q < 0 || window_tokens < 0 || sink_tokens < 0) return FP2_ERR_INVALID_ARG;
  if (num_seqs == 0 || total_q == 0) return FP2_OK;
  if (!on(q, 16) || !on(out, 16)) return FP2_ERR_INVALID_ARG;
  if (q_stride < (int64_t)c->prm.num_q_heads * kHeadDim || q_stride % 8 != 0) return FP2_ERR_INVALID_ARG;
  const int group = c->prm.num_q_heads / c->prm.num_kv_heads;
  if ((int64_t)group * total_q > 0x7fffffffll - 64) return FP2_ERR_CAPACITY;   // packed rows are 32-bit
  if ((s = check_device(c)) != FP2_OK) return s;
  uint8_t* ws = (uint8_t*)workspace;
  DecodeArgs a;
  a.q = (const uint8_t*)q;
  a.q_stride_bytes = q_stride * 2;
  a.cu = cu; a.lk = lk; a.page_table = page_table;
  a.k = (const uint8_t*)k; a.v = (const uint8_t*)v;
  a.k_scale = ks; a.v_scale = vs;
  a.out = (__nv_bfloat16*)out;
  a.lse = lse;
  a.part_o = (float*)(ws + c->ws_part_o);
  a.part_ml = ws + c->ws_part_ml;
  a.counters = (int32_t*)(ws + c->ws_counters);
  a.status = (int*)ws;
  a.total_q = total_q; a.num_q_heads = c->prm.num_q_heads; a.group = group;
  a.group_magic = group > 1 ? (uint32_t)(((1ull << 32) + group - 1) / group) : 0u;
  a.window = (int32_t)std::min<int64_t>(window_tokens, kMaxCacheTokens);   // (no position is that far away)
  a.sinks = window_tokens > 0 ? (int32_t)std::min<int64_t>(sink_tokens, kMaxCacheTokens) : 0;
  a.scale_log2 = c->scale_log2;
  a.g = geom(c, num_seqs);
  const int64_t rows = ((int64_t)group * total_q + num_seqs - 1) / num_seqs;
  // (no more CTAs than there can be items, one of 64 tokens for a tile of 8 rows at least)
  const int64_t tiles = ((int64_t)group * total_q / 8 + num_seqs) * c->prm.num_kv_heads;
  const int64_t blocks = (((int64_t)c->prm.max_pages_per_seq << c->page_shift) + 63) / 64 + kDecUnitCost;
  const int64_t grid = std::min<int64_t>(c->workers, tiles * blocks);
  return c->prm.format == FP2_CACHE_BF16       ? launch_decode<FMT_BF16>(rows, grid, stream, a)
         : c->prm.format == FP2_CACHE_FP8_HEAD ? launch_decode<FMT_FP8_HEAD>(rows, grid, stream, a)
                                               : launch_decode<FMT_FP8_PAGE>(rows, grid, stream, a);
}

extern "C" fp2_status fp2_cache_read_status(const fp2_cache* c, void* workspace, int32_t* h_words, fp2_stream stream) {
  if (!c || !on(workspace, 1024)) return FP2_ERR_INVALID_ARG;
  const fp2_status s = check_device(c);
  if (s != FP2_OK) return s;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  int32_t w[8];
  if (cudaMemcpyAsync(w, workspace, sizeof(w), cudaMemcpyDeviceToHost, st) != cudaSuccess) return FP2_ERR_CUDA;
  if (cudaStreamSynchronize(st) != cudaSuccess) return FP2_ERR_CUDA;
  if (cudaMemsetAsync(workspace, 0, sizeof(w), st) != cudaSuccess) return FP2_ERR_CUDA;
  if (h_words) memcpy(h_words, w, sizeof(w));
  return w[kCacheStBad] ? FP2_ERR_INVALID_ARG : FP2_OK;
}
