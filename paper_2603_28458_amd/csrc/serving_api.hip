// Host side of the calls around the indexer (include/hisa.h): argument validation, workspace carving and kernel launches
// of the paged cache's upkeep and of the attention that reads it.  Nothing here allocates or synchronises.
#include "../../include/hisa.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "api_common.h"
#include "attention_kernels.h"
#include "cache_kernels.h"

using namespace hisa;

namespace {

constexpr int kMaxHeads = 256, kMaxList = 65536, kMaxAppendD = 512;

constexpr float kLog2e = 1.44269504088896341f;
constexpr long kMaxThreads = (1L << 32) - 1;   // of a launch: the packet counts them in 32 bits

inline int elem_bytes(int dtype) { return dtype == HISA_F32 ? 4 : dtype == HISA_BF16 ? 2 : 1; }
inline bool overflows31(long a, long b) { return a * b >= (1L << 31); }   // (both below 2^31)

// What the append and the attention ask of a cache alike.
int check_cache(const hisa_cache* c, long align) {
  if (!c || !c->k) return HISA_ERR_NULL;
  if (c->dtype < HISA_F32 || c->dtype > HISA_FP8_E4M3) return HISA_ERR_DTYPE;
  if (c->n_pages < 1 || c->page < 1 || c->H_kv < 1 || c->H_kv > kMaxHeads || c->d < 1) return HISA_ERR_SHAPE;
  if (overflows31(c->n_pages, c->page)) return HISA_ERR_SHAPE;
  if (c->page_stride < 0 || c->token_stride < 0 || c->head_stride < 0) return HISA_ERR_SHAPE;
  if (c->dtype == HISA_FP8_E4M3 && (!c->k_scale || (c->v && !c->v_scale))) return HISA_ERR_NULL;
  if (!aligned16(c->k) || (c->v && !aligned16(c->v))) return HISA_ERR_ALIGN;
  if (c->page_stride % align || c->token_stride % align || c->head_stride % align) return HISA_ERR_ALIGN;
  return HISA_OK;
}

int check_attention(const hisa_queries* q, const hisa_cache* c, int32_t k) {
  if (!q || !q->q) return HISA_ERR_NULL;
  if (q->T < 1 || q->T > kMaxT || q->H < 1 || q->H > kMaxHeads) return HISA_ERR_SHAPE;
  if (!aligned16(q->q)) return HISA_ERR_ALIGN;
  if (!c) return HISA_ERR_NULL;
  int st = check_cache(c, 16 / (c->dtype >= HISA_F32 && c->dtype <= HISA_FP8_E4M3 ? elem_bytes(c->dtype) : 1));
  if (st) return st;
  if (!c->v || !c->block_table || !c->seq_len) return HISA_ERR_NULL;
  if (c->n_seq < 1 || c->n_seq > kMaxSeq || c->max_pages < 1 || q->H % c->H_kv) return HISA_ERR_SHAPE;
  if (c->page & (c->page - 1) || overflows31(c->max_pages, c->page)) return HISA_ERR_SHAPE;
  if (k < 0 || k > kMaxList) return HISA_ERR_SHAPE;
  if (c->weights != HISA_WEIGHTS_16BIT && c->weights != HISA_WEIGHTS_8BIT) return HISA_ERR_DTYPE;
  if (q->q_dtype == HISA_F32 && c->dtype == HISA_F32) {
    if (c->d < 4 || c->d % 4 || c->d > kF32MaxD) return HISA_ERR_SHAPE;
  } else if (q->q_dtype == HISA_BF16 && (c->dtype == HISA_BF16 || c->dtype == HISA_FP8_E4M3)) {
    if (c->d != 64 && c->d != 128) return HISA_ERR_SHAPE;
  } else {
    return HISA_ERR_DTYPE;
  }
  return HISA_OK;
}

// How a call is cut into workgroups; the same answer for the workspace and for the launch.  (Times: H = 64, H_kv = 8,
// d = 128, bf16 where nothing else is said.)
enum AttnKernel { ATTN_F32, ATTN_ROWS, ATTN_CHUNK };
struct AttnPlan {
  AttnKernel kernel;
  bool pair;          // ATTN_ROWS: 64 heads per workgroup, not 32
  bool rest;          // bf16, fp8: weights in two parts (the caller's choice)
  long units;         // tiles of query rows, of one KV head
  int splits;         // parts of their keys
  size_t ws_bytes;
};

constexpr long kCus = 256, kPartKeys = 256;

// Parts of the keys of `units` workgroups, of which `fit` run at a time, by the time until the last one is done.  A part
// costs as much as 512 keys beside its own (lists and ranges of 44 shapes, geometric mean: 128 38.0 us, 256 36.3, 512 35.5,
// 768 35.6, 1024 35.6; always filling the machine once 39.3).  uneven: sequences of a batch differ in length, which several
// rounds even out.
long parts(long units, long fit, long keys, long most, bool uneven) {
  long best = 0, last = 0;
  double least = 0;
  for (int j = 1; j <= 16; ++j) {            // (as many as j rounds hold)
    const long s = std::max(1L, std::min(most, j * fit / units));
    if (s == last) continue;
    last = s;
    const double rounds = (double)units * s / fit, one = (double)keys / s + 512;
    const double time = one * (rounds <= 1 ? 1. : uneven ? 0.88 * rounds + 0.4 : std::ceil(rounds));
    if (!best || time < least) least = time, best = s;
  }
  return best;
}

AttnPlan plan_attention(const hisa_queries* q, const hisa_cache* c, int32_t k) {
  AttnPlan p{};
  const long keys = k ? k : (long)c->max_pages * c->page;
  const long G = q->H / c->H_kv, T = q->T;
  long most = (keys + kPartKeys - 1) / kPartKeys, splits;
  // The second part costs nothing where a call waits for memory (32 tokens over up to 131072 keys 2563 and 2570 us, 1 over
  // 1000 12.6 and 12.5, 32 lists of 2048 19.8 and 20.4), and what a product costs where there are many rows: 1024 lists of
  // 2048 137 and 157 us, 1024 tokens behind 64K 1.95 and 2.68 ms, fp8 2.30 and 2.96.
  p.rest = c->weights == HISA_WEIGHTS_16BIT;
  // A few new tokens a sequence: one at a time reads their keys that many times, from L2 for the most part, with every
  // wave on keys of its own; together they read them once, but 32 rows are one wave's, and a tile of 64 keys takes it
  // 4000 cycles from scores to values.  Measured (one at a time, together), 64 sequences of 3000, 2 new tokens each: 167 and
  // 210 us, 4 each: 260 and 221, fp8 267 and 262; 32 of 8000, 2 each: 221 and 268, 4 each: 345 and 275, fp8 355 and 325; 64 heads on
  // one KV head, 64 sequences of 8000, 2 each: 89 and 152, fp8 4 each: 142 and 228; 200 of 500, 32 heads on 8, fp8, 4 each:
  // 173 and 186.
  // (The lengths are not known here, T counts padding and n_seq idle rows of the table: a chunk in a batch that is as large as
  // this is read token by token too, as often as it has tokens.  64 sequences of 8000 and one chunk of 64 of as many: 527 us,
  // in two calls 422; fp8 and a chunk of 192: 724 and 352; a table of 256 idle rows and a chunk of 512 behind 64K: 8.2 ms, with its
  // own row alone 1.4; fp8 and 1024: 17.4 and 3.1.  And a batch of single tokens padded to more rows takes the chunk kernel: 32
  // of 1000 32 us, in 256 rows 42; fp8 28 and 49.)
  const long few = c->dtype == HISA_FP8_E4M3 ? 4 : 2;
  if (c->dtype == HISA_F32) {
    p.kernel = ATTN_F32;
    p.units = k ? T * ((G + 31) / 32) : T * G / 32 + c->n_seq;
    most = (keys + 127) / 128;
    splits = parts(p.units * c->H_kv, (c->d > 128 ? 1 : 2) * kCus, keys, most, !k);
  } else if (k || T <= few * c->n_seq) {
    p.kernel = ATTN_ROWS;
    // (one gathering of the keys for up to 64 heads: lists of 2048, 64 heads on one KV head, 1024 queries 159 us, two
    // workgroups of 32 heads each 221; 32 queries 20.9 and 19.2)
    p.pair = G > 32;
    const long heads = p.pair ? 64 : 32;
    p.units = T * ((G + heads - 1) / heads);
    splits = parts(p.units * c->H_kv, (p.pair ? 1 : 2) * kCus, keys, most, !k);
  } else {
    p.kernel = ATTN_CHUNK;
    p.units = T * G / kChunkRows + c->n_seq;
    const long each = (T * G + (long)c->n_seq * kChunkRows - 1) / ((long)c->n_seq * kChunkRows);   // (if all were alike)
    splits = parts(each * c->n_seq * c->H_kv, kCus, keys, most, false);
  }
  p.splits = (int)splits;
  p.ws_bytes = splits > 1 ? (size_t)splits * T * q->H * (c->d + 2) * 4 : 0;
  return p;
}

AttnArgs attention_args(const hisa_queries* q, const hisa_cache* c, float scale, void* out, float* lse) {
  AttnArgs a{};
  a.q = q->q;
  a.q_seq = q->q_seq;
  a.q_pos = q->q_pos;
  a.q_lo = q->q_lo;
  a.k = c->k;
  a.v = c->v;
  a.k_scale = c->k_scale;
  a.v_scale = c->v_scale;
  a.table = c->block_table;
  a.seq_len = c->seq_len;
  a.out = out;
  a.lse = lse;
  a.page_stride = c->page_stride;
  a.token_stride = c->token_stride;
  a.head_stride = c->head_stride;
  a.scale_log2 = scale * kLog2e;
  a.T = q->T;
  a.H = q->H;
  a.H_kv = c->H_kv;
  a.G = q->H / c->H_kv;
  a.d = c->d;
  a.n_pages = c->n_pages;
  a.page_shift = __builtin_ctz(c->page);
  a.n_seq = c->n_seq;
  a.max_pages = c->max_pages;
  return a;
}

template <int D, int KDT, bool PAIR, bool LIST, bool REST>
int launch_rows(const AttnArgs& a, dim3 grid, hipStream_t st) {
  using Geo = RowGeom<D, KDT, PAIR>;
  constexpr auto kern = k_attn_rows<D, KDT, PAIR, LIST, REST>;
  if (Geo::kLds > 65536 && raise_lds_limit<kern>(Geo::kLds)) return HISA_ERR_LAUNCH;
  hipLaunchKernelGGL(kern, grid, dim3(64 * Geo::kWaves), Geo::kLds, st, a);
  return HISA_OK;
}

template <int D, int KDT, bool LIST, bool REST>
int launch_parts(const AttnArgs& a, const AttnPlan& p, dim3 grid, hipStream_t st) {
  if (p.kernel == ATTN_ROWS)
    return p.pair ? launch_rows<D, KDT, true, LIST, REST>(a, grid, st) : launch_rows<D, KDT, false, LIST, REST>(a, grid, st);
  if constexpr (!LIST) {
    constexpr auto kern = k_attn_chunk<D, KDT, REST>;
    constexpr int lds = ChunkGeom<D, KDT>::kLds;
    if (lds > 65536 && raise_lds_limit<kern>(lds)) return HISA_ERR_LAUNCH;
    hipLaunchKernelGGL(kern, grid, dim3(64 * kChunkWaves), lds, st, a);
  }
  return HISA_OK;
}

template <int D, int KDT, bool LIST>
int launch_mfma(const AttnArgs& a, const AttnPlan& p, dim3 grid, hipStream_t st) {
  return p.rest ? launch_parts<D, KDT, LIST, true>(a, p, grid, st) : launch_parts<D, KDT, LIST, false>(a, p, grid, st);
}

template <int D, bool LIST>
int launch_f32(const AttnArgs& a, dim3 grid, hipStream_t st) {
  constexpr auto kern = k_attn_f32<D, LIST>;
  constexpr int lds = F32Geom<D>::kLds;
  if (lds > 65536 && raise_lds_limit<kern>(lds)) return HISA_ERR_LAUNCH;
  hipLaunchKernelGGL(kern, grid, dim3(256), lds, st, a);
  return HISA_OK;
}

template <bool LIST>
int launch_attention(AttnArgs a, const AttnPlan& p, int dtype, hipStream_t st) {
  const long wgs = p.units * a.H_kv * a.splits;
  if (wgs * 512 > kMaxThreads) return HISA_ERR_SHAPE;
  const dim3 grid((unsigned)wgs);
  int status = HISA_OK;
  if (dtype == HISA_F32)
    status = a.d == 64    ? launch_f32<64, LIST>(a, grid, st)
             : a.d == 128 ? launch_f32<128, LIST>(a, grid, st)
                          : launch_f32<kF32MaxD, LIST>(a, grid, st);
  else if (dtype == HISA_BF16)
    status = a.d == 128 ? launch_mfma<128, 1, LIST>(a, p, grid, st) : launch_mfma<64, 1, LIST>(a, p, grid, st);
  else
    status = a.d == 128 ? launch_mfma<128, 2, LIST>(a, p, grid, st) : launch_mfma<64, 2, LIST>(a, p, grid, st);
  if (status) return status;
  if (a.splits > 1) {
    // more sets of lanes per row while that spares a trip to memory and the workgroup has them
    const int sets = 256 / (a.d / 4);
    int groups = 1;
    while (groups * 2 <= sets && groups * kJoinParts < a.splits) groups *= 2;
    const int rows = sets / groups;
    const dim3 jg((unsigned)(((long)a.T * a.H + rows - 1) / rows));
    if (dtype == HISA_F32)
      hipLaunchKernelGGL((k_attn_join<0, LIST>), jg, dim3(256), 0, st, a, groups);
    else
      hipLaunchKernelGGL((k_attn_join<1, LIST>), jg, dim3(256), 0, st, a, groups);
  }
  return launch_status();
}

int attention(const hisa_queries* q, const hisa_cache* c, const int32_t* q_start, const int32_t* list, int32_t k,
              float scale, void* out, float* lse, void* ws, size_t ws_bytes, void* stream) {
  const int st = check_attention(q, c, k);
  if (st) return st;
  if (!out || (k ? !list : !q_start)) return HISA_ERR_NULL;
  if (!aligned16(out)) return HISA_ERR_ALIGN;
  if (!(scale > 0.f) || !std::isfinite(scale * kLog2e)) return HISA_ERR_SHAPE;
  const AttnPlan p = plan_attention(q, c, k);
  if (p.ws_bytes && (!ws || ws_bytes < p.ws_bytes)) return HISA_ERR_WORKSPACE;
  if (p.ws_bytes && !aligned16(ws)) return HISA_ERR_ALIGN;
  AttnArgs a = attention_args(q, c, scale, out, lse);
  a.q_start = q_start;
  a.list = list;
  a.n_list = k;
  a.part = (float*)ws;
  a.splits = p.splits;
  hipStream_t s = (hipStream_t)stream;
  return k ? launch_attention<true>(a, p, c->dtype, s) : launch_attention<false>(a, p, c->dtype, s);
}

template <int SDT>
void launch_append(const AppendArgs& a, int dtype, dim3 grid, hipStream_t st) {
  if constexpr (SDT == HISA_F32)
    if (dtype == HISA_F32) {
      hipLaunchKernelGGL((k_cache_append<SDT, 0>), grid, dim3(256), 0, st, a);
      return;
    }
  if (dtype == HISA_BF16) hipLaunchKernelGGL((k_cache_append<SDT, 1>), grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL((k_cache_append<SDT, 2>), grid, dim3(256), 0, st, a);
}

}  // namespace

extern "C" {

int hisa_page_tables(const int32_t* ctx_len, const int32_t* new_len, int32_t n_seq, int32_t* block_table,
                     int32_t max_pages, int32_t page, const int32_t* free_pages, int32_t n_free, int32_t rows,
                     int32_t s_max, int32_t* seq_len, int32_t* q_start, int32_t* page_start, int32_t* q_seq,
                     int32_t* q_pos, int32_t* slots, int32_t* key_rows, void* stream) {
  if (!ctx_len || !new_len || !block_table || !seq_len || !q_start || !page_start || !q_seq || !q_pos || !slots)
    return HISA_ERR_NULL;
  if (n_free > 0 && !free_pages) return HISA_ERR_NULL;
  if (n_seq < 1 || n_seq > kMaxSeq || max_pages < 1 || page < 1 || n_free < 0 || rows < 1 || rows > kMaxT)
    return HISA_ERR_SHAPE;
  if (overflows31(n_seq, max_pages) || overflows31(max_pages, page)) return HISA_ERR_SHAPE;
  if (key_rows && (s_max < 1 || overflows31(n_seq, s_max))) return HISA_ERR_SHAPE;
  // (every workgroup reads the lengths that one of them would overwrite)
  if (seq_len == ctx_len || seq_len == new_len) return HISA_ERR_SHAPE;
  TableArgs a{ctx_len, new_len, free_pages, block_table, seq_len, q_start,   page_start, q_seq, q_pos,
              slots,   key_rows, n_seq,     max_pages,   page,    n_free,    rows,       s_max};
  hipStream_t st = (hipStream_t)stream;
  if (n_seq <= kTableThreads) {
    const unsigned wgs = (unsigned)((rows + kTableThreads - 1) / kTableThreads);
    hipLaunchKernelGGL(k_page_tables, dim3(wgs), dim3(kTableThreads), 0, st, a);
  } else {
    hipLaunchKernelGGL(k_page_scan, dim3(1), dim3(kTableThreads), 0, st, a);
    hipLaunchKernelGGL(k_page_rows, dim3((unsigned)((rows + 255) / 256)), dim3(256), 0, st, a);
  }
  return launch_status();
}

int hisa_cache_append(const hisa_cache* cache, const int32_t* slots, const void* k_new, const void* v_new,
                      int32_t src_dtype, int64_t src_stride, int32_t T, void* stream) {
  const int st = check_cache(cache, 8);
  if (st) return st;
  if (T == 0) return HISA_OK;
  if (!slots || !k_new || (v_new != nullptr) != (cache->v != nullptr)) return HISA_ERR_NULL;
  if (src_dtype != HISA_F32 && src_dtype != HISA_BF16) return HISA_ERR_DTYPE;
  if (src_dtype == HISA_BF16 && cache->dtype == HISA_F32) return HISA_ERR_DTYPE;
  if (T < 1 || T > kMaxT || cache->d % 8 || cache->d > kMaxAppendD) return HISA_ERR_SHAPE;
  if (src_stride < (int64_t)cache->H_kv * cache->d || src_stride >= (1L << 31)) return HISA_ERR_SHAPE;
  if (src_stride % 8 || !aligned16(k_new) || (v_new && !aligned16(v_new))) return HISA_ERR_ALIGN;
  AppendArgs a{};
  a.src[0] = k_new;
  a.src[1] = v_new;
  a.dst[0] = cache->k;
  a.dst[1] = cache->v;
  a.scale[0] = cache->k_scale;
  a.scale[1] = cache->v_scale;
  a.slots = slots;
  a.src_stride = src_stride;
  a.page_stride = cache->page_stride;
  a.token_stride = cache->token_stride;
  a.head_stride = cache->head_stride;
  a.T = T;
  a.R = cache->H_kv;
  a.d = cache->d;
  a.page = cache->page;
  a.lanes = 1;
  while (a.lanes * 8 < a.d) a.lanes *= 2;
  a.n_slots = (long)cache->n_pages * cache->page;
  const long rows = (long)T * a.R, per = 256 / a.lanes, wgs = (rows + per - 1) / per;
  if (wgs * 256 > kMaxThreads) return HISA_ERR_SHAPE;
  if (src_dtype == HISA_F32) launch_append<0>(a, cache->dtype, dim3((unsigned)wgs), (hipStream_t)stream);
  else launch_append<1>(a, cache->dtype, dim3((unsigned)wgs), (hipStream_t)stream);
  return launch_status();
}

int hisa_paged_attention(const hisa_queries* queries, const hisa_cache* cache, const int32_t* q_start,
                         float scale, void* out, float* lse, void* ws, size_t ws_bytes, void* stream) {
  return attention(queries, cache, q_start, nullptr, 0, scale, out, lse, ws, ws_bytes, stream);
}

int hisa_sparse_attention(const hisa_queries* queries, const hisa_cache* cache, const int32_t* topk_idx,
                          int32_t k, float scale, void* out, float* lse, void* ws, size_t ws_bytes,
                          void* stream) {
  if (k < 1) return HISA_ERR_SHAPE;
  return attention(queries, cache, nullptr, topk_idx, k, scale, out, lse, ws, ws_bytes, stream);
}

size_t hisa_attention_workspace_bytes(const hisa_queries* queries, const hisa_cache* cache, int32_t k) {
  if (check_attention(queries, cache, k)) return 0;
  return plan_attention(queries, cache, k).ws_bytes;
}

}  // extern "C"
