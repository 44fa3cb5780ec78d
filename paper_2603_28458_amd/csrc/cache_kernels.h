// Kernels that keep a paged cache: block tables and slot maps from request lengths, and the rows of new tokens.
#pragma once

#include "hisa_device.h"

namespace hisa {

// ---- block tables and slot maps ---------------------------------------------------------------
struct TableArgs {
  const int32_t* ctx_len;
  const int32_t* new_len;
  const int32_t* free_pages;
  int32_t* block_table;
  int32_t* seq_len;
  int32_t* q_start;
  int32_t* page_start;
  int32_t* q_seq;
  int32_t* q_pos;
  int32_t* slots;
  int32_t* key_rows;
  int n_seq, max_pages, page, n_free, rows, s_max;
};

constexpr int kTableThreads = 1024;

// A sequence as the tables see it: lengths that cannot lead out of any array.  Sums of new tokens stop at `rows`: adding
// with a ceiling is associative, so a scan may do it in any order.  Sums of pages stay below n_seq * max_pages, so 2^31.
struct TableSeq {
  int ctx, had, need;     // tokens cached, pages they fill, pages they and the new ones fill
  uint32_t fresh, grown;  // new tokens, new pages
  int len;
};

__device__ __forceinline__ TableSeq table_seq(const TableArgs& a, int n) {
  TableSeq s;
  const long cap = (long)a.max_pages * a.page;
  const int ctx = a.ctx_len[n], fresh = a.new_len[n];
  s.ctx = ctx < 0 ? 0 : ctx;
  const long f = fresh < 0 ? 0 : fresh;
  s.fresh = (uint32_t)(f < a.rows ? f : a.rows);
  const long total = s.ctx + f;
  const long end = total < cap ? total : cap, begin = s.ctx < cap ? s.ctx : cap;
  s.len = (int)end;
  s.had = (int)((begin + a.page - 1) / a.page);
  s.need = (int)((end + a.page - 1) / a.page);
  s.grown = (uint32_t)(s.need - s.had);
  return s;
}

__device__ __forceinline__ uint32_t add_to(uint32_t a, uint32_t b, uint32_t ceiling) {
  const uint32_t s = a + b;
  return s < ceiling ? s : ceiling;
}

// Exclusive prefix sums (of tokens with a ceiling) of one value pair per thread over the workgroup; the totals come back too.
__device__ __forceinline__ void table_scan(uint32_t& tok, uint32_t& pg, uint32_t& tok_all, uint32_t& pg_all,
                                           uint32_t ceiling, uint32_t (*part)[2]) {
  const int lane = lane_id(), wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  uint32_t t = tok, p = pg;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t tu = __shfl_up(t, o), pu = __shfl_up(p, o);
    if (lane >= o) {
      t = add_to(t, tu, ceiling);
      p += pu;
    }
  }
  if (lane == 63) {
    part[wave][0] = t;
    part[wave][1] = p;
  }
  uint32_t te = __shfl_up(t, 1), pe = __shfl_up(p, 1);
  if (lane == 0) te = pe = 0;
  __syncthreads();
  uint32_t tb = 0, pb = 0, ta = 0, pa = 0;
  for (int w = 0; w < waves; ++w) {
    if (w == wave) {
      tb = ta;
      pb = pa;
    }
    ta = add_to(ta, part[w][0], ceiling);
    pa += part[w][1];
  }
  __syncthreads();
  tok = add_to(tb, te, ceiling);
  pg = pb + pe;
  tok_all = ta;
  pg_all = pa;
}

// Last n in [0, n_seq) with start[n] <= x, for an ascending start[0] == 0.
template <class Start>
__device__ __forceinline__ int table_find(const Start& start, int n_seq, int x) {
  int lo = 0, hi = n_seq;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if ((int)start[mid] <= x) lo = mid;
    else hi = mid;
  }
  return lo;
}

// Pages taken from the free list, from number `first` on, every `step`-th.  (Where all new tokens have a row there are no
// more of them than rows, and threads: a new page holds a new token.  Where `rows` cuts the tokens short there may be any
// number, and each thread takes several.)
template <class Start>
__device__ __forceinline__ void table_pages(const TableArgs& a, const Start& page_start, int pages, uint32_t first,
                                            uint32_t step) {
  for (uint32_t e = first; e < (uint32_t)pages; e += step) {          // (both below 2^31)
    const int n = table_find(page_start, a.n_seq, (int)e);
    const TableSeq s = table_seq(a, n);
    const int j = s.had + (int)e - (int)page_start[n];
    if (j < s.need) a.block_table[(long)n * a.max_pages + j] = (int)e < a.n_free ? a.free_pages[e] : -1;
  }
}

// Token row e.
template <class Start>
__device__ __forceinline__ void table_row(const TableArgs& a, const Start& q_start, const Start& page_start, int tokens, int e) {
  if (e >= a.rows) return;
  int seq = 0, pos = -1, slot = -1, key_row = -1;
  if (e < tokens) {
    seq = table_find(q_start, a.n_seq, e);
    const TableSeq s = table_seq(a, seq);
    const long at_pos = (long)s.ctx + e - (int)q_start[seq];       // (a cached length may be any number)
    pos = at_pos < 0x7fffffff ? (int)at_pos : 0x7fffffff;
    if (pos < s.len) {
      const int j = pos / a.page;
      // the page of a new entry is looked up where the entry comes from: its write is not waited for
      const int f = (int)page_start[seq] + j - s.had;
      const int id = j < s.had ? a.block_table[(long)seq * a.max_pages + j] : f < a.n_free ? a.free_pages[f] : -1;
      const long at = (long)id * a.page + pos % a.page;
      if (id >= 0 && at < 1L << 31) slot = (int)at;
    }
    if (pos >= 0 && pos < a.s_max) key_row = seq * a.s_max + pos;
  }
  a.q_seq[e] = seq;
  a.q_pos[e] = pos;
  a.slots[e] = slot;
  if (a.key_rows) a.key_rows[e] = key_row;
}

// Up to kTableThreads sequences: every workgroup scans all of them into LDS and fills its own rows; the first one also
// writes the scans.  One launch: what such a call costs is the latency of its few dependent loads (32 sequences 4.5 us, 1000
// 5.7; with the two launches below 6.2 and 8.7).
static __global__ __launch_bounds__(kTableThreads) void k_page_tables(TableArgs a) {
  __shared__ uint32_t part[16][2];
  __shared__ uint32_t q_start[kTableThreads], page_start[kTableThreads];
  const int n = threadIdx.x;
  TableSeq s{};
  if (n < a.n_seq) s = table_seq(a, n);
  uint32_t tok = s.fresh, pg = s.grown, tok_all, pg_all;
  table_scan(tok, pg, tok_all, pg_all, (uint32_t)a.rows, part);
  q_start[n] = tok;
  page_start[n] = pg;
  if (blockIdx.x == 0) {
    if (n < a.n_seq) {
      a.seq_len[n] = s.len;
      a.q_start[n] = (int)tok;
      a.page_start[n] = (int)pg;
    }
    if (n == 0) {
      a.q_start[a.n_seq] = (int)tok_all;
      a.page_start[a.n_seq] = (int)pg_all;
    }
  }
  __syncthreads();
  const int e = blockIdx.x * kTableThreads + n;
  table_pages(a, page_start, (int)pg_all, e, gridDim.x * kTableThreads);
  table_row(a, q_start, page_start, (int)tok_all, e);
}

// More sequences: the scans by one workgroup (each thread a run of consecutive sequences), the rows by another launch.
static __global__ __launch_bounds__(kTableThreads) void k_page_scan(TableArgs a) {
  __shared__ uint32_t part[16][2];
  const int per = (a.n_seq + kTableThreads - 1) / kTableThreads;
  const int first = threadIdx.x * per, last = first + per < a.n_seq ? first + per : a.n_seq;
  uint32_t tok = 0, pg = 0, tok_all, pg_all;
  for (int n = first; n < last; ++n) {
    const TableSeq s = table_seq(a, n);
    tok = add_to(tok, s.fresh, (uint32_t)a.rows);
    pg += s.grown;
  }
  table_scan(tok, pg, tok_all, pg_all, (uint32_t)a.rows, part);
  for (int n = first; n < last; ++n) {
    const TableSeq s = table_seq(a, n);
    a.seq_len[n] = s.len;
    a.q_start[n] = (int)tok;
    a.page_start[n] = (int)pg;
    tok = add_to(tok, s.fresh, (uint32_t)a.rows);
    pg += s.grown;
  }
  if (threadIdx.x == 0) {
    a.q_start[a.n_seq] = (int)tok_all;
    a.page_start[a.n_seq] = (int)pg_all;
  }
}

static __global__ __launch_bounds__(256) void k_page_rows(TableArgs a) {
  const int e = blockIdx.x * 256 + threadIdx.x;
  table_pages(a, a.page_start, a.page_start[a.n_seq], e, gridDim.x * 256);
  table_row(a, a.q_start, a.page_start, a.q_start[a.n_seq], e);
}

// ---- new rows into the cache --------------------------------------------------------------------
struct AppendArgs {
  const void* src[2];   // keys, values (or NULL)
  void* dst[2];
  float* scale[2];
  const int32_t* slots;
  long src_stride, page_stride, token_stride, head_stride;
  int T, R, d, page;
  int lanes;            // lanes per row: a power of two, at least d / 8
  long n_slots;
};

struct Eight {
  float x[8];
};

__device__ __forceinline__ float bf16_low(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_high(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
  const bf16x2 p = {(__bf16)lo, (__bf16)hi};
  return __builtin_bit_cast(uint32_t, p);
}

template <int SDT>
__device__ __forceinline__ Eight load_eight(const void* src, long at) {
  Eight e;
  if constexpr (SDT == 0) {
    const float4* p = reinterpret_cast<const float4*>((const float*)src + at);
    const float4 a = p[0], b = p[1];
    e.x[0] = a.x, e.x[1] = a.y, e.x[2] = a.z, e.x[3] = a.w;
    e.x[4] = b.x, e.x[5] = b.y, e.x[6] = b.z, e.x[7] = b.w;
  } else {
    const uint4 a = *reinterpret_cast<const uint4*>((const uint16_t*)src + at);
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      e.x[2 * i] = bf16_low(w[i]);
      e.x[2 * i + 1] = bf16_high(w[i]);
    }
  }
  return e;
}

// x / b, correctly rounded, from y = 1 / b, correctly rounded: two corrections by the exact remainder (Markstein's), 5
// instructions where a division is a dozen.  Remainders are exact while |x| is above 2^-102 or the quotient below any use.
__device__ __forceinline__ float quotient(float x, float b, float y) {
  float q = x * y;
  q = __builtin_fmaf(__builtin_fmaf(-q, b, x), y, q);
  return __builtin_fmaf(__builtin_fmaf(-q, b, x), y, q);
}

// A row of d elements is held by a group of lanes, 8 elements each; scale: the group's largest finite magnitude / 448 by
// a correctly rounded division, as the codes are (a reciprocal would put some of them on the other side of a border).
// Bound by memory: every byte is moved once, 16 bytes a lane in, 4 to 32 out (16384 tokens of 8 heads of 128, keys and
// values: bf16 20.9 us, 6.4 TB/s; fp8 28.2 us, 3.6 TB/s: the arithmetic between a load and its store).
// Keys and values of a token and head are the same lanes' work, so that one's way to memory covers the other's arithmetic
// (each by lanes of its own: bf16 22.3 us, fp8 33.2).
template <int DDT>
__device__ __forceinline__ void write_eight(const AppendArgs& a, int arr, const Eight& e, int slot, int h, int part, long at) {
  const bool mine = part * 8 < a.d;
  if constexpr (DDT == 2) {
    float most = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float m = __builtin_fabsf(e.x[i]);
      most = m < __builtin_inff() && m > most ? m : most;
    }
    const auto other = [](auto permuted, float x) { return __uint_as_float(permuted(__float_as_uint(x))); };
    if (a.lanes > 1) most = fmaxf(most, other(dpp_perm<0xB1>, most));    // lane ^ 1
    if (a.lanes > 2) most = fmaxf(most, other(dpp_perm<0x4E>, most));    // lane ^ 2
    if (a.lanes > 4) most = fmaxf(most, other(dpp_perm<0x141>, most));   // 8 lanes mirrored: the other four
    if (a.lanes > 8) most = fmaxf(most, other(dpp_perm<0x140>, most));   // 16 lanes mirrored
    for (int x = 16; x < a.lanes; x <<= 1) most = fmaxf(most, __shfl_xor(most, x));
    float scale = most / 448.f;
    scale = most > 0.f ? fmaxf(scale, 1.17549435e-38f) : 1.f;
    if (part == 0) a.scale[arr][(long)slot * a.R + h] = scale;
    const float inverse = 1.f / scale;
    float y[8];
    if (scale < 0x1p-60f) {                  // (remainders would fall below the smallest number)
      asm volatile("");
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = e.x[i] / scale;
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = quotient(e.x[i], scale, inverse);
    }
    uint32_t w[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float z = fminf(fmaxf(y[i], -448.f), 448.f);
      const uint32_t one = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(z, z, 0, false) & 0xffu;
      w[i >> 2] |= (__builtin_fabsf(e.x[i]) < __builtin_inff() ? one : 0x7fu) << (8 * (i & 3));
    }
    if (mine) *reinterpret_cast<uint2*>((uint8_t*)a.dst[arr] + at) = make_uint2(w[0], w[1]);
  } else if constexpr (DDT == 1) {
    const uint4 w = make_uint4(bf16_pair(e.x[0], e.x[1]), bf16_pair(e.x[2], e.x[3]), bf16_pair(e.x[4], e.x[5]),
                               bf16_pair(e.x[6], e.x[7]));
    if (mine) *reinterpret_cast<uint4*>((uint16_t*)a.dst[arr] + at) = w;
  } else if (mine) {
    float4* out = reinterpret_cast<float4*>((float*)a.dst[arr] + at);
    out[0] = make_float4(e.x[0], e.x[1], e.x[2], e.x[3]);
    out[1] = make_float4(e.x[4], e.x[5], e.x[6], e.x[7]);
  }
}

template <int SDT, int DDT>
static __global__ __launch_bounds__(256) void k_cache_append(AppendArgs a) {
  const int per_wg = 256 / a.lanes, part = threadIdx.x & (a.lanes - 1);
  const uint32_t row = blockIdx.x * (uint32_t)per_wg + threadIdx.x / (uint32_t)a.lanes;   // (token, head)
  if (row >= (uint32_t)a.T * (uint32_t)a.R) return;                     // (below 2^30)
  const int t = (int)(row / (uint32_t)a.R), h = (int)(row - (uint32_t)t * (uint32_t)a.R);
  const int slot = a.slots[t];
  Eight e[2]{};
  if (part * 8 < a.d) {
    const long from = t * a.src_stride + (long)h * a.d + part * 8;
    e[0] = load_eight<SDT>(a.src[0], from);
    if (a.src[1]) e[1] = load_eight<SDT>(a.src[1], from);
  }
  if (slot < 0 || slot >= a.n_slots) return;
  const int p = slot / a.page, o = slot - p * a.page;
  const long at = p * a.page_stride + o * a.token_stride + h * a.head_stride + part * 8;
  write_eight<DDT>(a, 0, e[0], slot, h, part, at);
  if (a.src[1]) write_eight<DDT>(a, 1, e[1], slot, h, part, at);
}

}  // namespace hisa
