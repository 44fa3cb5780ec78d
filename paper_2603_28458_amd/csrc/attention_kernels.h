// Attention over a paged cache: of the new tokens of a batch over everything they see, and over a list of positions per
// query.  Softmax in one pass: a running maximum m, the sum l of exp2(x - m) and the weighted values, all in fp32, with
// x = log2(e) * scale * (q . k); parts of a row are joined by the same rule.
#pragma once

#include "hisa_device.h"

namespace hisa {

struct AttnArgs {
  const void* q;
  const int32_t* q_start;   // ranges: first token row of each sequence
  const int32_t* q_seq;     // lists: sequence of each query
  const int32_t* q_pos;
  const int32_t* q_lo;
  const int32_t* list;      // [T, n_list]
  const void* k;
  const void* v;
  const float* k_scale;
  const float* v_scale;
  const int32_t* table;
  const int32_t* seq_len;
  void* out;
  float* lse;
  float* part;              // [splits, T, H, d] weighted values, then [splits, T, H, 2] (m, l)
  long page_stride, token_stride, head_stride;
  float scale_log2;
  int T, H, H_kv, G, d, n_list;
  int n_pages, page_shift, n_seq, max_pages;
  int splits;
};

// Last n in [0, n_seq) with q_start[n] <= t; whether t is a row of it is the caller's to check.
__device__ __forceinline__ int seq_of_row(const int32_t* __restrict__ q_start, int n_seq, int t) {
  int lo = 0, hi = n_seq;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (q_start[mid] <= t) lo = mid;
    else hi = mid;
  }
  return lo;
}

__device__ __forceinline__ int clamp_len(const AttnArgs& a, int n) {
  const int len = a.seq_len[n];
  const long cap = (long)a.max_pages << a.page_shift;
  return len < 0 ? 0 : len < cap ? len : (int)cap;
}

// Slot of position s of sequence n (whose table row is given), or -1: its page is no page of the cache.
__device__ __forceinline__ long slot_of(const AttnArgs& a, const int32_t* __restrict__ table_row, int s) {
  const int id = table_row[s >> a.page_shift];
  return (uint32_t)id < (uint32_t)a.n_pages ? ((long)id << a.page_shift) + (s & ((1 << a.page_shift) - 1)) : -1;
}
__device__ __forceinline__ long row_of_slot(const AttnArgs& a, long slot) {
  return (slot >> a.page_shift) * a.page_stride + (slot & ((1 << a.page_shift) - 1)) * a.token_stride;
}

// Four elements at row + e, widened.
template <int DT>
__device__ __forceinline__ float4 load_four(const void* base, long at) {
  if constexpr (DT == 0) {
    return *reinterpret_cast<const float4*>((const float*)base + at);
  } else if constexpr (DT == 1) {
    const uint2 w = *reinterpret_cast<const uint2*>((const uint16_t*)base + at);
    return make_float4(__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xffff0000u), __uint_as_float(w.y << 16),
                       __uint_as_float(w.y & 0xffff0000u));
  } else {
    const int w = *reinterpret_cast<const int*>((const uint8_t*)base + at);
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
    return make_float4(lo[0], lo[1], hi[0], hi[1]);
  }
}

// One result row (or its part): o already holds the sum of the weighted values.
template <int QDT>
__device__ __forceinline__ void store_four(const AttnArgs& a, long row, int e, float4 o) {
  if constexpr (QDT == 0) {
    *reinterpret_cast<float4*>((float*)a.out + row * a.d + e) = o;
  } else {
    const bf16x2 lo = {(__bf16)o.x, (__bf16)o.y}, hi = {(__bf16)o.z, (__bf16)o.w};
    *reinterpret_cast<uint2*>((uint16_t*)a.out + row * a.d + e) =
        make_uint2(__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi));
  }
}

// The plain kernel: one query token, up to 8 heads of one KV head, one part of its keys per workgroup of 4 waves.  A
// wave takes every fourth tile of 64 keys: a key per lane for the scores, then 4 output columns per lane for the values.
constexpr int kPlainHeads = 8, kPlainMaxD = 256;

template <int QDT, int KDT, bool LIST>
static __global__ __launch_bounds__(256) void k_attn_plain(AttnArgs a) {
  __shared__ float qs[kPlainHeads][kPlainMaxD];
  __shared__ float ps[4][kPlainHeads][64];
  __shared__ long vrow[4][64];
  __shared__ float join_o[4][kPlainHeads][kPlainMaxD];
  __shared__ float join_ml[4][kPlainHeads][2];
  const int lane = lane_id(), wave = threadIdx.x >> 6;
  const int chunks = (a.G + kPlainHeads - 1) / kPlainHeads;
  long id = blockIdx.x;
  const int split = (int)(id % a.splits);
  id /= a.splits;
  const int chunk = (int)(id % chunks);
  id /= chunks;
  const int hk = (int)(id % a.H_kv), t = (int)(id / a.H_kv);
  const int h0 = hk * a.G + chunk * kPlainHeads;
  const int heads = a.G - chunk * kPlainHeads < kPlainHeads ? a.G - chunk * kPlainHeads : kPlainHeads;

  int n, begin = 0, end;
  if constexpr (LIST) {
    n = a.q_seq ? a.q_seq[t] : 0;
    end = (uint32_t)n < (uint32_t)a.n_seq ? a.n_list : 0;
    if (end == 0) n = 0;
  } else {
    n = seq_of_row(a.q_start, a.n_seq, t);
    if (t < a.q_start[n] || t >= a.q_start[n + 1]) return;       // nobody's row
    const int len = clamp_len(a, n);
    const int pos = a.q_pos ? a.q_pos[t] : a.seq_len[n] - a.q_start[n + 1] + t;
    end = pos < len ? pos + 1 : len;
    if (a.q_lo && a.q_lo[t] > 0) begin = a.q_lo[t];
  }
  const int len = clamp_len(a, n);
  const int32_t* __restrict__ row = a.table + (long)n * a.max_pages;
  if (a.splits > 1 && end > begin) {                              // this part: whole tiles of 64
    const long tiles = (end - (long)begin + 63) / 64;
    const int b0 = begin;
    begin = b0 + (int)(tiles * split / a.splits) * 64;
    const long stop = b0 + (tiles * (split + 1) / a.splits) * 64;
    end = stop < end ? (int)stop : end;
  }

  for (int i = threadIdx.x; i < heads * (a.d / 4); i += 256) {
    const int g = i / (a.d / 4), e = i % (a.d / 4) * 4;
    const float4 x = load_four<QDT>(a.q, ((long)t * a.H + h0 + g) * a.d + e);
    qs[g][e] = x.x * a.scale_log2;
    qs[g][e + 1] = x.y * a.scale_log2;
    qs[g][e + 2] = x.z * a.scale_log2;
    qs[g][e + 3] = x.w * a.scale_log2;
  }
  __syncthreads();

  float m[kPlainHeads], l[kPlainHeads];
  float4 o[kPlainHeads];
#pragma unroll
  for (int g = 0; g < kPlainHeads; ++g) {
    m[g] = neg_inf();
    l[g] = 0.f;
    o[g] = make_float4(0.f, 0.f, 0.f, 0.f);
  }
  const bool mine = lane * 4 < a.d;
  for (long tile = (long)begin + wave * 64; tile < end; tile += 256) {
    const int c = (int)tile + lane;
    long slot = -1;
    if (c < end) {
      const int s = LIST ? a.list[(long)t * a.n_list + c] : c;
      if (s >= 0 && s < len) slot = slot_of(a, row, s);
    }
    const long at = slot < 0 ? 0 : row_of_slot(a, slot) + hk * a.head_stride;
    float x[kPlainHeads];
#pragma unroll
    for (int g = 0; g < kPlainHeads; ++g) x[g] = 0.f;
    float vs = 1.f;
    if (slot >= 0) {
      for (int e = 0; e < a.d; e += 4) {
        const float4 kk = load_four<KDT>(a.k, at + e);
#pragma unroll
        for (int g = 0; g < kPlainHeads; ++g)
          x[g] = __builtin_fmaf(qs[g][e], kk.x,
                 __builtin_fmaf(qs[g][e + 1], kk.y, __builtin_fmaf(qs[g][e + 2], kk.z, __builtin_fmaf(qs[g][e + 3], kk.w, x[g]))));
      }
      if constexpr (KDT == 2) {
        const float ks = a.k_scale[slot * a.H_kv + hk];
        vs = a.v_scale[slot * a.H_kv + hk];
#pragma unroll
        for (int g = 0; g < kPlainHeads; ++g) x[g] *= ks;
      }
    }
    vrow[wave][lane] = slot < 0 ? -1 : at;
#pragma unroll
    for (int g = 0; g < kPlainHeads; ++g) {
      if (slot < 0) x[g] = neg_inf();
      float top = x[g];
      for (int s = 1; s < 64; s <<= 1) top = fmaxf(top, __shfl_xor(top, s));
      const float mn = fmaxf(m[g], top);
      const float base = mn == neg_inf() ? 0.f : mn;
      const float p = slot < 0 ? 0.f : __builtin_amdgcn_exp2f(x[g] - base);
      const float shrink = __builtin_amdgcn_exp2f(m[g] - base);
      float sum = p;
      for (int s = 1; s < 64; s <<= 1) sum += __shfl_xor(sum, s);
      l[g] = l[g] * shrink + sum;
      o[g].x *= shrink;
      o[g].y *= shrink;
      o[g].z *= shrink;
      o[g].w *= shrink;
      m[g] = mn;
      ps[wave][g][lane] = p * vs;
    }
    wave_lds_order();
    for (int j = 0; j < 64; ++j) {
      const long vat = vrow[wave][j];
      if (vat < 0 || !mine) continue;
      const float4 vv = load_four<KDT>(a.v, vat + lane * 4);
#pragma unroll
      for (int g = 0; g < kPlainHeads; ++g) {
        const float p = ps[wave][g][j];
        o[g].x = __builtin_fmaf(p, vv.x, o[g].x);
        o[g].y = __builtin_fmaf(p, vv.y, o[g].y);
        o[g].z = __builtin_fmaf(p, vv.z, o[g].z);
        o[g].w = __builtin_fmaf(p, vv.w, o[g].w);
      }
    }
    wave_lds_order();
  }
#pragma unroll
  for (int g = 0; g < kPlainHeads; ++g) {
    if (mine) *reinterpret_cast<float4*>(&join_o[wave][g][lane * 4]) = o[g];
    if (lane == 0) {
      join_ml[wave][g][0] = m[g];
      join_ml[wave][g][1] = l[g];
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < heads * (a.d / 4); i += 256) {
    const int g = i / (a.d / 4), e = i % (a.d / 4) * 4;
    float top = neg_inf();
    for (int w = 0; w < 4; ++w) top = fmaxf(top, join_ml[w][g][0]);
    const float base = top == neg_inf() ? 0.f : top;
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    float sum = 0.f;
    for (int w = 0; w < 4; ++w) {
      const float f = __builtin_amdgcn_exp2f(join_ml[w][g][0] - base);
      sum += f * join_ml[w][g][1];
      const float4 x = *reinterpret_cast<const float4*>(&join_o[w][g][e]);
      s.x = __builtin_fmaf(f, x.x, s.x);
      s.y = __builtin_fmaf(f, x.y, s.y);
      s.z = __builtin_fmaf(f, x.z, s.z);
      s.w = __builtin_fmaf(f, x.w, s.w);
    }
    const long r = (long)t * a.H + h0 + g;
    if (a.splits > 1) {
      const long pr = (long)split * a.T * a.H + r;
      *reinterpret_cast<float4*>(a.part + pr * a.d + e) = s;
      if (e == 0) {
        float* ml = a.part + (long)a.splits * a.T * a.H * a.d + pr * 2;
        ml[0] = top;
        ml[1] = sum;
      }
    } else {
      const float inv = sum == 0.f ? 0.f : 1.f / sum;
      store_four<QDT>(a, r, e, make_float4(s.x * inv, s.y * inv, s.z * inv, s.w * inv));
      if (e == 0 && a.lse) a.lse[r] = sum == 0.f ? neg_inf() : (base + log2f(sum)) * 0.693147180559945309f;
    }
  }
}

// Joins the parts of a row: 4 columns per lane, rows of a token in consecutive groups of lanes.
template <int QDT, bool LIST>
static __global__ __launch_bounds__(256) void k_attn_join(AttnArgs a) {
  const int per = a.d / 4;
  const long i = (long)blockIdx.x * 256 + threadIdx.x;
  const long r = i / per;
  const int e = (int)(i - r * per) * 4;
  if (r >= (long)a.T * a.H) return;
  if constexpr (!LIST) {
    const int t = (int)(r / a.H);
    if (t < a.q_start[0] || t >= a.q_start[a.n_seq]) return;
  }
  const float* ml = a.part + (long)a.splits * a.T * a.H * a.d;
  float top = neg_inf();
  for (int s = 0; s < a.splits; ++s) top = fmaxf(top, ml[((long)s * a.T * a.H + r) * 2]);
  const float base = top == neg_inf() ? 0.f : top;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  float sum = 0.f;
  for (int s = 0; s < a.splits; ++s) {
    const long pr = (long)s * a.T * a.H + r;
    const float l = ml[pr * 2 + 1];
    if (l == 0.f) continue;
    const float f = __builtin_amdgcn_exp2f(ml[pr * 2] - base);
    sum = __builtin_fmaf(f, l, sum);
    const float4 x = *reinterpret_cast<const float4*>(a.part + pr * a.d + e);
    o.x = __builtin_fmaf(f, x.x, o.x);
    o.y = __builtin_fmaf(f, x.y, o.y);
    o.z = __builtin_fmaf(f, x.z, o.z);
    o.w = __builtin_fmaf(f, x.w, o.w);
  }
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  store_four<QDT>(a, r, e, make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv));
  if (e == 0 && a.lse) a.lse[r] = sum == 0.f ? neg_inf() : (base + log2f(sum)) * 0.693147180559945309f;
}

}  // namespace hisa
