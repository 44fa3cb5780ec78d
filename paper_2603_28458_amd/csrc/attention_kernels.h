// Attention over a paged cache: of the new tokens of a batch over everything they see, and over a list of positions per
// query.  Softmax in one pass: a running maximum m, the sum l of exp2(x - m) and the weighted values, all in fp32, with
// x = log2(e) * scale * (q . k); parts of a row are joined by the same rule.
#pragma once

#include <utility>

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

// f(0), f(1), .. f(N - 1) with the number as a type: a loop that is written out whatever its size.
template <class F, int... I>
__device__ __forceinline__ void steps(F&& f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>{}), ...);
}

// Last n in [0, n_seq) for which `le(n)` holds (ascending: true up to it), by the whole wave, 64 candidates at a time; 0 if
// it holds for none.
template <class Le>
__device__ __forceinline__ int last_seq(int n_seq, Le le) {
  int lo = 0, hi = n_seq;
  while (hi - lo > 1) {
    const int step = (hi - lo + 63) / 64;
    const int n = lo + lane_id() * step;
    const uint64_t b = __builtin_amdgcn_ballot_w64(n < hi && le(n));
    lo += b ? (63 - __builtin_clzll(b)) * step : 0;
    hi = lo + step < hi ? lo + step : hi;
  }
  return lo;
}

__device__ __forceinline__ int clamp_len(const AttnArgs& a, int len) {
  const long cap = (long)a.max_pages << a.page_shift;
  return len < 0 ? 0 : len < cap ? len : (int)cap;
}

__device__ __forceinline__ float4 load_f32x4(const void* base, long at) {
  return *reinterpret_cast<const float4*>((const float*)base + at);
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

// ------------------------------------------------------------------------------------------
// Matrix-core path (bf16 queries, bf16 or fp8 rows, d = 64 or 128).  Everything is computed transposed, keys (then
// columns of the output) along the rows of the 32x32x16 MFMA and query rows along its columns: S^T = K Q^T, O^T = V^T P^T.
// A lane then holds 16 scores of ONE query row per 32 keys: the softmax needs one exchange between lanes l and l ^ 32 per
// tile, the row's maximum, sum and rescaling are per-lane numbers, and the weights are the second product's B operand as
// they stand (an MFMA takes the contraction index in any order as long as both operands use the same: slots 0..3 and 4..7
// of lane half h are keys 16 kk + 4 h + 0..3 and 16 kk + 8 + 4 h + 0..3, which is how the accumulator holds them).
// A query row is (token, head of the KV head's group), tokens outermost, so few tokens of a wide group fill a tile too.
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

// A tile of rows in LDS, bf16, D elements per row, in 16-byte chunks that are permuted inside each row so that the reads
// below meet no bank twice: keys are read 16 bytes per row by 32 consecutive rows, values 64 bytes of 4 consecutive rows
// per 32 lanes (the transposing read).  The permutations are exclusive ors, so a lane's address is one number of its own
// xor a constant of the step plus a constant: `read_key` and `read_value` are these numbers.
template <int D>
struct RowTile {
  static constexpr int kRowBytes = D * 2;
  __device__ static __forceinline__ int key_byte(int r, int c) {
    return r * kRowBytes + ((c ^ (D == 128 ? r & 15 : (r >> 1) & 7)) << 4);
  }
  __device__ static __forceinline__ int value_byte(int r, int c) {
    return r * kRowBytes + ((c ^ (D == 128 ? (r & 3) << 2 : ((r >> 1) & 1) << 2)) << 4);
  }
  __device__ static __forceinline__ int read_key() {
    const int lane = lane_id();
    return key_byte(lane & 31, lane >> 5);
  }
  __device__ static __forceinline__ int read_value() {
    const int lane = lane_id(), i = lane & 15;
    return value_byte(4 * (lane >> 5) + (i >> 2), ((lane >> 4) & 1) * 2 + ((i >> 1) & 1)) + (i & 1) * 8;
  }
  // A operand of the scores: key rows r0 .. r0 + 31 (r0 % 32 == 0), contraction step kk.
  __device__ static __forceinline__ bf16x8 key_operand(const unsigned char* tile, int read_key, int r0, int kk) {
    return as_bf16x8(*reinterpret_cast<const uint4*>(tile + (read_key ^ (kk << 5)) + r0 * kRowBytes));
  }
  // A operand of the output: columns 32 dt .. + 31, keys r0 .. r0 + 15 (r0 % 16 == 0) in the order of the weights' operand.
  __device__ static __forceinline__ bf16x8 value_operand(const unsigned char* tile, int read_value, int r0, int dt) {
    const unsigned char* p = tile + (read_value ^ (dt << 6)) + r0 * kRowBytes;
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)p);
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + 8 * kRowBytes));
    const s16x8 v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    return __builtin_bit_cast(bf16x8, v);
  }
};

// Keeps what is computed from x inside the loop where it is used: a lane's addresses of a tile's steps are cheaper
// computed again (one xor) than kept in a register each.
__device__ __forceinline__ int renewed(int x) {
  asm volatile("" : "+v"(x));
  return x;
}

// 16 stored bytes of a row as they go into a tile: bf16 as they are, fp8 widened (exactly) into two chunks.
__device__ __forceinline__ uint4 widen_fp8(uint32_t lo, uint32_t hi) {
  const uint2 a = fp8x4_to_bf16x4(lo), b = fp8x4_to_bf16x4(hi);
  return make_uint4(a.x, a.y, b.x, b.y);
}
template <int D, int KDT, bool VALUES>
__device__ __forceinline__ void store_chunk(unsigned char* tile, int r, int c, uint4 x) {
  using R = RowTile<D>;
  if constexpr (KDT == 2) {
    const uint4 a = widen_fp8(x.x, x.y), b = widen_fp8(x.z, x.w);
    *reinterpret_cast<uint4*>(tile + (VALUES ? R::value_byte(r, 2 * c) : R::key_byte(r, 2 * c))) = a;
    *reinterpret_cast<uint4*>(tile + (VALUES ? R::value_byte(r, 2 * c + 1) : R::key_byte(r, 2 * c + 1))) = b;
  } else {
    *reinterpret_cast<uint4*>(tile + (VALUES ? R::value_byte(r, c) : R::key_byte(r, c))) = x;
  }
}

__device__ __forceinline__ float max_halves(float x) {   // with lane ^ 32
  const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __builtin_elementwise_maximum(__uint_as_float(sw[0]), __uint_as_float(sw[1]));
}
__device__ __forceinline__ float add_halves(float x) {
  const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
}

// 32 query rows of a wave.
template <int D>
struct RowState {
  bf16x8 q[D / 16];      // B operand of the scores: row lane % 32
  f32x16 o[D / 32];      // O^T: column = row lane % 32, register i of tile dt = output column 32 dt + 8 (i/4) + 4 half + i%4
  float m, l;            // running maximum (x = scale_log2 * score) and this lane half's share of the sum
  int pos, lo;           // what the row sees

  __device__ __forceinline__ void clear() {
    m = neg_inf();
    l = 0.f;
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[dt][i] = 0.f;
  }
  __device__ __forceinline__ void load_q(const uint16_t* __restrict__ row) {
    const int half = lane_id() >> 5;
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) q[kk] = as_bf16x8(*reinterpret_cast<const uint4*>(row + kk * 16 + half * 8));
  }
};

// How far a row's maximum may grow before its sums are rescaled: weights stay below 2^8, far inside what fp32 sums and
// bf16 weights (whose precision is relative) hold, and most tiles need no pass over the accumulators.
constexpr float kSlack = 8.f;

// Hides the scores of the keys of a block of 32 whose bits are clear.
__device__ __forceinline__ void hide_keys(f32x16& s, uint32_t keys) {
  const uint32_t mine = keys >> (4 * (lane_id() >> 5));
#pragma unroll
  for (int i = 0; i < 16; ++i)
    if (!(mine >> (8 * (i >> 2) + (i & 3)) & 1u)) s[i] = neg_inf();
}

// The same for a block that begins at `base`, where rows see different keys: key r counts where bit r of `keys` is set and the row
// sees it.
template <int D>
__device__ __forceinline__ void hide(const RowState<D>& st, f32x16& s, uint32_t keys, int base) {
  const int half4 = 4 * (lane_id() >> 5);
  const uint32_t mine = keys >> half4;
  const int last = st.pos - base - half4, first = st.lo - base - half4;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int r = 8 * (i >> 2) + (i & 3);
    if (!(mine >> r & 1u) || r > last || r < first) s[i] = neg_inf();
  }
}

template <int NB>
__device__ __forceinline__ void scale_scores(f32x16 (&s)[NB], const float* ks) {   // fp8: the rows' scales
  const int half = lane_id() >> 5;
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float4 f = *reinterpret_cast<const float4*>(ks + b * 32 + 8 * j + 4 * half);
      s[b][4 * j] *= f.x;
      s[b][4 * j + 1] *= f.y;
      s[b][4 * j + 2] *= f.z;
      s[b][4 * j + 3] *= f.w;
    }
}

// Scores of NB blocks of 32 keys -> weights as B operands; updates m, l, o.  vs: scales of the value rows (fp8).
// A weight rounded to bf16 is off by up to 2^-8 of itself (1.6e-3 in the mean square), and so are the sums: as much as the
// result's own rounding adds, and more where few rows leave it no chance to average out (7 rows up to 1.7 times, 1024 rows
// 1.45).  A caller may choose that.  REST, which is what one gets otherwise: what is left of each weight goes to `rest`, for a
// second product of the values, with which the sums are as good as with weights in fp32 (to 2^-15).  It is cut and not rounded off, so that both parts have
// one sign, and never 0 where there is a weight: an infinite value stays what it is in both products.
__device__ __forceinline__ float cut_off(float w, uint32_t bits) {
  return __builtin_amdgcn_fmed3f(w - __uint_as_float(bits & 0xffff0000u), w, 1.17549435e-38f);
}
template <int D, int KDT, int NB, bool REST>
__device__ __forceinline__ void softmax_tile(RowState<D>& st, const f32x16 (&s)[NB], bf16x8 (&p)[2 * NB],
                                             bf16x8 (&rest)[2 * NB], float c, const float* vs) {
  const int half = lane_id() >> 5;
  // (the IEEE 754-2019 maximum: three operands an instruction, none of them quieted first as fmaxf's are; a NaN comes
  // through it, leaves m as it is and makes the row's sum NaN below)
  float top4[4];
#pragma unroll
  for (int x = 0; x < 4; ++x) {
    top4[x] = __builtin_elementwise_maximum(s[0][4 * x], s[0][4 * x + 1]);
    top4[x] = __builtin_elementwise_maximum(__builtin_elementwise_maximum(top4[x], s[0][4 * x + 2]), s[0][4 * x + 3]);
#pragma unroll
    for (int b = 1; b < NB; ++b) {
      top4[x] = __builtin_elementwise_maximum(__builtin_elementwise_maximum(top4[x], s[b][4 * x]), s[b][4 * x + 1]);
      top4[x] = __builtin_elementwise_maximum(__builtin_elementwise_maximum(top4[x], s[b][4 * x + 2]), s[b][4 * x + 3]);
    }
  }
  float top = __builtin_elementwise_maximum(__builtin_elementwise_maximum(top4[0], top4[1]), top4[2]);
  top = max_halves(__builtin_elementwise_maximum(top, top4[3])) * c;
  const bool grown = top > st.m + kSlack;
  if (__builtin_amdgcn_ballot_w64(grown)) {
    const float mn = grown ? top : st.m;     // (a row goes by its own scores, not by its neighbours')
    const float f = __builtin_amdgcn_exp2f(st.m - (mn == neg_inf() ? 0.f : mn));
    st.m = mn;
    st.l *= f;
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
      for (int i = 0; i < 16; ++i) st.o[dt][i] *= f;
  }
  const float off = st.m == neg_inf() ? 0.f : -st.m;
  float sum0 = 0.f, sum1 = 0.f;
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float w[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][4 * j + e], c, off));
      sum0 += w[0] + w[1];
      sum1 += w[2] + w[3];
      if constexpr (KDT == 2) {
        const float4 f = *reinterpret_cast<const float4*>(vs + b * 32 + 8 * j + 4 * half);
        w[0] *= f.x;
        w[1] *= f.y;
        w[2] *= f.z;
        w[3] *= f.w;
      }
#pragma unroll
      for (int e = 0; e < 4; e += 2) {
        const int at = 4 * (j & 1) + e;
        bf16x2 first = {(__bf16)w[e], (__bf16)w[e + 1]};
        if constexpr (REST) {
          const uint32_t x = __float_as_uint(w[e]), y = __float_as_uint(w[e + 1]);
          first = __builtin_bit_cast(bf16x2, (y & 0xffff0000u) | x >> 16);
          rest[2 * b + (j >> 1)][at] = (__bf16)cut_off(w[e], x);
          rest[2 * b + (j >> 1)][at + 1] = (__bf16)cut_off(w[e + 1], y);
        }
        p[2 * b + (j >> 1)][at] = first[0];
        p[2 * b + (j >> 1)][at + 1] = first[1];
      }
    }
  st.l += sum0 + sum1;
}

// O^T += V^T P^T over 32 keys.
template <int D, bool REST>
__device__ __forceinline__ void add_values(RowState<D>& st, const unsigned char* tile, int read_value, const bf16x8 (&p)[2],
                                           const bf16x8 (&rest)[2]) {
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      const bf16x8 v = RowTile<D>::value_operand(tile, read_value, 16 * kk, dt);
      st.o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, p[kk], st.o[dt], 0, 0, 0);
      if constexpr (REST) st.o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, rest[kk], st.o[dt], 0, 0, 0);
    }
}

// A value (or, fp8, its row's scale) that is infinite or NaN must not reach the rows that do not see it, and 0 * inf
// would.  Where some rows of a workgroup see less of a tile than others, such values go into the tile as zeros, and
// afterwards to the rows that see them (add_odd_values): rare enough to read the rows again.
__device__ __forceinline__ uint32_t odd_bf16(uint32_t w) {   // 0xffff over each bf16 that is inf or NaN
  return ((((w & 0x7fff7fffu) + 0x00800080u) & 0x80008000u) >> 15) * 0xffffu;
}
__device__ __forceinline__ uint32_t odd_fp8(uint32_t w) {    // 0xff over each code that is NaN
  return ((((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) >> 7) * 0xffu;
}
template <int KDT>
__device__ __forceinline__ bool drop_odd(uint4& x) {
  const uint4 odd = KDT == 2 ? make_uint4(odd_fp8(x.x), odd_fp8(x.y), odd_fp8(x.z), odd_fp8(x.w))
                             : make_uint4(odd_bf16(x.x), odd_bf16(x.y), odd_bf16(x.z), odd_bf16(x.w));
  x = make_uint4(x.x & ~odd.x, x.y & ~odd.y, x.z & ~odd.z, x.w & ~odd.w);
  return (odd.x | odd.y | odd.z | odd.w) != 0;
}

// The infinities and NaN among the values of the 64 positions from `base` on, added to the rows that see them (whatever
// their weight: it is not 0 in exact arithmetic).  offsets (bytes behind vbase, -1: none), slots: where the rows lie.
template <int D, int KDT>
__device__ __forceinline__ void add_odd_values(RowState<D>& st, const unsigned char* __restrict__ vbase, const long* offsets,
                                               const int* slots, const float* __restrict__ v_scale, int H_kv, int base) {
  const int half = lane_id() >> 5;
#pragma unroll 1
  for (int key = 0; key < 64; ++key) {
    const bool sees = base + key >= st.lo && base + key <= st.pos && offsets[key] >= 0;
    if (!__builtin_amdgcn_ballot_w64(sees)) continue;
    const unsigned char* row = vbase + offsets[key];
    const float scale = KDT == 2 ? v_scale[(long)slots[key] * H_kv] : 1.f;
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int e = dt * 32 + 8 * j + 4 * half;
        uint2 w;
        if constexpr (KDT == 2) w = fp8x4_to_bf16x4(*reinterpret_cast<const uint32_t*>(row + e));
        else w = *reinterpret_cast<const uint2*>(row + 2 * e);
        const float v[4] = {__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xffff0000u), __uint_as_float(w.y << 16),
                            __uint_as_float(w.y & 0xffff0000u)};
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const float y = KDT == 2 ? v[x] * scale : v[x];
          if (sees && !(__builtin_fabsf(y) < __builtin_inff())) st.o[dt][4 * j + x] += y;
        }
        __builtin_amdgcn_sched_barrier(0);
      }
  }
}

template <int D, int NB>
__device__ __forceinline__ void score_tile(const RowState<D>& st, const unsigned char* tile, int read_key, f32x16 (&s)[NB]) {
#pragma unroll
  for (int b = 0; b < NB; ++b) {
#pragma unroll
    for (int i = 0; i < 16; ++i) s[b][i] = 0.f;
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk)
      s[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(RowTile<D>::key_operand(tile, read_key, 32 * b, kk), st.q[kk], s[b], 0, 0, 0);
  }
}

// Scores of one tile of 64 keys and values of the one before, as one stream of D / 4 products.  The operands of the next
// eight are under way from LDS while one is multiplied: the order is pinned, because the compiler's own asks for four at
// most and the matrix unit then waits for LDS after every second product.  Consecutive products have different
// accumulators.
template <int D, bool REST, class Between>
__device__ __forceinline__ void products(RowState<D>& st, const unsigned char* kt, int read_key, f32x16 (&s)[2],
                                         const unsigned char* vt, int read_value, const bf16x8 (&p)[4],
                                         const bf16x8 (&rest)[4], Between between) {
  constexpr int kAhead = 6, kScores = D / 8, kTiles = D / 32;
  bf16x8 f[kAhead];
  auto operand = [&](int i) {
    return i < kScores ? RowTile<D>::key_operand(kt, read_key, 32 * (i & 1), i >> 1)
                       : RowTile<D>::value_operand(vt, read_value, 16 * ((i - kScores) / kTiles), (i - kScores) % kTiles);
  };
#pragma unroll
  for (int i = 0; i < kAhead; ++i) f[i] = operand(i);
#pragma unroll
  for (int i = 0; i < 2 * kScores; ++i) {
    const bf16x8 x = f[i % kAhead];
    if (i < kScores) {
      f32x16 c = s[i & 1];
      if (i < 2) {
#pragma unroll
        for (int e = 0; e < 16; ++e) c[e] = 0.f;
      }
      s[i & 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, st.q[i >> 1], c, 0, 0, 0);
    } else {
      const int j = i - kScores;
      st.o[j % kTiles] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, p[j / kTiles], st.o[j % kTiles], 0, 0, 0);
      if constexpr (REST)
        st.o[j % kTiles] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, rest[j / kTiles], st.o[j % kTiles], 0, 0, 0);
    }
    if (i + kAhead < 2 * kScores) f[i % kAhead] = operand(i + kAhead);
    between(i);
    __builtin_amdgcn_sched_barrier(0);
  }
}

// The workgroup's number such that the KV heads of the same keys follow each other on one XCD (workgroups go round the 8 of
// them): of fp8 rows 64 bytes are half a cache line, and one line holds the scales of 32 rows and heads.  64 sequences of
// 8000, 4 KV heads, fp8: d = 64 53 us, without 89; d = 128 123 and 117, 24 of 16000 and 8 heads 181 and 186, 200 of 500 23.4 and
// 24.1.  Rows of bf16 are whole lines and go the other way: 24 of 16000 272 and 265.
__device__ __forceinline__ uint32_t heads_together(const AttnArgs& a) {
  const uint32_t H = (uint32_t)a.H_kv, group = 8 * H, b = blockIdx.x, first = b - b % group;
  if (first + group > gridDim.x) return b;
  const uint32_t in = b - first;
  return first + (in & 7) * H + (in >> 3);
}

// What a query token sees of sequence n (ranges): clamped to the sequence, so that nothing behind it is read.
struct Seen {
  int lo, pos;
};
__device__ __forceinline__ Seen seen_by(const AttnArgs& a, int n, int len, int t, int t_end) {
  Seen s;
  const int pos = a.q_pos ? a.q_pos[t] : a.seq_len[n] - t_end + t;
  const int lo = a.q_lo ? a.q_lo[t] : 0;
  s.pos = pos < -1 ? -1 : pos < len ? pos : len - 1;     // (differences of positions fit 32 bits)
  s.lo = lo > 0 ? lo : 0;
  return s;
}
__device__ __forceinline__ int wave_max_int(int x) {
  return __builtin_amdgcn_readfirstlane((int)(wave_max((uint32_t)x ^ 0x80000000u) ^ 0x80000000u));
}
__device__ __forceinline__ int wave_min_int(int x) {
  return __builtin_amdgcn_readfirstlane((int)(wave_min((uint32_t)x ^ 0x80000000u) ^ 0x80000000u));
}

// A barrier of the workgroup that orders LDS alone: __syncthreads would also wait for every global load under way.
__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// The row tile `unit` of rows_per tile rows: sequence and first row in it, or -1.  Tiles are numbered so that sequence n
// begins at floor(q_start[n] * G / rows_per) + n: at most one number per sequence stays unused, and the grid needs T,
// n_seq and G alone.
struct RowUnit {
  int n, t_begin, t_end;   // sequence and its token rows
  int r0;                  // first row (token, head) of the tile, in the sequence
};
template <int ROWS>
__device__ __forceinline__ RowUnit find_unit(const AttnArgs& a, int unit) {
  const int lo = last_seq(a.n_seq, [&](int i) { return (long)a.q_start[i] * a.G / ROWS + i <= unit; });
  RowUnit u;
  u.n = lo;
  u.t_begin = a.q_start[lo];
  u.t_end = a.q_start[lo + 1];
  u.r0 = (unit - (int)((long)u.t_begin * a.G / ROWS + lo)) * ROWS;
  return u;
}

// Part `split` of the tiles begin .. end: consecutive runs of equal length, `least` tiles at least, so that the last parts
// of a short sequence are empty.
__device__ __forceinline__ void take_part(int& begin, int& end, int split, int splits, int least) {
  const uint32_t n = (uint32_t)(end - begin), share = (n + (uint32_t)splits - 1) / (uint32_t)splits;
  const uint32_t per = share < (uint32_t)least ? (uint32_t)least : share;
  const uint64_t first = (uint64_t)per * (uint32_t)split;
  const int e = end;
  begin = first < n ? begin + (int)first : e;
  end = e - begin > (int)per ? begin + (int)per : e;
}

// One result row: 4 columns at e of (t, h) row r, sums with maximum m and weight sum l.
template <int QDT, bool PART>
__device__ __forceinline__ void store_result(const AttnArgs& a, int split, long r, int D, int e, float4 o, float m, float l) {
  if constexpr (PART) {
    const long pr = (long)split * a.T * a.H + r;
    *reinterpret_cast<float4*>(a.part + pr * D + e) = o;
    if (e == 0) {
      float* ml = a.part + (long)a.splits * a.T * a.H * D + pr * 2;
      ml[0] = m;
      ml[1] = l;
    }
  } else {
    const float inv = l == 0.f ? 0.f : 1.f / l;
    store_four<QDT>(a, r, e, make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv));
    if (e == 0 && a.lse) a.lse[r] = l == 0.f ? neg_inf() : (m + log2f(l)) * 0.693147180559945309f;
  }
}

// ---- fp32 queries and rows ---------------------------------------------------------------------
// The same transposed products on the 32x32x2 fp32 MFMA (exact products, fp32 sums).  A workgroup takes 32 query rows of
// one KV head (tokens of one sequence times heads; lists: heads of one token) and a part of their keys; each of 4 waves
// works alone on every fourth tile of 32 keys, and the waves' results are joined at the end.  Operands come straight from
// memory: of a key row lane half h reads elements 8 kk + 4 h + 0..3 and spends them on four products (a contraction may
// take its index in any order), a value row is read 32 columns at a time by 32 lanes.  As the keys of a tile are used up the
// values take their registers, and the next keys theirs: each is under way for as long as the other is multiplied.  The
// scores' accumulator holds keys 8 j + 4 half + x in register 4 j + x, so product 4 j + x of the values takes those two keys
// and that register as it is.
// Bound by memory where a KV head's group is small (8 D bytes per key), by the fp32 matrix units where 32 rows are real.
// Measured, d = 128, 64 heads on 8: 32 tokens over 16384 keys each 0.80 ms, 4.7 TB/s; 800 over 3000 0.66 ms, 94 TFLOP/s.
constexpr int kF32MaxD = 256;

template <int D>
struct F32Geom {
  static constexpr int kQ = D * 128;                          // [D / 8][64] of 16 bytes
  static constexpr int kLoop = kQ + 4 * 256, kJoin = D * 512; // and row offsets [4][32]; or [4][D][32] to join
  static constexpr int kMl = kLoop > kJoin ? kLoop : kJoin, kLds = kMl + 4 * 256;
};

template <int D, bool LIST>
static __global__ __launch_bounds__(256, D > 128 ? 1 : 2) void k_attn_f32(AttnArgs a) {
  using Geo = F32Geom<D>;
  constexpr int kSteps = D / 8, kCols = D / 32;
  constexpr int kKeep = kSteps < 16 ? kSteps : 16, kRows = D > 128 ? 8 : 16;   // key steps, value rows in registers
  constexpr bool kPart = D == kF32MaxD;                       // rows may be shorter than D
  extern __shared__ __align__(16) unsigned char lds[];
  const int lane = lane_id(), half = lane >> 5, col = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  float4* qs = reinterpret_cast<float4*>(lds);
  long* row_at = reinterpret_cast<long*>(lds + Geo::kQ) + wave * 32;
  float* join = reinterpret_cast<float*>(lds + Geo::kMl);     // [wave][32][2]

  uint32_t id = blockIdx.x;
  const int hk = (int)(id % (uint32_t)a.H_kv);
  id /= (uint32_t)a.H_kv;
  const int split = (int)(id % (uint32_t)a.splits), unit = (int)(id / (uint32_t)a.splits);
  int n, len, r0, rows, t_begin, begin, end;                  // tiles of 32 keys (list entries)
  int t_end = 0;
  if constexpr (LIST) {
    const int head_tiles = (a.G + 31) / 32;
    t_begin = unit / head_tiles;
    r0 = (unit - t_begin * head_tiles) * 32;
    rows = a.G;
    n = a.q_seq ? a.q_seq[t_begin] : 0;
    const bool none = (uint32_t)n >= (uint32_t)a.n_seq;
    n = none ? 0 : n;
    len = none ? 0 : clamp_len(a, a.seq_len[n]);
    begin = 0;
    end = (a.n_list + 31) / 32;
  } else {
    const RowUnit u = find_unit<32>(a, unit);
    n = u.n;
    t_begin = u.t_begin;
    t_end = u.t_end;
    r0 = u.r0;
    rows = (t_end - t_begin) * a.G;
    if (r0 < 0 || r0 >= rows || t_begin < 0 || t_end > a.T) return;
    len = clamp_len(a, a.seq_len[n]);
  }
  int qr = r0 + col;
  const bool mine = qr < rows;
  if (!mine) qr = rows - 1;                                   // (columns beyond the last row repeat it and are not stored)
  const int t = t_begin + qr / a.G;
  const long row = (long)t * a.H + hk * a.G + qr % a.G;
  Seen seen{0, 0x7fffffff};
  int pos_min = 0x7fffffff, lo_max = 0, pos_max = 0x7fffffff, lo_min = 0;
  if constexpr (!LIST) {
    seen = seen_by(a, n, len, t, t_end);
    pos_min = wave_min_int(seen.pos);
    pos_max = wave_max_int(seen.pos);
    lo_min = wave_min_int(seen.lo);
    lo_max = wave_max_int(seen.lo);
    begin = lo_min >> 5;
    end = (pos_max >> 5) + 1;                                 // (a position may be the last one below 2^31)
    if (pos_max < 0 || end < begin) end = begin;
  }
  if (a.splits > 1) take_part(begin, end, split, a.splits, 4);   // of at least one tile per wave

  for (int kk = wave; kk < kSteps; kk += 4) {
    const int e = kk * 8 + half * 4;
    qs[kk * 64 + lane] = !kPart || e < a.d ? load_f32x4(a.q, row * a.d + e) : make_float4(0.f, 0.f, 0.f, 0.f);
  }

  const int32_t* __restrict__ table = a.table + (long)n * a.max_pages;
  const int cap_last = (int)(((long)a.max_pages << a.page_shift) - 1);
  auto position = [&](int tile) {            // of key `col` of a tile (or one that is no position)
    if (tile >= end) return -1;
    const int c = tile * 32 + col;
    if constexpr (LIST) return c < a.n_list ? a.list[(long)t * a.n_list + c] : -1;
    else return c;
  };
  auto page_of = [&](int s) {
    const int in = s < 0 ? 0 : s > cap_last ? cap_last : s;
    return table[in >> a.page_shift];
  };
  uint32_t valid;                            // keys of the tile that there are
  long at;                                   // of key `col` (a row that is none: the pool's first, read and cleared)
  auto locate = [&](int s, int page) {
    const bool ok = (LIST ? s >= 0 && s < len : s >= lo_min && s <= pos_max) && (uint32_t)page < (uint32_t)a.n_pages;
    valid = (uint32_t)__builtin_amdgcn_ballot_w64(ok);
    at = ok ? page * a.page_stride + (s & ((1 << a.page_shift) - 1)) * a.token_stride : 0;
  };
  const float* __restrict__ kbase = (const float*)a.k + hk * a.head_stride + half * 4;
  const float* __restrict__ vbase = (const float*)a.v + hk * a.head_stride;
  float4 kx[kKeep];
  float vx[kRows][kCols];
  auto request_key = [&](int kk) {
    kx[kk % kKeep] = load_f32x4(kbase, at + (kPart && kk * 8 + half * 4 >= a.d ? -half * 4 : kk * 8));   // (beyond a row: not used)
  };
  auto key_of = [&](int i) { return 8 * (i >> 2) + 4 * half + (i & 3); };   // of register i
  auto request_value = [&](int i) {
    const float* v = vbase + row_at[key_of(i)];
#pragma unroll
    for (int dt = 0; dt < kCols; ++dt) vx[i % kRows][dt] = v[kPart && dt * 32 + col >= a.d ? 0 : dt * 32 + col];
  };
  auto leave_rows = [&]() {                  // for request_value
    wave_lds_order();
    if (half == 0) row_at[col] = at;
    wave_lds_order();
  };

  int tile = begin + wave;
  int s_next = position(tile + 4), s_after = position(tile + 8);
  {
    const int s = position(tile), page = page_of(s);
    locate(s, page);
  }
  int p_next = page_of(s_next);
#pragma unroll
  for (int kk = 0; kk < kKeep; ++kk) request_key(kk);
  leave_rows();
  float m = neg_inf(), l = 0.f;
  f32x16 o[kCols];
#pragma unroll
  for (int dt = 0; dt < kCols; ++dt)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[dt][i] = 0.f;
  __syncthreads();                           // (the queries)
  for (; tile < end; tile += 4) {
    const int base = tile * 32;
    const uint32_t keys = valid;
    const bool mixed = !LIST && (base + 31 > pos_min || base < lo_max);
    f32x16 s;
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
    for (int kk = 0; kk < kSteps; ++kk) {
      const float4 q = qs[kk * 64 + lane];
      float4 k = kx[kk % kKeep];
      if (kPart && kk * 8 + half * 4 >= a.d) k = make_float4(0.f, 0.f, 0.f, 0.f);
      s = __builtin_amdgcn_mfma_f32_32x32x2f32(k.x, q.x, s, 0, 0, 0);
      s = __builtin_amdgcn_mfma_f32_32x32x2f32(k.y, q.y, s, 0, 0, 0);
      s = __builtin_amdgcn_mfma_f32_32x32x2f32(k.z, q.z, s, 0, 0, 0);
      s = __builtin_amdgcn_mfma_f32_32x32x2f32(k.w, q.w, s, 0, 0, 0);
      if (kk + kKeep < kSteps) request_key(kk + kKeep);
      const int f = kk + kKeep - kSteps;
#pragma unroll
      for (int i = f < 0 ? 0 : f * kRows / kKeep; i < (f + 1) * kRows / kKeep; ++i) request_value(i);
      __builtin_amdgcn_sched_barrier(0);
    }
    locate(s_next, p_next);
    s_next = s_after;
    p_next = page_of(s_next);
    s_after = position(tile + 12);

    float top = neg_inf();
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int key = key_of(i);
      const bool in = (keys >> key & 1u) && (LIST || (base + key >= seen.lo && base + key <= seen.pos));
      s[i] = in ? s[i] * a.scale_log2 : neg_inf();
      top = __builtin_elementwise_maximum(top, s[i]);
    }
    top = max_halves(top);
    const bool grown = top > m + kSlack;
    if (__builtin_amdgcn_ballot_w64(grown)) {
      const float mn = grown ? top : m;
      const float f = __builtin_amdgcn_exp2f(m - (mn == neg_inf() ? 0.f : mn));
      m = mn;
      l *= f;
#pragma unroll
      for (int dt = 0; dt < kCols; ++dt)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[dt][i] *= f;
    }
    const float off = m == neg_inf() ? 0.f : m;
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      s[i] = __builtin_amdgcn_exp2f(s[i] - off);
      sum += s[i];
    }
    l += sum;

    const bool clean = keys != 0xffffffffu || mixed;
    bool odd = false;                        // (as in the tiles of bf16: what some rows must not meet is added apart)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      float (&v)[kCols] = vx[i % kRows];
      if (clean) {
        const bool there = keys >> key_of(i) & 1u;
#pragma unroll
        for (int dt = 0; dt < kCols; ++dt) {
          const bool bad = mixed && !(__builtin_fabsf(v[dt]) < __builtin_inff());
          odd |= there && bad;
          if (!there || bad) v[dt] = 0.f;
        }
      }
#pragma unroll
      for (int dt = 0; dt < kCols; ++dt) o[dt] = __builtin_amdgcn_mfma_f32_32x32x2f32(v[dt], s[i], o[dt], 0, 0, 0);
      if (i + kRows < 16) request_value(i + kRows);
      const int f = i + kRows - 16;
#pragma unroll
      for (int kk = f < 0 ? 0 : f * kKeep / kRows; kk < (f + 1) * kKeep / kRows; ++kk) request_key(kk);
      __builtin_amdgcn_sched_barrier(0);
    }
    if (__builtin_amdgcn_ballot_w64(odd)) {
      for (int key = 0; key < 32; ++key) {
        const bool in = (keys >> key & 1u) && base + key >= seen.lo && base + key <= seen.pos;
        const float* v = vbase + row_at[key];
#pragma unroll
        for (int dt = 0; dt < kCols; ++dt)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int e = dt * 32 + 8 * j + 4 * half;
            if (kPart && e >= a.d) continue;
            const float4 x = *reinterpret_cast<const float4*>(v + e);
            const float y[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
            for (int c = 0; c < 4; ++c)
              if (in && !(__builtin_fabsf(y[c]) < __builtin_inff())) o[dt][4 * j + c] += y[c];
          }
      }
    }
    leave_rows();
  }

  l = add_halves(l);
  if (half == 0) {
    join[(wave * 32 + col) * 2] = m;
    join[(wave * 32 + col) * 2 + 1] = l;
  }
  __syncthreads();
  float top = neg_inf(), sum = 0.f;
#pragma unroll
  for (int w = 0; w < 4; ++w) top = fmaxf(top, join[(w * 32 + col) * 2]);
  const float base = top == neg_inf() ? 0.f : top;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const float* ml = join + (w * 32 + col) * 2;
    sum = __builtin_fmaf(__builtin_amdgcn_exp2f(ml[0] - base), ml[1], sum);
  }
  float* part = reinterpret_cast<float*>(lds);                // [wave][D][32]
  const float f = __builtin_amdgcn_exp2f(m - base);
#pragma unroll
  for (int dt = 0; dt < kCols; ++dt)
#pragma unroll
    for (int i = 0; i < 16; ++i) part[(wave * D + dt * 32 + key_of(i)) * 32 + col] = o[dt][i] * f;
  __syncthreads();
  if (!mine) return;
  for (int e = (threadIdx.x >> 5) * 4; e < a.d; e += 32) {
    float y[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      y[c] = 0.f;
#pragma unroll
      for (int w = 0; w < 4; ++w) y[c] += part[(w * D + e + c) * 32 + col];
    }
    const float4 x = make_float4(y[0], y[1], y[2], y[3]);
    if (a.splits > 1) store_result<0, true>(a, split, row, a.d, e, x, top, sum);
    else store_result<0, false>(a, split, row, a.d, e, x, top, sum);
  }
}

// ---- one token at a time, over a range or a list: keys split over the waves -----------------------
// A workgroup takes one token, up to 32 heads of one KV head's group (64: PAIR) and a part of the keys.  Each of 4 waves
// works alone on its own tiles of 32 keys (every fourth): later tiles' rows are on their way into registers while the
// present one, in the wave's own LDS, is multiplied; the waves' results are joined at the end.  With PAIR a wave has a
// second one beside it on its SIMD: one brings the keys of their tile, the other the values, and each multiplies 32 of the
// heads, so that wider groups gather every row once and still leave each SIMD two waves.  All rows see the same keys, so a
// row outside is a row of zeros and a score of -inf for everybody.  Bound by memory: 4 D bytes (bf16) per key and KV head,
// whatever the number of heads.  Measured, d = 128: one token of 32 sequences of up to 131072, 64 heads on 8 KV heads, 2.54
// ms, 5.9 TB/s; of 200 short ones, 4 KV heads, fp8, 0.45 ms, 5.0 TB/s (a workgroup there is a quarter start and end); 1024
// lists of 2048, 64 heads on one KV head, 157 us (6.8 TB/s gathered, from L2 for the most part; weights of 8 bits 137).
constexpr int kRowWaves = 4;

template <int D, int KDT, bool PAIR>
struct RowGeom {
  static constexpr int kCpr = D * (KDT == 2 ? 1 : 2) / 16;   // stored 16-byte chunks of a row
  static constexpr int kRpi = 64 / kCpr;                     // rows per load instruction
  static constexpr int kNi = 32 / kRpi;                      // load instructions per 32 rows
  static constexpr int kLoads = PAIR ? kNi : 2 * kNi;        // of a wave per tile
  static constexpr int kDepth = PAIR || KDT == 2 || D == 64 ? 2 : 1;   // tiles under way: two where the registers allow it
  static constexpr int kTile = 32 * D * 2;                   // LDS bytes of 32 keys, or values
  static constexpr int kStage = 2 * kTile + (KDT == 2 ? 256 : 0);
  static constexpr int kStages = PAIR ? 2 : 1;
  static constexpr int kWaves = PAIR ? 2 * kRowWaves : kRowWaves;
  // rings, then per wave 32 row offsets, then per wave (m, l) of 32 rows
  static constexpr int kOffsets = kRowWaves * kStages * kStage, kJoin = kOffsets + kWaves * 256;
  static constexpr int kLds = kJoin + kWaves * 256;
};

template <int D, int KDT, bool PAIR, bool LIST, bool REST>
static __global__ __launch_bounds__(PAIR ? 512 : 256, 2) void k_attn_rows(AttnArgs a) {
  using Geo = RowGeom<D, KDT, PAIR>;
  extern __shared__ __align__(16) unsigned char lds[];
  const int lane = lane_id(), half = lane >> 5, col = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lead = wave & 3, second = PAIR ? wave >> 2 : 0;
  unsigned char* ring = lds + lead * Geo::kStages * Geo::kStage;
  long* row_at = reinterpret_cast<long*>(lds + Geo::kOffsets) + wave * 32;
  float* join = reinterpret_cast<float*>(lds + Geo::kJoin);                    // [wave][32][2]

  uint32_t id = KDT == 2 ? heads_together(a) : blockIdx.x;
  const int hk = (int)(id % (uint32_t)a.H_kv);
  id /= (uint32_t)a.H_kv;
  const int split = (int)(id % (uint32_t)a.splits);
  const int unit = (int)(id / (uint32_t)a.splits);
  constexpr int kHeads = PAIR ? 64 : 32;
  const int head_tiles = (a.G + kHeads - 1) / kHeads;
  const int t = unit / head_tiles, r0 = (unit - t * head_tiles) * kHeads + second * 32;
  int n, len, lo = 0, pos = 0, begin, end;      // tiles of 32 keys (list entries); range tiles begin at multiples of 32
  if constexpr (LIST) {
    n = a.q_seq ? a.q_seq[t] : 0;
    const bool none = (uint32_t)n >= (uint32_t)a.n_seq;
    n = none ? 0 : n;
    len = none ? 0 : clamp_len(a, a.seq_len[n]);
    begin = 0;
    end = (a.n_list + 31) / 32;
  } else {
    // (one token per sequence is the common batch: everything about sequence t is asked for at once, and only if t is not
    // its token is the right one searched: 200 sequences of 500 35.8 us, with a search first 36.6)
    n = t < a.n_seq ? t : a.n_seq - 1;
    int t_begin = a.q_start[n], t_end = a.q_start[n + 1], had = a.seq_len[n];
    const int q_pos = a.q_pos ? a.q_pos[t] : 0, q_lo = a.q_lo ? a.q_lo[t] : 0;
    if (t < t_begin || t >= t_end) {
      n = last_seq(a.n_seq, [&](int i) { return a.q_start[i] <= t; });
      t_begin = a.q_start[n];
      t_end = a.q_start[n + 1];
      if (t < t_begin || t >= t_end) return;
      had = a.seq_len[n];
    }
    len = clamp_len(a, had);
    pos = a.q_pos ? q_pos : had - t_end + t;
    pos = pos < len ? pos : len - 1;
    lo = q_lo > 0 ? q_lo : 0;
    begin = lo >> 5;
    end = (pos >> 5) + 1;                       // (a position may be the last one below 2^31)
    if (pos < 0 || end < begin) end = begin;
  }
  if (a.splits > 1) take_part(begin, end, split, a.splits, 8);      // of at least two tiles per wave
  const int32_t* __restrict__ table = a.table + (long)n * a.max_pages;
  const int cap_last = (int)(((long)a.max_pages << a.page_shift) - 1);

  // position of key `col` of a tile (or one that is no position), and the table's entry for it, whatever it is
  auto position = [&](int tile) {
    if (tile >= end) return -1;
    const int c = tile * 32 + col;
    if constexpr (LIST) return c < a.n_list ? a.list[(long)t * a.n_list + c] : -1;
    else return c;
  };
  auto page_of = [&](int s) {
    const int in = s < 0 ? 0 : s > cap_last ? cap_last : s;
    return table[in >> a.page_shift];
  };
  auto counts = [&](int s, int page) {
    const bool seen = LIST ? s >= 0 && s < len : s >= lo && s <= pos;
    return seen && (uint32_t)page < (uint32_t)a.n_pages;
  };
  constexpr int kBytes = KDT == 2 ? 1 : 2;
  const unsigned char* __restrict__ kbase = (const unsigned char*)a.k + hk * a.head_stride * kBytes + lane % Geo::kCpr * 16;
  const unsigned char* __restrict__ vbase = (const unsigned char*)a.v + hk * a.head_stride * kBytes + lane % Geo::kCpr * 16;
  // loads of a tile: keys, then values (PAIR: the keys by the first wave, the values by the second)
  auto is_value = [&](int i) { return PAIR ? second == 1 : i >= Geo::kNi; };
  auto row_of = [&](int i) { return i % Geo::kNi * Geo::kRpi + lane / Geo::kCpr; };
  uint4 x[Geo::kDepth][Geo::kLoads];
  float scale[Geo::kDepth];
  uint32_t valid[Geo::kDepth];                  // rows of the tile in registers that there are
  // (A row that is none is read from the first row of the pool and cleared on its way into LDS: no load waits for a branch.)
  auto request = [&](auto slot_number, int s, int page) {
    constexpr int d = slot_number;
    const bool ok = counts(s, page);
    const int o = s & ((1 << a.page_shift) - 1);
    valid[d] = (uint32_t)__builtin_amdgcn_ballot_w64(ok);
    long at[Geo::kNi];
    if (!LIST && a.page_shift >= 5 && valid[d] == 0xffffffffu) {
      // the whole tile lies in one page: one address and a lane's part of it
      const int o0 = __builtin_amdgcn_readfirstlane(o), page0 = __builtin_amdgcn_readfirstlane(page);
      const long first = (page0 * a.page_stride + o0 * a.token_stride) * kBytes;
      const long mine = lane / Geo::kCpr * a.token_stride * kBytes, step = Geo::kRpi * a.token_stride * kBytes;
#pragma unroll
      for (int i = 0; i < Geo::kNi; ++i) at[i] = first + i * step + mine;
    } else {
      const long row = ok ? (page * a.page_stride + o * a.token_stride) * kBytes : 0;
      if (half == 0) row_at[col] = row;
      wave_lds_order();
#pragma unroll
      for (int i = 0; i < Geo::kNi; ++i) at[i] = row_at[row_of(i)];
      wave_lds_order();
    }
#pragma unroll
    for (int i = 0; i < Geo::kLoads; ++i)
      x[d][i] = *reinterpret_cast<const uint4*>((is_value(i) ? vbase : kbase) + at[i % Geo::kNi]);
    if constexpr (KDT == 2) {
      const long slot = ok ? ((long)page << a.page_shift) + o : 0;
      // lanes 0 .. 31 the keys' scales, 32 .. 63 the values' (PAIR: each wave its own, twice)
      scale[d] = ((PAIR ? second : half) ? a.v_scale : a.k_scale)[slot * a.H_kv + hk];
      scale[d] = ok ? scale[d] : 0.f;
    }
  };
  auto deposit = [&](auto slot_number, unsigned char* kt, unsigned char* vt) {
    constexpr int d = slot_number;
    if (valid[d] != 0xffffffffu) {
#pragma unroll
      for (int i = 0; i < Geo::kLoads; ++i)
        if (!(valid[d] >> row_of(i) & 1)) x[d][i] = make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < Geo::kLoads; ++i) {
      if (is_value(i)) store_chunk<D, KDT, true>(vt, row_of(i), lane % Geo::kCpr, x[d][i]);
      else store_chunk<D, KDT, false>(kt, row_of(i), lane % Geo::kCpr, x[d][i]);
    }
    if constexpr (KDT == 2) {
      float* sc = reinterpret_cast<float*>(vt + Geo::kTile);                   // 32 key scales, 32 value scales
      if (!PAIR) sc[lane] = scale[d];
      else if (half == 0) sc[second * 32 + col] = scale[d];
    }
  };

  // page lookups run one tile ahead of the rows, list entries two
  int tile = begin + lead, s_next, p_next, s_after;
  RowState<D> st;
  {
    constexpr int kD = Geo::kDepth;
    int s[kD + 2], p[kD + 1];
#pragma unroll
    for (int i = 0; i < kD + 2; ++i) s[i] = position(tile + i * kRowWaves);
#pragma unroll
    for (int i = 0; i < kD + 1; ++i) p[i] = page_of(s[i]);
    steps([&](auto d) { request(d, s[d], p[d]); }, std::make_integer_sequence<int, kD>{});
    s_next = s[kD];
    p_next = p[kD];
    s_after = s[kD + 1];
    int r = r0 + col;                           // (columns beyond the last head repeat it and are not stored)
    if (r >= a.G) r = a.G - 1;
    st.clear();
    st.load_q((const uint16_t*)a.q + ((long)t * a.H + hk * a.G + r) * D);
  }
  const int read_key = RowTile<D>::read_key(), read_value = RowTile<D>::read_value();
  int turn = 0;
  auto iterate = [&](auto slot_number) {
    constexpr int d = slot_number;
    unsigned char* kt = ring + (PAIR ? turn * Geo::kStage : 0);
    unsigned char* vt = kt + Geo::kTile;
    const float* sc = reinterpret_cast<const float*>(vt + Geo::kTile);
    const uint32_t keys = valid[d];
    deposit(slot_number, kt, vt);
    if constexpr (PAIR) lds_barrier();
    else wave_lds_order();
    request(slot_number, s_next, p_next);
    s_next = s_after;
    p_next = page_of(s_next);
    s_after = position(tile + (Geo::kDepth + 2) * kRowWaves);
    if (!PAIR || tile < end) {
      f32x16 s[1];
      bf16x8 p[2], rest[2];
      score_tile<D, 1>(st, kt, renewed(read_key), s);
      if constexpr (KDT == 2) scale_scores<1>(s, sc);
      if (keys != 0xffffffffu) {
        asm volatile("");                       // (a branch, not selects for every tile)
        hide_keys(s[0], keys);
      }
      softmax_tile<D, KDT, 1, REST>(st, s, p, rest, a.scale_log2, sc + 32);
      add_values<D, REST>(st, vt, renewed(read_value), p, rest);
    }
    if constexpr (!PAIR) wave_lds_order();
    tile += kRowWaves;
    turn ^= 1;
  };
  // (with PAIR all waves go round together, whether they have a tile left or not)
  auto more = [&]() { return PAIR ? tile - lead < end : tile < end; };
  while (more())
    steps(
        [&](auto d) {
          if (more()) iterate(d);
        },
        std::make_integer_sequence<int, Geo::kDepth>{});

  // the waves' shares of every row, joined
  float* part = reinterpret_cast<float*>(lds);                  // [wave][D][32]
  const float l = add_halves(st.l);
  if (half == 0) {
    join[(wave * 32 + col) * 2] = st.m;
    join[(wave * 32 + col) * 2 + 1] = l;
  }
  __syncthreads();
  const int first = second * kRowWaves;                         // the waves with the same rows
  float top = neg_inf();
#pragma unroll
  for (int w = 0; w < kRowWaves; ++w) top = fmaxf(top, join[((first + w) * 32 + col) * 2]);
  const float base = top == neg_inf() ? 0.f : top;
  float sum = 0.f;
#pragma unroll
  for (int w = 0; w < kRowWaves; ++w) {
    const float* ml = join + ((first + w) * 32 + col) * 2;
    sum = __builtin_fmaf(__builtin_amdgcn_exp2f(ml[0] - base), ml[1], sum);
  }
  const float f = __builtin_amdgcn_exp2f(st.m - base);
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int i = 0; i < 16; ++i)
      part[(wave * D + dt * 32 + 8 * (i >> 2) + 4 * half + (i & 3)) * 32 + col] = st.o[dt][i] * f;
  __syncthreads();
  const int r = r0 + col;
  if (r < a.G) {
    const long row = (long)t * a.H + hk * a.G + r;
#pragma unroll
    for (int j = 0; j < D / 32; ++j) {
      const int e = ((threadIdx.x >> 5 & 7) * (D / 32) + j) * 4;
      float y[4];
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        y[c] = 0.f;
#pragma unroll
        for (int w = 0; w < kRowWaves; ++w) y[c] += part[((first + w) * D + e + c) * 32 + col];
      }
      const float4 o = make_float4(y[0], y[1], y[2], y[3]);
      if (a.splits > 1) store_result<1, true>(a, split, row, D, e, o, top, sum);
      else store_result<1, false>(a, split, row, D, e, o, top, sum);
    }
  }
}

// ---- many rows per sequence ----------------------------------------------------------------------
// A workgroup of 8 waves takes 256 query rows of one KV head (32 per wave) and a part of their keys, in tiles of 64 keys
// that all waves multiply from LDS.  Bound by the matrix units (4 D flop per visible pair) and, for d = 64, by the vector
// units that make the weights; a second part of the weights (REST) is half as many products again.  Measured: 1024 tokens
// behind 64K, 64 heads on 8, d = 128, 2.7 ms, 0.81 PFLOP/s (fp8 3.0 ms; weights of 8 bits 2.0 and 2.3 ms); eleven prompts of 2777
// tokens at most, windows of 1024, 32 heads on 2, d = 64, fp8, 0.63 ms, 0.36 (8 bits 0.52).  Each SIMD holds two waves, one
// of the first four (group 0) and one of the last four (group 1).  In interval i, between two barriers, group 0 turns its
// scores of tile i into weights, then runs its products for tile i + 1 (scores of tile i + 1, values of tile i), while
// group 1 runs its products for tile i, then turns those scores into weights: one computes while the other multiplies, and
// neither waits for the other half way.  Keys of tile i are thus read in intervals i - 1 (group 0) and i (group 1), values
// of tile i in intervals i and i + 1.
//
// Rows go from memory to LDS without passing registers (there are none left to hold a tile that is under way for as long as
// HBM takes).  What is asked for in one interval has arrived when the next one ends.
//   bf16  interval i asks for keys of tile i + 3 and values of tile i + 2, into four buffers each, in their final places:
//         keys of tile i - 1 were last read in interval i - 1, values of tile i - 2 as well.
//   fp8   interval i asks for keys of tile i + 4 and values of tile i + 3, as stored, into three buffers in which a thread
//         finds its own 16 bytes again; in interval i + 2 it widens them into three tile buffers: keys of tile i + 4 take
//         that of tile i + 1, last read in interval i + 1, values of tile i + 3 that of tile i, last read there too.
// The requests are written as instructions of their own, and waited for by count: from its own builtins the compiler would
// wait for all of them before every read of LDS.
constexpr int kChunkWaves = 8, kChunkRows = 32 * kChunkWaves, kChunkKeys = 64;

template <int D, int KDT>
struct ChunkGeom {
  static constexpr int kCpr = D * (KDT == 2 ? 1 : 2) / 16;            // stored 16-byte chunks of a row
  static constexpr int kPerThread = 2 * kChunkKeys * kCpr / 512;      // of keys and values per thread and step
  static constexpr int kTile = kChunkKeys * D * 2;
  static constexpr int kBuffers = KDT == 2 ? 3 : 4;
  static constexpr int kRaw = 2 * kChunkKeys * kCpr * 16;             // stored bytes of a step
  static constexpr int kRings = kBuffers * 2 * kTile + (KDT == 2 ? 3 * kRaw : 0);
  // and: offsets [8][64] of 8 bytes, masks [8] of 8, pages [8][64] and slots [8][64] of 4, odd [8], scales [8][2][64] (fp8)
  static constexpr int kLds = kRings + 8 * kChunkKeys * 16 + 8 * 8 + 8 * 4 + (KDT == 2 ? 8 * 2 * kChunkKeys * 4 : 0);
};

// 16 or 4 bytes per lane from `src` to LDS byte lds + 16 (or 4) * lane.  m0 is the compiler's, which takes no clobber of it:
// it gets back what was there.
__device__ __forceinline__ void dma16(uint32_t lds, const void* src) {
  int was;
  asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, off\n\ts_mov_b32 m0, %0" :
               "=&s"(was) : "s"(__builtin_amdgcn_readfirstlane((int)lds)), "v"(src) : "memory");
}
__device__ __forceinline__ void dma4(uint32_t lds, const void* src) {
  int was;
  asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %2, off\n\ts_mov_b32 m0, %0" :
               "=&s"(was) : "s"(__builtin_amdgcn_readfirstlane((int)lds)), "v"(src) : "memory");
}
template <int N>
__device__ __forceinline__ void dma_left() {   // until at most N requests of this wave are under way
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

template <int D, int KDT, bool REST>
static __global__ __launch_bounds__(512, 2) void k_attn_chunk(AttnArgs a) {
  using Geo = ChunkGeom<D, KDT>;
  extern __shared__ __align__(16) unsigned char lds[];
  const int lane = lane_id(), half = lane >> 5, col = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), group = wave >> 2;

  uint32_t id = blockIdx.x;
  const int hk = (int)(id % (uint32_t)a.H_kv);
  id /= (uint32_t)a.H_kv;
  const int split = (int)(id % (uint32_t)a.splits);
  const RowUnit u = find_unit<kChunkRows>(a, (int)(id / (uint32_t)a.splits));
  const int n = u.n, t_begin = u.t_begin, t_end = u.t_end;
  const int r0 = u.r0, rows = (t_end - t_begin) * a.G;
  if (r0 < 0 || r0 >= rows || t_begin < 0 || t_end > a.T) return;
  const int len = clamp_len(a, a.seq_len[n]);
  const int32_t* __restrict__ table = a.table + (long)n * a.max_pages;

  // what this wave's rows see, and what the whole tile of rows sees
  RowState<D> st;
  int qr = r0 + wave * 32 + col;
  const bool mine = qr < rows;
  if (!mine) qr = rows - 1;
  const int t = t_begin + qr / a.G, h = hk * a.G + qr % a.G;
  {
    const Seen s = seen_by(a, n, len, t, t_end);
    st.pos = s.pos;
    st.lo = s.lo;
  }
  int wg_pos = -1, wg_lo = 0x7fffffff, wg_pos_min = 0x7fffffff, wg_lo_max = 0;
  {
    const int last = r0 + kChunkRows - 1 < rows - 1 ? r0 + kChunkRows - 1 : rows - 1;
    for (int i = r0 / a.G + lane; i <= last / a.G; i += 64) {
      const Seen s = seen_by(a, n, len, t_begin + i, t_end);
      wg_pos = s.pos > wg_pos ? s.pos : wg_pos;
      wg_lo = s.lo < wg_lo ? s.lo : wg_lo;
      wg_pos_min = s.pos < wg_pos_min ? s.pos : wg_pos_min;
      wg_lo_max = s.lo > wg_lo_max ? s.lo : wg_lo_max;
    }
  }
  st.clear();
  st.load_q((const uint16_t*)a.q + ((long)t * a.H + h) * D);
  wg_pos_min = wave_min_int(wg_pos_min);
  wg_lo_max = wave_max_int(wg_lo_max);
  wg_pos = wave_max_int(wg_pos);
  wg_lo = wave_min_int(wg_lo);
  const int pos_min = wave_min_int(st.pos), lo_max = wave_max_int(st.lo);

  int begin = wg_lo / kChunkKeys, end = wg_pos / kChunkKeys + 1;
  if (wg_pos < 0 || end < begin) end = begin;
  if (a.splits > 1) {
    take_part(begin, end, split, a.splits, 4);
  }

  // Wave 0 finds out where the rows of a tile lie, five tiles ahead, and leaves it in LDS for all: byte offsets (-1: nobody
  // sees the row, or its page is none), fp8 slots, and a mask of the rows that are there; eight tiles of each.
  constexpr int kBytes = KDT == 2 ? 1 : 2;
  long* offsets = reinterpret_cast<long*>(lds + Geo::kRings);                          // [8][64]
  uint64_t* masks = reinterpret_cast<uint64_t*>(offsets + 8 * kChunkKeys);             // [8]
  int* pages = reinterpret_cast<int*>(masks + 8);                                      // [8][64]
  int* slots = pages + 8 * kChunkKeys;                                                 // [8][64]
  int* odd = slots + 8 * kChunkKeys;                                                   // [8]: tile with values dropped
  float* scales = reinterpret_cast<float*>(odd + 8);                                   // [8][2][64] (fp8)
  if (threadIdx.x < 8) odd[threadIdx.x] = -1;
  // first position of a tile; of those behind the last one, which are asked about too, perhaps beyond 2^31 and negative
  auto first_of = [](int tile) { return (int)((uint32_t)tile * kChunkKeys); };
  auto seen_row = [&](int tile) {            // of this lane
    const int s = first_of(tile) | lane;
    return tile < end && s >= wg_lo && s <= wg_pos;
  };
  auto page_entry = [&](int tile) {          // (an entry that there is, whatever the tile)
    return table + (seen_row(tile) ? (first_of(tile) | lane) >> a.page_shift : 0);
  };
  auto publish = [&](int tile, int page) {
    const int o = (first_of(tile) | lane) & ((1 << a.page_shift) - 1);
    const bool ok = seen_row(tile) && (uint32_t)page < (uint32_t)a.n_pages;
    const uint64_t mask = __builtin_amdgcn_ballot_w64(ok);
    offsets[(tile & 7) * kChunkKeys + lane] = ok ? (page * a.page_stride + o * a.token_stride) * kBytes : -1;
    if constexpr (KDT == 2) slots[(tile & 7) * kChunkKeys + lane] = ok ? (page << a.page_shift) + o : -1;
    if (lane == 0) masks[tile & 7] = mask;
  };
  auto mask_of = [&](int tile) {
    const uint64_t m = masks[tile & 7];
    return (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(m >> 32)) << 32 |
           (uint32_t)__builtin_amdgcn_readfirstlane((int)m);
  };

  // this thread's chunks of a step (keys of one tile and values of the tile before it): chunk i * 512 + thread, keys first
  constexpr int kHalf = kChunkKeys * Geo::kCpr;
  static_assert(kHalf == 256 || kHalf % 512 == 0, "keys and values meet between waves");
  auto is_value = [&](int i) { return kHalf < 512 ? wave >= 4 : i * 512 >= kHalf; };
  const int row0 = (kHalf < 512 ? (int)threadIdx.x % kHalf : (int)threadIdx.x) / Geo::kCpr;
  auto row_of = [&](int i) { return row0 + (kHalf < 512 ? 0 : i * 512 % kHalf / Geo::kCpr); };
  // bf16: the chunk of a row that lies at this thread's place of a tile
  const int col0 = threadIdx.x % Geo::kCpr;
  const int kcol = KDT == 2 ? col0 : RowTile<D>::key_byte(row0, col0) / 16 % Geo::kCpr;
  const int vcol = KDT == 2 ? col0 : RowTile<D>::value_byte(row0, col0) / 16 % Geo::kCpr;
  const unsigned char* __restrict__ kbase = (const unsigned char*)a.k + hk * a.head_stride * kBytes + kcol * 16;
  const unsigned char* __restrict__ vbase = (const unsigned char*)a.v + hk * a.head_stride * kBytes + vcol * 16;
  const uint32_t lds0 = lds_address(lds);
  // buffer of a tile: its number modulo four (bf16), or modulo three, counted from `begin` on (fp8)
  auto after = [](int r) { return KDT == 2 ? (r == 2 ? 0 : r + 1) : (r + 1) & 3; };
  auto before = [](int r) { return KDT == 2 ? (r == 0 ? 2 : r - 1) : (r + 3) & 3; };
  auto key_tile = [&](int ring) { return ring * 2 * Geo::kTile; };
  auto value_tile = [&](int ring) { return ring * 2 * Geo::kTile + Geo::kTile; };
  constexpr int kRawAt = Geo::kBuffers * 2 * Geo::kTile;
  // byte of chunk i (its wave's first) of the step with the keys of the tile of buffer r; fp8: in the raw buffer
  auto place = [&](int i, int r) {
    if (KDT == 2) return kRawAt + r * Geo::kRaw + (i * 512 + wave * 64) * 16;
    return is_value(i) ? value_tile(before(r)) + (i * 512 - kHalf + wave * 64) * 16 : key_tile(r) + (i * 512 + wave * 64) * 16;
  };
  struct Where {
    long at[Geo::kPerThread];
    int slot;
  };
  auto where = [&](int tile) {              // of the step with the keys of `tile`
    Where w;
#pragma unroll
    for (int i = 0; i < Geo::kPerThread; ++i)
      w.at[i] = offsets[((tile - is_value(i)) & 7) * kChunkKeys + row_of(i)];
    if constexpr (KDT == 2) w.slot = slots[(tile & 7) * kChunkKeys + lane];
    return w;
  };
  // (a row that is none is read from the first row of the pool, and cleared once it is there)
  auto request = [&](int tile, const Where& w, int r, int page_tile) {
    if (wave == 0) dma4(lds0 + (uint32_t)((unsigned char*)(pages + (page_tile & 7) * kChunkKeys) - lds), page_entry(page_tile));
    if (KDT == 2 && wave < 2)
      dma4(lds0 + (uint32_t)((unsigned char*)(scales + ((tile & 7) * 2 + wave) * kChunkKeys) - lds),
           (wave == 0 ? a.k_scale : a.v_scale) + (long)(w.slot < 0 ? 0 : w.slot) * a.H_kv + hk);
#pragma unroll
    for (int i = 0; i < Geo::kPerThread; ++i)
      dma16(lds0 + place(i, r), (is_value(i) ? vbase : kbase) + (w.at[i] < 0 ? 0 : w.at[i]));
  };
  auto step_arrived = [&]() {               // the step before the last one that was requested
    constexpr int n = Geo::kPerThread + (KDT == 2);
    if (wave == 0) dma_left<n + 1>();
    else if (wave == 1) dma_left<n>();
    else dma_left<Geo::kPerThread>();
  };
  auto mixed = [&](int tile) { return (first_of(tile) | (kChunkKeys - 1)) > wg_pos_min || first_of(tile) < wg_lo_max; };
  // chunk i of an arrived step: cleared where its row is none, and of infinities and NaN in a mixed tile
  auto cleaned = [&](int i, uint4 x, uint64_t km, uint64_t vm, int tile) {
    if (!((is_value(i) ? vm : km) >> row_of(i) & 1)) x = make_uint4(0, 0, 0, 0);
    if (is_value(i) && mixed(tile - 1) && drop_odd<KDT>(x)) odd[(tile - 1) & 7] = tile - 1;
    return x;
  };
  // What an arrived step (keys of `tile`, in buffer r) still needs: bf16 only where there is something to clean, fp8 to be
  // widened, from raw buffer `raw`.
  auto finish = [&](int tile, int r, int raw, uint64_t km, uint64_t vm) {
    const bool clean = (km & vm) != ~0ull || mixed(tile - 1);
    if constexpr (KDT == 1) {
      if (clean) {
#pragma unroll
        for (int i = 0; i < Geo::kPerThread; ++i) {
          uint4* p = reinterpret_cast<uint4*>(lds + place(i, r)) + lane;
          *p = cleaned(i, *p, km, vm, tile);
        }
      }
    } else {
      if (wave == 1) {
        float* sc = scales + ((tile & 7) * 2 + 1) * kChunkKeys + lane;
        if (!(km >> lane & 1)) *sc = 0.f;
        else if (mixed(tile) && !(__builtin_fabsf(*sc) < __builtin_inff())) {
          *sc = 0.f;
          odd[tile & 7] = tile;
        }
      }
#pragma unroll
      for (int i = 0; i < Geo::kPerThread; ++i) {
        uint4 x = reinterpret_cast<const uint4*>(lds + place(i, raw))[lane];
        if (clean) x = cleaned(i, x, km, vm, tile);
        if (is_value(i)) store_chunk<D, 2, true>(lds + value_tile(before(r)), row_of(i), col0, x);
        else store_chunk<D, 2, false>(lds + key_tile(r), row_of(i), col0, x);
      }
    }
  };

  const int read_key = RowTile<D>::read_key(), read_value = RowTile<D>::read_value();
  if (wave == 0) {
    int first[6];
#pragma unroll
    for (int i = 0; i < 6; ++i) first[i] = *page_entry(begin + i);
#pragma unroll
    for (int i = 0; i < 5; ++i) publish(begin + i, first[i]);
    pages[((begin + 5) & 7) * kChunkKeys + lane] = first[5];
    masks[(begin - 1) & 7] = 0;              // (the first step has keys and no values)
    offsets[((begin - 1) & 7) * kChunkKeys + lane] = -1;
  }
  lds_barrier();
  // r: buffer of the present tile; fp8: raw buffer of the step that is widened for the next one
  int r = KDT == 2 ? 0 : begin & 3;
  request(begin, where(begin), r, begin + 6);
  request(begin + 1, where(begin + 1), after(r), begin + 6);
  if constexpr (KDT == 2) request(begin + 2, where(begin + 2), after(after(r)), begin + 6);
  dma_left<0>();
  finish(begin, r, r, mask_of(begin), 0);
  finish(begin + 1, after(r), after(r), mask_of(begin + 1), mask_of(begin));
  if (group == 1) request(begin + 2 + (KDT == 2), where(begin + 2 + (KDT == 2)), KDT == 2 ? r : after(after(r)), 0);
  lds_barrier();
  if (__builtin_amdgcn_readfirstlane(r0 + wave * 32 >= rows)) {
    // A wave without rows goes through the loop below for its share of the tiles alone and leaves the others the machine.
    if (group == 1) lds_barrier();
    if (KDT == 2 && group == 1) finish(begin + 2, after(after(r)), after(after(r)), mask_of(begin + 2), mask_of(begin + 1));
    // (the pages of later tiles are wave 0's business, which has rows)
    auto bring = [&](int tile, int to) { request(tile, where(tile), KDT == 2 ? to : tile & 3, 0); };
    bring(begin + group + 2 + (KDT == 2), group == 1 ? after(r) : r);
    if (group == 0) lds_barrier();
    for (int tile = begin; tile < end; ++tile) {
      const int r1 = after(r), r2 = after(r1);
      const uint64_t km = mask_of(tile + 2), vm = mask_of(tile + 1);
      if (KDT == 1 && group == 1) {
        step_arrived();
        finish(tile + 2, r2, 0, km, vm);
      }
      if (group == 1) lds_barrier();
      if constexpr (KDT == 2) {
        step_arrived();
        if (group == 0) finish(tile + 2, r2, r2, km, vm);
        else finish(tile + 3, r, r, mask_of(tile + 3), km);
      }
      bring(tile + 3 + group + (KDT == 2), group == 0 ? r1 : r2);
      if (KDT == 1 && group == 0) {
        step_arrived();
        finish(tile + 2, r2, 0, km, vm);
      }
      if (group == 0) lds_barrier();
      r = r1;
    }
    dma_left<0>();
    return;
  }
  f32x16 s[2];
  bf16x8 p[4], rest[4];
  if (group == 1) lds_barrier();
  score_tile<D, 2>(st, lds + key_tile(r), renewed(read_key), s);
  {
    // (fp8: what group 1 widens here, and group 0 between the products for the next tile, came with the third request)
    const int tile = begin + group;
    const Where at = where(tile + 2 + (KDT == 2));
    if (KDT == 2 && group == 1) finish(begin + 2, after(after(r)), after(after(r)), mask_of(begin + 2), mask_of(begin + 1));
    const int to = KDT == 2 ? (group == 1 ? after(r) : r) : (tile + 2) & 3;
    request(tile + 2 + (KDT == 2), at, to, begin + 6 + (KDT == 2));
  }
  if (group == 0) lds_barrier();
  for (int tile = begin; tile < end; ++tile) {
    const int base = tile * kChunkKeys, r1 = after(r), r2 = after(r1);
    const uint64_t mask = mask_of(tile), km = mask_of(tile + 2), vm = mask_of(tile + 1);
    {
      const float* sc = scales + (tile & 7) * 2 * kChunkKeys;
      if constexpr (KDT == 2) scale_scores<2>(s, sc);
      if (mask != ~0ull || base + kChunkKeys - 1 > pos_min || base < lo_max) {
        asm volatile("");                  // (a branch, not 32 selects for every tile)
        hide(st, s[0], (uint32_t)mask, base);
        hide(st, s[1], (uint32_t)(mask >> 32), base + 32);
      }
      softmax_tile<D, KDT, 2, REST>(st, s, p, rest, a.scale_log2, sc + kChunkKeys);
    }
    // (the weights are made here and not, as the compiler would have it, between the products that need them)
#pragma unroll
    for (int i = 0; i < 4; ++i) asm volatile("" : "+v"(p[i]));
    if constexpr (REST)
#pragma unroll
      for (int i = 0; i < 4; ++i) asm volatile("" : "+v"(rest[i]));
    asm volatile("" : "+v"(st.l));
    if (wave == 0) publish(tile + 5, pages[((tile + 5) & 7) * kChunkKeys + lane]);
    if (group == 1) {
      if constexpr (KDT == 1) {
        step_arrived();
        finish(tile + 2, r2, 0, km, vm);
      }
      lds_barrier();
    }
    // products for the next tile (behind the last one there are keys of nobody, whose scores are not looked at)
    __builtin_amdgcn_sched_barrier(0);
    const bool dropped = __builtin_amdgcn_readfirstlane(odd[tile & 7]) == tile;
    const int asked = tile + 3 + group + (KDT == 2);
    if constexpr (KDT == 2) {
      // group 0 is in interval `tile`, group 1 in the next one: keys of tile + 2, of tile + 3
      step_arrived();
      if (group == 0) finish(tile + 2, r2, r2, km, vm);
      else finish(tile + 3, r, r, mask_of(tile + 3), km);
    }
    Where at;
    constexpr int kProducts = D / 4;
    __builtin_amdgcn_s_setprio(3);           // (the wave that multiplies goes first: 0.5 % at 1024 new tokens behind 64K)
    products<D, REST>(st, lds + key_tile(r1), renewed(read_key), s, lds + value_tile(r), renewed(read_value), p, rest,
                      [&](int i) {
      if (i == 1) at = where(asked);
      // (fp8: the buffer of the step before the one that is widened now)
      if (i == kProducts / 4) request(asked, at, KDT == 2 ? (group == 0 ? r1 : r2) : asked & 3, tile + 7 + (KDT == 2));
    });
    __builtin_amdgcn_s_setprio(0);
    if (dropped)
      add_odd_values<D, KDT>(st, (const unsigned char*)a.v + hk * a.head_stride * kBytes, offsets + (tile & 7) * kChunkKeys,
                             slots + (tile & 7) * kChunkKeys, a.v_scale + hk, a.H_kv, base);
    if (group == 0) {
      if constexpr (KDT == 1) {
        step_arrived();
        finish(tile + 2, r2, 0, km, vm);
      }
      lds_barrier();
    }
    r = r1;
  }
  dma_left<0>();                           // (LDS is somebody else's once the workgroup has ended)

  if (!mine) return;
  const float l = add_halves(st.l);
  const long row = (long)t * a.H + h;
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int e = dt * 32 + 8 * j + 4 * half;
      const float4 o = make_float4(st.o[dt][4 * j], st.o[dt][4 * j + 1], st.o[dt][4 * j + 2], st.o[dt][4 * j + 3]);
      if (a.splits > 1) store_result<1, true>(a, split, row, D, e, o, st.m, l);
      else store_result<1, false>(a, split, row, D, e, o, st.m, l);
    }
}

// Joins the parts of a row: 4 columns per lane, 8 parts asked for at once (what this costs is the way to memory, once per
// 8 parts), `groups` sets of lanes per row that share its parts and meet in LDS.  (One token over 130000 keys, 64 heads on
// one KV head, 128 parts: with one set per row and a part at a time the call took 341 us, so 42.)
constexpr int kJoinParts = 8;

struct Joined {
  float4 o;
  float m, l;
};
__device__ __forceinline__ void join_part(Joined& j, float f, float4 o, float l) {
  j.l = __builtin_fmaf(f, l, j.l);
  j.o.x = __builtin_fmaf(f, o.x, j.o.x);
  j.o.y = __builtin_fmaf(f, o.y, j.o.y);
  j.o.z = __builtin_fmaf(f, o.z, j.o.z);
  j.o.w = __builtin_fmaf(f, o.w, j.o.w);
}

template <int QDT, bool LIST>
static __global__ __launch_bounds__(256) void k_attn_join(AttnArgs a, int groups) {
  __shared__ float4 group_o[256];
  __shared__ float2 group_ml[256];
  const int per = a.d / 4, rows = 256 / per / groups;         // lanes of a set, rows of this workgroup
  const int set = threadIdx.x / per, e = (threadIdx.x - set * per) * 4, group = set % groups;
  const long r = (long)blockIdx.x * rows + set / groups, all = (long)a.T * a.H;
  bool mine = set < rows * groups && r < all;
  if constexpr (!LIST) {
    const int t = (int)(r / a.H);
    mine = mine && t >= a.q_start[0] && t < a.q_start[a.n_seq];
  }
  Joined j{make_float4(0.f, 0.f, 0.f, 0.f), neg_inf(), 0.f};
  if (mine) {
    const float2* ml = reinterpret_cast<const float2*>(a.part + a.splits * all * a.d);
    for (int first = group * kJoinParts; first < a.splits; first += groups * kJoinParts) {
      float2 x[kJoinParts];
      float4 o[kJoinParts];
#pragma unroll
      for (int i = 0; i < kJoinParts; ++i) {
        const long pr = (first + i < a.splits ? first + i : a.splits - 1) * all + r;
        x[i] = ml[pr];
        o[i] = *reinterpret_cast<const float4*>(a.part + pr * a.d + e);
      }
      float top = j.m;
#pragma unroll
      for (int i = 0; i < kJoinParts; ++i) top = fmaxf(top, x[i].x);
      const float base = top == neg_inf() ? 0.f : top, f = __builtin_amdgcn_exp2f(j.m - base);
      j = Joined{make_float4(j.o.x * f, j.o.y * f, j.o.z * f, j.o.w * f), top, j.l * f};
#pragma unroll
      for (int i = 0; i < kJoinParts; ++i)
        if (first + i < a.splits) join_part(j, __builtin_amdgcn_exp2f(x[i].x - base), o[i], x[i].y);
    }
  }
  if (groups > 1) {
    group_o[threadIdx.x] = j.o;
    group_ml[threadIdx.x] = make_float2(j.m, j.l);
    __syncthreads();
    if (group != 0) return;
    float top = j.m;
    for (int g = 1; g < groups && mine; ++g) top = fmaxf(top, group_ml[threadIdx.x + g * per].x);
    const float base = top == neg_inf() ? 0.f : top, f = __builtin_amdgcn_exp2f(j.m - base);
    j = Joined{make_float4(j.o.x * f, j.o.y * f, j.o.z * f, j.o.w * f), top, j.l * f};
    for (int g = 1; g < groups && mine; ++g) {
      const float2 x = group_ml[threadIdx.x + g * per];
      join_part(j, __builtin_amdgcn_exp2f(x.x - base), group_o[threadIdx.x + g * per], x.y);
    }
  }
  if (!mine) return;
  const float inv = j.l == 0.f ? 0.f : 1.f / j.l;
  store_four<QDT>(a, r, e, make_float4(j.o.x * inv, j.o.y * inv, j.o.z * inv, j.o.w * inv));
  if (e == 0 && a.lse) a.lse[r] = j.l == 0.f ? neg_inf() : (j.m + log2f(j.l)) * 0.693147180559945309f;
}

}  // namespace hisa
