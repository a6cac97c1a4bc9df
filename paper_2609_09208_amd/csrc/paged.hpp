// What the kernels of the paged cache share: where a sequence's tokens stand, its new rows,
// queries as score operands, and the values' fp16 numbers.
#pragma once

#include "encode_rows.hpp"
#include "head_rows.hpp"
#include "page_ranges.hpp"
#include "pot_device.hpp"
#include "pot_launch.hpp"

namespace potattn {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

// Loads past the caches, of what a call reads once.
__device__ __forceinline__ uint4 stream16(const void* p) {
  const u32x4v v = __builtin_nontemporal_load(static_cast<const u32x4v*>(p));
  return make_uint4(v.x, v.y, v.z, v.w);
}

// A group's rows of the pool are counted by groups: row8 = row / 8, below 2^31.
// First cache row / 8 of group `group` of a sequence for a kv head: group `in` of its page;
// -1 where the table has no such page. table: the sequence's entries.
__device__ __forceinline__ int group_row8(const PagesArg& p, const int32_t* table, int kvh, int group) {
  const uint32_t page = page_of_group((uint32_t)group, p.div);
  if (group < 0 || page >= (uint32_t)p.table_len) return -1;
  const int32_t at = table[page];
  if ((uint32_t)at >= (uint32_t)p.n_pages) return -1;
  return (at * p.Hkv + kvh) * p.page_groups + (group - (int)page * p.page_groups);
}

__device__ __forceinline__ NewTokens sequence_tokens(const PackedRows& r, int b, int most_new,
                                                     int most_len) {
  return new_tokens(r.cu_new[b], r.cu_new[b + 1], r.seq_lens[b], r.n, most_new, most_len);
}

// 8 natural elements of a row (16-byte aligned) as floats. Every lane of a row takes part.
__device__ __forceinline__ void load8(const void* base, int64_t at, int chunk, int type,
                                      float (&x)[8]) {
  if (type == POT_FP32) to_floats<POT_FP32, kNeighbours>(load_row<POT_FP32, kNeighbours>(base, at, chunk), x);
  else if (type == POT_BF16) to_floats<POT_BF16, kNeighbours>(load_row<POT_BF16, kNeighbours>(base, at, chunk), x);
  else to_floats<POT_FP16, kNeighbours>(load_row<POT_FP16, kNeighbours>(base, at, chunk), x);
}

// Weights, references and factors (Reference).
constexpr float kWeightShift = 7.0f, kMostWeight = 15.0f, kNoReference = -3e38f, kLeastFactor = 1e-30f;
constexpr float kFarReference = 0x1p20f;  // fp32's steps there are 1/8

// Walsh-Hadamard rotation of a row over its 8 lanes (lane g: elements 8g .. 8g + 7), fp64
// stages of span 1 .. 32, one rounding to fp32.
__device__ __forceinline__ void rotate_hadamard(float (&x)[8], int lane) {
  double v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = (double)x[i];
#pragma unroll
  for (int h = 1; h < 8; h <<= 1)
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if ((i & h) == 0) {
        const double p = v[i], q = v[i + h];
        v[i] = p + q;
        v[i + h] = p - q;
      }
  const double s1 = butterfly_sign<1>(lane), s2 = butterfly_sign<2>(lane), s4 = butterfly_sign<4>(lane);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    v[i] = butterfly<1>(v[i], s1);
    v[i] = butterfly<2>(v[i], s2);
    v[i] = butterfly<4>(v[i], s4);
    x[i] = (float)(v[i] * 0.125);
  }
}

// The INT8 query of a row over its 8 lanes as fp16 integers, in the order of decode_weights
// (elements 0 4 1 5 2 6 3 7 of the lane's 8), and its score factor: with the weights' 2^-8
// taken back, sum * scale * factor is the score times log2 e.
__device__ __forceinline__ uint4 quantised_query(float (&x)[8], int hadamard, int lane, float* factor) {
  if (hadamard) rotate_hadamard(x, lane);
  float top = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(x[i]));
  top = max_over_8_lanes(top);
  int q[8];
  const float inv = 127.0f / top;  // correctly rounded divisions
#pragma unroll
  for (int i = 0; i < 8; ++i) q[i] = top == 0.0f ? 0 : quantize_int8(x[i], inv);
  *factor = fmaxf(__fmul_rn(top / 127.0f, log2e_f32()) * 32.0f, kLeastFactor);
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = pack_half((float)q[i], (float)q[i + 4]);
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// Code dword w (nibble n: element n) and its mantissa planes' bytes (bit n: element n) as the
// fp16 weights sigma (1 + j / 2^K) 2^(-8 - e), in the order 0 4 1 5 2 6 3 7: sign bit, exponent
// field 7 - e, the mantissa bits on top of fp16's; the zero code (e = 7) is exponent field 0,
// where the mantissa bits are taken off whatever they are. The numbers' high bytes are looked up,
// four codes an operation: 12 operations for 8 codes at K = 0.
__device__ __forceinline__ uint32_t spread_nibbles(uint32_t x) {  // bit n of 8 to bit 4n
  x = (x | (x << 12)) & 0x000F000Fu;
  x = (x | (x << 6)) & 0x03030303u;
  return (x | (x << 3)) & 0x11111111u;
}
template <int K>
__device__ __forceinline__ half8 paged_weights(uint32_t w, const uint32_t* planes) {
  constexpr uint32_t kLut0 = 0x1014181Cu, kLut1 = 0x0004080Cu, kTop = 0x80808080u;
  const uint32_t even = w & 0x07070707u, odd = (w >> 4) & 0x07070707u;
  const uint32_t be = __builtin_amdgcn_perm(kLut1, kLut0, even) | ((w << 4) & kTop);
  const uint32_t bo = __builtin_amdgcn_perm(kLut1, kLut0, odd) | (w & kTop);
  uint32_t v[4] = {__builtin_amdgcn_perm(0u, be, 0x020C000Cu), __builtin_amdgcn_perm(0u, bo, 0x020C000Cu),
                   be & 0xFF00FF00u, bo & 0xFF00FF00u};
  if constexpr (K > 0) {
    // bytes of ones where the code is not zero, spread over the halves
    const uint32_t me = __builtin_amdgcn_perm(0x00FFFFFFu, 0xFFFFFFFFu, even);
    const uint32_t mo = __builtin_amdgcn_perm(0x00FFFFFFu, 0xFFFFFFFFu, odd);
    const uint32_t keep[4] = {__builtin_amdgcn_perm(0u, me, 0x02020000u), __builtin_amdgcn_perm(0u, mo, 0x02020000u),
                              __builtin_amdgcn_perm(0u, me, 0x03030101u), __builtin_amdgcn_perm(0u, mo, 0x03030101u)};
    uint32_t j = spread_nibbles(planes[0]);  // nibble n: element n's mantissa
#pragma unroll
    for (int b = 1; b < K; ++b) j |= spread_nibbles(planes[b]) << b;
    constexpr uint32_t kField = (((1u << K) - 1) << (10 - K)) * 0x10001u;
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      const int sh = 10 - K - 4 * n;
      const uint32_t m = sh >= 0 ? j << (sh >= 0 ? sh : 0) : j >> (sh < 0 ? -sh : 0);
      v[n] |= m & (kField & keep[n]);
    }
  }
  return __builtin_bit_cast(half8, make_uint4(v[0], v[1], v[2], v[3]));
}

// fp16 values z + s n of 8 tokens, each rounded once (a packed multiply-add), from the tokens'
// n (bytes of w0, w1, below 16) and their steps and minima, two a dword.
__device__ __forceinline__ uint4 int4_values(uint32_t w0, uint32_t w1, const uint4& s, const uint4& z) {
  constexpr uint32_t kExp = 0x64646464u;  // a byte under it: 1024 + n
  const uint32_t n4[4] = {__builtin_amdgcn_perm(kExp, w0, 0x04010400u),
                          __builtin_amdgcn_perm(kExp, w0, 0x04030402u),
                          __builtin_amdgcn_perm(kExp, w1, 0x04010400u),
                          __builtin_amdgcn_perm(kExp, w1, 0x04030402u)};
  const uint32_t s4[4] = {s.x, s.y, s.z, s.w}, z4[4] = {z.x, z.y, z.z, z.w};
  uint32_t r[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const half2v c = {(_Float16)-1024.0f, (_Float16)-1024.0f};
    const half2v n = __builtin_bit_cast(half2v, n4[i]) + c;
    r[i] = __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(n, __builtin_bit_cast(half2v, s4[i]),
                                                                  __builtin_bit_cast(half2v, z4[i])));
  }
  return make_uint4(r[0], r[1], r[2], r[3]);
}

// Tokens at or past `end` of the 8 from `first` on to 0: whatever the cache holds there cannot
// reach the sums.
__device__ __forceinline__ uint4 mask_tokens(uint4 v, int first, int end) {
  uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i)
    w[i] &= ((first + 2 * i < end) ? 0x0000FFFFu : 0u) | ((first + 2 * i + 1 < end) ? 0xFFFF0000u : 0u);
  return make_uint4(w[0], w[1], w[2], w[3]);
}

__device__ __forceinline__ SeenKeys seen_keys(const PagedAttendArgs& a, int place, int end, int t0) {
  return seen_keys(place, end, t0, a.window, a.n_sink);
}
// y where bit e of the mask is set, minus infinity elsewhere.
__device__ __forceinline__ float if_seen(float y, uint32_t mask, int e) {
  const uint32_t all = (uint32_t)__builtin_amdgcn_sbfe((int)mask, e, 1);
  return __uint_as_float((__float_as_uint(y) & all) | (0xFF800000u & ~all));
}

// Values that are infinite or NaN, in tiles of which some query sees a part only: their product
// with a weight of 0 would be NaN where they are not seen. They go into the sums as 0; after the
// last tile, the matrix cores count them for the keys that a query sees (a path that no ordinary
// cache takes: it reads the values again).
__device__ __forceinline__ uint32_t special_mask(uint32_t w) {
  return ((w & 0x7C00u) == 0x7C00u ? 0x0000FFFFu : 0u) | ((w & 0x7C000000u) == 0x7C000000u ? 0xFFFF0000u : 0u);
}
__device__ __forceinline__ bool has_special(const uint4& v) {
  return (special_mask(v.x) | special_mask(v.y) | special_mask(v.z) | special_mask(v.w)) != 0;
}
__device__ __forceinline__ uint4 without_special(const uint4& v) {
  return make_uint4(v.x & ~special_mask(v.x), v.y & ~special_mask(v.y), v.z & ~special_mask(v.z),
                    v.w & ~special_mask(v.w));
}
__device__ __forceinline__ half8 special_marks(const uint4& v) {  // 1 where a value is special
  constexpr uint32_t kOne = 0x3C003C00u;
  return __builtin_bit_cast(half8, make_uint4(kOne & special_mask(v.x), kOne & special_mask(v.y),
                                              kOne & special_mask(v.z), kOne & special_mask(v.w)));
}
// What the counted values make of a sum.
__device__ __forceinline__ float special_sum(float count) {
  return count > 0.0f ? __builtin_nanf("") : 0.0f;
}
// The fp16 values of dimension d of the 8 tokens of a group of cache rows.
template <int VF>
__device__ __forceinline__ uint4 group_values(const PagesArg& p, int row8, int d) {
  if constexpr (VF == POT_VALUES_INT4) {
    const uint8_t* rec = p.values + (int64_t)row8 * kI4GroupBytes;
    const uint2 n = *reinterpret_cast<const uint2*>(rec + 16 * (d & 15) + 8 * (d >> 5));
    const int sh = (d & 16) ? 4 : 0;
    return int4_values((n.x >> sh) & 0x0F0F0F0Fu, (n.y >> sh) & 0x0F0F0F0Fu,
                       *reinterpret_cast<const uint4*>(rec + kI4Steps),
                       *reinterpret_cast<const uint4*>(rec + kI4Minima));
  } else {
    return *reinterpret_cast<const uint4*>(p.values + (int64_t)row8 * (16 * kDim) + 16 * d);
  }
}

// Weights of fp32 as fp16 operands: rounded to nearest, and what that left, rounded in turn.
__device__ __forceinline__ uint32_t low_part(float a, float b, uint32_t hi) {
  const half2v h = __builtin_bit_cast(half2v, hi);
  return pack_half(a - (float)h.x, b - (float)h.y);
}

// A row's output from its weighted sums, 4 neighbouring elements, in the output's type.
__device__ __forceinline__ void store_out4(void* out, int64_t at, int type, float a, float b, float c,
                                           float d) {
  if (type == POT_FP32)
    *reinterpret_cast<float4*>(static_cast<float*>(out) + at) = make_float4(a, b, c, d);
  else if (type == POT_BF16)
    *reinterpret_cast<uint2*>(static_cast<uint16_t*>(out) + at) = make_uint2(pack_bf16(a, b), pack_bf16(c, d));
  else
    *reinterpret_cast<uint2*>(static_cast<uint16_t*>(out) + at) = make_uint2(pack_half(a, b), pack_half(c, d));
}

// A query's reference m (a sum times its scale), and b = 7 - m c as rounded: a key's weight is
// 2^(y c + b), y its sum times its scale, c the query's factor. What b's rounding leaves is the
// same for all weights, and a new reference takes the old sums with it by 2^(b - b_old), so it
// does not matter, until b is so large that a weight of 2^7 could leave fp16's range: then the
// difference y - m is taken first (far, for a wave).
//
// The reference rises, to a tile's largest y, when that key's weight would be over 2^15; it is
// 2^7 then, so fp16's normal numbers reach 2^-21 of the largest weight at the least. A key that is
// not seen has y = minus infinity and weight 0: factors are at least kLeastFactor, and b is 0 as
// long as there is no reference.
struct Reference {
  float m = kNoReference, b = 0.0f;
  bool far = false;  // uniform
};
// y as weight_of takes it.
template <int N>
__device__ __forceinline__ void far_sums(const Reference& r, float (&y)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) y[i] -= r.m;
}
__device__ __forceinline__ float weight_shift(const Reference& r) { return r.far ? kWeightShift : r.b; }
__device__ __forceinline__ float weight_of(float y, float c, float shift) {
  return __builtin_amdgcn_exp2f(__builtin_fmaf(y, c, shift));
}
// Whether the reference has to rise for a largest y of `top` (or there is none), for the wave.
__device__ __forceinline__ bool must_rise(const Reference& r, float top, float c) {
  const float x = r.far ? __builtin_fmaf(top - r.m, c, kWeightShift) : __builtin_fmaf(top, c, r.b);
  return __any(x > kMostWeight || r.m == kNoReference);
}
// 2^((m - M) c) of two references.
__device__ __forceinline__ float between(float m, float M, float c) {
  return __builtin_amdgcn_exp2f((m - M) * c);
}
// Raises the reference to `top`, the largest y of the query in the tile; returns what the sums
// are to be multiplied by.
__device__ __forceinline__ float raise(Reference& r, float top, float c) {
  const float to = fmaxf(r.m, top);
  const float b = to == kNoReference ? 0.0f : __builtin_fmaf(-to, c, kWeightShift);
  const bool far = r.far || __any(fabsf(b) >= kFarReference);
  float f = r.far ? (r.m - to) * c : far ? __builtin_fmaf(-to, c, kWeightShift - r.b) : b - r.b;
  f = r.m == kNoReference ? 0.0f : __builtin_amdgcn_exp2f(f);
  r.m = to;
  r.b = b;
  r.far = far;
  return f;
}
// What takes sums to the weights 2^(y c - m c + 7) of the exact reference, for a merge with others.
__device__ __forceinline__ float exact_reference(const Reference& r, float c) {
  return r.far || r.m == kNoReference
             ? 1.0f : __builtin_amdgcn_exp2f(-__builtin_fmaf(r.m, c, r.b - kWeightShift));
}

// A row's partials of S key ranges (`next` floats apart) as one by a wave, of which lane l takes
// dimensions 4 (l % 16) ..+3 of ranges l / 16, 4 + l / 16 ..; the quotients in every lane.
struct Merged {
  float o[4];
};
__device__ __forceinline__ float over_rows(float v) {  // sum over the wave's 16-lane rows
  const auto r16 = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(r16[0]) + __uint_as_float(r16[1]);
  const auto r32 = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r32[0]) + __uint_as_float(r32[1]);
}
__device__ __forceinline__ Merged merge_parts(const float* part, int next, int S, int lane) {
  const int grp = lane >> 4, d = 4 * (lane & 15);
  float M = kNoReference, c = 0.0f, L = 0.0f;
  f32x4 O = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int s0 = 0; s0 < S; s0 += 16) {
    f32x4 w[4], o[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float* p = part + (int64_t)min(s0 + 4 * i + grp, S - 1) * next;
      w[i] = *reinterpret_cast<const f32x4*>(p + kDim);
      o[i] = *reinterpret_cast<const f32x4*>(p + d);
    }
    c = w[0][2];
    float top = M;
#pragma unroll
    for (int i = 0; i < 4; ++i) top = fmaxf(top, w[i][0]);
    const auto r16 = __builtin_amdgcn_permlane16_swap(__float_as_uint(top), __float_as_uint(top), false, false);
    top = fmaxf(__uint_as_float(r16[0]), __uint_as_float(r16[1]));
    const auto r32 = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
    top = fmaxf(__uint_as_float(r32[0]), __uint_as_float(r32[1]));
    const float f0 = between(M, top, c);
    L *= f0;
    O *= f0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float f = s0 + 4 * i + grp < S ? between(w[i][0], top, c) : 0.0f;
      L += f * w[i][1];
      O += f * o[i];
    }
    M = top;
  }
  L = over_rows(L);
  const float inv = L == 0.0f ? 0.0f : 1.0f / L;
  Merged g;
#pragma unroll
  for (int i = 0; i < 4; ++i) g.o[i] = over_rows(O[i]) * inv;
  return g;
}

}  // namespace potattn
