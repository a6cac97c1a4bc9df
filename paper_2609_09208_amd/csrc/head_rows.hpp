// Rows of a projection in registers: 64 elements over 8 lanes, 8 rows a wave. Loads and stores
// of the three types, RMS norm and position rotation (the kernels that use them:
// norm_rope.hip, paged_append.hip).
// Angles: position * inv_freq / 2 pi in fp64, whose whole turns are taken off exactly,
// then sine and cosine by their series on an eighth of a turn in fp32.
#pragma once

#include <type_traits>

#include "pot_device.hpp"

namespace potattn {

// How a head's elements are paired.
//  kFullHalves: (i, i + 32). kNeighbours: (2i, 2i + 1), the first rot_dim elements.
//  kHalves: (i, i + rot_dim / 2) of any rot_dim, the partners through LDS.
enum PairMode : int { kFullHalves = 0, kNeighbours = 1, kHalves = 2 };

template <int DT>
constexpr int kElemBytes = DT == POT_FP32 ? 4 : 2;

// What lane g (0 .. 7) of a row works on in its registers 0 .. 7: elements 8g .. 8g + 7,
// or for kFullHalves 4p .. 4p + 3 and 32 + 4p .. 32 + 4p + 3 with p = quad_of(g).
//
// Rows of 16-bit numbers move 16 bytes a lane all the same: lane g < 4 has elements
// 8g .. 8g + 7 and lane 7 - g the same of the upper half, and the two exchange a half each
// in one DPP step (two 8-byte pieces a lane instead cost 8% at 32768 tokens).
__device__ __forceinline__ int quad_of(int g) { return g < 4 ? 2 * g : 2 * (7 - g) + 1; }
constexpr int kMirror8 = 0x141;  // row_half_mirror: lane g reads lane 7 - g of its 8
// Lanes of the banks in MASK take src of their mirror lane, the others keep own.
template <int MASK>
__device__ __forceinline__ uint32_t take_mirror(uint32_t own, uint32_t src) {
  return (uint32_t)__builtin_amdgcn_update_dpp((int)own, (int)src, kMirror8, 0xF, MASK, false);
}
constexpr int kLowBanks = 0x5, kHighBanks = 0xA;  // lanes g < 4 and g >= 4
__device__ __forceinline__ void exchange_quads(uint2& lo, uint2& hi) {
  const uint2 a = lo, b = hi;
  lo = make_uint2(take_mirror<kHighBanks>(a.x, b.x), take_mirror<kHighBanks>(a.y, b.y));
  hi = make_uint2(take_mirror<kLowBanks>(b.x, a.x), take_mirror<kLowBanks>(b.y, a.y));
}

// A lane's 8 elements as loaded: two pieces of 4.
template <int DT>
struct RawRow {
  std::conditional_t<DT == POT_FP32, uint4, uint2> p[2];
};
template <int DT, int MODE>
__device__ __forceinline__ RawRow<DT> load_row(const void* base, int64_t at, int g) {
  // at: the row's first element
  using Piece = std::conditional_t<DT == POT_FP32, uint4, uint2>;
  const char* p = static_cast<const char*>(base) + at * kElemBytes<DT>;
  RawRow<DT> r;
  if constexpr (DT == POT_FP32) {
    p += MODE == kFullHalves ? 16 * quad_of(g) : 32 * g;
    r.p[0] = *reinterpret_cast<const Piece*>(p);
    r.p[1] = *reinterpret_cast<const Piece*>(p + (MODE == kFullHalves ? 128 : 16));
  } else {
    p += 16 * (MODE == kFullHalves && g >= 4 ? 11 - g : g);
    const uint4 v = *reinterpret_cast<const uint4*>(p);
    r.p[0] = make_uint2(v.x, v.y);
    r.p[1] = make_uint2(v.z, v.w);
  }
  return r;
}
__device__ __forceinline__ float from_half_bits(uint32_t u) {
  return __half2float(__ushort_as_half((unsigned short)u));
}
// The 8 elements to work on; every lane of the row takes part.
template <int DT, int MODE>
__device__ __forceinline__ void to_floats(RawRow<DT> r, float (&x)[8]) {
  if constexpr (MODE == kFullHalves && DT != POT_FP32) exchange_quads(r.p[0], r.p[1]);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    if constexpr (DT == POT_FP32) {
      const uint32_t w[4] = {r.p[h].x, r.p[h].y, r.p[h].z, r.p[h].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) x[4 * h + i] = __uint_as_float(w[i]);
    } else {
      const uint32_t w[2] = {r.p[h].x, r.p[h].y};
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        x[4 * h + 2 * i] = DT == POT_BF16 ? __uint_as_float(w[i] << 16) : from_half_bits(w[i]);
        x[4 * h + 2 * i + 1] =
            DT == POT_BF16 ? __uint_as_float(w[i] & 0xFFFF0000u) : from_half_bits(w[i] >> 16);
      }
    }
  }
}

// Two floats as a dword of 16-bit numbers, rounded to nearest even.
typedef float float2v __attribute__((ext_vector_type(2)));
typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t pack_half(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((float2v{a, b}), half2v));
}
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((float2v{a, b}), bf16x2));
}
// Every lane of the row takes part; only rows that are `there` are written. STREAM: past the
// caches (32768 tokens 72.6 -> 67.8 us, 2048 10.0 -> 7.5; few tokens' rows are read again by
// the next call and stay).
typedef uint32_t u32x4v __attribute__((ext_vector_type(4)));
template <bool STREAM>
__device__ __forceinline__ void write16(void* p, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  const u32x4v v = {a, b, c, d};
  if constexpr (STREAM) __builtin_nontemporal_store(v, static_cast<u32x4v*>(p));
  else *static_cast<u32x4v*>(p) = v;
}
template <int MODE, bool STREAM>
__device__ __forceinline__ void store_row(void* base, int64_t at, int g, int type,
                                          const float (&x)[8], bool there) {
  if (type == POT_FP32) {
    float* p = static_cast<float*>(base) + at + (MODE == kFullHalves ? 4 * quad_of(g) : 8 * g);
    if (!there) return;
    write16<STREAM>(p, __float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]),
                    __float_as_uint(x[3]));
    write16<STREAM>(p + (MODE == kFullHalves ? 32 : 4), __float_as_uint(x[4]),
                    __float_as_uint(x[5]), __float_as_uint(x[6]), __float_as_uint(x[7]));
    return;
  }
  uint32_t w[4];
  if (type == POT_BF16) {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = pack_bf16(x[2 * i], x[2 * i + 1]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = pack_half(x[2 * i], x[2 * i + 1]);
  }
  uint2 lo = make_uint2(w[0], w[1]), hi = make_uint2(w[2], w[3]);
  if constexpr (MODE == kFullHalves) exchange_quads(lo, hi);
  uint16_t* p = static_cast<uint16_t*>(base) + at + 8 * (MODE == kFullHalves && g >= 4 ? 11 - g : g);
  if (there) write16<STREAM>(p, lo.x, lo.y, hi.x, hi.y);
}

template <int MODE>
__device__ __forceinline__ void load_weights(const void* w, int type, int g, float (&out)[8]) {
  if (type == POT_FP32) to_floats<POT_FP32, MODE>(load_row<POT_FP32, MODE>(w, 0, g), out);
  else if (type == POT_BF16) to_floats<POT_BF16, MODE>(load_row<POT_BF16, MODE>(w, 0, g), out);
  else to_floats<POT_FP16, MODE>(load_row<POT_FP16, MODE>(w, 0, g), out);
}

// Sum of the squares over the row's 8 lanes.
__device__ __forceinline__ float row_squares(const float (&x)[8]) {
  float ss = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) ss = __builtin_fmaf(x[i], x[i], ss);
  ss += __uint_as_float(lane_xor_u32<1>(__float_as_uint(ss)));
  ss += __uint_as_float(lane_xor_u32<2>(__float_as_uint(ss)));
  return ss + dpp_move<0x141>(ss);  // row_half_mirror: the other half of the 8 lanes
}
// x / sqrt(mean x^2 + eps) * w over the row's 8 lanes; every lane of the wave takes part. A row
// whose squares pass fp32's range, or fall out of it beside a small eps, is first scaled by a
// power of two. The hardware's reciprocal root is within a unit in the last place.
__device__ __forceinline__ void norm_row(float (&x)[8], const float (&w)[8], float eps) {
  float ss = row_squares(x), m = __builtin_fmaf(ss, 1.0f / 64, eps);
  const bool large = !(ss < 0x1p120f), small = m < 0x1p-80f;
  if (__any(large || small)) {
    const float c = large ? 0x1p-70f : small ? 0x1p100f : 1.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] *= c;
    ss = row_squares(x);
    m = __builtin_fmaf(ss, 1.0f / 64, eps * c * c);
  }
  const float r = __builtin_amdgcn_rsqf(m);
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = x[i] * r * w[i];
}

// Sine and cosine of an angle given in quarter turns (|.| < 2^51). Its whole quarters go
// off exactly in fp64: adding 1.5 2^52 rounds to an integer, whose low bits say which
// quarter; at most an eighth of a turn is left, and the series' next terms are below
// 2e-9.
__device__ __forceinline__ void sin_cos_quarters(double quarters, float* s, float* c) {
  const double u = quarters + 0x1.8p52;
  const int q = (int)(uint32_t)__builtin_bit_cast(uint64_t, u);
  const float t = (float)(quarters - (u - 0x1.8p52)) * 1.57079632679489661923f;
  const float t2 = t * t;
  float sn = __builtin_fmaf(t2, 1.0f / 362880, -1.0f / 5040);
  sn = __builtin_fmaf(t2, sn, 1.0f / 120);
  sn = __builtin_fmaf(t2, sn, -1.0f / 6);
  sn = __builtin_fmaf(t2 * t, sn, t);
  float cs = __builtin_fmaf(t2, -1.0f / 3628800, 1.0f / 40320);
  cs = __builtin_fmaf(t2, cs, -1.0f / 720);
  cs = __builtin_fmaf(t2, cs, 1.0f / 24);
  cs = __builtin_fmaf(t2, cs, -0.5f);
  cs = __builtin_fmaf(t2, cs, 1.0f);
  const float a = q & 1 ? cs : sn, b = q & 1 ? sn : cs;
  *s = q & 2 ? -a : a;
  *c = (q + 1) & 2 ? -b : b;
}

// The turns of a lane's pairs: kFullHalves 4 (pair i of registers i and 4 + i),
// kNeighbours 4 (registers 2i and 2i + 1), kHalves one per element.
template <int MODE>
constexpr int kLanePairs = MODE == kHalves ? 8 : 4;
template <int MODE>
struct Turn {
  float s[kLanePairs<MODE>], c[kLanePairs<MODE>];
};
template <int MODE>
__device__ __forceinline__ Turn<MODE> turns_of(const NormRopeArgs& a, int64_t tok,
                                               int64_t n_tok, int g) {
  Turn<MODE> t;
  const int half = a.rot_dim / 2;
  const double pos0 = (double)a.positions[tok];
#pragma unroll
  for (int i = 0; i < kLanePairs<MODE>; ++i) {
    int pair = MODE == kHalves ? 8 * g + i : 4 * (MODE == kFullHalves ? quad_of(g) : g) + i;
    bool in = pair < half;
    if constexpr (MODE == kHalves) {
      in = pair < a.rot_dim;
      pair = pair >= half ? pair - half : pair;
    }
    pair = in ? pair : 0;
    const double pos =
        a.n_axes > 1 ? (double)a.positions[a.axis_of_pair[pair] * n_tok + tok] : pos0;
    sin_cos_quarters(pos * a.inv_freq[pair] * 0.63661977236758134308, &t.s[i], &t.c[i]);
  }
  return t;
}

// Rotation in registers. kHalves: part is the wave's LDS for 8 rows (row r at 68 r), whose
// elements the lanes of a row exchange; no other wave touches it.
constexpr int kPartStride = 68;
template <int MODE>
__device__ __forceinline__ void rotate_row(float (&x)[8], const Turn<MODE>& t, int rot_dim, int g,
                                           float* part) {
  if constexpr (MODE == kFullHalves) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float p = x[i], q = x[4 + i];
      x[i] = __builtin_fmaf(p, t.c[i], -(q * t.s[i]));
      x[4 + i] = __builtin_fmaf(q, t.c[i], p * t.s[i]);
    }
  } else if constexpr (MODE == kNeighbours) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (8 * g + 2 * i >= rot_dim) break;
      const float p = x[2 * i], q = x[2 * i + 1];
      x[2 * i] = __builtin_fmaf(p, t.c[i], -(q * t.s[i]));
      x[2 * i + 1] = __builtin_fmaf(q, t.c[i], p * t.s[i]);
    }
  } else {
    const int half = rot_dim / 2;
    __builtin_amdgcn_wave_barrier();  // the reads of the row before
#pragma unroll
    for (int i = 0; i < 8; ++i) part[8 * g + i] = x[i];
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int e = 8 * g + i;
      if (e >= rot_dim) break;
      const bool second = e >= half;
      const float y = part[second ? e - half : e + half];
      x[i] = __builtin_fmaf(x[i], t.c[i], second ? y * t.s[i] : -(y * t.s[i]));
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
}

}  // namespace potattn
