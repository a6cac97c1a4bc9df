// Key rows to codes in registers: 8 lanes to a row, 8 elements to a lane, a code word each
// (encode.hip has the scheme; paged_append.hip uses it too).
#pragma once

#include "pot_device.hpp"

namespace potattn {

// Maximum over the 8 lanes of an aligned group (lane & ~7) of non-negative,
// non-NaN floats, compared as their bit patterns: swap neighbours, swap
// pairs, then the mirror image inside each half row (a maximum does not care
// which lane of the other quad it meets).
template <int kCtrl>
__device__ __forceinline__ uint32_t dpp_u32(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_mov_dpp((int)x, kCtrl, 0xF, 0xF, true);
}
__device__ __forceinline__ float max_over_8_lanes(float v) {
  constexpr int kQuadSwap1 = 0xB1, kQuadSwap2 = 0x4E, kRowHalfMirror = 0x141;
  uint32_t b = __float_as_uint(v);
  b = max(b, dpp_u32<kQuadSwap1>(b));
  b = max(b, dpp_u32<kQuadSwap2>(b));
  return __uint_as_float(max(b, dpp_u32<kRowHalfMirror>(b)));
}

// Scales whose reciprocal takes the fast path: [2^-126, 2^126] (no NaN,
// sign, infinity or subnormal reciprocal), by one unsigned compare.
__device__ __forceinline__ bool recip_in_range(float s) {
  return __float_as_uint(s) - 0x00800000u <= 0x7E800000u - 0x00800000u;
}

// RN(1 / s) for s in [2^-126, 2^126]: v_rcp_f32 is within one ulp, and one
// Newton step with fused multiply-adds then rounds correctly for every start
// within an ulp, except for an all-ones mantissa, s = (2 - 2^-23) 2^k, where
// the step can land on a tie: there 1/s = 2^-(k+1) (1 + 2^-24 + 2^-48 ...)
// rounds to 2^-(k+1) (1 + 2^-23), whose bits are 0x7E800001 minus the
// exponent field of s. (Checked over every mantissa of one binade and every
// start within an ulp.)
__device__ __forceinline__ float recip_rn(float s) {
  const float r0 = __builtin_amdgcn_rcpf(s);
  const float r1 = __builtin_fmaf(__builtin_fmaf(-s, r0, 1.0f), r0, r0);
  const uint32_t sb = __float_as_uint(s);
  return ((sb & 0x007FFFFFu) == 0x007FFFFFu) ? __uint_as_float(0x7E800001u - (sb & 0x7F800000u))
                                               : r1;
}

// Clamp to [0, 1] with NaN mapped to 0: folds into the producing
// instruction's clamp bit (the DX10 clamp mode, on for compute kernels).
__device__ __forceinline__ float clamp01(float x) { return __builtin_amdgcn_fmed3f(x, 0.0f, 1.0f); }

// Nibble masks of 8 signs: nibble i of the result is 0xF where bytes a (signs
// 0..3) and b (signs 4..7), each 0x00 or 0xFF, say sign i is set.
__device__ __forceinline__ uint32_t sign_nibbles(uint32_t a, uint32_t b) {
  const uint32_t even = __builtin_amdgcn_perm(b, a, 0x06040200u);  // signs 0 2 4 6
  const uint32_t odd = __builtin_amdgcn_perm(b, a, 0x07050301u);   // signs 1 3 5 7
  return (even & 0x0F0F0F0Fu) | (odd & 0xF0F0F0F0u);
}

// PoT-4 code word of 8 elements from their clamped ratios c_i = min(RN(|x_i|
// / s), 1) (0 for NaN) and sign masks. With c = (1 + M 2^-23) 2^(E-127) and
// the cut point RD(sqrt 2) = 1 + Mc 2^-23, the log-nearest exponent is
// e = 127 - (E + [M > Mc]) and the ratio is at or below the zero cut
// RD(sqrt 2) 2^-(E_max+1) exactly when E + [M > Mc] <= 127 - (E_max + 1).
// Adding 2^23 - 1 - Mc to the bits carries into the exponent exactly when
// M > Mc, so G = clamp((bits + 2^23 - 1 - Mc - (120 << 23)) >> 23, 0, 7)
// is 0 for zero and 7 - e otherwise (E_max = 6, c <= 1 saturates at e = 0).
// The word holds 7 - G per nibble, with the sign bit where G > 0.
__device__ __forceinline__ uint32_t pot4_word(const float (&c)[8], uint32_t sgn, uint32_t cst) {
  uint32_t w = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int t = (int)(__float_as_uint(c[i]) + cst) >> 23;
    const uint32_t gi = (uint32_t)min(max(t, 0), 7);
    w |= gi << (4 * i);
  }
  return (w ^ 0x77777777u) | (sgn & (w + 0x77777777u) & 0x88888888u);
}

// PoT-Mk code word and mantissa-plane bytes of 8 elements from their clamped
// half ratios v_i = min(RN(|x_i| / (2 s)), 1) (0 for NaN): ratios up to 2 on
// the unit interval, so that caller scales with |x| / s in [1, 2) still see
// their mantissa. With v = (1 + M 2^-23) 2^(E-127) and m = 1 + M 2^-23, the top
// K bits of M are j0, t = floor(m 2^k) = 2^k + j0, and m lies above the cut
// between grid points j0 and j0 + 1, RD(sqrt(t (t + 1)) / 2^k), exactly when
// (m 2^k)^2 > t (t + 1) (the root is irrational), which one fused multiply-add
// decides by its sign. E and j0 stand next to each other in v's bits, so adding
// that decision to the bits above them carries from the last grid point into
// the next binade by itself: u = (E - 119) 2^k + j0 + [above], clamped to 2^k
// .. 2^(k+3) - 1 (ratios past the top value and below the smallest magnitude)
// and 0 for a ratio at or below the zero cut, holds 7 - e above the mantissa.
// (Deciding exponent and mantissa apart took about 20 operations per element,
// this 14: 2 M rows k = 1 85 -> 81, k = 4 109 -> 96 us.) The u's are packed a byte
// each (bytes of a: elements 0..3, of b: 4..7), so exponents and mantissas come
// apart four at a time, and the mantissa nibbles (bit i of plane b: bit b of
// element i's j) become plane bytes by two exchanges of bits between bytes, all
// planes at once (a nibble each and a bit gather per plane: k = 1 80, k = 4 95 us;
// now 77 and 83).
// Returns the code word (signs as in pot4_word); byte b of planes is plane b's,
// bytes from K on hold no plane.
template <int K>
__device__ __forceinline__ uint32_t potmk_word(const float (&v)[8], uint32_t sgn,
                                               uint32_t zc_half, uint32_t& planes) {
  constexpr int n = 1 << K;
  uint32_t a = 0, b = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t vb = __float_as_uint(v[i]);
    const float mn = __uint_as_float((vb & 0x007FFFFFu) | ((127u + K) << 23));  // m 2^k
    const float t = truncf(mn);                  // 2^k + j0
    const float p = __builtin_fmaf(t, t, t);     // t (t + 1) <= 992, exact
    const int above = __builtin_fmaf(mn, mn, -p) > 0.0f ? 1 : 0;
    const int q = ((int)(vb - (119u << 23)) >> (23 - K)) + above;
    uint32_t u = (uint32_t)min(max(q, n), 8 * n - 1);
    u = vb > zc_half ? u : 0u;
    if (i < 4) a |= u << (8 * i);
    else b |= u << (8 * i - 32);
  }
  const uint32_t even = __builtin_amdgcn_perm(b, a, 0x06040200u);
  const uint32_t odd = __builtin_amdgcn_perm(b, a, 0x07050301u);
  const uint32_t w = ((even >> K) & 0x07070707u) | (((odd >> K) & 0x07070707u) << 4);
  // bit 8c + 4h + b of x: bit b of element 4h + c; exchange index bit 0 with 3, 1 with 4
  uint32_t x = (a & 0x0F0F0F0Fu) | ((b << 4) & 0xF0F0F0F0u);
  uint32_t t = (x ^ (x >> 7)) & 0x00AA00AAu;
  x ^= t ^ (t << 7);
  t = (x ^ (x >> 14)) & 0x0000CCCCu;
  planes = x ^ t ^ (t << 14);
  return (w ^ 0x77777777u) | (sgn & (w + 0x77777777u) & 0x88888888u);
}

// 8 elements 8g .. 8g + 7 (g = lane % 8) of a row from their fp16 words, with
// the optional rotation over the row's 8 lanes: butterflies over bits 0..2 of
// the element in registers, over bits 0..2 of g across lanes; fp16 inputs keep
// every fp64 sum exact.
template <bool HAD>
__device__ __forceinline__ void unpack_row(const uint32_t (&w4)[4], int lane, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __half2float(__ushort_as_half((unsigned short)(w4[i] & 0xFFFFu)));
    x[2 * i + 1] = __half2float(__ushort_as_half((unsigned short)(w4[i] >> 16)));
  }
  if constexpr (HAD) {
    const double sign1 = butterfly_sign<1>(lane), sign2 = butterfly_sign<2>(lane),
                 sign4 = butterfly_sign<4>(lane);
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
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = butterfly<1>(v[i], sign1);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = butterfly<2>(v[i], sign2);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = butterfly<4>(v[i], sign4);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (float)(v[i] * 0.125);
  }
}

// The plane bytes of each lane of a quad (byte b: plane b; code words 4h .. 4h + 3 of a row)
// to one dword of plane j in lane j: a 4 x 4 byte transpose by two DPP moves
// and byte permutes, for one dword store per lane. (With a byte store per lane
// and plane 2 M rows at k = 4 took 117 us, so 108.)
__device__ __forceinline__ uint32_t quad_planes(uint32_t w, int lane) {
  w = __builtin_amdgcn_perm(lane_xor_u32<1>(w), w, lane & 1 ? 0x03070105u : 0x06020400u);
  return __builtin_amdgcn_perm(lane_xor_u32<2>(w), w, lane & 2 ? 0x03020706u : 0x05040100u);
}

// The bits-to-G offset of pot4_word (Mc from the fp32 cut point) and half the
// zero cut.
struct CutBits {
  uint32_t cst, zc_half;
};
__device__ __forceinline__ CutBits cut_bits(const EncodeTables& tab) {
  return {0x007FFFFFu - (__float_as_uint(tab.cut[0]) & 0x007FFFFFu) - (120u << 23),
          __float_as_uint(tab.zero_cut) - (1u << 23)};
}

// Sign nibbles of 8 fp32 numbers (selector 9 / 11: bit 31 of the low / high
// source, 12: zero byte).
__device__ __forceinline__ uint32_t float_signs(const float* x) {
  uint32_t xb[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) xb[i] = __float_as_uint(x[i]);
  return sign_nibbles(__builtin_amdgcn_perm(xb[1], xb[0], 0x0C0C0B09u) |
                          __builtin_amdgcn_perm(xb[3], xb[2], 0x0B090C0Cu),
                      __builtin_amdgcn_perm(xb[5], xb[4], 0x0C0C0B09u) |
                          __builtin_amdgcn_perm(xb[7], xb[6], 0x0B090C0Cu));
}

// A row's scale as its elements use it.
// The clamped ratio c = min(RN(|x| / ss), 1) per element (ss = s for PoT-4, 2 s
// for PoT-Mk), NaN -> 0 (zero code), comes from one correctly rounded reciprocal
// per row; other scales (zero, negative, NaN, infinite, or too small or too
// large for a normal reciprocal) divide instead. The quotient q = RN(|x| r) is
// clamped too: min(q, 1) is still within an ulp of a quotient below 1, any q >=
// 1 gives c >= 1, and an infinite or NaN q (infinite or NaN x) cannot poison
// the residual.
struct RowScale {
  float s, ss, r;
  bool fast;
};
template <int K>
__device__ __forceinline__ RowScale row_scale(float s) {
  const float ss = K == 0 ? s : 2.0f * s;
  return {s, ss, recip_rn(ss), recip_in_range(ss)};
}

// Code word and plane bytes (byte b: plane b) of 8 elements.
template <int K>
__device__ __forceinline__ uint32_t encode_word(const float* x, const RowScale& sc, uint32_t sgn,
                                                const CutBits& cut, uint32_t& planes) {
  float c[8];
  if (sc.fast) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float a = fabsf(x[i]);
      const float q = clamp01(a * sc.r);
      c[i] = clamp01(__builtin_fmaf(__builtin_fmaf(-q, sc.ss, a), sc.r, q));
    }
  } else {
    // (|x| / 2) / s rounds as |x| / (2 s) and stays finite-safe for huge s
#pragma unroll
    for (int i = 0; i < 8; ++i)
      c[i] = (sc.s > 0.0f) ? clamp01((K == 0 ? fabsf(x[i]) : fabsf(x[i]) * 0.5f) / sc.s) : 0.0f;
  }
  if constexpr (K == 0) return pot4_word(c, sgn, cut.cst);
  else return potmk_word<K>(c, sgn, cut.zc_half, planes);
}

}  // namespace potattn
