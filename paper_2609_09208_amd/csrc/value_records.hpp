// A record of the 4-bit value store from 8 tokens' rows in registers (values_int4.hip,
// paged_append.hip).
#pragma once

#include "row_groups.hpp"

namespace potattn {

// A token's n over its 8 lanes as the bytes that the record has them in: lane g gets columns
// 8 (g % 2) + 4 (g / 2 % 2) + j (j = 0 .. 3, byte j) of half g / 4. Its step and minimum too.
__device__ __forceinline__ uint32_t record_columns(const uint4 v, int lane, uint16_t* step_out,
                                                   float* lo_out) {
  const int g = lane & 7;
  const uint32_t w4[4] = {v.x, v.y, v.z, v.w};
  float x[8];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    x[2 * k] = __half2float(__ushort_as_half((unsigned short)(w4[k] & 0xFFFFu)));
    x[2 * k + 1] = __half2float(__ushort_as_half((unsigned short)(w4[k] >> 16)));
  }
  // the maximum of x and of -x over the token's 8 lanes; fmaxf passes over NaN
  float hi = x[0], nlo = -x[0];
#pragma unroll
  for (int k = 1; k < 8; ++k) {
    hi = fmaxf(hi, x[k]);
    nlo = fmaxf(nlo, -x[k]);
  }
  hi = fmaxf(hi, dpp_move<0xB1>(hi));
  nlo = fmaxf(nlo, dpp_move<0xB1>(nlo));
  hi = fmaxf(hi, dpp_move<0x4E>(hi));
  nlo = fmaxf(nlo, dpp_move<0x4E>(nlo));
  hi = fmaxf(hi, dpp_move<0x141>(hi));
  nlo = fmaxf(nlo, dpp_move<0x141>(nlo));
  // infinite ends are the largest finite numbers; infinite elements then come out as n = 0
  // or 15 by the median below
  const bool any = hi == hi;
  hi = any ? __builtin_amdgcn_fmed3f(hi, -65504.0f, 65504.0f) : 0.0f;
  const float lo = any ? __builtin_amdgcn_fmed3f(-nlo, -65504.0f, 65504.0f) : 0.0f;
  const uint16_t step = value_step_i4(lo, hi);
  const float inv = step_reciprocal(__half2float(__ushort_as_half(step)));
  // n as the low byte of 1.5 2^23 + n: the addition rounds to nearest even; the median of
  // a NaN and 0 .. 15 is 0
  uint32_t m[8], b[2];
#pragma unroll
  for (int k = 0; k < 8; ++k)
    m[k] = __float_as_uint(__builtin_amdgcn_fmed3f(__fmul_rn(x[k] - lo, inv), 0.0f, 15.0f) +
                           12582912.0f);
#pragma unroll
  for (int h = 0; h < 2; ++h)
    b[h] = __builtin_amdgcn_perm(
        __builtin_amdgcn_perm(m[4 * h + 3], m[4 * h + 2], 0x0C0C0400u),
        __builtin_amdgcn_perm(m[4 * h + 1], m[4 * h], 0x0C0C0400u), 0x05040100u);
  // bytes of dimension pairs (c, c + 16): lane bit 1 is that of the 16
  const bool upper = (g & 2) != 0;
  const uint32_t got = lane_xor_u32<2>(upper ? b[0] : b[1]);
  *step_out = step;
  *lo_out = lo;
  return upper ? (got | (b[1] << 4)) : (b[0] | (got << 4));
}

// A record of 8 tokens by a wave. Lane l has dimensions 8g .. 8g + 7 (g = l % 8) of token
// l / 8, 16 bytes; a group is one contiguous KiB. Its 8 lanes find the token's minimum and
// maximum. The n of lanes g and g ^ 2 (dimensions 16 apart) share bytes: each of the two
// makes four of the eight (one exchange), and two exchanges over the token's low bits then
// give every lane a dword of four tokens, 4 bytes of the record's 256. t: the lane's token
// in the range, first: that of its dword's first; n_tok for uint32 comparisons, full: all
// eight are there (uniform).
__device__ __forceinline__ void store_record(const uint4 v, uint8_t* __restrict__ out, int lane,
                                             bool full, int t, int first, uint32_t n_tok) {
  const int g = lane & 7, u = lane >> 3;
  uint16_t step;
  float lo;
  const uint32_t d = transpose_tokens(record_columns(v, lane, &step, &lo), lane);
  const int at = record_offset(lane);
  if (full) {
    *reinterpret_cast<uint32_t*>(out + at) = d;
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if ((uint32_t)(first + k) < n_tok) out[at + k] = (uint8_t)(d >> (8 * k));
  }
  // lane g = 0 has the token's step, g = 1 its minimum
  const uint16_t sz = g == 0 ? step : __half_as_ushort(__float2half_rn(lo));
  if (g < 2 && (full || (uint32_t)t < n_tok))
    *reinterpret_cast<uint16_t*>(out + kI4Steps + 16 * g + 2 * u) = sz;
}

}  // namespace potattn
