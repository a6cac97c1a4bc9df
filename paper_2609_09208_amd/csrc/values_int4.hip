// The 4-bit value store: rows in, records of 8 tokens out (layout and rounding in
// pot_device.hpp). 128 bytes read and 36 written per token: the memory stream.
#include "pot_device.hpp"
#include "row_groups.hpp"

namespace potattn {

// One wave per token: for one token of each sequence, which would leave seven lanes of eight
// of a record's wave idle (and for the append of the decode kernels).
__global__ __launch_bounds__(kBlock) void store_tokens_i4_kernel(
    const uint16_t* __restrict__ src, RowRange r, uint8_t* __restrict__ v_u4) {
  const uint32_t n = (uint32_t)(r.n_seq * r.n_tok), n_tok = (uint32_t)r.n_tok;
  for (uint32_t i = first_wave(); i < n; i += wave_stride()) {
    const uint32_t s = i / n_tok;
    store_value_token_i4_wave(src + (int64_t)i * kDim, v_u4 + s * r.t_cap * (kI4GroupBytes / 8),
                              r.t0 + (i - s * n_tok));
  }
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
  uint32_t d = upper ? (got | (b[1] << 4)) : (b[0] | (got << 4));
  d = transpose_tokens(d, lane);
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

// A wave takes up to REC records of a sequence, their rows requested together. The
// arithmetic, 130 operations a record, is as long as the stream, and indices and addresses
// are 70 more: four records a wave from kManyRecords on (2 M rows 68 us, one record a wave
// 80; 262144 11.9 and 12.7; 131072, with too few waves for four 9.1 and 8.1).
constexpr int64_t kManyRecords = 32768;
template <int REC>
__global__ __launch_bounds__(kBlock) void store_values_i4_kernel(
    const uint16_t* __restrict__ src, RowRange r, uint8_t* __restrict__ v_u4) {
  const int lane = lane_id(), u = lane >> 3;
  const uint32_t per_seq = (uint32_t)((r.n_groups + REC - 1) / REC);
  const uint32_t n = (uint32_t)r.n_seq * per_seq, n_tok = (uint32_t)r.n_tok;
  for (uint32_t i = first_wave(); i < n; i += wave_stride()) {
    const uint32_t seq = __builtin_amdgcn_readfirstlane(i / per_seq);
    const int64_t s = seq, g0 = (int64_t)(i - seq * per_seq) * REC;  // of the range
    const int records = (int)min((int64_t)REC, r.n_groups - g0);
    // first token of the first record, in the range (above -8)
    const int t_first = (int)((r.g_first + g0) * 8 - r.t0);
    const uint16_t* rows = src + (s * r.n_tok + t_first) * kDim;
    uint8_t* out = v_u4 + (s * (r.t_cap / 8) + r.g_first + g0) * kI4GroupBytes;
    uint4 v[REC];
    if (t_first >= 0 && (uint32_t)t_first + 8 * REC <= n_tok) {
#pragma unroll
      for (int c = 0; c < REC; ++c)
        v[c] = *reinterpret_cast<const uint4*>(rows + c * 8 * kDim + lane * 8);
#pragma unroll
      for (int c = 0; c < REC; ++c)
        store_record(v[c], out + c * kI4GroupBytes, lane, true, 0, 0, 0);
      continue;
    }
    for (int c = 0; c < records; ++c) {
      const int t = t_first + 8 * c + u;
      v[0] = make_uint4(0u, 0u, 0u, 0u);
      if ((uint32_t)t < n_tok) v[0] = *reinterpret_cast<const uint4*>(rows + c * 8 * kDim + lane * 8);
      store_record(v[0], out + c * kI4GroupBytes, lane, false, t, t_first + 8 * c + 4 * (lane >> 5),
                   n_tok);
    }
  }
}

hipError_t launch_store_values_i4(const uint16_t* src, int64_t n_seq, int64_t n_tok,
                                  int64_t t_cap, int64_t t0, uint8_t* v_u4, hipStream_t stream) {
  const RowRange r = row_range(n_seq, n_tok, t_cap, t0);
  if (n_tok == 1)
    hipLaunchKernelGGL(store_tokens_i4_kernel, blocks_of(n_seq * n_tok), dim3(kBlock), 0, stream,
                       src, r, v_u4);
  else if (n_seq * r.n_groups < kManyRecords)
    hipLaunchKernelGGL((store_values_i4_kernel<1>), blocks_of(n_seq * r.n_groups), dim3(kBlock), 0,
                       stream, src, r, v_u4);
  else
    hipLaunchKernelGGL((store_values_i4_kernel<4>), blocks_of(n_seq * ((r.n_groups + 3) / 4)),
                       dim3(kBlock), 0, stream, src, r, v_u4);
  return hipGetLastError();
}

}  // namespace potattn
