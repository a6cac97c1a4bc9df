// The 4-bit value store: rows in, records of 8 tokens out (layout and rounding in
// pot_device.hpp). 128 bytes read and 36 written per token: the memory stream.
#include "pot_device.hpp"
#include "row_groups.hpp"
#include "value_records.hpp"

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
