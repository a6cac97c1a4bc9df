// Rows t0 .. t0 + n_tok - 1 of every sequence of a cache by groups of 8 tokens, and the
// byte exchange between the 4-bit records' order and tokens' order.
#pragma once

#include "pot_device.hpp"

namespace potattn {

struct RowRange {
  int64_t n_seq, n_tok, t_cap, t0, g_first, n_groups;
};
static inline RowRange row_range(int64_t n_seq, int64_t n_tok, int64_t t_cap, int64_t t0) {
  return {n_seq, n_tok, t_cap, t0, t0 / 8, (t0 + n_tok - 1) / 8 - t0 / 8 + 1};
}

// The waves of a launch in order, and their number: a dispatch holds 2^32 work-items, so
// its waves step over longer ranges.
__device__ __forceinline__ uint32_t first_wave() {
  return blockIdx.x * (kBlock / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
}
__device__ __forceinline__ uint32_t wave_stride() { return gridDim.x * (kBlock / 64); }
static inline dim3 blocks_of(int64_t waves) {
  const int64_t blocks = (waves + kBlock / 64 - 1) / (kBlock / 64), most = 1 << 20;
  return dim3((uint32_t)(blocks < most ? blocks : most));
}

// Lane l = 8 u + g, u the token, has the bytes of four dimension pairs j = 0 .. 3 of its
// token; afterwards lane bits 4 and 3 are j, bit 5 the upper four tokens, and its bytes are
// those four tokens. Its own inverse: one exchange of byte index bit 1 with lane bit 4
// (v_permlane16_swap) and one of bit 0 with lane bit 3 (row_ror:8).
__device__ __forceinline__ uint32_t transpose_tokens(uint32_t d, int lane) {
  const auto r = __builtin_amdgcn_permlane16_swap(d, d, false, false);
  // r[0]: the even row's dword in both rows, r[1]: the odd row's
  d = __builtin_amdgcn_perm(r[1], r[0], (lane >> 4) & 1 ? 0x07060302u : 0x05040100u);
  return __builtin_amdgcn_perm(lane_xor_u32<8>(d), d, (lane >> 3) & 1 ? 0x03070105u : 0x06020400u);
}
// Where that dword stands in its record: lane g works on the byte columns 8 (g % 2) +
// 4 (g / 2 % 2) + j of half g / 4.
__device__ __forceinline__ int record_offset(int lane) {
  const int g = lane & 7, j = 2 * ((lane >> 4) & 1) + ((lane >> 3) & 1);
  return 16 * (8 * (g & 1) + 4 * ((g >> 1) & 1) + j) + 8 * (g >> 2) + 4 * (lane >> 5);
}

}  // namespace potattn
