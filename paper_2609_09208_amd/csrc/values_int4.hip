// The 4-bit value store: rows in, groups of 8 tokens out (layout and rounding in
// pot_device.hpp). 128 bytes read and 36 written per token: the memory stream.
#include "pot_device.hpp"

namespace potattn {

// One wave per token.
__global__ __launch_bounds__(kBlock) void store_tokens_i4_kernel(
    const uint16_t* __restrict__ src, int64_t n, int64_t n_tok, int64_t t_cap, int64_t t0,
    uint8_t* __restrict__ v_u4) {
  const int64_t stride = (int64_t)gridDim.x * (kBlock / 64);
  for (int64_t i = (int64_t)blockIdx.x * (kBlock / 64) +
                   __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
       i < n; i += stride) {
    const int64_t s = i / n_tok;
    store_value_token_i4_wave(src + i * kDim, v_u4 + s * t_cap * (kI4GroupBytes / 8),
                              t0 + (i - s * n_tok));
  }
}

hipError_t launch_store_values_i4(const uint16_t* src, int64_t n_seq, int64_t n_tok,
                                  int64_t t_cap, int64_t t0, uint8_t* v_u4, hipStream_t stream) {
  const int64_t n = n_seq * n_tok;
  const dim3 grid((uint32_t)((n + 3) / 4 < 8192 ? (n + 3) / 4 : 8192));
  hipLaunchKernelGGL(store_tokens_i4_kernel, grid, dim3(kBlock), 0, stream, src, n, n_tok, t_cap,
                     t0, v_u4);
  return hipGetLastError();
}

}  // namespace potattn
