// Cache rows back to dense fp16 rows.
#include "pot_device.hpp"

namespace potattn {

struct LoadRange {
  int64_t n_seq, n_tok, t_cap, t0;
};

// One wave per row, a lane per element.
template <int K>
__global__ __launch_bounds__(kBlock) void load_keys_kernel(
    const uint8_t* __restrict__ codes_se, const uint8_t* __restrict__ codes_m,
    const float* __restrict__ key_scale, LoadRange r, int hadamard, uint16_t* __restrict__ out) {
  const int lane = lane_id();
  const int64_t n = r.n_seq * r.n_tok, stride = (int64_t)gridDim.x * (kBlock / 64);
  for (int64_t i = (int64_t)blockIdx.x * (kBlock / 64) +
                   __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
       i < n; i += stride) {
    const int64_t s = i / r.n_tok, row = s * r.t_cap + r.t0 + (i - s * r.n_tok);
    const int f = (codes_se[row * 32 + lane / 2] >> (4 * (lane & 1))) & 15;
    int j = 0;
    for (int b = 0; b < K; ++b)
      j |= ((codes_m[row * 8 * K + 8 * b + lane / 8] >> (lane & 7)) & 1) << b;
    float x = 0.0f;
    if ((f & 7) != kZeroField)
      x = __fmul_rn(key_scale[row],
                    __builtin_amdgcn_ldexpf((float)((1 << K) + j) * (f & 8 ? -1.0f : 1.0f), -K - (f & 7)));
    if (hadamard) x = (float)(wave_fwht64((double)x) * 0.125);
    out[i * kDim + lane] = __half_as_ushort(__float2half_rn(x));
  }
}

__global__ __launch_bounds__(kBlock) void load_values_kernel(
    int fmt, const void* __restrict__ cache, const int8_t* __restrict__ v_exp, LoadRange r,
    uint16_t* __restrict__ out) {
  const int64_t n = r.n_seq * r.n_tok * kDim, stride = (int64_t)gridDim.x * kBlock;
  for (int64_t e = (int64_t)blockIdx.x * kBlock + threadIdx.x; e < n; e += stride) {
    const int64_t i = e / kDim, s = i / r.n_tok, t = r.t0 + (i - s * r.n_tok);
    const int d = (int)(e % kDim), u = (int)(t % 8);
    const int64_t at = (s * r.t_cap + t - u) * kDim + d * 8 + u;
    float x;
    if (fmt == 0) {
      out[e] = static_cast<const uint16_t*>(cache)[at];
      continue;
    } else if (fmt == 1) {
      x = __builtin_amdgcn_ldexpf((float)(static_cast<const uint8_t*>(cache)[at] - 128),
                                  -v_exp[s * r.t_cap + t]);
    } else {
      const uint8_t* g = static_cast<const uint8_t*>(cache) + (s * r.t_cap + t - u) / 8 * kI4GroupBytes;
      const int b = g[16 * (d & 15) + 8 * (d >> 5) + u];
      const float st = __half2float(reinterpret_cast<const __half*>(g + kI4Steps)[u]);
      const float z = __half2float(reinterpret_cast<const __half*>(g + kI4Minima)[u]);
      x = __builtin_fmaf((float)(d & 16 ? b >> 4 : b & 15), st, z);
    }
    out[e] = __half_as_ushort(__float2half_rn(x));
  }
}

static dim3 grid_for(int64_t blocks) { return dim3((uint32_t)(blocks < 16384 ? blocks : 16384)); }

hipError_t launch_load_keys(int mant_bits, int hadamard, const uint8_t* codes_se,
                            const uint8_t* codes_m, const float* key_scale, int64_t n_seq,
                            int64_t n_tok, int64_t t_cap, int64_t t0, uint16_t* k,
                            hipStream_t stream) {
  const LoadRange r{n_seq, n_tok, t_cap, t0};
  const dim3 grid = grid_for((n_seq * n_tok + 3) / 4);
  switch (mant_bits) {
#define POT_CASE(KK)                                                                             \
  case KK:                                                                                       \
    hipLaunchKernelGGL((load_keys_kernel<KK>), grid, dim3(kBlock), 0, stream, codes_se, codes_m, \
                       key_scale, r, hadamard, k);                                               \
    break;
    POT_CASE(0) POT_CASE(1) POT_CASE(2) POT_CASE(3) POT_CASE(4)
#undef POT_CASE
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

hipError_t launch_load_values(int fmt, const void* cache, const int8_t* v_exp, int64_t n_seq,
                              int64_t n_tok, int64_t t_cap, int64_t t0, uint16_t* v,
                              hipStream_t stream) {
  const LoadRange r{n_seq, n_tok, t_cap, t0};
  hipLaunchKernelGGL(load_values_kernel, grid_for((n_seq * n_tok * kDim + 255) / 256),
                     dim3(kBlock), 0, stream, fmt, cache, v_exp, r, v);
  return hipGetLastError();
}

}  // namespace potattn
