// RMS norm of queries and keys per head and the position rotation in one pass over a
// projection's rows, written as the cache writers and the decode calls take them.
#include <hip/hip_bf16.h>

#include "pot_device.hpp"

namespace potattn {

__device__ __forceinline__ float load_elem(const void* p, int64_t i, int dtype) {
  if (dtype == POT_FP32) return static_cast<const float*>(p)[i];
  const uint16_t u = static_cast<const uint16_t*>(p)[i];
  return dtype == POT_BF16 ? __uint_as_float((uint32_t)u << 16) : __half2float(__ushort_as_half(u));
}
__device__ __forceinline__ uint16_t to_bf16(float x) {
  return __builtin_bit_cast(uint16_t, __float2bfloat16(x));
}

// One wave per row, a lane per element.
__global__ __launch_bounds__(kBlock) void norm_rope_kernel(const NormRopeArgs a) {
  const int lane = lane_id(), heads = a.Hq + 2 * a.Hkv;
  const int64_t n = (int64_t)a.B * a.S * heads, stride = (int64_t)gridDim.x * (kBlock / 64);
  for (int64_t i = (int64_t)blockIdx.x * (kBlock / 64) +
                   __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
       i < n; i += stride) {
    const int64_t tok = i / heads, b = tok / a.S, t = tok - b * a.S;
    int h = (int)(i - tok * heads);
    const int kind = h < a.Hq ? 0 : h < a.Hq + a.Hkv ? 1 : 2;
    h -= kind == 0 ? 0 : kind == 1 ? a.Hq : a.Hq + a.Hkv;
    const RowsIn& in = kind == 0 ? a.q : kind == 1 ? a.k : a.v;
    if (in.data == nullptr) continue;
    float x = load_elem(in.data, b * in.stride_b + t * in.stride_s + h * in.stride_h + lane, a.dtype);
    const void* w = kind == 0 ? a.q_weight : kind == 1 ? a.k_weight : nullptr;
    if (w != nullptr) {
      float ss = x * x;
      for (int o = 32; o >= 1; o >>= 1) ss += __shfl_xor(ss, o, 64);
      x = x * (1.0f / sqrtf(ss * (1.0f / 64) + a.eps)) * load_elem(w, lane, a.weight_dtype);
    }
    if (kind < 2 && a.rot_dim > 0) {
      const int half = a.rot_dim / 2;
      const bool in_rot = lane < a.rot_dim;
      const int pair = !in_rot ? 0 : a.neighbours ? lane / 2 : lane % half;
      const bool second = a.neighbours ? (lane & 1) : lane >= half;
      const int other = !in_rot ? lane : a.neighbours ? lane ^ 1 : second ? lane - half : lane + half;
      const double turns = (double)a.positions[((int64_t)a.axis_of_pair[pair] * a.B + b) * a.S + t] *
                           a.inv_freq[pair] * 0.15915494309189533577;
      double sn, cs;
      sincospi(2.0 * (turns - rint(turns)), &sn, &cs);
      const float y = __shfl(x, other, 64);
      if (in_rot) x = second ? x * (float)cs + y * (float)sn : x * (float)cs - y * (float)sn;
    }
    const int64_t H = kind == 0 ? a.Hq : a.Hkv, at = ((b * H + h) * a.S + t) * kDim + lane;
    if (kind == 0 && a.q_out_dtype == POT_FP32) static_cast<float*>(a.q_out)[at] = x;
    else if (kind == 0 && a.q_out_dtype == POT_BF16) static_cast<uint16_t*>(a.q_out)[at] = to_bf16(x);
    else (kind == 0 ? static_cast<uint16_t*>(a.q_out) : kind == 1 ? a.k_out : a.v_out)[at] =
        __half_as_ushort(__float2half_rn(x));
  }
}

hipError_t launch_norm_rope(const NormRopeArgs& a, hipStream_t stream) {
  const int64_t blocks = ((int64_t)a.B * a.S * (a.Hq + 2 * a.Hkv) + 3) / 4;
  hipLaunchKernelGGL(norm_rope_kernel, dim3((uint32_t)(blocks < 16384 ? blocks : 16384)),
                     dim3(kBlock), 0, stream, a);
  return hipGetLastError();
}

}  // namespace potattn
