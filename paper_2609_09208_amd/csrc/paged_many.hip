// Many rows over a paged cache: the kernels of every key format and value format, and the merge
// of their key ranges.
#include "paged_many.hpp"

namespace potattn {

// O = sum_s 2^((m_s - M) c) o_s / sum_s 2^((m_s - M) c) l_s over the key ranges s of 16 rows.
__global__ __launch_bounds__(256) void paged_many_merge_kernel(const PagedAttendArgs a) {
  const int R = 32 * a.plan.many_waves, S = a.plan.many_splits;
  const int piece = blockIdx.x % (R / 16), kvh = blockIdx.y, index = blockIdx.x / (R / 16);
  const RowTile at = find_tile(a, index, R);
  if (at.b < 0) return;
  const NewTokens t = sequence_tokens(a.packed, at.b, a.max_new, a.max_len);
  const int in = 16 * piece + threadIdx.x / 16, r = at.tile * R + in, d = 4 * (threadIdx.x & 15);
  if (r >= t.n * a.G) return;
  const float* part = a.many_part + (((int64_t)index * a.pages.Hkv + kvh) * S * R + in) * kPartial;
  const int64_t next = (int64_t)R * kPartial;
  float M = kNoReference;
  for (int s = 0; s < S; ++s) M = fmaxf(M, part[s * next + kDim]);
  float L = 0.0f;
  f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int s = 0; s < S; ++s) {
    const f32x4 w = *reinterpret_cast<const f32x4*>(part + s * next + kDim);
    if (w[1] == 0.0f) continue;
    const float f = between(w[0], M, w[2]);
    L += f * w[1];
    o += f * *reinterpret_cast<const f32x4*>(part + s * next + d);
  }
  const int tok = r / a.G, head = a.q_head(kvh * a.G + (r - tok * a.G));
  const float inv = L == 0.0f ? 0.0f : 1.0f / L;
  store_out4(a.out, ((int64_t)(t.first + tok) * a.Hq + head) * kDim + d, a.out_dtype, o[0] * inv,
             o[1] * inv, o[2] * inv, o[3] * inv);
}

template <int VF, int NW>
static hipError_t launch_k(const PagedAttendArgs& a, hipStream_t stream) {
  switch (a.mant_bits) {
    case 0: return launch_many<0, VF, NW>(a, stream);
    case 1: return launch_many<1, VF, NW>(a, stream);
    case 2: return launch_many<2, VF, NW>(a, stream);
    case 3: return launch_many<3, VF, NW>(a, stream);
    default: return launch_many<4, VF, NW>(a, stream);
  }
}

hipError_t launch_paged_many(const PagedAttendArgs& a, hipStream_t stream) {
  const hipError_t e = a.plan.many_waves == 8
                           ? (a.value_format == POT_VALUES_INT4 ? launch_k<POT_VALUES_INT4, 8>(a, stream)
                                                                : launch_k<POT_VALUES_FP16, 8>(a, stream))
                           : (a.value_format == POT_VALUES_INT4 ? launch_k<POT_VALUES_INT4, 4>(a, stream)
                                                                : launch_k<POT_VALUES_FP16, 4>(a, stream));
  if (e != hipSuccess || a.plan.many_splits == 1) return e;
  hipLaunchKernelGGL(paged_many_merge_kernel,
                     dim3((uint32_t)(a.plan.many_tiles * (2 * a.plan.many_waves)), (uint32_t)a.pages.Hkv),
                     dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace potattn
