// Few rows over a paged cache: the kernels of every key format and value format, and the merge
// of their key ranges.
#include "paged_few.hpp"

namespace potattn {

// O = sum_s 2^((m_s - M) c) o_s / sum_s 2^((m_s - M) c) l_s over the key ranges s of a row.
__global__ __launch_bounds__(256) void paged_few_merge_kernel(const PagedAttendArgs a) {
  const int kvh = blockIdx.x, b = blockIdx.y, S = a.plan.few_splits;
  const NewTokens t = sequence_tokens(a.packed, b, a.max_new, a.max_len);
  if (t.n == 0 || t.n > a.plan.few_limit || t.n * a.G > a.plan.few_limit) return;
  const int r = threadIdx.x / 16, d = 4 * (threadIdx.x & 15);
  if (r >= t.n * a.G) return;
  const float* part = a.few_part + (((int64_t)b * a.pages.Hkv + kvh) * S * kFewRows + r) * kPartial;
  constexpr int kNext = kFewRows * kPartial;
  float M = kNoReference;
  for (int s = 0; s < S; ++s) M = fmaxf(M, part[(int64_t)s * kNext + kDim]);
  float L = 0.0f;
  f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int s = 0; s < S; ++s) {
    const f32x4 w = *reinterpret_cast<const f32x4*>(part + (int64_t)s * kNext + kDim);
    if (w[1] == 0.0f) continue;
    const float f = between(w[0], M, w[2]);
    L += f * w[1];
    o += f * *reinterpret_cast<const f32x4*>(part + (int64_t)s * kNext + d);
  }
  const int tok = r / a.G, head = a.q_head(kvh * a.G + (r - tok * a.G));
  const float inv = L == 0.0f ? 0.0f : 1.0f / L;
  store_out4(a.out, ((int64_t)(t.first + tok) * a.Hq + head) * kDim + d, a.out_dtype, o[0] * inv,
             o[1] * inv, o[2] * inv, o[3] * inv);
}

template <int VF>
static hipError_t launch_k(const PagedAttendArgs& a, hipStream_t stream) {
  switch (a.mant_bits) {
    case 0: return launch_few<0, VF>(a, stream);
    case 1: return launch_few<1, VF>(a, stream);
    case 2: return launch_few<2, VF>(a, stream);
    case 3: return launch_few<3, VF>(a, stream);
    default: return launch_few<4, VF>(a, stream);
  }
}

hipError_t launch_paged_few(const PagedAttendArgs& a, hipStream_t stream) {
  const hipError_t e = a.value_format == POT_VALUES_INT4 ? launch_k<POT_VALUES_INT4>(a, stream)
                                                         : launch_k<POT_VALUES_FP16>(a, stream);
  if (e != hipSuccess || a.plan.few_splits == 1) return e;
  hipLaunchKernelGGL(paged_few_merge_kernel, dim3((uint32_t)a.pages.Hkv, (uint32_t)a.packed.B), dim3(256),
                     0, stream, a);
  return hipGetLastError();
}

}  // namespace potattn
