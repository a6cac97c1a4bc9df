// Few rows over a paged cache: the kernels of every key format and value format, and the merge
// of their key ranges.
#include "paged_few.hpp"

namespace potattn {

// O = sum_s 2^((m_s - M) c) o_s / sum_s 2^((m_s - M) c) l_s over the key ranges s of a row: a wave
// per row, 4 ranges at a time by its 16-lane rows, of 4 dimensions a lane. Every load of 16 ranges
// is under way before the first is used.
__global__ __launch_bounds__(256) void paged_few_merge_kernel(const PagedAttendArgs a) {
  const int kvh = blockIdx.x / (kFewRows / 4), b = blockIdx.y, S = a.plan.few_splits;
  const NewTokens t = sequence_tokens(a.packed, b, a.max_new, a.max_len);
  if (t.n == 0 || t.n > a.plan.few_limit || t.n * a.G > a.plan.few_limit) return;
  const int lane = threadIdx.x & 63;
  const int r = 4 * (blockIdx.x % (kFewRows / 4)) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (r >= t.n * a.G) return;
  const float* part = a.few_part + (((int64_t)b * a.pages.Hkv + kvh) * S * kFewRows + r) * kPartial;
  constexpr int kNext = kFewRows * kPartial;
  const Merged g = merge_parts(part, kNext, S, lane);
  if (lane >= 16) return;
  const int tok = r / a.G, head = a.q_head(kvh * a.G + (r - tok * a.G));
  store_out4(a.out, ((int64_t)(t.first + tok) * a.Hq + head) * kDim + 4 * lane, a.out_dtype, g.o[0], g.o[1],
             g.o[2], g.o[3]);
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
  hipLaunchKernelGGL(paged_few_merge_kernel, dim3((uint32_t)a.pages.Hkv * (kFewRows / 4), (uint32_t)a.packed.B), dim3(256),
                     0, stream, a);
  return hipGetLastError();
}

}  // namespace potattn
