// Many rows over a paged cache: the kernels of every key format and value format, and the merge
// of their key ranges.
#include "paged_many.hpp"

namespace potattn {

// The same merge for the rows of a row tile, a wave per row. A row tile's rows are shared out among its
// pieces, kMergeParts workgroups for each.
constexpr int kMergeParts = 4;
__global__ __launch_bounds__(256) void paged_many_merge_kernel(const PagedAttendArgs a) {
  const int R = a.plan.many_rows, Hkv = a.pages.Hkv;
  const int index = blockIdx.x / kMergeParts, kvh = blockIdx.y;
  const int4 rec = a.many_pieces[index];
  const int b = rec.x, tile = rec.y, S = rec.z, first = rec.w;
  // bounds that do not ascend can ask for more pieces than there is room for
  if (b < 0 || S <= 1 || first < 0 || index < first || index >= first + S ||
      first + S > a.plan.many_tiles + a.plan.many_extra)
    return;
  const NewTokens t = sequence_tokens(a.packed, b, a.max_new, a.max_len);
  const int lane = threadIdx.x & 63, rows = min(R, t.n * a.G - tile * R);
  const int share = (index - first) * kMergeParts + blockIdx.x % kMergeParts, shares = S * kMergeParts;
  const int end = min(rows, (share + 1) * R / shares);
  const float* part = a.many_part + ((int64_t)first * Hkv + kvh) * R * kPartial;
  for (int in = share * R / shares + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); in < end; in += 4) {
    const Merged g = merge_parts(part + in * kPartial, Hkv * R * kPartial, S, lane);
    if (lane >= 16) continue;
    const int r = tile * R + in, tok = r / a.G, head = a.q_head(kvh * a.G + (r - tok * a.G));
    store_out4(a.out, ((int64_t)(t.first + tok) * a.Hq + head) * kDim + 4 * lane, a.out_dtype, g.o[0], g.o[1],
               g.o[2], g.o[3]);
  }
}

template <int VF, int R>
static hipError_t launch_k(const PagedAttendArgs& a, hipStream_t stream) {
  switch (a.mant_bits) {
    case 0: return launch_many<0, VF, R>(a, stream);
    case 1: return launch_many<1, VF, R>(a, stream);
    case 2: return launch_many<2, VF, R>(a, stream);
    case 3: return launch_many<3, VF, R>(a, stream);
    default: return launch_many<4, VF, R>(a, stream);
  }
}

template <int VF>
static hipError_t launch_rows(const PagedAttendArgs& a, hipStream_t stream) {
  return a.plan.many_rows == 256 ? launch_k<VF, 256>(a, stream) : launch_k<VF, 128>(a, stream);
}

hipError_t launch_paged_many(const PagedAttendArgs& a, hipStream_t stream) {
  const hipError_t e = a.value_format == POT_VALUES_INT4 ? launch_rows<POT_VALUES_INT4>(a, stream)
                                                         : launch_rows<POT_VALUES_FP16>(a, stream);
  if (e != hipSuccess || a.plan.many_extra == 0) return e;
  hipLaunchKernelGGL(paged_many_merge_kernel,
                     dim3((uint32_t)((a.plan.many_tiles + a.plan.many_extra) * kMergeParts), (uint32_t)a.pages.Hkv),
                     dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace potattn
