// Decode kernels: values in 4 bits, shift-accumulate scores and PoT-4 codes decoded to
// fp16 weights.
#include "decode_kernel.hpp"

namespace potattn {

template hipError_t launch_mode_vf<kScorePot, 3>(int, int, bool, const DecodeArgs&, hipStream_t,
                                                 hipEvent_t, hipEvent_t);
template hipError_t launch_mode_vf<kScoreDs4a, 3>(int, int, bool, const DecodeArgs&, hipStream_t,
                                                 hipEvent_t, hipEvent_t);

}  // namespace potattn
