// RMS norm of queries and keys per head and the position rotation in one pass over a
// projection's rows, written as the cache writers and the decode calls take them.
//
//   y = x / sqrt(mean x^2 + eps) * w,   (a, b) -> (a cos f - b sin f, b cos f + a sin f)
//
// A row is one head of one token: 64 elements over 8 lanes, 8 rows a wave. The bound is
// the memory stream (every row read and written once); the sum of squares takes three
// DPP steps, and where the halves of a head are paired over its full width a lane works
// on four elements of either half, so that pairs meet in registers. Halves of a part of the
// head meet through LDS and make every angle twice: 32768 tokens of bf16 66.2 us with 32 and
// 67.0 with 48 elements turned, against 65.8 with all 64.
#include "head_rows.hpp"
#include "pot_device.hpp"

namespace potattn {
// Many tokens: a wave takes 8 tokens, a row of 8 lanes each, and goes through a chunk of
// heads, so that the turns (fp64 angles, series) are made once for all of them. Writes
// are 8 tokens of a head side by side.
template <int DT, int MODE>
__global__ __launch_bounds__(kBlock) void norm_rope_tokens_kernel(const NormRopeArgs a,
                                                                  int heads, int chunk,
                                                                  int n_chunks) {
  __shared__ float part[MODE == kHalves ? kBlock / 64 * 8 * kPartStride : 1];
  const int lane = lane_id(), g = lane & 7, row = lane >> 3;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t unit = (int64_t)blockIdx.x * (kBlock / 64) + wave;
  const int64_t n_tok = (int64_t)a.B * a.S;
  const int64_t group = unit / n_chunks;
  if (group * 8 >= n_tok) return;
  const int h_first = (int)(unit - group * n_chunks) * chunk, h_end = min(h_first + chunk, heads);
  const int64_t tok = min(group * 8 + row, n_tok - 1);
  const bool there = group * 8 + row < n_tok;
  const int64_t b = (uint64_t)tok / (uint32_t)a.S, s = tok - b * a.S;
  float* my_part = part + (MODE == kHalves ? (wave * 8 + row) * kPartStride : 0);

  const int qk_end = a.Hq + a.Hkv;
  const bool turns = a.rot_dim > 0 && h_first < qk_end;
  Turn<MODE> t{};
  // Heads lo .. hi - 1 of the chunk belong to one part of the projection, whose first
  // head is `first`; kAhead rows are under way while one is worked on.
  constexpr int kAhead = 2;
  auto part_of = [&](const RowsIn& in, const void* weight, void* out, int out_type, int first,
                     int H, bool turn, bool make_turns) {
    const int lo = max(h_first, first) - first, hi = min(h_end, first + H) - first;
    if (lo >= hi || out == nullptr) return;
    const int64_t src = b * in.stride_b + s * in.stride_s;
    int64_t dst = ((b * H + lo) * a.S + s) * kDim;
    RawRow<DT> ahead[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
      ahead[i] = load_row<DT, MODE>(in.data, src + min(lo + i, hi - 1) * in.stride_h, g);
    float w[8];
    if (weight != nullptr) load_weights<MODE>(weight, a.weight_dtype, g, w);
    if (make_turns) t = turns_of<MODE>(a, tok, n_tok, g);
    for (int h = lo; h < hi; h += kAhead) {
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        if (h + i >= hi) break;  // uniform
        float x[8];
        to_floats<DT, MODE>(ahead[i], x);
        ahead[i] = load_row<DT, MODE>(in.data, src + min(h + i + kAhead, hi - 1) * in.stride_h, g);
        if (weight != nullptr) norm_row(x, w, a.eps);
        if (turn) rotate_row<MODE>(x, t, a.rot_dim, g, my_part);
        store_row<MODE, true>(out, dst, g, out_type, x, there);
        dst += (int64_t)a.S * kDim;
      }
    }
  };
  const bool q_rows = h_first < a.Hq;
  part_of(a.q, a.q_weight, a.q_out, a.q_out_dtype, 0, a.Hq, turns, turns && q_rows);
  part_of(a.k, a.k_weight, a.k_out, POT_FP16, a.Hq, a.Hkv, turns, turns && !q_rows);
  part_of(a.v, nullptr, a.v_out, POT_FP16, qk_end, a.Hkv, false, false);
}

// Few tokens: a wave takes 8 heads of one token.
template <int DT, int MODE>
__global__ __launch_bounds__(64) void norm_rope_heads_kernel(const NormRopeArgs a, int heads,
                                                             int n_groups) {
  __shared__ float part[MODE == kHalves ? 8 * kPartStride : 1];
  const int lane = lane_id(), g = lane & 7, row = lane >> 3;
  const int64_t tok = blockIdx.x / (uint32_t)n_groups;
  const int h = (int)(blockIdx.x - tok * n_groups) * 8 + row;
  const int64_t b = (uint64_t)tok / (uint32_t)a.S, s = tok - b * a.S;
  const int kind = h < a.Hq ? 0 : h < a.Hq + a.Hkv ? 1 : 2;
  const int hh = h - (kind == 0 ? 0 : kind == 1 ? a.Hq : a.Hq + a.Hkv);
  const void* data = kind == 0 ? a.q.data : kind == 1 ? a.k.data : a.v.data;
  const int64_t sb = kind == 0 ? a.q.stride_b : kind == 1 ? a.k.stride_b : a.v.stride_b;
  const int64_t ss = kind == 0 ? a.q.stride_s : kind == 1 ? a.k.stride_s : a.v.stride_s;
  const int64_t sh = kind == 0 ? a.q.stride_h : kind == 1 ? a.k.stride_h : a.v.stride_h;
  const void* wp = kind == 0 ? a.q_weight : kind == 1 ? a.k_weight : nullptr;
  void* out = kind == 0 ? a.q_out : kind == 1 ? (void*)a.k_out : (void*)a.v_out;
  const bool there = h < heads && data != nullptr;
  RawRow<DT> raw{};
  if (there) raw = load_row<DT, MODE>(data, b * sb + s * ss + hh * sh, g);
  // the lanes of a row go together, but rows differ: everything that exchanges between
  // lanes is done by all of them
  const void* any = a.q_weight != nullptr ? a.q_weight : a.k_weight;
  float w[8];
  if (any != nullptr) load_weights<MODE>(wp != nullptr ? wp : any, a.weight_dtype, g, w);
  Turn<MODE> t{};
  const bool turns = a.rot_dim > 0 && kind < 2 && there;
  if (turns) t = turns_of<MODE>(a, tok, (int64_t)a.B * a.S, g);
  float x[8], y[8];
  to_floats<DT, MODE>(raw, x);
  if (any != nullptr) {
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = x[i];
    norm_row(y, w, a.eps);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = wp != nullptr ? y[i] : x[i];
  }
  if (a.rot_dim > 0) {
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = x[i];
    rotate_row<MODE>(y, t, a.rot_dim, g, part + (MODE == kHalves ? row * kPartStride : 0));
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = turns ? y[i] : x[i];
  }
  const int64_t at = ((b * (kind == 0 ? a.Hq : a.Hkv) + hh) * a.S + s) * kDim;
  // q's type where a wave has rows of both is another than k's and v's
  if (__any(kind == 0))
    store_row<MODE, false>(out, at, g, a.q_out_dtype, x, there && kind == 0);
  if (__any(kind != 0)) store_row<MODE, false>(out, at, g, POT_FP16, x, there && kind != 0);
}

// Which kernel: tokens by eights once the work of the angles, made once a token, is more than
// the chain through a wave's heads. us, by eights and by heads, bf16: 32 + 4 + 4 heads 512
// tokens 4.7 and 4.8, 1024 5.2 and 6.6, 2048 7.8 and 10.5, 128 3.9 and 3.5; 8 + 1 + 1 heads 512
// 3.8 and 3.6, 1024 4.1 and 4.2, 2048 4.7 and 5.7; half of a head turned 512 6.2 and 5.9, 1024
// 6.8 and 8.5.
constexpr int64_t kManyTokens = 1024;
constexpr int64_t kTargetWaves = 4096;

template <int DT, int MODE>
static hipError_t launch_mode(const NormRopeArgs& a, hipStream_t stream) {
  const int heads = a.Hq + 2 * a.Hkv;
  const int64_t n_tok = (int64_t)a.B * a.S;
  if (n_tok < kManyTokens) {
    const int n_groups = (heads + 7) / 8;
    hipLaunchKernelGGL((norm_rope_heads_kernel<DT, MODE>), dim3((uint32_t)(n_tok * n_groups)),
                       dim3(64), 0, stream, a, heads, n_groups);
  } else {
    const int64_t groups = (n_tok + 7) / 8;
    // four waves a SIMD, or as many as heads allow
    int64_t n_chunks = (kTargetWaves + groups - 1) / groups;
    n_chunks = n_chunks < heads ? n_chunks : heads;
    const int chunk = (int)((heads + n_chunks - 1) / n_chunks);
    n_chunks = (heads + chunk - 1) / chunk;
    const int64_t blocks = (groups * n_chunks + kBlock / 64 - 1) / (kBlock / 64);
    hipLaunchKernelGGL((norm_rope_tokens_kernel<DT, MODE>), dim3((uint32_t)blocks), dim3(kBlock),
                       0, stream, a, heads, chunk, (int)n_chunks);
  }
  return hipGetLastError();
}
template <int DT>
static hipError_t launch_type(const NormRopeArgs& a, hipStream_t stream) {
  if (a.neighbours || a.rot_dim == 0) return launch_mode<DT, kNeighbours>(a, stream);
  return a.rot_dim == 64 ? launch_mode<DT, kFullHalves>(a, stream)
                         : launch_mode<DT, kHalves>(a, stream);
}

hipError_t launch_norm_rope(const NormRopeArgs& a, hipStream_t stream) {
  switch (a.dtype) {
    case POT_FP16: return launch_type<POT_FP16>(a, stream);
    case POT_BF16: return launch_type<POT_BF16>(a, stream);
    default: return launch_type<POT_FP32>(a, stream);
  }
}

}  // namespace potattn
