// New tokens into a paged cache: the rows of a QKV projection, of sequences of any number of new
// tokens side by side, normed and rotated as norm_rope.hip does it; queries go out, keys are
// encoded and values stored in the pages where their tokens belong, in the same pass (a row is
// the same 8 lanes in all three steps).
//
// Bound: the stream of many tokens (rows in, queries out: 9/10 of the bytes at 32 + 4 + 4 heads);
// of few a chain of round trips: the sequence's bounds, its length and page, the row. Measured (32 + 4 + 4
// heads): 1 token 5 us, 64 sequences of one 6, 8192 tokens bf16 to k = 4 and fp16 values 19.5 (97 MB with what
// reads them back: 4 TB/s; VALU busy for 60% of the time that the CUs are); 2300 tokens of fp32 with rotated
// keys, k = 2, 16 + 8 + 8 heads, 15.5 (VALU 51%, the encoder's divisions and both rotations most of it, in few
// waves that wait for the same chain).
#include "encode_rows.hpp"
#include "head_rows.hpp"
#include "paged.hpp"
#include "value_records.hpp"

namespace potattn {

// Where a packed row belongs.
struct Token {
  int b;      // sequence, -1: none, the row is not touched
  int place;  // in the sequence; negative: stored nowhere
};
// Row t0 + `in` of a wave's rows t0 .. t0 + N - 1 (`in` differs by lane, 0 .. N - 1). Every lane
// takes part: a lane reads one sequence's end, and a row's sequence is the number of ends at or
// before it. Of more than 64 sequences, 64 ends find the part that row t0's is in, and so on.
template <int N>
__device__ __forceinline__ Token find_token(const PackedRows& r, int t0, int in, int lane) {
  int first = 0;  // sequences that end at or before row t0, at least
  for (int span = r.B; span > 64;) {
    const int step = (span + 63) / 64, e = min(first + (lane + 1) * step, r.B);  // ascending
    const int n = (int)__builtin_popcountll(__ballot(r.cu_new[e] <= t0));
    first = min(first + n * step, r.B);
    span = min(step, r.B - first);
  }
  int before = first;
  for (int b0 = first; b0 < r.B; b0 += 64) {
    const int b = b0 + lane, end = b < r.B ? r.cu_new[b + 1] : INT32_MAX;
    uint64_t past = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      past = __ballot(b < r.B && end <= t0 + i);
      before += in == i ? (int)__builtin_popcountll(past) : 0;
    }
    if (past != ~0ull) break;
  }
  const int tok = t0 + in;
  if (tok >= r.n || before >= r.B || tok < r.cu_new[before]) return {-1, -1};
  const int len = min(max(r.seq_lens[before], 0), 1 << 24);
  return {before, len - (r.cu_new[before + 1] - tok)};
}

// A lane's 8 elements as loaded, of any type.
struct AnyRow {
  uint4 p[2];
};
template <int MODE>
__device__ __forceinline__ AnyRow load_any(const void* base, int64_t at, int g, int type) {
  AnyRow r;
  if (type == POT_FP32) {
    const RawRow<POT_FP32> v = load_row<POT_FP32, MODE>(base, at, g);
    r.p[0] = v.p[0];
    r.p[1] = v.p[1];
  } else {
    const RawRow<POT_FP16> v = load_row<POT_FP16, MODE>(base, at, g);
    r.p[0] = make_uint4(v.p[0].x, v.p[0].y, v.p[1].x, v.p[1].y);
    r.p[1] = make_uint4(0u, 0u, 0u, 0u);
  }
  return r;
}
template <int MODE>
__device__ __forceinline__ void any_to_floats(const AnyRow& r, int type, float (&x)[8]) {
  if (type == POT_FP32) {
    to_floats<POT_FP32, MODE>(RawRow<POT_FP32>{{r.p[0], r.p[1]}}, x);
    return;
  }
  const uint2 a = make_uint2(r.p[0].x, r.p[0].y), b = make_uint2(r.p[0].z, r.p[0].w);
  if (type == POT_BF16) to_floats<POT_BF16, MODE>(RawRow<POT_BF16>{{a, b}}, x);
  else to_floats<POT_FP16, MODE>(RawRow<POT_FP16>{{a, b}}, x);
}

// Lanes g >= 4 of a row take the value of the lane opposite in their quad.
__device__ __forceinline__ uint32_t turn_high_quad(uint32_t v) {
  constexpr int kReverse = 0x1B;
  return (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, kReverse, 0xF, kHighBanks, false);
}
// The row as fp16, lane g having elements 8g .. 8g + 7 whatever the pairing.
template <int MODE>
__device__ __forceinline__ uint4 natural_halves(const float (&x)[8]) {
  uint2 lo = make_uint2(pack_half(x[0], x[1]), pack_half(x[2], x[3]));
  uint2 hi = make_uint2(pack_half(x[4], x[5]), pack_half(x[6], x[7]));
  if constexpr (MODE == kFullHalves) {
    exchange_quads(lo, hi);  // lanes g >= 4 have piece 11 - g: turned round in their quad
    lo = make_uint2(turn_high_quad(lo.x), turn_high_quad(lo.y));
    hi = make_uint2(turn_high_quad(hi.x), turn_high_quad(hi.y));
  }
  return make_uint4(lo.x, lo.y, hi.x, hi.y);
}

// An encoded key over its 8 lanes: lane g's code word and, in lanes g % 4 < K, half of plane g % 4.
struct EncodedKey {
  uint32_t word, planes;
  float scale;
};
template <int K, bool HAD>
__device__ __forceinline__ EncodedKey encode_key(const uint4& raw, int lane, const CutBits& cut) {
  const uint32_t w4[4] = {raw.x, raw.y, raw.z, raw.w};
  float x[8];
  unpack_row<HAD>(w4, lane, x);
  float s = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) s = fmaxf(s, fabsf(x[i]));
  s = max_over_8_lanes(s);
  const uint32_t sgn = HAD ? float_signs(x)
                           : sign_nibbles(__builtin_amdgcn_perm(w4[1], w4[0], 0x0B0A0908u),
                                          __builtin_amdgcn_perm(w4[3], w4[2], 0x0B0A0908u));
  uint32_t planes = 0;
  EncodedKey e;
  e.word = encode_word<K>(x, row_scale<K>(s), sgn, cut, planes);
  e.planes = 0;
  if constexpr (K > 0) e.planes = quad_planes(planes, lane);
  e.scale = s;
  return e;
}

// Keys and values of rows into the pages: row8 the group of 8 cache rows, u the row in it; rows
// that are not `there` are not written. Every lane of the wave takes part.
template <int K>
__device__ __forceinline__ void store_key(const PagedAppendArgs& a, const CutBits& cut, const uint4& raw,
                                          int row8, int u, int lane, bool there) {
  const EncodedKey e = a.hadamard ? encode_key<K, true>(raw, lane, cut) : encode_key<K, false>(raw, lane, cut);
  if (!there) return;
  const int g = lane & 7;
  const int64_t row = (int64_t)row8 * 8 + u;
  *reinterpret_cast<uint32_t*>(a.pages.codes_se + row * (kDim / 2) + 4 * g) = e.word;
  if constexpr (K > 0) {
    if ((g & 3) < K)
      *reinterpret_cast<uint32_t*>(a.pages.codes_m + row * 8 * K + 8 * (g & 3) + 4 * (g >> 2)) = e.planes;
  }
  if (g == 0) a.pages.key_scale[row] = e.scale;
}
// whole: the wave's 8 rows are the 8 tokens of one group, in order (uniform).
__device__ __forceinline__ void store_value(const PagedAppendArgs& a, const uint4& raw, int row8, int u,
                                            int lane, bool there, bool whole) {
  const int g = lane & 7;
  if (a.value_format == POT_VALUES_INT4) {
    uint8_t* rec = a.pages.values + (int64_t)row8 * kI4GroupBytes;
    if (whole) {
      store_record(raw, rec, lane, true, 0, 0, 0);
      return;
    }
    uint16_t step;
    float lo;
    const uint32_t d = record_columns(raw, lane, &step, &lo);
    if (!there) return;
    uint8_t* at = rec + 16 * (8 * (g & 1) + 4 * ((g >> 1) & 1)) + 8 * (g >> 2) + u;
#pragma unroll
    for (int j = 0; j < 4; ++j) at[16 * j] = (uint8_t)(d >> (8 * j));
    const uint16_t sz = g == 0 ? step : __half_as_ushort(__float2half_rn(lo));
    if (g < 2) *reinterpret_cast<uint16_t*>(rec + kI4Steps + 16 * g + 2 * u) = sz;
    return;
  }
  if (!there) return;
  uint16_t* at = reinterpret_cast<uint16_t*>(a.pages.values) + (int64_t)row8 * (8 * kDim) + 64 * g + u;
  const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    at[16 * i] = (uint16_t)w[i];
    at[16 * i + 8] = (uint16_t)(w[i] >> 16);
  }
}

// The group of cache rows of a token for kv head 0 (-1: its page is not there); a kv head's
// stands page_groups further on.
__device__ __forceinline__ int token_row8(const PagesArg& p, const Token& t) {
  return t.b < 0 || t.place < 0 ? -1 : group_row8(p, p.table + (int64_t)t.b * p.table_len, 0, t.place >> 3);
}

template <int MODE>
__device__ __forceinline__ Turn<MODE> turns_at(const NormRopeArgs& a, int64_t tok, int place, int g) {
  if (a.positions != nullptr) return turns_of<MODE>(a, tok, a.S, g);
  Turn<MODE> t;
  const int half = a.rot_dim / 2;
#pragma unroll
  for (int i = 0; i < kLanePairs<MODE>; ++i) {
    int pair = MODE == kHalves ? 8 * g + i : 4 * (MODE == kFullHalves ? quad_of(g) : g) + i;
    bool in = pair < half;
    if constexpr (MODE == kHalves) {
      in = pair < a.rot_dim;
      pair = pair >= half ? pair - half : pair;
    }
    sin_cos_quarters((double)place * a.inv_freq[in ? pair : 0] * 0.63661977236758134308, &t.s[i], &t.c[i]);
  }
  return t;
}

// Many tokens: a wave takes 8 rows of one head after another, 8 lanes each, through a chunk of
// heads, so that places, pages and turns are found once for all of them.
template <int K, int MODE>
__global__ __launch_bounds__(kBlock) void paged_append_tokens_kernel(const PagedAppendArgs a, int heads,
                                                                     int chunk, int n_chunks) {
  __shared__ float part[MODE == kHalves ? kBlock / 64 * 8 * kPartStride : 1];
  const NormRopeArgs& n = a.rows;
  const int lane = lane_id(), g = lane & 7, row = lane >> 3;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int unit = blockIdx.x * (kBlock / 64) + wave, group = unit / n_chunks;
  if (group * 8 >= n.S) return;
  const int h_first = (unit - group * n_chunks) * chunk, h_end = min(h_first + chunk, heads);
  const Token t = find_token<8>(a.packed, group * 8, row, lane);
  const int tok = min(group * 8 + row, n.S - 1);
  float* my_part = part + (MODE == kHalves ? (wave * 8 + row) * kPartStride : 0);
  const CutBits cut = cut_bits(a.tab);
  const int qk_end = n.Hq + n.Hkv;
  const int row8 = h_end > n.Hq ? token_row8(a.pages, t) : -1;
  const int u = t.place & 7;
  // the wave's rows are a group's 8 tokens: each lane's group is its neighbour row's, and its
  // place in it is the row
  const int first8 = __builtin_amdgcn_readfirstlane(row8);
  const bool whole = __all(row8 >= 0 && row8 == first8 && u == row);
  const bool turns = n.rot_dim > 0 && h_first < qk_end;
  Turn<MODE> turn{};
  if (turns) turn = turns_at<MODE>(n, tok, t.place, g);
  constexpr int kAhead = 2;
  auto part_of = [&](const RowsIn& in, const void* weight, int first, int H, auto emit) {
    const int lo = max(h_first, first) - first, hi = min(h_end, first + H) - first;
    if (lo >= hi) return;
    const int64_t src = tok * in.stride_s;
    AnyRow ahead[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
      ahead[i] = load_any<MODE>(in.data, src + min(lo + i, hi - 1) * in.stride_h, g, n.dtype);
    float w[8];
    if (weight != nullptr) load_weights<MODE>(weight, n.weight_dtype, g, w);
    for (int h = lo; h < hi; h += kAhead) {
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        if (h + i >= hi) break;  // uniform
        float x[8];
        any_to_floats<MODE>(ahead[i], n.dtype, x);
        ahead[i] = load_any<MODE>(in.data, src + min(h + i + kAhead, hi - 1) * in.stride_h, g, n.dtype);
        if (weight != nullptr) norm_row(x, w, n.eps);
        emit(h + i, x);
      }
    }
  };
  if (n.q.data != nullptr)
    part_of(n.q, n.q_weight, 0, n.Hq, [&](int h, float (&x)[8]) {
      if (turns) rotate_row<MODE>(x, turn, n.rot_dim, g, my_part);
      store_row<MODE, true>(n.q_out, ((int64_t)tok * n.Hq + h) * kDim, g, n.q_out_dtype, x, t.b >= 0);
    });
  part_of(n.k, n.k_weight, n.Hq, n.Hkv, [&](int h, float (&x)[8]) {
    if (turns) rotate_row<MODE>(x, turn, n.rot_dim, g, my_part);
    store_key<K>(a, cut, natural_halves<MODE>(x), row8 + h * a.pages.page_groups, u, lane, row8 >= 0);
  });
  part_of(n.v, nullptr, qk_end, n.Hkv, [&](int h, float (&x)[8]) {
    store_value(a, natural_halves<MODE>(x), row8 + h * a.pages.page_groups, u, lane, row8 >= 0, whole);
  });
}

// Few tokens: a wave takes 8 heads of one token.
template <int K, int MODE>
__global__ __launch_bounds__(64) void paged_append_heads_kernel(const PagedAppendArgs a, int heads,
                                                                int n_groups) {
  __shared__ float part[MODE == kHalves ? 8 * kPartStride : 1];
  const NormRopeArgs& n = a.rows;
  const int lane = lane_id(), g = lane & 7, row = lane >> 3;
  const int tok = blockIdx.x / (uint32_t)n_groups;
  const int h = (int)(blockIdx.x - tok * n_groups) * 8 + row;
  const int kind = h < n.Hq ? 0 : h < n.Hq + n.Hkv ? 1 : 2;
  const int hh = h - (kind == 0 ? 0 : kind == 1 ? n.Hq : n.Hq + n.Hkv);
  const RowsIn qi = n.q, ki = n.k, vi = n.v;
  const void *qw = n.q_weight, *kw = n.k_weight;
  const void* data = kind == 0 ? qi.data : kind == 1 ? ki.data : vi.data;
  const int64_t ss = kind == 0 ? qi.stride_s : kind == 1 ? ki.stride_s : vi.stride_s;
  const int64_t sh = kind == 0 ? qi.stride_h : kind == 1 ? ki.stride_h : vi.stride_h;
  const void* wp = kind == 0 ? qw : kind == 1 ? kw : nullptr;
  const bool there = h < heads && data != nullptr;
  AnyRow raw{};
  if (there) raw = load_any<MODE>(data, tok * ss + hh * sh, g, n.dtype);
  const void* any = qw != nullptr ? qw : kw;
  float w[8];
  if (any != nullptr) load_weights<MODE>(wp != nullptr ? wp : any, n.weight_dtype, g, w);
  const Token t = find_token<1>(a.packed, tok, 0, lane);
  if (t.b < 0) return;  // uniform
  Turn<MODE> turn{};
  const bool turns = n.rot_dim > 0 && kind < 2 && there;
  if (turns) turn = turns_at<MODE>(n, tok, t.place, g);
  float x[8], y[8];
  any_to_floats<MODE>(raw, n.dtype, x);
  if (any != nullptr) {
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = x[i];
    norm_row(y, w, n.eps);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = wp != nullptr ? y[i] : x[i];
  }
  if (n.rot_dim > 0) {
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = x[i];
    rotate_row<MODE>(y, turn, n.rot_dim, g, part + (MODE == kHalves ? row * kPartStride : 0));
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = turns ? y[i] : x[i];
  }
  if (__any(there && kind == 0))
    store_row<MODE, false>(n.q_out, ((int64_t)tok * n.Hq + hh) * kDim, g, n.q_out_dtype, x, there && kind == 0);
  if (!__any(there && kind != 0)) return;
  const int first = token_row8(a.pages, t), row8 = first + hh * a.pages.page_groups;
  const uint4 halves = natural_halves<MODE>(x);
  if (__any(there && kind == 1))
    store_key<K>(a, cut_bits(a.tab), halves, row8, t.place & 7, lane, there && kind == 1 && first >= 0);
  if (__any(there && kind == 2))
    store_value(a, halves, row8, t.place & 7, lane, there && kind == 2 && first >= 0, false);
}

// Which kernel (32 + 4 + 4 heads, 4-bit values): 512 tokens 9.6 us by tokens and 9.8 by heads, 1000 10.7 and
// 11.5, 4000 17.7 and 24.4. Waves of the former: 8192 tokens, k = 4, with fp16 values, read back, 25.0 us with
// 4096, 27.1 with 2048, 28.7 with 8192.
constexpr int kManyTokens = 512;
constexpr int kTargetWaves = 4096;

template <int K, int MODE>
static hipError_t launch_mode(const PagedAppendArgs& a, hipStream_t stream) {
  const int heads = a.rows.Hq + 2 * a.rows.Hkv, n_tok = a.rows.S;
  if (n_tok < kManyTokens) {
    const int n_groups = (heads + 7) / 8;
    hipLaunchKernelGGL((paged_append_heads_kernel<K, MODE>), dim3((uint32_t)(n_tok * n_groups)), dim3(64), 0,
                       stream, a, heads, n_groups);
  } else {
    const int groups = (n_tok + 7) / 8;
    int n_chunks = (kTargetWaves + groups - 1) / groups;
    n_chunks = n_chunks < heads ? n_chunks : heads;
    const int chunk = (heads + n_chunks - 1) / n_chunks;
    n_chunks = (heads + chunk - 1) / chunk;
    const int64_t blocks = ((int64_t)groups * n_chunks + kBlock / 64 - 1) / (kBlock / 64);
    hipLaunchKernelGGL((paged_append_tokens_kernel<K, MODE>), dim3((uint32_t)blocks), dim3(kBlock), 0, stream,
                       a, heads, chunk, n_chunks);
  }
  return hipGetLastError();
}
template <int K>
static hipError_t launch_pairs(const PagedAppendArgs& a, hipStream_t stream) {
  if (a.rows.neighbours || a.rows.rot_dim == 0) return launch_mode<K, kNeighbours>(a, stream);
  return a.rows.rot_dim == 64 ? launch_mode<K, kFullHalves>(a, stream) : launch_mode<K, kHalves>(a, stream);
}

hipError_t launch_paged_append(const PagedAppendArgs& a, hipStream_t stream) {
  switch (a.tab.mant_bits) {
    case 0: return launch_pairs<0>(a, stream);
    case 1: return launch_pairs<1>(a, stream);
    case 2: return launch_pairs<2>(a, stream);
    case 3: return launch_pairs<3>(a, stream);
    default: return launch_pairs<4>(a, stream);
  }
}

}  // namespace potattn
