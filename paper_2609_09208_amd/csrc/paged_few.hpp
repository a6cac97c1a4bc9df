// Attention over a paged cache for sequences with up to 16 rows (new tokens x query heads of a
// kv head): single tokens, drafts. Grid (key ranges, kv heads, sequences), four waves; a wave
// streams 64-key tiles of its own, as the decode kernel does, and the waves meet at the end.
//
// Per tile: scores S^T = K Q^T by v_mfma_f32_16x16x32_f16 (codes as fp16 weights, the INT8
// queries as fp16 integers: exact sums), rows of K in such an order that a lane ends up with
// the scores of one query and 8 consecutive keys of either half tile, which are then the
// operand of O^T = V^T P^T as they stand; a query's reference, sum and outputs are its lanes'
// own, so a rise of the reference is 16 products a lane. The reference rises only when weights
// would leave fp16's range.
//
// Tiles that every query sees in full take a loop without a test of keys; the others (the
// sequence's end, the window's, pages that are not there) go through the same code with them.
//
// Bound: the stream with fp16 values (164 bytes a key: 64 x 8192 keys 63 us, 5.5 TB/s; with a window
// of 4096 33, 30 in one range); with 4-bit values (72 bytes) VALU issue, 71 - 74% busy of 345
// operations a tile, most of them the operands' (64 x 16384 keys 62 us, 4.9 TB/s; 64 x 8192 34). Pages
// cost nothing: pages of 128 and of 32768 keys differ by 1%.
#pragma once

#include "paged.hpp"

namespace potattn {

constexpr int kFewWaves = 4;

template <int VF>
struct FewValues {  // by half tile
  uint4 f[2][4];
};
template <>
struct FewValues<POT_VALUES_INT4> {
  uint4 f[2], s[2], z[2];
};

// Value of lane `from` (any lane).
__device__ __forceinline__ int lane_value(int v, int from) {
  return __builtin_amdgcn_ds_bpermute(from << 2, v);
}

// UNI: a tile lies in one page (page sizes of whole tiles). LOW: the weights' rounding goes into
// the products too (outputs of 32 bits). EIGHT: no sequence has more than 8 rows. The columns of the
// products are 16 all the same, so columns 8 .. 15 take the same queries to a tile's other 32 keys:
// scores K_0 [Q 0] + K_1 [0 Q], then half the scales, weights and references a lane; the weights meet
// both halves' values, and of the two products a lane keeps its half's.
template <int K, int VF, bool UNI, bool LOW, bool EIGHT>
__global__ __launch_bounds__(64 * kFewWaves) __attribute__((amdgpu_waves_per_eu(
    few_simd_waves(K, UNI, EIGHT))))
void paged_few_kernel(const PagedAttendArgs a) {
  constexpr int NW = kFewWaves, R = kFewRows;
  __shared__ uint4 sq[R][8];
  __shared__ float sc[R], sm[NW][R], sl[NW][R];
  __shared__ __attribute__((aligned(16))) float so[NW][R][kDim];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int split = blockIdx.x, kvh = blockIdx.y, b = blockIdx.z;
  const NewTokens t = sequence_tokens(a.packed, b, a.max_new, a.max_len);
  if (t.n == 0 || t.n > a.plan.few_limit || t.n * a.G > a.plan.few_limit) return;
  const int rows = t.n * a.G, p_first = t.place, p_last = t.place + t.n - 1;
  const SeenTiles seen = seen_tiles(p_first, p_last, t.len, a.window, a.n_sink);
  const TileRun run = split_tiles(seen.tiles, split, a.plan.few_splits);
  const int32_t* table = a.pages.table + (int64_t)b * a.pages.table_len;
  const int col = lane & 15, grp = lane >> 4;
  constexpr int kHalves = EIGHT ? 1 : 2;  // half tiles that a lane has weights of
  const int half = EIGHT ? col >> 3 : 0, query = EIGHT ? col & 7 : col;

  // The rows of a tile's groups: of the first one (UNI, uniform), or of group lane % 8 in each
  // lane; -1 where there is no page. Tiles past the run: the last one again.
  auto rows_of = [&](int j) -> int {
    const int g = tile_start(seen, min(j, run.end - 1)) / 8;
    return group_row8(a.pages, table, kvh, UNI ? g : g + (lane & 7));
  };
  // Row of group g (0 .. 7, by lane) of a tile; groups without a page read row 0, which is there.
  auto row_at = [&](int rows8, int g) -> int64_t {
    return UNI ? max(rows8, 0) + g : max(lane_value(rows8, g), 0);
  };

  // a wave's loads of a tile: codes of keys 32 kb + 8 (col / 4) + 4 s + col % 4, dimensions
  // 16 grp ..+15; scales and values of keys 32 kb + 8 grp ..+7
  uint2 kc[2][2];
  uint32_t kp[2][2][K > 0 ? K : 1];
  float4 ks[kHalves][2];
  FewValues<VF> vr;
  auto load_keys = [&](int rows8) {
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      const int64_t row = row_at(rows8, 4 * kb + (col >> 2)) * 8 + (col & 3);
      const uint8_t* c = a.pages.codes_se + row * 32 + 8 * grp;
#pragma unroll
      for (int s = 0; s < 2; ++s) kc[kb][s] = *reinterpret_cast<const uint2*>(c + 128 * s);
      if constexpr (K > 0) {
        const uint8_t* m = a.pages.codes_m + row * 8 * K + 2 * grp;
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int p = 0; p < K; ++p)
            kp[kb][s][p] = *reinterpret_cast<const uint16_t*>(m + 32 * K * s + 8 * p);
      }
    }
  };
  auto load_values = [&](int rows8) {
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      const int64_t row8 = row_at(rows8, 4 * kb + grp);
      if (kb < kHalves) {
        const int64_t mine = EIGHT ? row_at(rows8, 4 * half + grp) : row8;
        const float4* sp = reinterpret_cast<const float4*>(a.pages.key_scale + mine * 8);
        ks[kb][0] = sp[0];
        ks[kb][1] = sp[1];
      }
      if constexpr (VF == POT_VALUES_INT4) {
        const uint8_t* rec = a.pages.values + row8 * kI4GroupBytes;
        vr.f[kb] = stream16(rec + 16 * col);
        vr.s[kb] = *reinterpret_cast<const uint4*>(rec + kI4Steps);
        vr.z[kb] = *reinterpret_cast<const uint4*>(rec + kI4Minima);
      } else {
        const uint8_t* v = a.pages.values + row8 * (16 * kDim) + 16 * col;
#pragma unroll
        for (int nb = 0; nb < 4; ++nb) vr.f[kb][nb] = stream16(v + 256 * nb);
      }
    }
  };
  int j = run.first + wave;
  int rows_now = -1, rows_next = -1;
  if (j < run.end) {
    rows_now = rows_of(j);
    load_keys(rows_now);
    load_values(rows_now);
    rows_next = rows_of(j + NW);
  }

  if (wave < R / 8) {
    const int r = 8 * wave + (lane >> 3);
    float x[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
    if (r < rows) {
      const int tok = r / a.G, head = a.q_head(kvh * a.G + (r - tok * a.G));
      load8(a.q, (t.first + tok) * a.q_stride_t + head * a.q_stride_h, lane & 7, a.dtype, x);
    }
    float factor;
    sq[r][lane & 7] = quantised_query(x, a.hadamard, lane, &factor);
    if ((lane & 7) == 0) sc[r] = factor;
  }
  __syncthreads();
  half8 q[3 - kHalves][2];  // of each half tile's keys
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    const uint4 w = sq[query][2 * grp + s], none = make_uint4(0u, 0u, 0u, 0u);
    q[0][s] = __builtin_bit_cast(half8, half == 0 ? w : none);
    if constexpr (EIGHT) q[1][s] = __builtin_bit_cast(half8, half == 1 ? w : none);
  }
  const float c = sc[query];

  f32x4 acc[3 - kHalves][4];  // EIGHT: of either half tile's values
#pragma unroll
  for (int h = 0; h < 3 - kHalves; ++h)
#pragma unroll
    for (int nb = 0; nb < 4; ++nb) acc[h][nb] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  Reference ref;
  float l = 0.0f;

  auto place_of_col = [&]() { return p_first + (query < rows ? query : 0) / a.G; };
  bool special = false;  // a tile in part held special values (paged.hpp)

  auto tile = [&](auto part_tag, int t0) {
    constexpr bool PART = decltype(part_tag)::value;
    float y[kHalves][8];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      f32x4 d[2] = {{0.0f, 0.0f, 0.0f, 0.0f}, {0.0f, 0.0f, 0.0f, 0.0f}};
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          uint32_t pl[K > 0 ? K : 1];
#pragma unroll
          for (int p = 0; p < K; ++p) pl[p] = h ? kp[kb][s][p] >> 8 : kp[kb][s][p] & 0xFFu;
          f32x4& at = d[EIGHT ? 0 : kb];
          at = __builtin_amdgcn_mfma_f32_16x16x32_f16(paged_weights<K>(h ? kc[kb][s].y : kc[kb][s].x, pl),
                                                      q[EIGHT ? kb : 0][h], at, 0, 0, 0);
        }
#pragma unroll
      for (int kb = 0; kb < kHalves; ++kb)
#pragma unroll
        for (int i = 0; i < 4; ++i) y[kb][4 * s + i] = d[kb][i];
    }
    // the codes have become operands: the next tile's may come
    const int rows_tile = rows_now;
    load_keys(rows_next);
    rows_now = rows_next;
    rows_next = rows_of(j + 2 * NW);
#pragma unroll
    for (int kb = 0; kb < kHalves; ++kb)
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const float4 sv = ks[kb][s];
        y[kb][4 * s] *= sv.x;
        y[kb][4 * s + 1] *= sv.y;
        y[kb][4 * s + 2] *= sv.z;
        y[kb][4 * s + 3] *= sv.w;
      }
    int end[2] = {0, 0};
    if constexpr (PART) {
      const SeenKeys sk = seen_keys(a, place_of_col(), seen.end, t0 + 8 * grp);
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        const bool there = (UNI ? rows_tile : lane_value(rows_tile, 4 * kb + grp)) >= 0;
        end[kb] = there ? seen.end : 0;
        if constexpr (!EIGHT) {
          const uint32_t mask = there ? seen_bits(sk, 32 * kb) : 0u;
#pragma unroll
          for (int i = 0; i < 8; ++i) y[kb][i] = if_seen(y[kb][i], mask, i);
        }
      }
      if constexpr (EIGHT) {
        const uint32_t mask = end[half] > 0 ? seen_bits(sk, 32 * half) : 0u;
#pragma unroll
        for (int i = 0; i < 8; ++i) y[0][i] = if_seen(y[0][i], mask, i);
      }
    }
    float top = fmaxf(y[0][0], y[0][1]);
#pragma unroll
    for (int i = 2; i < 8 * kHalves; ++i) top = fmaxf(top, y[i >> 3][i & 7]);
    const auto r16 = __builtin_amdgcn_permlane16_swap(__float_as_uint(top), __float_as_uint(top), false, false);
    top = fmaxf(__uint_as_float(r16[0]), __uint_as_float(r16[1]));
    const auto r32 = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
    top = fmaxf(__uint_as_float(r32[0]), __uint_as_float(r32[1]));
    if (must_rise(ref, top, c)) {
      const float f = raise(ref, top, c);
#pragma unroll
      for (int h = 0; h < 3 - kHalves; ++h)
#pragma unroll
        for (int nb = 0; nb < 4; ++nb) acc[h][nb] *= f;
      l *= f;
    }
    if (ref.far) {  // uniform
#pragma unroll
      for (int kb = 0; kb < kHalves; ++kb) far_sums(ref, y[kb]);
    }
    const float shift = weight_shift(ref);
    uint32_t hi[kHalves][4], lo[kHalves][4];
    float tile_l = 0.0f;  // the tile's weights go onto l together: each alone would be rounded at l's size
#pragma unroll
    for (int kb = 0; kb < kHalves; ++kb)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float p0 = weight_of(y[kb][2 * i], c, shift), p1 = weight_of(y[kb][2 * i + 1], c, shift);
        hi[kb][i] = pack_half(p0, p1);
        if constexpr (LOW) {
          tile_l += p0;
          tile_l += p1;
        } else {  // of the weights as they are multiplied
          const half2v ones = {(_Float16)1.0f, (_Float16)1.0f};
          tile_l = __builtin_amdgcn_fdot2(__builtin_bit_cast(half2v, hi[kb][i]), ones, tile_l, false);
        }
        if constexpr (LOW) lo[kb][i] = low_part(p0, p1, hi[kb][i]);
      }
    l += tile_l;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      const int at = EIGHT ? 0 : kb;  // of the weights
      const half8 ph = __builtin_bit_cast(half8, make_uint4(hi[at][0], hi[at][1], hi[at][2], hi[at][3]));
      half8 pl{};
      if constexpr (LOW) pl = __builtin_bit_cast(half8, make_uint4(lo[at][0], lo[at][1], lo[at][2], lo[at][3]));
#pragma unroll
      for (int nb = 0; nb < 4; ++nb) {
        uint4 u;
        if constexpr (VF == POT_VALUES_INT4) {
          const uint4 w = vr.f[kb];
          const uint32_t w0 = nb < 2 ? w.x : w.z, w1 = nb < 2 ? w.y : w.w;
          u = int4_values((nb & 1 ? w0 >> 4 : w0) & 0x0F0F0F0Fu, (nb & 1 ? w1 >> 4 : w1) & 0x0F0F0F0Fu,
                          vr.s[kb], vr.z[kb]);
        } else {
          u = vr.f[kb][nb];
        }
        if constexpr (PART) {
          u = mask_tokens(u, t0 + 32 * kb + 8 * grp, end[kb]);
          special |= has_special(u);
          u = without_special(u);
        }
        const half8 v = __builtin_bit_cast(half8, u);
        f32x4& sum = acc[EIGHT ? kb : 0][nb];
        sum = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, ph, sum, 0, 0, 0);
        if constexpr (LOW) sum = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, pl, sum, 0, 0, 0);
      }
    }
    load_values(rows_now);
    j += NW;
  };
  auto whole = [&](int t0, int rows8) {
    return whole_tile(seen, p_first, p_last, t0, a.window, a.n_sink) && (UNI ? rows8 >= 0 : __all(rows8 >= 0));
  };
#pragma nounroll
  while (j < run.end) {
    int t0 = tile_start(seen, j);
#pragma nounroll
    while (whole(t0, rows_now)) {
      tile(std::false_type{}, t0);
      if (j >= run.end) break;
      t0 = tile_start(seen, j);
    }
    if (j < run.end) tile(std::true_type{}, t0);
  }
  if (__any(special)) {
#pragma nounroll
    for (j = run.first + wave; j < run.end; j += NW) {
      const int t0 = tile_start(seen, j), rows8 = rows_of(j);
      if (whole(t0, rows8)) continue;
      const SeenKeys sk = seen_keys(a, place_of_col(), seen.end, t0 + 8 * grp);
#pragma nounroll
      for (int kb = 0; kb < 2; ++kb) {
        const int g = 4 * kb + grp, row8 = UNI ? (rows8 < 0 ? -1 : rows8 + g) : lane_value(rows8, g);
        const uint32_t mask = row8 >= 0 ? seen_bits(sk, 32 * kb) : 0u;
        half8 ones;
#pragma unroll
        for (int i = 0; i < 8; ++i) ones[i] = (mask >> i) & 1 ? (_Float16)1.0f : (_Float16)0.0f;
#pragma unroll
        for (int nb = 0; nb < 4; ++nb) {
          uint4 v = make_uint4(0u, 0u, 0u, 0u);
          if (row8 >= 0) v = mask_tokens(group_values<VF>(a.pages, row8, 16 * nb + col), t0 + 8 * g, seen.end);
          const f32x4 n = __builtin_amdgcn_mfma_f32_16x16x32_f16(special_marks(v), ones, f32x4{0.0f, 0.0f, 0.0f, 0.0f}, 0, 0, 0);
#pragma unroll
          for (int i = 0; i < 4; ++i) acc[0][nb][i] += special_sum(n[i]);  // EIGHT: those of half 0 count
        }
      }
    }
  }

  // ---- the waves' sums -------------------------------------------------------------------
  {
    const auto r16 = __builtin_amdgcn_permlane16_swap(__float_as_uint(l), __float_as_uint(l), false, false);
    l = __uint_as_float(r16[0]) + __uint_as_float(r16[1]);
    const auto r32 = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
    l = __uint_as_float(r32[0]) + __uint_as_float(r32[1]);
  }
  const float f = exact_reference(ref, c);
  l *= f;
#pragma unroll
  for (int nb = 0; nb < 4; ++nb) {
    if constexpr (EIGHT) acc[0][nb] = half == 0 ? acc[0][nb] : acc[1][nb];
    acc[0][nb] *= f;
  }
  if (lane < R) {
    sm[wave][col] = ref.m;
    sl[wave][col] = l;
  }
#pragma unroll
  for (int nb = 0; nb < 4; ++nb)
    *reinterpret_cast<f32x4*>(&so[wave][col][16 * nb + 4 * grp]) = acc[0][nb];
  __syncthreads();
  const int r = tid / 16, d = 4 * (tid & 15);
  if (r >= rows) return;
  const float cr = sc[r];
  float M = sm[0][r];
#pragma unroll
  for (int w = 0; w < NW; ++w)
#pragma unroll
    for (int h = 0; h < 3 - kHalves; ++h) M = fmaxf(M, sm[w][r + 8 * h]);
  float L = 0.0f;
  f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int w = 0; w < NW; ++w)
#pragma unroll
    for (int h = 0; h < 3 - kHalves; ++h) {
      const float fw = between(sm[w][r + 8 * h], M, cr);
      L += fw * sl[w][r + 8 * h];
      o += fw * *reinterpret_cast<const f32x4*>(&so[w][r + 8 * h][d]);
    }
  if (a.plan.few_splits == 1) {
    const int tok = r / a.G, head = a.q_head(kvh * a.G + (r - tok * a.G));
    const float inv = L == 0.0f ? 0.0f : 1.0f / L;
    store_out4(a.out, ((int64_t)(t.first + tok) * a.Hq + head) * kDim + d, a.out_dtype, o[0] * inv,
               o[1] * inv, o[2] * inv, o[3] * inv);
    return;
  }
  float* part = a.few_part + ((((int64_t)b * a.pages.Hkv + kvh) * a.plan.few_splits + split) * R + r) * kPartial;
  *reinterpret_cast<f32x4*>(part + d) = o;
  if (d == 0) *reinterpret_cast<f32x4*>(part + kDim) = f32x4{M, L, cr, 0.0f};
}

template <int K, int VF, bool UNI, bool LOW>
void launch_few_rows(const PagedAttendArgs& a, dim3 grid, hipStream_t stream) {
  if (a.plan.few_limit <= 8)
    hipLaunchKernelGGL((paged_few_kernel<K, VF, UNI, LOW, true>), grid, dim3(64 * kFewWaves), 0, stream, a);
  else
    hipLaunchKernelGGL((paged_few_kernel<K, VF, UNI, LOW, false>), grid, dim3(64 * kFewWaves), 0, stream, a);
}
template <int K, int VF>
hipError_t launch_few(const PagedAttendArgs& a, hipStream_t stream) {
  const dim3 grid((uint32_t)a.plan.few_splits, (uint32_t)a.pages.Hkv, (uint32_t)a.packed.B);
  const bool uni = a.pages.page_groups % (kWTile / 8) == 0;
  if (a.out_dtype == POT_FP32) {
    if (uni) launch_few_rows<K, VF, true, true>(a, grid, stream);
    else launch_few_rows<K, VF, false, true>(a, grid, stream);
  } else {
    if (uni) launch_few_rows<K, VF, true, false>(a, grid, stream);
    else launch_few_rows<K, VF, false, false>(a, grid, stream);
  }
  return hipGetLastError();
}

}  // namespace potattn
