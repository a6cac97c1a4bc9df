// Attention over a paged cache for sequences with up to 16 rows (new tokens x query heads of a
// kv head): single tokens, drafts. Grid (key ranges, kv heads, sequences), four waves; a wave
// streams 64-key tiles of its own, as the decode kernel does, and the waves meet at the end.
//
// Per tile: scores S^T = K Q^T by v_mfma_f32_16x16x32_f16 (codes as fp16 weights, the INT8
// queries as fp16 integers: exact sums), rows of K in such an order that a lane ends up with
// the scores of one query and 8 consecutive keys of either half tile, which are then the
// operand of O^T = V^T P^T as they stand; a query's reference, sum and outputs are its lanes'
// own, so a rise of the reference is 16 products a lane. Weights go in as fp16 numbers and what
// rounding left of them. The reference rises only when a weight would leave fp16's range.
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

template <int K, int VF>
__global__ __launch_bounds__(64 * kFewWaves) void paged_few_kernel(const PagedAttendArgs a) {
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

  // a wave's loads of a tile: codes of keys 32 kb + 8 (col / 4) + 4 s + col % 4, dimensions
  // 16 grp ..+15; scales and values of keys 32 kb + 8 grp ..+7
  uint2 kc[2][2];
  uint32_t kp[2][2][K > 0 ? K : 1];
  float4 ks[2][2];
  FewValues<VF> vr;
  bool there[2];
  auto load_keys = [&](int j) {
    const int g0 = tile_start(seen, j) / 8;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      const int g = g0 + 4 * kb + (col >> 2);
      const int64_t row8 = g * 8 < seen.end ? group_row8(a.pages, table, kvh, g) : -1;
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        kc[kb][s] = make_uint2(0u, 0u);
#pragma unroll
        for (int p = 0; p < K; ++p) kp[kb][s][p] = 0u;
        if (row8 >= 0) {
          const int64_t row = row8 * 8 + 4 * s + (col & 3);
          kc[kb][s] = *reinterpret_cast<const uint2*>(a.pages.codes_se + row * 32 + 8 * grp);
#pragma unroll
          for (int p = 0; p < K; ++p)
            kp[kb][s][p] = *reinterpret_cast<const uint16_t*>(a.pages.codes_m + row * 8 * K + 8 * p + 2 * grp);
        }
      }
    }
  };
  auto load_values = [&](int j) {
    const int g0 = tile_start(seen, j) / 8;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      const int g = g0 + 4 * kb + grp;
      const int64_t row8 = g * 8 < seen.end ? group_row8(a.pages, table, kvh, g) : -1;
      there[kb] = row8 >= 0;
      const uint4 none = make_uint4(0u, 0u, 0u, 0u);
      ks[kb][0] = ks[kb][1] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      if constexpr (VF == POT_VALUES_INT4) {
        vr.f[kb] = vr.s[kb] = vr.z[kb] = none;
      } else {
#pragma unroll
        for (int nb = 0; nb < 4; ++nb) vr.f[kb][nb] = none;
      }
      if (row8 >= 0) {
        const float4* sp = reinterpret_cast<const float4*>(a.pages.key_scale + row8 * 8);
        ks[kb][0] = sp[0];
        ks[kb][1] = sp[1];
        if constexpr (VF == POT_VALUES_INT4) {
          const uint8_t* rec = a.pages.values + row8 * kI4GroupBytes;
          vr.f[kb] = *reinterpret_cast<const uint4*>(rec + 16 * col);
          vr.s[kb] = *reinterpret_cast<const uint4*>(rec + kI4Steps);
          vr.z[kb] = *reinterpret_cast<const uint4*>(rec + kI4Minima);
        } else {
#pragma unroll
          for (int nb = 0; nb < 4; ++nb)
            vr.f[kb][nb] = *reinterpret_cast<const uint4*>(a.pages.values + row8 * (16 * kDim) + 256 * nb + 16 * col);
        }
      }
    }
  };
  int j = run.first + wave;
  if (j < run.end) {
    load_keys(j);
    load_values(j);
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
  half8 q[2];
#pragma unroll
  for (int s = 0; s < 2; ++s) q[s] = __builtin_bit_cast(half8, sq[col][2 * grp + s]);
  const float c = sc[col];
  const int place = p_first + (col < rows ? col : 0) / a.G;

  f32x4 acc[4];
#pragma unroll
  for (int nb = 0; nb < 4; ++nb) acc[nb] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  float m = -INFINITY, l = 0.0f;
  while (j < run.end) {
    const int t0 = tile_start(seen, j);
    float y[2][8];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        f32x4 d = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          uint32_t pl[K > 0 ? K : 1];
#pragma unroll
          for (int p = 0; p < K; ++p) pl[p] = kp[kb][s][p] >> (8 * h);
          d = __builtin_amdgcn_mfma_f32_16x16x32_f16(paged_weights<K>(h ? kc[kb][s].y : kc[kb][s].x, pl),
                                                     q[h], d, 0, 0, 0);
        }
        const float4 sv = ks[kb][s];
        y[kb][4 * s] = d[0] * sv.x;
        y[kb][4 * s + 1] = d[1] * sv.y;
        y[kb][4 * s + 2] = d[2] * sv.z;
        y[kb][4 * s + 3] = d[3] * sv.w;
      }
    const int jn = j + NW;
    if (jn < run.end) load_keys(jn);
    const bool part = !all_seen(p_first, p_last, t0, a.window, a.n_sink) || __any(!there[0] || !there[1]);
    if (part) {
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int key = t0 + 32 * kb + 8 * grp + i;
          if (!(there[kb] && key < seen.end && sees(place, key, a.window, a.n_sink))) y[kb][i] = -INFINITY;
        }
    }
    float top = y[0][0];
#pragma unroll
    for (int i = 1; i < 16; ++i) top = fmaxf(top, y[i >> 3][i & 7]);
    const auto r16 = __builtin_amdgcn_permlane16_swap(__float_as_uint(top), __float_as_uint(top), false, false);
    top = fmaxf(__uint_as_float(r16[0]), __uint_as_float(r16[1]));
    const auto r32 = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
    top = fmaxf(__uint_as_float(r32[0]), __uint_as_float(r32[1]));
    const bool rises = top > m && (m == -INFINITY || (top - m) * c > kMostRise);
    if (__any(rises)) {
      const float to = rises ? top : m, f = between(m, to, c);
#pragma unroll
      for (int nb = 0; nb < 4; ++nb) acc[nb] *= f;
      l *= f;
      m = to;
    }
    uint32_t hi[2][4], lo[2][4];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      float p[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) p[i] = paged_weight(y[kb][i], m, c);
      if (part) {
#pragma unroll
        for (int i = 0; i < 8; ++i) p[i] = y[kb][i] == -INFINITY ? 0.0f : p[i];
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        l += p[2 * i];
        l += p[2 * i + 1];
        hi[kb][i] = pack_half(p[2 * i], p[2 * i + 1]);
        lo[kb][i] = low_part(p[2 * i], p[2 * i + 1], hi[kb][i]);
      }
    }
    auto fragment = [&](int kb, int nb) -> half8 {
      uint4 v;
      if constexpr (VF == POT_VALUES_INT4) {
        const uint4 w = vr.f[kb];
        const uint32_t w0 = nb < 2 ? w.x : w.z, w1 = nb < 2 ? w.y : w.w;
        v = int4_values((nb & 1 ? w0 >> 4 : w0) & 0x0F0F0F0Fu, (nb & 1 ? w1 >> 4 : w1) & 0x0F0F0F0Fu,
                        vr.s[kb], vr.z[kb]);
      } else {
        v = vr.f[kb][nb];
      }
      return __builtin_bit_cast(half8, part ? mask_tokens(v, t0 + 32 * kb + 8 * grp, seen.end) : v);
    };
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      const half8 ph = __builtin_bit_cast(half8, make_uint4(hi[kb][0], hi[kb][1], hi[kb][2], hi[kb][3]));
      const half8 pl = __builtin_bit_cast(half8, make_uint4(lo[kb][0], lo[kb][1], lo[kb][2], lo[kb][3]));
#pragma unroll
      for (int nb = 0; nb < 4; ++nb) {
        half8 v = fragment(kb, nb);
        if (part && __any(has_special(__builtin_bit_cast(uint4, v)))) {
          half8 marks, ones;
          split_special(v, &v, &marks);
#pragma unroll
          for (int i = 0; i < 8; ++i) ones[i] = y[kb][i] == -INFINITY ? (_Float16)0.0f : (_Float16)1.0f;
          const f32x4 n = __builtin_amdgcn_mfma_f32_16x16x32_f16(marks, ones, f32x4{0.0f, 0.0f, 0.0f, 0.0f}, 0, 0, 0);
#pragma unroll
          for (int i = 0; i < 4; ++i) acc[nb][i] += special_sum(n[i]);
        }
        acc[nb] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, ph, acc[nb], 0, 0, 0);
        acc[nb] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, pl, acc[nb], 0, 0, 0);
      }
    }
    if (jn < run.end) load_values(jn);
    j = jn;
  }

  // ---- the waves' sums -------------------------------------------------------------------
  {
    const auto r16 = __builtin_amdgcn_permlane16_swap(__float_as_uint(l), __float_as_uint(l), false, false);
    l = __uint_as_float(r16[0]) + __uint_as_float(r16[1]);
    const auto r32 = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
    l = __uint_as_float(r32[0]) + __uint_as_float(r32[1]);
  }
  if (lane < R) {
    sm[wave][col] = m;
    sl[wave][col] = l;
  }
#pragma unroll
  for (int nb = 0; nb < 4; ++nb)
    *reinterpret_cast<f32x4*>(&so[wave][col][16 * nb + 4 * grp]) = acc[nb];
  __syncthreads();
  const int r = tid / 16, d = 4 * (tid & 15);
  if (r >= rows) return;
  const float cr = sc[r];
  float M = sm[0][r];
#pragma unroll
  for (int w = 1; w < NW; ++w) M = fmaxf(M, sm[w][r]);
  float L = 0.0f;
  f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int w = 0; w < NW; ++w) {
    const float f = between(sm[w][r], M, cr);
    L += f * sl[w][r];
    o += f * *reinterpret_cast<const f32x4*>(&so[w][r][d]);
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

template <int K, int VF>
hipError_t launch_few(const PagedAttendArgs& a, hipStream_t stream) {
  hipLaunchKernelGGL((paged_few_kernel<K, VF>),
                     dim3((uint32_t)a.plan.few_splits, (uint32_t)a.pages.Hkv, (uint32_t)a.packed.B),
                     dim3(64 * kFewWaves), 0, stream, a);
  return hipGetLastError();
}

}  // namespace potattn
