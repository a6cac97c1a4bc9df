// Attention over a paged cache for sequences with many rows (new tokens x query heads of a kv
// head): chunks of prompts. A workgroup takes a tile of R rows of one sequence and kv head, 32 a
// wave, and goes through the 64-key tiles that some of its rows see; the keys' codes and the values
// become fp16 operands in LDS once for all its waves, the next tile's loads under way meanwhile.
//
// Scores S^T = K Q^T by v_mfma_f32_32x32x16_f16 (codes as fp16 weights, the INT8 queries as fp16
// integers: exact sums), the rows of K in such an order that a lane ends up with the scores of
// one query and 8 consecutive keys of every 16: the operand of O^T = V^T P^T as they stand. A
// query's reference, sum and outputs are its two lanes' own. The reference rises only when weights
// would leave fp16's range.
//
// Bound: VALU issue. Of 32 rows and 64 keys a wave has 16 matrix instructions and 216 operations (at k = 1
// and fp16 values; 331 at k = 4 and 4 bits): two products, an exponential and its half of a maximum, of a
// pack and of a sum a score, then the tile's staging. Counted over whole calls, with the tiles at the
// diagonal and the window's ends, 16.8 VALU instructions a matrix instruction, itself among them, and 28.2.
// VALU is 74% busy in both, the matrix cores 32% and 19%; four waves a SIMD, for which the queries stand in
// LDS (one row block a wave at 128 registers; when this took 410 us, two blocks at 256 took 430, two blocks
// whose weights and products alternate 560, 16 waves a workgroup 399 but more on short calls). 8192 tokens of
// 32 + 4 heads, k = 1, fp16 values: 417 us, 660 TFLOP/s; 2 x 2048 tokens with a window of 1000, k = 4, 4 bits:
// 81 us.
#pragma once

#include "paged.hpp"

namespace potattn {

// What a sequence asks for: its row tiles, and the 64-key tiles that the last of them sees.
struct ManyShape {
  int rows, keys;
};
__device__ __forceinline__ ManyShape many_shape(const PagedAttendArgs& a, int b, int R) {
  if (b >= a.packed.B) return {0, 0};
  const NewTokens t = sequence_tokens(a.packed, b, a.max_new, a.max_len);
  const int rows = t.n * a.G;
  if (t.n <= a.plan.few_limit && rows <= a.plan.few_limit) return {0, 0};
  const int n = (rows + R - 1) / R;
  return {n, max(1, seen_tiles(t.place + (n - 1) * R / a.G, t.place + t.n - 1, t.len, a.window, a.n_sink).tiles)};
}
__device__ __forceinline__ int wave_scan(int v, int lane) {  // sums up to and with the lane's
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int u = __shfl_up(v, o, 64);
    v += lane >= o ? u : 0;
  }
  return v;
}

// A workgroup's piece: row tile `tile` of sequence b, key range `split` of `splits`. A row tile's
// keys are split when the row tiles do not fill the chip (many_extra > 0): into ranges of equal
// length for all sequences (piece_range), the shortest (to the step) for which kManyPieces of them take
// the whole work; a short sequence's rows stay whole. Pieces count from the last sequence's last: a
// prompt's late tiles, which see the most keys, come first. A row tile's pieces are first .. first +
// splits - 1. b < 0: there is no piece i. Every thread of the workgroup takes part, a sequence a thread.
struct RowPiece {
  int b, tile, split, splits, first;
};
template <int NW>
struct FindScratch {
  int64_t sums[2][NW];
  RowPiece found;
};
template <int NW>
__device__ __forceinline__ RowPiece find_piece(const PagedAttendArgs& a, int i, int R, FindScratch<NW>& sh) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const ManyShape mine = many_shape(a, tid, R);
  auto shape = [&](int b0) { return b0 == 0 ? mine : many_shape(a, b0 + tid, R); };
  auto over_group = [&](auto& v) {  // each of the thread's numbers summed over the workgroup
    constexpr int N = sizeof(v) / sizeof(v[0]);
#pragma unroll
    for (int i = 0; i < N; ++i) {
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) v[i] += __shfl_xor((long long)v[i], o, 64);
      if (lane == 0) sh.sums[i][wave] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      v[i] = 0;
#pragma unroll
      for (int w = 0; w < NW; ++w) v[i] += sh.sums[i][w];
    }
    __syncthreads();
  };
  const int extra = a.plan.many_extra;
  int64_t all[2] = {0, 0};  // work, row tiles
  if (extra > 0) {
    for (int b0 = 0; b0 < a.packed.B; b0 += 64 * NW) {
      const ManyShape m = shape(b0);
      all[0] += (int64_t)m.rows * m.keys;
      all[1] += m.rows;
    }
    over_group(all);
  }
  const PieceRange plan = piece_range(extra, (int64_t)a.packed.n * a.G / R, all[0], all[1], [&](int range) {
    int64_t n[1] = {0};
    for (int b0 = 0; b0 < a.packed.B; b0 += 64 * NW) {
      const ManyShape m = shape(b0);
      n[0] += pieces_of(m.rows, m.keys, range);
    }
    over_group(n);
    return n[0];
  });
  const int64_t total = plan.total;
  if (tid == 0) sh.found.b = -1;
  const int64_t at = total - 1 - i;
  int64_t before = 0;  // pieces of the sequences before
  for (int b0 = 0; b0 < a.packed.B && at >= before; b0 += 64 * NW) {  // uniform
    const ManyShape m = shape(b0);
    const int n = pieces_of(m.rows, m.keys, plan.range), sum = wave_scan(n, lane);
    if (lane == 63) sh.sums[0][wave] = sum;
    __syncthreads();
    int64_t start = before + sum - n;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      start += w < wave ? sh.sums[0][w] : 0;
      before += sh.sums[0][w];
    }
    if (at >= start && at < start + n) {
      const int S = n / m.rows, j = (int)(at - start), tile = j / S;
      sh.found = {b0 + tid, tile, j - tile * S, S, (int)(total - (start + (int64_t)(tile + 1) * S))};
    }
    __syncthreads();
  }
  __syncthreads();
  const RowPiece p = sh.found;
  return {__builtin_amdgcn_readfirstlane(p.b), __builtin_amdgcn_readfirstlane(p.tile),
          __builtin_amdgcn_readfirstlane(p.split), __builtin_amdgcn_readfirstlane(p.splits),
          __builtin_amdgcn_readfirstlane(p.first)};
}

template <int VF>
struct ManyStage {  // what a lane loads of a group of 8 keys
  uint32_t code, plane[4];
  float scale;
  uint4 v;
};
template <>
struct ManyStage<POT_VALUES_INT4> {
  uint32_t code, plane[4];
  float scale;
  uint2 n;
  uint32_t s, z;  // two of the 8 steps and minima, those of lane % 4
};
// The four lanes' dwords in each of them.
__device__ __forceinline__ uint4 quad_dwords(uint32_t x) {
  return make_uint4(__builtin_amdgcn_mov_dpp(x, 0x00, 0xF, 0xF, true), __builtin_amdgcn_mov_dpp(x, 0x55, 0xF, 0xF, true),
                    __builtin_amdgcn_mov_dpp(x, 0xAA, 0xF, 0xF, true), __builtin_amdgcn_mov_dpp(x, 0xFF, 0xF, 0xF, true));
}


// R: rows of a tile. LOW: what rounding to fp16 leaves of the weights goes into the products too. Outputs of
// 32 bits have it. For outputs of 16 bits that rounding (half a step of fp16) is no larger than the output's
// own: their error against 64 bits is 1.7e-3 of the outputs' size for bf16, as with weights of 32 bits, and
// 2.5e-4 for fp16 (2.1e-4 with weights of 32 bits); LOW takes 8192 tokens from 417 us to 536 and 512 on 8192
// keys from 74 to 87.
template <int K, int VF, int R, bool LOW>
__global__ __launch_bounds__(2 * R) __attribute__((amdgpu_waves_per_eu(R == 128 ? 3 : 4)))
void paged_many_kernel(const PagedAttendArgs a) {
  constexpr int NW = R / 32, kGroups = 8 / NW;  // groups a wave stages
  struct Tile {
    uint4 k[8 * 65];  // chunk d (dimensions 8d ..+7) of key j at 65 d + j
    uint4 v[8 * 64];  // tokens 8g ..+7 of dimension d at 64 g + d
  };
  __shared__ Tile tiles[2];
  __shared__ __attribute__((aligned(16))) float scales[2][64];
  __shared__ __attribute__((aligned(16))) int flags[2][8];  // of a group: 1 not there, 2 holds special values
  __shared__ uint4 queries[R * 9];  // chunk d of row r at 9 r + d; a wave's own rows
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int Hkv = a.pages.Hkv, kvh = blockIdx.x % Hkv, index = blockIdx.x / Hkv;
  __shared__ FindScratch<NW> scratch;
  const RowPiece at = find_piece(a, index, R, scratch);
  if (a.plan.many_extra > 0 && kvh == 0 && tid == 0)
    a.many_pieces[index] = make_int4(at.b, at.tile, at.splits, at.first);
  if (at.b < 0) return;
  const NewTokens t = sequence_tokens(a.packed, at.b, a.max_new, a.max_len);
  const int rows = t.n * a.G, r0 = at.tile * R;
  const int last = min(r0 + R, rows) - 1;
  const int wg_first = t.place + r0 / a.G, wg_last = t.place + last / a.G;
  const SeenTiles seen = seen_tiles(wg_first, wg_last, t.len, a.window, a.n_sink);
  const TileRun run = split_tiles(seen.tiles, at.split, at.splits);
  const int32_t* table = a.pages.table + (int64_t)at.b * a.pages.table_len;
  const int col = lane & 31, half = lane >> 5;
  const int wr0 = r0 + 32 * wave;  // the wave's first row

  // ---- staging: wave w has groups w, w + NW .. of the tile --------------------------------
  ManyStage<VF> st[kGroups];
  int st_row[kGroups], next_row[kGroups];  // first cache row / 8, -1: not there
  auto find_rows = [&](int j) {
    const int g0 = tile_start(seen, min(j, run.end - 1)) / 8;
#pragma unroll
    for (int i = 0; i < kGroups; ++i) {
      const int g = g0 + wave + NW * i;
      next_row[i] = g * 8 < seen.end ? group_row8(a.pages, table, kvh, g) : -1;
    }
  };
  auto load = [&]() {  // the groups of next_row; those not there read row 0
#pragma unroll
    for (int i = 0; i < kGroups; ++i) {
      st_row[i] = next_row[i];
      // uniform, and said to be: addresses in scalar registers, a lane's offset once
      const int64_t row8 = __builtin_amdgcn_readfirstlane(max(next_row[i], 0));
      st[i].code = reinterpret_cast<const uint32_t*>(a.pages.codes_se + row8 * 256)[lane];
      const uint8_t* planes = a.pages.codes_m + row8 * (64 * K);
#pragma unroll
      for (int p = 0; p < K; ++p) st[i].plane[p] = planes[(uint32_t)((lane >> 3) * 8 * K + (lane & 7)) + 8 * p];
      st[i].scale = (a.pages.key_scale + row8 * 8)[lane & 7];
      if constexpr (VF == POT_VALUES_INT4) {
        const uint8_t* rec = a.pages.values + row8 * kI4GroupBytes;
        st[i].n = *reinterpret_cast<const uint2*>(rec + (uint32_t)(16 * (lane & 15) + 8 * (lane >> 5)));
        st[i].s = reinterpret_cast<const uint32_t*>(rec + kI4Steps)[lane & 3];
        st[i].z = reinterpret_cast<const uint32_t*>(rec + kI4Minima)[lane & 3];
      } else {
        st[i].v = reinterpret_cast<const uint4*>(a.pages.values + row8 * (16 * kDim))[lane];
      }
    }
  };
  auto stage = [&](int t0, int buf) {
    const bool part = !whole_tile(seen, wg_first, wg_last, t0, a.window, a.n_sink);
#pragma unroll
    for (int i = 0; i < kGroups; ++i) {
      const int g = wave + NW * i, key = 8 * g + (lane >> 3), d = lane & 7;
      tiles[buf].k[65 * d + key] = __builtin_bit_cast(uint4, paged_weights<K>(st[i].code, st[i].plane));
      if (lane < 8) scales[buf][8 * g + lane] = st[i].scale;
      uint4 v;
      if constexpr (VF == POT_VALUES_INT4) {
        const int sh = (lane & 16) ? 4 : 0;
        v = int4_values((st[i].n.x >> sh) & 0x0F0F0F0Fu, (st[i].n.y >> sh) & 0x0F0F0F0Fu,
                        quad_dwords(st[i].s), quad_dwords(st[i].z));
      } else {
        v = st[i].v;
      }
      int flag = st_row[i] >= 0 ? 0 : 1;
      if (part || flag) {  // uniform
        v = mask_tokens(v, t0 + 8 * g, flag ? 0 : seen.end);
        if (__any(has_special(v))) {
          flag |= 2;
          v = without_special(v);
        }
      }
      tiles[buf].v[64 * g + lane] = v;
      if (lane == 0) flags[buf][g] = flag;
    }
  };
  if (run.first < run.end) {
    find_rows(run.first);
    load();
    find_rows(run.first + 1);
  }

  // ---- queries: 8 rows of the wave at a time, 8 lanes each ---------------------------------
  uint4* sq = queries + wave * 32 * 9;
  float c = 0.0f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int rw = 8 * i + (lane >> 3), r = wr0 + rw;
    float x[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
    if (r < rows) {
      const int tok = r / a.G, head = a.q_head(kvh * a.G + (r - tok * a.G));
      load8(a.q, (int64_t)(t.first + tok) * a.q_stride_t + head * a.q_stride_h, lane & 7, a.dtype, x);
    }
    float factor;
    sq[rw * 9 + (lane & 7)] = quantised_query(x, a.hadamard, lane, &factor);
    // row 8 i + lane / 8 has its factor in 8 lanes; lane col wants that of row col
    const float got = __shfl(factor, 8 * (col & 7), 64);
    if ((col >> 3) == i) c = got;
  }
  const bool active = wr0 < rows;
  const int w_first = t.place + min(wr0, last) / a.G, w_last = t.place + min(wr0 + 31, last) / a.G;
  const int place = t.place + min(wr0 + col, last) / a.G;

  f32x16 acc[2];
  Reference ref;
  float l = 0.0f;
#pragma unroll
  for (int i = 0; i < 16; ++i) acc[0][i] = acc[1][i] = 0.0f;

  const half2v kOnes = {(_Float16)1.0f, (_Float16)1.0f};
  auto compute = [&](bool part, int t0, int buf) {
    // Places in LDS. Where a tile's loads take the most registers they are made anew for each tile: kept
    // through the loop, they leave reloads from memory behind the loads under way (2 x 2048 tokens with a window
    // of 1000, k = 4, 4 bits: 82 us, kept 85; 8192 tokens, k = 1, fp16 values: 438, kept 431).
    int ln = lane;
    if constexpr (K > 0 && VF == POT_VALUES_INT4) asm volatile("" : "+v"(ln));
    const int col = ln & 31, half = ln >> 5;
    // row of K for the lane: key 16 (col / 16) + 8 (col / 4 % 2) + 4 (col / 8 % 2) + col % 4
    const int krow = (col & 16) | ((col & 4) << 1) | ((col & 8) >> 1) | (col & 3);
    const Tile& T = tiles[buf];
    f32x16 s[2];
#pragma unroll
    for (int i = 0; i < 16; ++i) s[0][i] = s[1][i] = 0.0f;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int step = 0; step < 4; ++step) {
        const int d = 2 * step + half;
        const half8 kv = __builtin_bit_cast(half8, T.k[65 * d + 32 * kb + krow]);
        const half8 q = __builtin_bit_cast(half8, sq[9 * col + d]);
        s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_f16(kv, q, s[kb], 0, 0, 0);
      }
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const float4* sp = reinterpret_cast<const float4*>(&scales[buf][32 * kb + 16 * u + 8 * half]);
        const float4 a0 = sp[0], a1 = sp[1];
        const float sv[8] = {a0.x, a0.y, a0.z, a0.w, a1.x, a1.y, a1.z, a1.w};
#pragma unroll
        for (int i = 0; i < 8; ++i) s[kb][8 * u + i] *= sv[i];
      }
    if (part) {  // uniform
      const SeenKeys sk = seen_keys(a, place, seen.end, t0 + 8 * half);
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const uint32_t mask = flags[buf][4 * kb + 2 * u + half] & 1 ? 0u : seen_bits(sk, 32 * kb + 16 * u);
#pragma unroll
          for (int i = 0; i < 8; ++i) s[kb][8 * u + i] = if_seen(s[kb][8 * u + i], mask, i);
        }
    }
    float top = fmaxf(s[0][0], s[0][1]);
#pragma unroll
    for (int i = 2; i < 32; ++i) top = fmaxf(top, s[i >> 4][i & 15]);
    const auto r32 = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
    top = fmaxf(__uint_as_float(r32[0]), __uint_as_float(r32[1]));
    if (must_rise(ref, top, c)) {
      const float f = raise(ref, top, c);
      acc[0] *= f;
      acc[1] *= f;
      l *= f;
    }
    if (ref.far) {  // uniform
      s[0] -= ref.m;
      s[1] -= ref.m;
    }
    const float shift = weight_shift(ref);
    float tile_l = 0.0f;  // the tile's weights go onto l together: each alone would be rounded at l's size
#pragma unroll
    for (int b = 0; b < 4; ++b) {  // 16 keys at a time
      const int kb = b >> 1, e0 = 8 * (b & 1);
      uint32_t hi[4], lo[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float p0 = weight_of(s[kb][e0 + 2 * i], c, shift), p1 = weight_of(s[kb][e0 + 2 * i + 1], c, shift);
        hi[i] = pack_half(p0, p1);
        if constexpr (LOW) {
          tile_l += p0;
          tile_l += p1;
          lo[i] = low_part(p0, p1, hi[i]);
        } else {  // of the weights as they are multiplied
          tile_l = __builtin_amdgcn_fdot2(__builtin_bit_cast(half2v, hi[i]), kOnes, tile_l, false);
        }
      }
#pragma unroll
      for (int nb = 0; nb < 2; ++nb) {
        const half8 v = __builtin_bit_cast(half8, T.v[64 * (2 * b + half) + 32 * nb + col]);
        const half8 ph = __builtin_bit_cast(half8, make_uint4(hi[0], hi[1], hi[2], hi[3]));
        acc[nb] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v, ph, acc[nb], 0, 0, 0);
        if constexpr (LOW) {
          const half8 pl = __builtin_bit_cast(half8, make_uint4(lo[0], lo[1], lo[2], lo[3]));
          acc[nb] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v, pl, acc[nb], 0, 0, 0);
        }
      }
    }
    l += tile_l;
  };
  bool special = false;  // a tile in part held special values (paged.hpp); uniform
  auto tile = [&](int t0, int buf) {
    if (!active || none_seen(w_first, w_last, t0, a.window, a.n_sink)) return;
    const int4 f0 = *reinterpret_cast<const int4*>(&flags[buf][0]);
    const int4 f1 = *reinterpret_cast<const int4*>(&flags[buf][4]);
    const int any = __builtin_amdgcn_readfirstlane(f0.x | f0.y | f0.z | f0.w | f1.x | f1.y | f1.z | f1.w);
    compute(!whole_tile(seen, w_first, w_last, t0, a.window, a.n_sink) || (any & 1), t0, buf);
    special |= (any & 2) != 0;
  };

  int buf = 0;
  if (run.first < run.end) stage(tile_start(seen, run.first), 0);
  // a barrier a tile: it stands between the staging of a place and its use, and between its use
  // and its next staging, which comes a tile later
#pragma nounroll
  for (int j = run.first; j < run.end; ++j) {
    __syncthreads();
    if (j + 1 < run.end) {
      load();
      find_rows(j + 2);
    }
    tile(tile_start(seen, j), buf);
    if (j + 1 < run.end) stage(tile_start(seen, j + 1), buf ^ 1);
    buf ^= 1;
  }

  if (special) {
#pragma nounroll
    for (int j = run.first; j < run.end; ++j) {
      const int t0 = tile_start(seen, j);
      if (whole_tile(seen, wg_first, wg_last, t0, a.window, a.n_sink)) continue;
      const SeenKeys sk = seen_keys(a, place, seen.end, t0 + 8 * half);
#pragma nounroll
      for (int b = 0; b < 4; ++b) {
        const int g = 2 * b + half;
        const int row8 = t0 + 8 * g < seen.end ? group_row8(a.pages, table, kvh, t0 / 8 + g) : -1;
        const uint32_t mask = row8 >= 0 ? seen_bits(sk, 16 * b) : 0u;
        half8 ones;
#pragma unroll
        for (int i = 0; i < 8; ++i) ones[i] = (mask >> i) & 1 ? (_Float16)1.0f : (_Float16)0.0f;
#pragma unroll
        for (int nb = 0; nb < 2; ++nb) {
          uint4 v = make_uint4(0u, 0u, 0u, 0u);
          if (row8 >= 0) v = mask_tokens(group_values<VF>(a.pages, row8, 32 * nb + col), t0 + 8 * g, seen.end);
          f32x16 n;
#pragma unroll
          for (int i = 0; i < 16; ++i) n[i] = 0.0f;
          n = __builtin_amdgcn_mfma_f32_32x32x16_f16(special_marks(v), ones, n, 0, 0, 0);
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[nb][i] += special_sum(n[i]);
        }
      }
    }
  }

  const auto r32 = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
  l = __uint_as_float(r32[0]) + __uint_as_float(r32[1]);
  const int row = wr0 + col;
  if (row >= rows) return;
  if (at.splits == 1) {
    const int tok = row / a.G, head = a.q_head(kvh * a.G + (row - tok * a.G));
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    const int64_t base = ((int64_t)(t.first + tok) * a.Hq + head) * kDim + 4 * half;
#pragma unroll
    for (int nb = 0; nb < 2; ++nb)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        store_out4(a.out, base + 32 * nb + 8 * i, a.out_dtype, acc[nb][4 * i] * inv, acc[nb][4 * i + 1] * inv,
                   acc[nb][4 * i + 2] * inv, acc[nb][4 * i + 3] * inv);
    return;
  }
  const float f = exact_reference(ref, c);
  float* part = a.many_part + (((int64_t)index * Hkv + kvh) * R + (row - r0)) * kPartial;
#pragma unroll
  for (int nb = 0; nb < 2; ++nb)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *reinterpret_cast<f32x4*>(part + 32 * nb + 8 * i + 4 * half) =
          f32x4{acc[nb][4 * i] * f, acc[nb][4 * i + 1] * f, acc[nb][4 * i + 2] * f, acc[nb][4 * i + 3] * f};
  if (half == 0) *reinterpret_cast<f32x4*>(part + kDim) = f32x4{ref.m, l * f, c, 0.0f};
}

template <int K, int VF, int R>
hipError_t launch_many(const PagedAttendArgs& a, hipStream_t stream) {
  const dim3 grid((uint32_t)((a.plan.many_tiles + a.plan.many_extra) * a.pages.Hkv));
  if (a.out_dtype == POT_FP32)
    hipLaunchKernelGGL((paged_many_kernel<K, VF, R, true>), grid, dim3(2 * R), 0, stream, a);
  else
    hipLaunchKernelGGL((paged_many_kernel<K, VF, R, false>), grid, dim3(2 * R), 0, stream, a);
  return hipGetLastError();
}

}  // namespace potattn
