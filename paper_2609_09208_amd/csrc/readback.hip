// Cache rows back to dense fp16 rows. Every code byte is read once and every row written
// once, 128 bytes: the memory stream bounds these kernels, the writes most of it.
#include "pot_device.hpp"
#include "row_groups.hpp"

namespace potattn {

typedef float float2v __attribute__((ext_vector_type(2)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef _Float16 half8v __attribute__((ext_vector_type(8)));

__device__ __forceinline__ uint32_t pack_half(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((float2v{a, b}), half2v));
}

// Rows are written past the caches: nothing of the launch reads them again, and the codes
// keep their room (2 M rows of 4-bit values 77.6 -> 50.6 us, INT8 83.7 -> 72.5).
typedef uint32_t u32x4v __attribute__((ext_vector_type(4)));
__device__ __forceinline__ void write_row_part(uint16_t* p, uint32_t a, uint32_t b, uint32_t c,
                                               uint32_t d) {
  __builtin_nontemporal_store((u32x4v{a, b, c, d}), reinterpret_cast<u32x4v*>(p));
}

// The upper half of the wave's a for the lower half's b.
__device__ __forceinline__ void swap32(uint32_t& a, uint32_t& b) {
  const auto r = __builtin_amdgcn_permlane32_swap(a, b, false, false);
  a = r[0];
  b = r[1];
}

// Cache row of row i of the range (the range's rows in order).
__device__ __forceinline__ int64_t cache_row(const RowRange& r, uint32_t i) {
  const uint32_t s = i / (uint32_t)r.n_tok;
  return s * r.t_cap + r.t0 + (i - s * (uint32_t)r.n_tok);
}

// ---- keys ------------------------------------------------------------------------
// The 8 elements of one code dword as fp16 numbers sigma (1 + j / 2^K) 2^-e (0 for the
// zero code). The high byte of such a number depends on the code's four bits alone up to
// the mantissa's top two: v_perm_b32 looks four of them up at once. Mantissa bits are
// spread from a plane's byte to the four even or odd elements by a multiplication (of every
// second bit: the sums' carries end in the gaps).
template <int K>
__device__ __forceinline__ void codes_to_half(uint32_t w, const uint32_t* plane, uint32_t (&out)[4]) {
  // bytes e = 0 .. 7: (15 - e) << 2, the exponent field of 2^-e; 0 at e = 7
  constexpr uint32_t kLut0 = 0x3034383Cu, kLut1 = 0x0024282Cu;
  // all ones where e != 7
  constexpr uint32_t kSome1 = 0x00FFFFFFu;
  const uint32_t sel[2] = {w & 0x07070707u, (w >> 4) & 0x07070707u};  // even, odd elements
  uint32_t hi[2], lo[2] = {0u, 0u};
#pragma unroll
  for (int o = 0; o < 2; ++o) {
    hi[o] = __builtin_amdgcn_perm(kLut1, kLut0, sel[o]);
    if constexpr (K > 0) {
      uint32_t m = 0;
#pragma unroll
      for (int b = 0; b < K; ++b) {
        // bit 2 i + o of the plane byte to bit 8 i
        const uint32_t bits = __umul24((plane[b] >> o) & 0x55u, 0x41041u) & 0x01010101u;
        const int at = 9 - (K - 1 - b);  // its place in the fp16 number
        if (at >= 8) m |= bits << (at - 8);
        else lo[o] |= bits << at;
      }
      const uint32_t some = __builtin_amdgcn_perm(kSome1, 0xFFFFFFFFu, sel[o]);
      hi[o] |= m & some;
      lo[o] &= some;
    }
    hi[o] |= (o ? w : w << 4) & 0x80808080u;
  }
  if constexpr (K <= 2) {
    // byte pairs (0, high byte) of elements 2c and 2c + 1
#pragma unroll
    for (int c = 0; c < 4; ++c)
      out[c] = __builtin_amdgcn_perm(hi[1], hi[0], 0x040C000Cu + 0x01000100u * c);
  } else {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t sel2 = h ? 0x07030602u : 0x05010400u;  // (low, high) of two elements
      const uint32_t ev = __builtin_amdgcn_perm(hi[0], lo[0], sel2);
      const uint32_t od = __builtin_amdgcn_perm(hi[1], lo[1], sel2);
      out[2 * h] = __builtin_amdgcn_perm(od, ev, 0x05040100u);
      out[2 * h + 1] = __builtin_amdgcn_perm(od, ev, 0x07060302u);
    }
  }
}
// s times a number that is 0 for the zero code, whatever s is.
__device__ __forceinline__ float scaled(float w, float s) { return w == 0.0f ? 0.0f : w * s; }

struct KeysIn {
  const uint8_t* codes_se;
  const uint8_t* codes_m;
  const float* key_scale;
};

// Eight rows a wave: lane l has elements 8 (l % 8) ..+7 of row l / 8. Where all its scales
// are fp16 numbers (row maxima of fp16 keys are) one packed multiplication rounds the
// product as the fp32 one and its conversion do. 2.1 M rows, k = 0 to 4: 47, 62, 68, 68 and
// 71 us, 5.6 to 7.2 TB/s (plane bytes by one a lane, eight of a row side by side).
template <int K>
__global__ __launch_bounds__(kBlock) void load_keys_kernel(const KeysIn in, RowRange r,
                                                           uint16_t* __restrict__ out) {
  const int lane = lane_id(), g = lane & 7;
  const uint32_t n = (uint32_t)(r.n_seq * r.n_tok);
  for (uint32_t wave = first_wave(); wave * 8 < n; wave += wave_stride()) {
    const uint32_t i = wave * 8 + (lane >> 3);
    if (i >= n) return;
    const int64_t row = cache_row(r, i);
    const uint32_t w = reinterpret_cast<const uint32_t*>(in.codes_se)[row * 8 + g];
    const float s = in.key_scale[row];
    uint32_t plane[K > 0 ? K : 1];
#pragma unroll
    for (int b = 0; b < K; ++b) plane[b] = in.codes_m[row * 8 * K + 8 * b + g];
    uint32_t h[4];
    codes_to_half<K>(w, plane, h);
    const _Float16 s16 = (_Float16)s;
    uint32_t y[4];
    if (__all((float)s16 == s && fabsf(s) < 65505.0f)) {
#pragma unroll
      for (int c = 0; c < 4; ++c)
        y[c] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(half2v, h[c]) * half2v{s16, s16});
    } else {
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const half2v v = __builtin_bit_cast(half2v, h[c]);
        y[c] = pack_half(scaled((float)v.x, s), scaled((float)v.y, s));
      }
    }
    write_row_part(out + (int64_t)i * kDim + 8 * g, y[0], y[1], y[2], y[3]);
  }
}

// Rotated back, sixteen rows a wave, on the matrix cores: +-1 times the codes' numbers is
// exact in fp32 (integers below 2^17 in units of 2^-10), so s / 8 times the sum is one
// rounding more than the definition's last. B: lane l has elements 16 (l / 16) ..+15 of row
// l % 16, 8 to a K-block. A = H with its rows in the order that gives lane l those same
// elements of the result: one 8-byte load of codes and 32 bytes written per lane.
//
// H's signs: row m = 16 (col / 4) + 4 nb + col % 4 against column 16 blk + 8 kb + j. Bit 3
// (kb) meets nb's high bit, where the second K-block is negated; bit 2 (of j) meets nb's
// low bit; the rest is the lane's. Two fragments do for all eight. (One byte or dword load
// per K-block and plane, and a fragment for each nb: 64 x 32768 rows 109 us at k = 0 and 4.)
template <int K>
__global__ __launch_bounds__(kBlock) void load_keys_rotated_kernel(const KeysIn in, RowRange r,
                                                                   uint16_t* __restrict__ out) {
  const int lane = lane_id(), col = lane & 15, blk = lane >> 4;
  const uint32_t n = (uint32_t)(r.n_seq * r.n_tok);
  constexpr uint32_t kSigns = 0x80008000u;
  const uint32_t base = 0x3C003C00u ^ (__popc((col >> 2) & blk) & 1 ? kSigns : 0u) ^
                        (col & 1 ? 0x80000000u : 0u);
  const uint32_t next = base ^ (col & 2 ? kSigns : 0u);  // j = 2, 3
  const half8v h[2] = {
      __builtin_bit_cast(half8v, make_uint4(base, next, base, next)),
      __builtin_bit_cast(half8v, make_uint4(base, next, base ^ kSigns, next ^ kSigns))};
  for (uint32_t wave = first_wave(); wave * 16 < n; wave += wave_stride()) {
    const uint32_t i = wave * 16 + col;
    const bool there = i < n;
    const int64_t row = cache_row(r, there ? i : n - 1);
    const uint2 codes = reinterpret_cast<const uint2*>(in.codes_se)[row * 4 + blk];
    uint32_t planes[K > 0 ? K : 1];  // 16 bits of each plane
    if constexpr (K == 4) {
      // one plane a lane, and a 4 x 4 transpose of 16-bit parts over the row's four lanes
      const uint2 p = reinterpret_cast<const uint2*>(in.codes_m)[row * 4 + blk];
      uint32_t part[2] = {p.x, p.y};
      swap32(part[0], part[1]);
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const auto t = __builtin_amdgcn_permlane16_swap(part[c], part[c], false, false);
        const uint32_t d = __builtin_amdgcn_perm(t[1], t[0], blk & 1 ? 0x07060302u : 0x05040100u);
        planes[2 * c] = d & 0xFFFFu;
        planes[2 * c + 1] = d >> 16;
      }
    } else {
#pragma unroll
      for (int b = 0; b < K; ++b)
        planes[b] = reinterpret_cast<const uint16_t*>(in.codes_m)[(row * K + b) * 4 + blk];
    }
    const float s = in.key_scale[row] * 0.125f;
    uint32_t x[2][4];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      uint32_t plane[K > 0 ? K : 1];
#pragma unroll
      for (int b = 0; b < K; ++b) plane[b] = planes[b] >> (8 * kb);
      codes_to_half<K>(kb ? codes.y : codes.x, plane, x[kb]);
    }
    const half8v w0 = __builtin_bit_cast(half8v, make_uint4(x[0][0], x[0][1], x[0][2], x[0][3]));
    const half8v w1 = __builtin_bit_cast(half8v, make_uint4(x[1][0], x[1][1], x[1][2], x[1][3]));
    const half8v w1n = __builtin_bit_cast(half8v, make_uint4(x[1][0] ^ kSigns, x[1][1] ^ kSigns,
                                                             x[1][2] ^ kSigns, x[1][3] ^ kSigns));
    float4v d[4];
#pragma unroll
    for (int nb = 0; nb < 4; ++nb) {
      const float4v zero = {0.0f, 0.0f, 0.0f, 0.0f};
      d[nb] = __builtin_amdgcn_mfma_f32_16x16x32_f16(h[nb & 1], w0, zero, 0, 0, 0);
      d[nb] = __builtin_amdgcn_mfma_f32_16x16x32_f16(h[nb & 1], nb < 2 ? w1 : w1n, d[nb], 0, 0, 0);
    }
    uint32_t y[8];
    if (__all(fabsf(s) < __builtin_inff())) {
#pragma unroll
      for (int c = 0; c < 8; ++c)
        y[c] = pack_half(d[c / 2][2 * (c & 1)] * s, d[c / 2][2 * (c & 1) + 1] * s);
    } else {
#pragma unroll
      for (int c = 0; c < 8; ++c)
        y[c] = pack_half(scaled(d[c / 2][2 * (c & 1)], s), scaled(d[c / 2][2 * (c & 1) + 1], s));
    }
    // two exchanges over the row's four lanes: each of the two stores then writes half a
    // row of 64 contiguous bytes
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const auto t = __builtin_amdgcn_permlane16_swap(y[c], y[4 + c], false, false);
      y[c] = t[0];
      y[4 + c] = t[1];
    }
#pragma unroll
    for (int c = 0; c < 4; ++c) swap32(y[c], y[4 + c]);
    if (there) {
      uint16_t* p = out + (int64_t)i * kDim + 8 * blk;
      write_row_part(p, y[0], y[1], y[2], y[3]);
      write_row_part(p + 32, y[4], y[5], y[6], y[7]);
    }
  }
}

// ---- values ----------------------------------------------------------------------
// One wave per group of 8 tokens; lane l ends up with dimensions 8 (l % 8) ..+7 of token
// l / 8, so that a whole group is written as one contiguous KiB.

// fp16: lane l loads the 8 tokens of dimension 8 (l % 8) + l / 8; an 8 x 8 transpose of
// 16-bit numbers, one exchange per bit of the token, gives it 8 dimensions of token l / 8.
// (Gathers of 2 bytes at a stride of 16: 2 M rows 133 us, 1-byte ones of INT8 values 144.)
__device__ __forceinline__ uint4 value_row_f16(const uint16_t* v, int64_t g8, int lane) {
  const uint4 q = *reinterpret_cast<const uint4*>(v + g8 * 8 * kDim + (lane & 7) * 64 + (lane >> 3) * 8);
  uint32_t w[4] = {q.x, q.y, q.z, q.w};  // tokens 2c and 2c + 1
  swap32(w[0], w[2]);
  swap32(w[1], w[3]);
#pragma unroll
  for (int c = 0; c < 4; c += 2) {
    const auto r = __builtin_amdgcn_permlane16_swap(w[c], w[c + 1], false, false);
    w[c] = r[0];
    w[c + 1] = r[1];
  }
  const uint32_t sel = (lane >> 3) & 1 ? 0x03020706u : 0x05040100u;
#pragma unroll
  for (int c = 0; c < 4; ++c) w[c] = __builtin_amdgcn_perm(lane_xor_u32<8>(w[c]), w[c], sel);
  return make_uint4(w[0], w[1], w[2], w[3]);
}
// INT8: the same of bytes v^ + 128. (u - 128) 2^-g is exact in fp32, also as a multiply-add,
// and rounded once.
__device__ __forceinline__ uint4 value_row_i8(const uint8_t* v, int64_t g8, int exp, int lane) {
  const uint2 q = *reinterpret_cast<const uint2*>(v + g8 * 8 * kDim + (lane & 7) * 64 + (lane >> 3) * 8);
  uint32_t w[2] = {q.x, q.y};
  swap32(w[0], w[1]);
  const float unit = __builtin_amdgcn_ldexpf(1.0f, -exp), off = -128.0f * unit;
  uint32_t y[4];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint32_t d = transpose_tokens(w[h], lane);
#pragma unroll
    for (int c = 0; c < 2; ++c)
      y[2 * h + c] = pack_half(__builtin_fmaf((float)((d >> (16 * c)) & 0xFFu), unit, off),
                               __builtin_fmaf((float)((d >> (16 * c + 8)) & 0xFFu), unit, off));
  }
  return make_uint4(y[0], y[1], y[2], y[3]);
}
// 4 bits: a dword of the record per lane, the store's exchanges backwards.
__device__ __forceinline__ uint4 value_row_i4(const uint8_t* rec, int lane) {
  const int g = lane & 7, u = lane >> 3;
  uint32_t d = *reinterpret_cast<const uint32_t*>(rec + record_offset(lane));
  const float st = __half2float(*reinterpret_cast<const __half*>(rec + kI4Steps + 2 * u));
  const float z = __half2float(*reinterpret_cast<const __half*>(rec + kI4Minima + 2 * u));
  d = transpose_tokens(d, lane);
  const uint32_t got = lane_xor_u32<2>(d);
  const bool upper = (g & 2) != 0;  // dimensions of the bytes' high halves
  const uint32_t n[2] = {(upper ? got >> 4 : d) & 0x0F0F0F0Fu, (upper ? d >> 4 : got) & 0x0F0F0F0Fu};
  uint32_t w[4];
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    const uint32_t b = n[c / 2] >> (16 * (c & 1));
    w[c] = pack_half(__builtin_fmaf((float)(b & 0xFFu), st, z),
                     __builtin_fmaf((float)((b >> 8) & 0xFFu), st, z));
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

template <int FMT>
__global__ __launch_bounds__(kBlock) void load_values_kernel(const void* __restrict__ cache,
                                                             const int8_t* __restrict__ v_exp,
                                                             RowRange r,
                                                             uint16_t* __restrict__ out) {
  const int lane = lane_id();
  const uint32_t n = (uint32_t)(r.n_seq * r.n_groups), per_seq = (uint32_t)r.n_groups;
  for (uint32_t i = first_wave(); i < n; i += wave_stride()) {
    const uint32_t seq = i / per_seq;
    const int64_t s = seq, g8 = s * (r.t_cap / 8) + r.g_first + (i - seq * per_seq);
    const int64_t t = (r.g_first + (i - seq * per_seq)) * 8 + (lane >> 3) - r.t0;
    uint4 w;
    if constexpr (FMT == 0) w = value_row_f16(static_cast<const uint16_t*>(cache), g8, lane);
    else if constexpr (FMT == 1)
      w = value_row_i8(static_cast<const uint8_t*>(cache), g8, v_exp[g8 * 8 + (lane >> 3)], lane);
    else w = value_row_i4(static_cast<const uint8_t*>(cache) + g8 * kI4GroupBytes, lane);
    if (t >= 0 && t < r.n_tok)
      write_row_part(out + (s * r.n_tok + t) * kDim + 8 * (lane & 7), w.x, w.y, w.z, w.w);
  }
}

hipError_t launch_load_keys(int mant_bits, int hadamard, const uint8_t* codes_se,
                            const uint8_t* codes_m, const float* key_scale, int64_t n_seq,
                            int64_t n_tok, int64_t t_cap, int64_t t0, uint16_t* k,
                            hipStream_t stream) {
  const RowRange r = row_range(n_seq, n_tok, t_cap, t0);
  const KeysIn in{codes_se, codes_m, key_scale};
  const int64_t n = n_seq * n_tok;
  auto go = [&](auto k_tag) {
    constexpr int KK = decltype(k_tag)::value;
    if (hadamard)
      hipLaunchKernelGGL((load_keys_rotated_kernel<KK>), blocks_of((n + 15) / 16), dim3(kBlock), 0,
                         stream, in, r, k);
    else
      hipLaunchKernelGGL((load_keys_kernel<KK>), blocks_of((n + 7) / 8), dim3(kBlock), 0, stream, in,
                         r, k);
  };
  switch (mant_bits) {
    case 0: go(std::integral_constant<int, 0>{}); break;
    case 1: go(std::integral_constant<int, 1>{}); break;
    case 2: go(std::integral_constant<int, 2>{}); break;
    case 3: go(std::integral_constant<int, 3>{}); break;
    case 4: go(std::integral_constant<int, 4>{}); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

hipError_t launch_load_values(int fmt, const void* cache, const int8_t* v_exp, int64_t n_seq,
                              int64_t n_tok, int64_t t_cap, int64_t t0, uint16_t* v,
                              hipStream_t stream) {
  const RowRange r = row_range(n_seq, n_tok, t_cap, t0);
  const dim3 grid = blocks_of(n_seq * r.n_groups);
  if (fmt == 0)
    hipLaunchKernelGGL((load_values_kernel<0>), grid, dim3(kBlock), 0, stream, cache, v_exp, r, v);
  else if (fmt == 1)
    hipLaunchKernelGGL((load_values_kernel<1>), grid, dim3(kBlock), 0, stream, cache, v_exp, r, v);
  else
    hipLaunchKernelGGL((load_values_kernel<2>), grid, dim3(kBlock), 0, stream, cache, v_exp, r, v);
  return hipGetLastError();
}

}  // namespace potattn
