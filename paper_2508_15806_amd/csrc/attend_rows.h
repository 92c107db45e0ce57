// Rows of a cache as MFMA operands in a wave's registers, and what the kernels of attention over a cache share.
#ifndef SLKV_ATTEND_ROWS_H
#define SLKV_ATTEND_ROWS_H

#include "cache.h"
#include "device_utils.h"

namespace slkv {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// x / y for 0 <= x < 2^21, y > 0: (x + 1/2) / y is at least 1 / (2 y) from a whole number, and what reciprocal and product are off by, 2^-22 of it, is less.
__device__ __forceinline__ int divide(int x, int y) { return (int)(((float)x + 0.5f) * __builtin_amdgcn_rcpf((float)y)); }

template <int KIND, int D>
struct Attend {
  typedef typename Kind<KIND>::wide wide;
  static constexpr bool kF32 = KIND == SLKV_F32;
  static constexpr int kTiles = kF32 ? 1 : 2;          // K tiles of 16 rows a step
  static constexpr int kStep = 16 * kTiles;
  static constexpr int kEach = 4 * kTiles;             // rows of a step that a lane group holds
  static constexpr int kVD = D / 16;                   // dims of a row of V that a lane holds
  static constexpr int kRowBytes = D * Kind<KIND>::kBits / 8;
  static constexpr int kScales = D / kScaleBlock;
  static constexpr int kKWords = kRowBytes / 16;       // words of a row of K that a lane holds (a quarter of the row)
  static constexpr int kVWords = kF32 ? kVD : (kVD * Kind<KIND>::kBits + 31) / 32;   // words of a row of V that a lane holds
  // Reference of fp16 weights: they reach 2^15, so that those down to 2^-26 of the largest keep all their bits.
  static constexpr float kBelow = KIND == SLKV_F16 ? 12.f : 0.f, kBelowPower = KIND == SLKV_F16 ? 0x1p-12f : 1.f;
  static constexpr float kAbove = KIND == SLKV_F16 ? 15.f : 8.f;   // a product this far above the reference moves it

  struct KRegs { uint32_t w[kTiles][kKWords]; uint32_t s[kTiles]; };
  struct VRegs { uint32_t w[kEach][kVWords]; uint32_t s[kEach]; };

  // The rows of a part as buffers: what is beyond their end reads as 0, whatever is there.  The lane's place moves by whole steps; tiles and rows of a step are
  // constant offsets of the loads.
  struct Rows { __amdgpu_buffer_rsrc_t k, v, ks, vs; };
  struct Place { uint32_t k, v, ks, vs; };

  static __device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer(const unsigned char* p, int64_t first, int rows, int row_bytes) {
    return __builtin_amdgcn_make_buffer_rsrc((void*)(p + first * row_bytes), 0, rows * row_bytes, 0x00027000);
  }
  template <class ARGS>
  static __device__ __forceinline__ Rows rows_of(const ARGS& a, int64_t first, int rows) {
    Rows r;
    r.k = buffer(a.k, first, rows, kRowBytes);
    r.v = buffer(a.v, first, rows, kRowBytes);
    if constexpr (KIND == SLKV_BF16_KV_MXFP4) {
      r.ks = buffer(a.k_scale, first, rows, kScales);
      r.vs = buffer(a.v_scale, first, rows, kScales);
    }
    return r;
  }
  static __device__ __forceinline__ Place place_of(int step, int lane) {
    const int c = lane & 15, g = lane >> 4;
    const uint32_t krow = step * kStep + c / 4 * kEach + c % 4, vrow = step * kStep + g * kEach;
    Place p;
    p.k = krow * kRowBytes + g * (KIND == SLKV_BF16_KV_MXFP4 ? kRowBytes / 4 : 16);
    p.v = vrow * kRowBytes + c * (kRowBytes / 16);
    p.ks = krow * kScales + g * kScales / 4;
    p.vs = vrow * kScales + c * kVD / kScaleBlock;
    return p;
  }
  static __device__ __forceinline__ void advance(Place& p, int steps) {
    p.k += steps * kStep * kRowBytes;
    p.v += steps * kStep * kRowBytes;
    if constexpr (KIND == SLKV_BF16_KV_MXFP4) {
      p.ks += steps * kStep * kScales;
      p.vs += steps * kStep * kScales;
    }
  }

  // dims that lane group g multiplies in product p (of 8 dims; fp32: one dim each)
  static __device__ __forceinline__ int dim_of(int p, int g) {
    if constexpr (kF32) return p / 4 * 16 + g * 4 + p % 4;
    else if constexpr (KIND == SLKV_BF16_KV_FP8) return p / 2 * 64 + g * 16 + p % 2 * 8;
    else if constexpr (KIND == SLKV_BF16_KV_MXFP4) return g * (D / 4) + p * 8;
    else return p * 32 + g * 8;
  }

  static __device__ __forceinline__ void load_k(KRegs& r, const Rows& rows, const Place& p) {
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      if constexpr (KIND == SLKV_BF16_KV_MXFP4) {
        if constexpr (kKWords == 4) *(u32x4*)r.w[t] = __builtin_amdgcn_raw_buffer_load_b128(rows.k, p.k + t * 4 * kRowBytes, 0, 0);
        else *(u32x2*)r.w[t] = __builtin_amdgcn_raw_buffer_load_b64(rows.k, p.k + t * 4 * kRowBytes, 0, 0);
        r.s[t] = __builtin_amdgcn_raw_buffer_load_b8(rows.ks, p.ks + t * 4 * kScales, 0, 0);
      } else {
#pragma unroll
        for (int i = 0; i < kKWords / 4; ++i)
          *(u32x4*)(r.w[t] + i * 4) = __builtin_amdgcn_raw_buffer_load_b128(rows.k, p.k + t * 4 * kRowBytes + i * 64, 0, 0);
      }
    }
  }

  static __device__ __forceinline__ void load_v(VRegs& r, const Rows& rows, const Place& p) {
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
      const uint32_t at = p.v + j * kRowBytes;
      if constexpr (kRowBytes / 16 == 2) {
        r.w[j][0] = __builtin_amdgcn_raw_buffer_load_b16(rows.v, at, 0, 0);
      } else if constexpr (kVWords == 1) {
        r.w[j][0] = __builtin_amdgcn_raw_buffer_load_b32(rows.v, at, 0, 0);
      } else if constexpr (kVWords == 2) {
        *(u32x2*)r.w[j] = __builtin_amdgcn_raw_buffer_load_b64(rows.v, at, 0, 0);
      } else {
#pragma unroll
        for (int i = 0; i < kVWords / 4; ++i) *(u32x4*)(r.w[j] + i * 4) = __builtin_amdgcn_raw_buffer_load_b128(rows.v, at + i * 16, 0, 0);
      }
      if constexpr (KIND == SLKV_BF16_KV_MXFP4) r.s[j] = __builtin_amdgcn_raw_buffer_load_b8(rows.vs, p.vs + j * kScales, 0, 0);
    }
  }

  // One element of V, for the values that are not finite.
  template <class ARGS>
  static __device__ float value(const ARGS& a, int64_t row, int dim) {
    const unsigned char* p = a.v + row * kRowBytes;
    if constexpr (kF32) return ((const float*)p)[dim];
    else if constexpr (KIND == SLKV_BF16) return __uint_as_float((uint32_t)((const uint16_t*)p)[dim] << 16);
    else if constexpr (KIND == SLKV_F16) return (float)((const _Float16*)p)[dim];
    else if constexpr (KIND == SLKV_BF16_KV_FP8) return __uint_as_float(fp8_pair<false>(p[dim]) << 16);
    else return __uint_as_float(fp4_pair<0>(dim % 2 ? p[dim / 2] >> 4 : p[dim / 2], scale_of(a.v_scale[row * kScales + dim / kScaleBlock])) << 16);
  }

  static __device__ __forceinline__ f32x4 mfma(u32x4 x, u32x4 y, f32x4 c) {
    if constexpr (KIND == SLKV_F16)
      return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, x), __builtin_bit_cast(f16x8, y), c, 0, 0, 0);
    else
      return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, y), c, 0, 0, 0);
  }

  // Operand p of a tile of K: 8 wide elements.
  static __device__ __forceinline__ u32x4 k_operand(const KRegs& r, int t, int p) {
    if constexpr (KIND == SLKV_BF16_KV_MXFP4) {
      const float s = scale_of(r.s[t]);
      const uint32_t c = r.w[t][p];
      return u32x4{fp4_pair<0>(c, s), fp4_pair<1>(c, s), fp4_pair<2>(c, s), fp4_pair<3>(c, s)};
    } else if constexpr (KIND == SLKV_BF16_KV_FP8) {
      const uint32_t c0 = r.w[t][p * 2], c1 = r.w[t][p * 2 + 1];
      return u32x4{fp8_pair<false>(c0), fp8_pair<true>(c0), fp8_pair<false>(c1), fp8_pair<true>(c1)};
    } else {
      return u32x4{r.w[t][p * 4], r.w[t][p * 4 + 1], r.w[t][p * 4 + 2], r.w[t][p * 4 + 3]};
    }
  }

  // Pair U of row j of the lane's block of V: wide elements of dims c kVD + 2 U and the next.
  template <int U>
  static __device__ __forceinline__ uint32_t v_pair(const VRegs& r, int j) {
    if constexpr (KIND == SLKV_BF16_KV_MXFP4) return fp4_pair<U>(r.w[j][0], scale_of(r.s[j]));
    else if constexpr (KIND == SLKV_BF16_KV_FP8) return fp8_pair<U % 2 == 1>(r.w[j][U / 2]);
    else return r.w[j][U];
  }

  // Pairs of wide elements with 0 in the place of infinities and NaN.
  static __device__ __forceinline__ u32x4 finite(u32x4 x) {
    constexpr uint32_t kExp = KIND == SLKV_F16 ? 0x7c00u : 0x7f80u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t w = x[i];
      x[i] = ((w & kExp) == kExp ? 0u : w & 0xffffu) | ((w >> 16 & kExp) == kExp ? 0u : w & 0xffff0000u);
    }
    return x;
  }

  // Two weights as a pair of 16-bit numbers and the pair of what these leave of them.
  static __device__ __forceinline__ void split(float x, float y, uint32_t& hi, uint32_t& lo) {
    if constexpr (KIND == SLKV_F16) {
      const f16x2 h = __builtin_convertvector((f32x2{x, y}), f16x2);
      hi = __builtin_bit_cast(uint32_t, h);
      lo = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{x - (float)h[0], y - (float)h[1]}), f16x2));
    } else {
      const uint32_t xb = __float_as_uint(x), yb = __float_as_uint(y);
      hi = __builtin_amdgcn_perm(yb, xb, 0x07060302u);
      lo = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{x - __uint_as_float(xb & 0xffff0000u), y - __uint_as_float(yb & 0xffff0000u)}), bf16x2));
    }
  }
};

template <int KIND>
__device__ __forceinline__ void store_out(unsigned char* dst, f32x4 o) {   // four neighbouring outputs
  if constexpr (KIND == SLKV_F32) {
    *(f32x4*)dst = o;
  } else if constexpr (KIND == SLKV_F16) {
    typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
    *(f16x4*)dst = __builtin_convertvector(o, f16x4);
  } else {
    typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
    *(bf16x4*)dst = __builtin_convertvector(o, bf16x4);
  }
}

// Over `share` neighbouring lanes, 4 to 64, in every lane.
template <class OP>
__device__ __forceinline__ float reduce_lanes(float v, int share, OP op) {
  auto move = [&](auto ctrl) __attribute__((always_inline)) { return __uint_as_float(dpp_move<decltype(ctrl)::value>(0u, __float_as_uint(v))); };
  using std::integral_constant;
  v = op(v, move(integral_constant<int, 0xb1>{}));     // quad_perm 1, 0, 3, 2
  v = op(v, move(integral_constant<int, 0x4e>{}));     // quad_perm 2, 3, 0, 1
  if (share >= 8) v = op(v, move(integral_constant<int, 0x141>{}));    // row_half_mirror
  if (share >= 16) v = op(v, move(integral_constant<int, 0x140>{}));   // row_mirror
  if (share >= 32) v = op(v, __shfl_xor(v, 16));
  if (share >= 64) v = op(v, __shfl_xor(v, 32));
  return v;
}

}  // namespace slkv
#endif
