// What the calls on a cache share: the segments of a launch as a kernel argument, element types and their conversions.
#ifndef SLKV_CACHE_H
#define SLKV_CACHE_H

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "slkv_internal.h"

namespace slkv {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

constexpr int kScaleBlock = 32;      // MXFP4 elements that share an exponent

// Segments seg0 .. seg0 + nseg - 1 of a call.  w[r][i]: of segment seg0 + i, for each r what the launch's kernel says.  The arguments are at most 4 KiB, so a
// call with more segments than a table holds makes several launches; the small table spares the ordinary call the larger one's 3.5 KB of arguments.
template <int N, int WORDS>
struct SegWords {
  static constexpr int kSegs = N;
  int32_t nseg, seg0;
  int32_t w[WORDS][N + 1];
};
constexpr int kFewSegs = 64, kManySegs3 = 290;

__device__ __forceinline__ int rows_in_use(const int32_t* lengths, int seg, int room) {
  return lengths ? min(max(lengths[seg], 0), room) : room;
}

// Elements of K and V.
template <int KIND>
struct Kind;
template <>
struct Kind<SLKV_F32> { typedef float wide; static constexpr int kBits = 32; };
template <>
struct Kind<SLKV_BF16> { typedef __bf16 wide; static constexpr int kBits = 16; };
template <>
struct Kind<SLKV_F16> { typedef _Float16 wide; static constexpr int kBits = 16; };
template <>
struct Kind<SLKV_BF16_KV_FP8> { typedef __bf16 wide; static constexpr int kBits = 8; };
template <>
struct Kind<SLKV_BF16_KV_MXFP4> { typedef __bf16 wide; static constexpr int kBits = 4; };

inline int kind_bits(int dtype) { return dtype == SLKV_F32 ? 32 : dtype == SLKV_BF16_KV_FP8 ? 8 : dtype == SLKV_BF16_KV_MXFP4 ? 4 : 16; }
inline int wide_bytes(int dtype) { return dtype == SLKV_F32 ? 4 : 2; }

// 2^(e - 127) as the operand of the converters, which read its exponent field: 0 stands for 2^-127, 255 for NaN.
__device__ __forceinline__ float scale_of(uint32_t e) { return __uint_as_float(e << 23); }

// Two neighbouring values as a pair of bfloat16.
template <int BYTE>
__device__ __forceinline__ uint32_t fp4_pair(uint32_t codes, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, BYTE));
}
template <bool HIGH>
__device__ __forceinline__ uint32_t fp8_pair(uint32_t codes) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, 1.f, HIGH));
}

// f on the dtype as a compile-time constant.
template <class F>
auto with_kind(int dtype, F f) {
  using std::integral_constant;
  switch (dtype) {
    case SLKV_F32: return f(integral_constant<int, SLKV_F32>{});
    case SLKV_BF16: return f(integral_constant<int, SLKV_BF16>{});
    case SLKV_F16: return f(integral_constant<int, SLKV_F16>{});
    case SLKV_BF16_KV_FP8: return f(integral_constant<int, SLKV_BF16_KV_FP8>{});
  }
  return f(integral_constant<int, SLKV_BF16_KV_MXFP4>{});
}

inline slkv_status launch_status(const char* what) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? SLKV_OK : fail(SLKV_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

}  // namespace slkv
#endif
