// Attention of the latest tokens over a cache (slkv_attend_cache).
//
// A KV head's R = (Hq/Hkv)*T queries share its rows, so a row is read once for all of them.  A workgroup takes a part of a segment's rows, its waves
// take steps of 32 rows (fp32: 16) in turn, and every wave keeps, per query, a reference exponent, the sum of exp2(x - reference) and the
// weighted sum of the values; waves and parts are put together at the end.
//
// With MFMA operands of 16 keys by 32 dims the products x = K q come out as D[key][query]: lane l holds query l % 16 and the keys 4 g + i, g = l / 16, of each
// of the step's two tiles.  The product with the values wants P as [key][query] with 8 keys of a lane group g: the very registers, if the
// tiles' rows are dealt to keys so that group g holds the keys 8 g .. 8 g + 7 of the step.  Of V a lane needs, for each of these 8 keys, one value
// per product; it loads D/16 neighbouring ones of every key (16 lanes cover a row) and turns the 8 x D/16 block around in its registers, so that product m
// covers the dims c * D/16 + m.  Nothing goes through LDS until the end, and dims may be dealt to K's operands in any order that q follows.
#include "cache.h"
#include "device_utils.h"
#include "launch.h"

namespace slkv {

constexpr int kAttendWaves = 4, kAttendThreads = kAttendWaves * kWave;
constexpr int kTileRows = 32;        // rows of a tile of stored logits, and what parts of a segment are a multiple of
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

template <int N>
using AttendTab = SegWords<N, 2>;    // w[0] room of the segment (first row), w[1] parts before it (of the call)

struct AttendArgs {
  const unsigned char *k, *v, *k_scale, *v_scale, *q;
  unsigned char* out;
  const int32_t* lengths;
  float* lse;
  const float* w_in;
  float* w_out;
  float* part_o;                     // [part][R][D] sums of a part, relative to its reference
  float* part_ml;                    // [part][2][R] reference (log2), sum
  float* logits;                     // x in log2 units: tiles of [R][32 rows]
  int32_t T, R;
  int32_t row0;                      // first row of the call's rooms; logits of segment s, row j: tile (start - row0) / 32 + s + j / 32
  float c_log2;                      // log2(e) / sqrt(d)
};

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// Rows of a part: ceil(n / parts) rounded up to tiles, so that the work is spread over the same workgroups whatever the length is.
__device__ __forceinline__ int part_rows(int n, int parts) { return ((n + parts - 1) / parts + kTileRows - 1) / kTileRows * kTileRows; }

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
  static constexpr float kBelow = KIND == SLKV_F16 ? 12.f : 0.f;
  static constexpr float kAbove = KIND == SLKV_F16 ? 15.f : 8.f;   // a product this far above the reference moves it

  struct KRegs { uint32_t w[kTiles][kKWords]; uint32_t s[kTiles]; };
  struct VRegs { uint32_t w[kEach][kVWords]; uint32_t s[kEach]; };

  // dims that lane group g multiplies in product p (of 8 dims; fp32: one dim each)
  static __device__ __forceinline__ int dim_of(int p, int g) {
    if constexpr (kF32) return p / 4 * 16 + g * 4 + p % 4;
    else if constexpr (KIND == SLKV_BF16_KV_FP8) return p / 2 * 64 + g * 16 + p % 2 * 8;
    else if constexpr (KIND == SLKV_BF16_KV_MXFP4) return g * (D / 4) + p * 8;
    else return p * 32 + g * 8;
  }

  static __device__ __forceinline__ void load_k(KRegs& r, const AttendArgs& a, int64_t base, int key0, int last, int lane) {
    const int rho = lane & 15, g = lane >> 4;
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      const int64_t row = base + min(key0 + rho / 4 * kEach + t * 4 + rho % 4, last);
      const unsigned char* p = a.k + row * kRowBytes;
      if constexpr (KIND == SLKV_BF16_KV_MXFP4) {
        if constexpr (kKWords == 4) *(u32x4*)r.w[t] = *(const u32x4*)(p + g * 16);
        else *(u32x2*)r.w[t] = *(const u32x2*)(p + g * 8);
        r.s[t] = a.k_scale[row * kScales + g * kScales / 4];
      } else {
#pragma unroll
        for (int i = 0; i < kKWords / 4; ++i) *(u32x4*)(r.w[t] + i * 4) = *(const u32x4*)(p + i * 64 + g * 16);
      }
    }
  }

  static __device__ __forceinline__ void load_v(VRegs& r, const AttendArgs& a, int64_t base, int key0, int last, int lane) {
    const int c = lane & 15, g = lane >> 4;
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
      const int64_t row = base + min(key0 + g * kEach + j, last);
      const unsigned char* p = a.v + row * kRowBytes + c * (kRowBytes / 16);
      if constexpr (kRowBytes / 16 == 2) {
        r.w[j][0] = *(const uint16_t*)p;
      } else if constexpr (kVWords == 1) {
        r.w[j][0] = *(const uint32_t*)p;
      } else if constexpr (kVWords == 2) {
        *(u32x2*)r.w[j] = *(const u32x2*)p;
      } else {
#pragma unroll
        for (int i = 0; i < kVWords / 4; ++i) *(u32x4*)(r.w[j] + i * 4) = *(const u32x4*)(p + i * 16);
      }
      if constexpr (KIND == SLKV_BF16_KV_MXFP4) r.s[j] = a.v_scale[row * kScales + c * kVD / kScaleBlock];
    }
  }

  // One element of V, for the values that are not finite.
  static __device__ float value(const AttendArgs& a, int64_t row, int dim) {
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

  // Row j of the lane's block of V as kVD / 2 pairs of wide elements.
  static __device__ __forceinline__ void v_pairs(const VRegs& r, int j, uint32_t (&o)[kVD / 2]) {
    if constexpr (KIND == SLKV_BF16_KV_MXFP4) {
      const float s = scale_of(r.s[j]);
      o[0] = fp4_pair<0>(r.w[j][0], s);
      o[1] = fp4_pair<1>(r.w[j][0], s);
      if constexpr (kVD == 8) {
        o[2] = fp4_pair<2>(r.w[j][0], s);
        o[3] = fp4_pair<3>(r.w[j][0], s);
      }
    } else if constexpr (KIND == SLKV_BF16_KV_FP8) {
#pragma unroll
      for (int i = 0; i < kVD / 4; ++i) {
        o[i * 2] = fp8_pair<false>(r.w[j][i]);
        o[i * 2 + 1] = fp8_pair<true>(r.w[j][i]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < kVD / 2; ++i) o[i] = r.w[j][i];
    }
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

// RT: tiles of 16 queries.
template <int KIND, int D, int RT, class TAB>
__global__ __launch_bounds__(kAttendThreads, RT == 4 ? 1 : 2) void attend_kernel(const AttendArgs a, const TAB tab) {
  using A = Attend<KIND, D>;
  constexpr int kProducts = A::kF32 ? D / 4 : D / 32, kVD = A::kVD, kEach = A::kEach;
  __shared__ float sh_o[kAttendWaves][16][D + 4];
  __shared__ float sh_m[kAttendWaves][16 * RT], sh_l[kAttendWaves][16 * RT], sh_lse[16 * RT];
  const int part_id = (int)blockIdx.x + tab.w[1][0];
  const int i = find_segment_wave(tab.nseg, part_id, [&](int s) { return tab.w[1][s]; });
  const int seg = tab.seg0 + i, parts = tab.w[1][i + 1] - tab.w[1][i], part = part_id - tab.w[1][i];
  const int start = tab.w[0][i];
  const int n = rows_in_use(a.lengths, seg, tab.w[0][i + 1] - start);
  const int each = part_rows(n, parts);
  const int begin = part * each, end = min(n, begin + each);
  if (begin >= end && part > 0) return;
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave)), lane = threadIdx.x % kWave;
  const int rq = lane & 15, g = lane >> 4, R = a.R, T = a.T;
  const int64_t base = start;

  u32x4 q[RT][A::kF32 ? 1 : kProducts];
  float qf[RT][A::kF32 ? kProducts : 1];
  int sees[RT];                                        // rows that the lane's query sees
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int r = rt * 16 + rq;
    sees[rt] = r < R ? min(end, n - T + 1 + r % T) : 0;
    const unsigned char* p = a.q + ((int64_t)seg * R + min(r, R - 1)) * (D * (int)sizeof(typename A::wide));
    if constexpr (A::kF32) {
#pragma unroll
      for (int u = 0; u < kProducts / 4; ++u) *(f32x4*)&qf[rt][u * 4] = *(const f32x4*)(p + A::dim_of(u * 4, g) * 4);
    } else {
#pragma unroll
      for (int u = 0; u < kProducts; ++u) q[rt][u] = *(const u32x4*)(p + A::dim_of(u, g) * 2);
    }
  }
  const int64_t tile_seg = (int64_t)(start - a.row0) / kTileRows + seg;

  float ref[RT], sum[RT];
  f32x4 acc[RT][kVD];
  // The weights go into the products with the values as two 16-bit numbers each, which leaves 2^-16 of a weight (one number: 2^-9 of each, as much again as
  // the rounding of the output).  An infinite value would make NaN of the second one's zero, and values of rows that a query does not see would reach it through
  // a weight of zero: sums that come out not finite are taken again, with such values kept out of the second number's products and, where not every query
  // sees the row, out of both.
  bool careful = false;
  for (;;) {
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      ref[rt] = -INFINITY;
      sum[rt] = 0.f;
#pragma unroll
      for (int m = 0; m < kVD; ++m) acc[rt][m] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    for (int key0 = begin + wave * A::kStep; key0 < end; key0 += kAttendWaves * A::kStep) {
      typename A::KRegs kr;
      typename A::VRegs vr;
      A::load_k(kr, a, base, key0, end - 1, lane);
      A::load_v(vr, a, base, key0, end - 1, lane);
      f32x4 x[RT][A::kTiles];
#pragma unroll
      for (int t = 0; t < A::kTiles; ++t) {
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) x[rt][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int u = 0; u < kProducts; ++u) {
          if constexpr (A::kF32) {
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) x[rt][t] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kr.w[t][u]), qf[rt][u], x[rt][t], 0, 0, 0);
          } else {
            const u32x4 ko = A::k_operand(kr, t, u);
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) x[rt][t] = A::mfma(ko, q[rt][u], x[rt][t]);
          }
        }
      }
      const int mine = key0 + g * kEach;               // the lane's rows: mine .. mine + kEach - 1
      const bool tail = key0 + A::kStep > min(end, n - T + 1);
      float p[RT][kEach];
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        float top = -INFINITY;
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
          p[rt][j] = x[rt][j / 4][j % 4] * a.c_log2;
          if (tail && mine + j >= sees[rt]) p[rt][j] = -INFINITY;
          top = fmaxf(top, p[rt][j]);
        }
        if (a.logits && rt * 16 + rq < R) {
          float* l = a.logits + ((tile_seg + key0 / kTileRows) * R + rt * 16 + rq) * kTileRows + mine % kTileRows;
#pragma unroll
          for (int j = 0; j < kEach; j += 4) *(f32x4*)(l + j) = f32x4{p[rt][j], p[rt][j + 1], p[rt][j + 2], p[rt][j + 3]};
        }
        if (__ballot(top > ref[rt] + A::kAbove)) {
          top = fmaxf(top, __shfl_xor(top, 16));
          top = fmaxf(top, __shfl_xor(top, 32));
          const float now = fmaxf(ref[rt], top - A::kBelow);
          const float f = ref[rt] == -INFINITY ? 0.f : exp2_fast(ref[rt] - now);
          // (sums of a NaN stay one)
          sum[rt] *= f;
#pragma unroll
          for (int m = 0; m < kVD; ++m) acc[rt][m] *= f;
          ref[rt] = now;
        }
        const float at = ref[rt] == -INFINITY ? 0.f : ref[rt];
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
          p[rt][j] = exp2_fast(p[rt][j] - at);
          sum[rt] += p[rt][j];
        }
      }
      // rows beyond the end were loaded from the last one
      if (key0 + A::kStep > end) {
#pragma unroll
        for (int j = 0; j < kEach; ++j)
          if (mine + j >= end) {
#pragma unroll
            for (int u = 0; u < A::kVWords; ++u) vr.w[j][u] = 0;
            if constexpr (KIND == SLKV_BF16_KV_MXFP4) vr.s[j] = 127;
          }
      }
      if (careful && tail) {
        // rows that not every query sees: one at a time, to the queries that see it
        const int from = max(key0, n - T + 1), to = min(key0 + A::kStep, end);
        for (int key = from; key < to; ++key) {
          const int holder = (key - key0) / kEach, which = (key - key0) % kEach;
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) {
            float w = 0.f;
#pragma unroll
            for (int j = 0; j < kEach; ++j)
              if (j == which) w = p[rt][j];
            w = __shfl(w, holder * 16 + rq);
            if (key < sees[rt]) {
#pragma unroll
              for (int m = 0; m < kVD; ++m)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[rt][m][e] += w * A::value(a, base + key, (g * 4 + e) * kVD + m);
            }
          }
        }
#pragma unroll
        for (int j = 0; j < kEach; ++j)
          if (mine + j >= from) {
#pragma unroll
            for (int u = 0; u < A::kVWords; ++u) vr.w[j][u] = 0;
            if constexpr (KIND == SLKV_BF16_KV_MXFP4) vr.s[j] = 127;
          }
      }
      if constexpr (A::kF32) {
#pragma unroll
        for (int m = 0; m < kVD; ++m)
#pragma unroll
          for (int j = 0; j < kEach; ++j)
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
              acc[rt][m] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(vr.w[j][m]), p[rt][j], acc[rt][m], 0, 0, 0);
      } else {
        uint32_t pair[kEach][kVD / 2];
#pragma unroll
        for (int j = 0; j < kEach; ++j) A::v_pairs(vr, j, pair[j]);
        u32x4 hi[RT], lo[RT];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            uint32_t h, l;
            A::split(p[rt][2 * j], p[rt][2 * j + 1], h, l);
            hi[rt][j] = h;
            lo[rt][j] = l;
          }
#pragma unroll
        for (int m = 0; m < kVD; ++m) {
          u32x4 vo;
#pragma unroll
          for (int j = 0; j < 4; ++j)
            vo[j] = __builtin_amdgcn_perm(pair[2 * j + 1][m / 2], pair[2 * j][m / 2], m % 2 ? 0x07060302u : 0x05040100u);
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) acc[rt][m] = A::mfma(vo, hi[rt], acc[rt][m]);
          if (careful) vo = A::finite(vo);
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) acc[rt][m] = A::mfma(vo, lo[rt], acc[rt][m]);
        }
      }
    }
    if (careful) break;
    bool finite = true;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
      for (int m = 0; m < kVD; ++m)
#pragma unroll
        for (int e = 0; e < 4; ++e) finite = finite && fabsf(acc[rt][m][e]) < INFINITY;
    if (!__ballot(!finite)) break;
    careful = true;
  }

  // the waves' references and sums
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    float l = sum[rt];
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (g == 0) {
      sh_m[wave][rt * 16 + rq] = ref[rt];
      sh_l[wave][rt * 16 + rq] = l;
    }
  }
  __syncthreads();
  const int rows_each = max(each, 1), active = (n + rows_each - 1) / rows_each;
  const bool whole = active <= 1;
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    float top = -INFINITY, total = 0.f;
#pragma unroll
    for (int w = 0; w < kAttendWaves; ++w) top = fmaxf(top, sh_m[w][rt * 16 + rq]);
    float mine = 0.f;
#pragma unroll
    for (int w = 0; w < kAttendWaves; ++w) {
      const float m = sh_m[w][rt * 16 + rq], l = sh_l[w][rt * 16 + rq];
      // (a wave that saw nothing has a sum of 0, or NaN where a product was NaN)
      const float f = m == -INFINITY ? 1.f : exp2_fast(m - top);
      total += l * f;
      if (w == wave) mine = f;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
#pragma unroll
      for (int m = 0; m < kVD; ++m) sh_o[wave][rq][(g * 4 + e) * kVD + m] = acc[rt][m][e] * mine;
    }
    const int r = rt * 16 + rq;
    if (wave == 0 && g == 0 && r < R) {
      if (whole) {
        const float lse2 = total > 0.f ? top + __builtin_amdgcn_logf(total) : (n - T + 1 + r % T > 0 ? NAN : INFINITY);
        sh_lse[r] = lse2;
        if (a.lse) a.lse[(int64_t)seg * R + r] = lse2 == INFINITY && !(total > 0.f) ? -INFINITY : lse2 * kLn2;
      } else {
        float* ml = a.part_ml + (int64_t)part_id * 2 * R;
        ml[r] = top;
        ml[R + r] = total;
      }
      sh_l[0][r] = total;
    }
    __syncthreads();
    for (int idx = threadIdx.x; idx < 16 * D / 4; idx += kAttendThreads) {
      const int r16 = idx / (D / 4), d0 = idx % (D / 4) * 4, row = rt * 16 + r16;
      if (row >= R) continue;
      f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < kAttendWaves; ++w) o += *(const f32x4*)&sh_o[w][r16][d0];
      if (!whole) {
        *(f32x4*)(a.part_o + ((int64_t)part_id * R + row) * D + d0) = o;
        continue;
      }
      const float l = sh_l[0][row];
      const bool none = n - T + 1 + row % T <= 0;
      const float inv = 1.f / l;
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = none ? 0.f : l > 0.f ? o[e] * inv : NAN;
      unsigned char* dst = a.out + ((int64_t)seg * R + row) * (D * (int)sizeof(typename A::wide));
      if constexpr (A::kF32) {
        *(f32x4*)(dst + d0 * 4) = o;
      } else if constexpr (KIND == SLKV_F16) {
        typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
        *(f16x4*)(dst + d0 * 2) = __builtin_convertvector(o, f16x4);
      } else {
        typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
        *(bf16x4*)(dst + d0 * 2) = __builtin_convertvector(o, bf16x4);
      }
    }
    __syncthreads();
  }
  if (!whole || !a.w_out) return;
  __threadfence_block();
  __syncthreads();
  for (int j = threadIdx.x; j < n; j += kAttendThreads) {
    float w = a.w_in ? a.w_in[base + j] : 0.f;
    const float* l = a.logits + (tile_seg + j / kTileRows) * R * kTileRows + j % kTileRows;
    float s = 0.f;
    for (int r = 0; r < R; ++r) s += exp2_fast(l[r * kTileRows] - sh_lse[r]);
    a.w_out[base + j] = w + s;
  }
}

// Segments of more than one part: the parts put together, in their order, and the weights.  Part p of a segment finishes the queries p, p + active, .. and
// the weights of its own rows; every workgroup adds up the references and sums of all parts, R pairs each.
template <int KIND, int D, class TAB>
__global__ __launch_bounds__(kAttendThreads) void attend_join_kernel(const AttendArgs a, const TAB tab) {
  using A = Attend<KIND, D>;
  __shared__ float sh_m[64], sh_l[64], sh_lse[64];
  __shared__ float sh_o[kAttendThreads / (D / 4)][D];
  const int part_id = (int)blockIdx.x + tab.w[1][0];
  const int i = find_segment_wave(tab.nseg, part_id, [&](int s) { return tab.w[1][s]; });
  const int seg = tab.seg0 + i, first = tab.w[1][i], parts = tab.w[1][i + 1] - first, part = part_id - first;
  const int start = tab.w[0][i];
  const int n = rows_in_use(a.lengths, seg, tab.w[0][i + 1] - start);
  const int each = part_rows(n, parts);
  const int active = each ? (n + each - 1) / each : 0;
  if (active <= 1 || part >= active) return;
  const int R = a.R, T = a.T, wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
  const float* ml = a.part_ml + (int64_t)first * 2 * R;
  for (int r = wave; r < R; r += kAttendWaves) {
    float top = -INFINITY, l = 0.f;
    for (int p = lane; p < active; p += kWave) top = fmaxf(top, ml[p * 2 * R + r]);
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
    for (int p = lane; p < active; p += kWave) {
      const float m = ml[p * 2 * R + r];
      l += ml[p * 2 * R + R + r] * (m == -INFINITY ? 1.f : exp2_fast(m - top));
    }
    l = wave_sum(l);
    if (lane == 0) {
      const bool none = n - T + 1 + r % T <= 0;
      const float lse2 = l > 0.f ? top + __builtin_amdgcn_logf(l) : none ? INFINITY : NAN;
      sh_m[r] = top;
      sh_l[r] = l;
      sh_lse[r] = lse2;
      if (part == 0 && a.lse) a.lse[(int64_t)seg * R + r] = none ? -INFINITY : lse2 * kLn2;
    }
  }
  __syncthreads();
  constexpr int kLanes = D / 4, kGroups = kAttendThreads / kLanes;
  const int d0 = threadIdx.x % kLanes * 4, grp = threadIdx.x / kLanes;
  for (int r = part; r < R; r += active) {
    f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int p = grp; p < active; p += kGroups) {
      const float m = ml[p * 2 * R + r];
      const float f = m == -INFINITY ? 1.f : exp2_fast(m - sh_m[r]);
      o += *(const f32x4*)(a.part_o + ((int64_t)(first + p) * R + r) * D + d0) * f;
    }
    *(f32x4*)&sh_o[grp][d0] = o;
    __syncthreads();
    if ((int)threadIdx.x < D) {
      float s = 0.f;
#pragma unroll
      for (int w = 0; w < kGroups; ++w) s += sh_o[w][threadIdx.x];
      const float l = sh_l[r];
      s = n - T + 1 + r % T <= 0 ? 0.f : l > 0.f ? s / l : NAN;
      ((typename A::wide*)a.out)[((int64_t)seg * R + r) * D + threadIdx.x] = (typename A::wide)s;
    }
    __syncthreads();
  }
  if (!a.w_out) return;
  const int64_t tile_seg = (int64_t)(start - a.row0) / kTileRows + seg;
  const int end = min(n, (part + 1) * each);
  for (int j = part * each + (int)threadIdx.x; j < end; j += kAttendThreads) {
    const float w = a.w_in ? a.w_in[(int64_t)start + j] : 0.f;
    const float* l = a.logits + (tile_seg + j / kTileRows) * R * kTileRows + j % kTileRows;
    float s = 0.f;
    for (int r = 0; r < R; ++r) s += exp2_fast(l[r * kTileRows] - sh_lse[r]);
    a.w_out[(int64_t)start + j] = w + s;
  }
}

// ------------------------------------------------------------------ host

struct AttendPlan {
  int64_t rows_each;                 // room rows of a part, about
  int64_t parts;                     // of the whole call
  bool split;                        // some segment has more than one
  size_t off_ml, off_o, off_logits, bytes;
};

static int64_t parts_of(const slkv_cache_desc* d, int64_t s, int64_t rows_each) {
  return std::max<int64_t>(1, (d->h_offsets[s + 1] - d->h_offsets[s] + rows_each - 1) / rows_each);
}

static AttendPlan plan_attend(const slkv_cache_desc* d, int T, bool weights) {
  AttendPlan p;
  const int64_t S = (int64_t)d->B * d->Hkv, rows = d->h_offsets[S] - d->h_offsets[0];
  const int64_t R = (int64_t)(d->Hq / d->Hkv) * T;
  constexpr int64_t kPlaces = 2 * 256, kLeast = kAttendWaves * 32;
  p.rows_each = std::max(kLeast, ((rows + kPlaces - 1) / kPlaces + kTileRows - 1) / kTileRows * kTileRows);
  p.parts = 0;
  for (int64_t s = 0; s < S; ++s) p.parts += parts_of(d, s, p.rows_each);
  p.split = p.parts > S;
  size_t at = 0;
  auto take = [&](int64_t floats) {
    const size_t off = at;
    at += ((size_t)floats * sizeof(float) + 255) / 256 * 256;
    return off;
  };
  p.off_ml = take(p.split ? p.parts * 2 * R : 0);
  p.off_o = take(p.split ? p.parts * R * d->d : 0);
  p.off_logits = take(weights ? (rows / kTileRows + S + 1) * kTileRows * R : 0);
  p.bytes = std::max<size_t>(at, 16);
  return p;
}

static slkv_status attend_checks(const slkv_cache_desc* desc, int32_t T) {
  slkv_status st = validate_cache_desc(desc);
  if (st != SLKV_OK) return st;
  if (T < 1) return fail(SLKV_ERR_BAD_ARG, "T must be >= 1");
  if (T > 64 || desc->Hq / desc->Hkv * T > 64) return fail(SLKV_ERR_UNSUPPORTED, "(Hq/Hkv)*T = %lld queries > 64", (long long)(desc->Hq / desc->Hkv) * T);
  return SLKV_OK;
}

}  // namespace slkv

using namespace slkv;

extern "C" slkv_status slkv_attend_workspace_bytes(const slkv_cache_desc* desc, int32_t T, int32_t want_weights, size_t* bytes) {
  clear_error();
  if (!bytes) return fail(SLKV_ERR_NULL, "bytes is NULL");
  slkv_status st = attend_checks(desc, T);
  if (st != SLKV_OK) return st;
  *bytes = plan_attend(desc, T, want_weights != 0).bytes;
  return SLKV_OK;
}

extern "C" slkv_status slkv_attend_cache(const slkv_cache_desc* desc, const slkv_cache* cache, int32_t T, const void* d_q, void* d_out,
                                         float* d_lse, float* d_weight_out, void* d_workspace, size_t workspace_bytes, void* hip_stream) {
  clear_error();
  slkv_status st = attend_checks(desc, T);
  if (st != SLKV_OK) return st;
  if ((st = validate_cache(desc, cache)) != SLKV_OK) return st;
  if (!d_q || !d_out || !d_workspace) return fail(SLKV_ERR_NULL, "a required device pointer is NULL");
  const void* ptrs[] = {d_q, d_out, d_lse, d_weight_out, d_workspace};
  for (const void* ptr : ptrs)
    if ((uintptr_t)ptr % 16) return fail(SLKV_ERR_BAD_ARG, "device pointer %p not 16-byte aligned", ptr);
  const AttendPlan p = plan_attend(desc, T, d_weight_out != nullptr);
  if (p.parts >= (int64_t(1) << 31)) return fail(SLKV_ERR_BAD_ARG, "too many parts");
  if (workspace_bytes < p.bytes) return fail(SLKV_ERR_WORKSPACE, "workspace %zu < %zu bytes", workspace_bytes, p.bytes);
  unsigned char* ws = (unsigned char*)d_workspace;
  const int64_t S = (int64_t)desc->B * desc->Hkv;
  AttendArgs a;
  a.k = (const unsigned char*)cache->d_k;
  a.v = (const unsigned char*)cache->d_v;
  a.k_scale = (const unsigned char*)cache->d_k_scale;
  a.v_scale = (const unsigned char*)cache->d_v_scale;
  a.q = (const unsigned char*)d_q;
  a.out = (unsigned char*)d_out;
  a.lengths = cache->d_lengths;
  a.lse = d_lse;
  a.w_in = cache->d_weight;
  a.w_out = d_weight_out;
  a.part_ml = (float*)(ws + p.off_ml);
  a.part_o = (float*)(ws + p.off_o);
  a.logits = d_weight_out ? (float*)(ws + p.off_logits) : nullptr;
  a.T = T;
  a.R = desc->Hq / desc->Hkv * T;
  a.row0 = (int32_t)desc->h_offsets[0];
  a.c_log2 = kLog2e / std::sqrt((float)desc->d);
  hipStream_t const stream = (hipStream_t)hip_stream;

  int64_t before = 0;                                  // parts of the segments of earlier tables
  auto launch = [&](auto tab, int64_t s0, int64_t ns) {
    using TAB = decltype(tab);
    tab.nseg = (int32_t)ns;
    tab.seg0 = (int32_t)s0;
    int64_t at = before;
    bool split = false;
    for (int64_t i = 0; i <= ns; ++i) {
      tab.w[0][i] = (int32_t)desc->h_offsets[s0 + i];
      tab.w[1][i] = (int32_t)at;
      if (i == ns) break;
      const int64_t parts = parts_of(desc, s0 + i, p.rows_each);
      split = split || parts > 1;
      at += parts;
    }
    const dim3 grid((unsigned)(at - before)), block(kAttendThreads);
    before = at;
    with_kind(desc->dtype, [&](auto kind) {
      auto with_dim = [&](auto dim) {
        constexpr int kKind = decltype(kind)::value, kDim = decltype(dim)::value;
        {
          ScopedKernelTimer timer(SLKV_K_ATTEND);
          if (a.R <= 16) SLKV_LAUNCH((attend_kernel<kKind, kDim, 1, TAB>), grid, block, 0, stream, a, tab);
          else if (a.R <= 32) SLKV_LAUNCH((attend_kernel<kKind, kDim, 2, TAB>), grid, block, 0, stream, a, tab);
          else SLKV_LAUNCH((attend_kernel<kKind, kDim, 4, TAB>), grid, block, 0, stream, a, tab);
        }
        if (split) {
          ScopedKernelTimer timer(SLKV_K_ATTEND_JOIN);
          SLKV_LAUNCH((attend_join_kernel<kKind, kDim, TAB>), grid, block, 0, stream, a, tab);
        }
      };
      if (desc->d == 64) with_dim(std::integral_constant<int, 64>{});
      else with_dim(std::integral_constant<int, 128>{});
    });
  };
  if (S <= kFewSegs) launch(AttendTab<kFewSegs>{}, 0, S);
  else
    for (int64_t s0 = 0; s0 < S; s0 += kManySegs2) launch(AttendTab<kManySegs2>{}, s0, std::min<int64_t>(kManySegs2, S - s0));
  return launch_status("attend");
}
