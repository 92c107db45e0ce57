// Attention of tiles of queries over tiles of rows that are staged in LDS: what slkv_attend_prompt and slkv_attend_tree share.
//
// The G = Hq/Hkv heads that share a KV head's rows are put together: query row r of a segment (sequence, KV head) is token r / G, head r % G, so that a tile of
// 32 rows covers 32/G neighbouring tokens and the mask cuts few of its keys.  A workgroup is WQ x WK waves; a wave holds 32 query rows in
// registers, and takes every WK'th 32 rows of a staged tile of keys.
//
// x = K q with MFMA operands of 32 keys by 16 dims comes out as D[key][query]: lane l holds query l % 32 and, of 32 keys, 8 (i / 4) + 4 (l / 32) + i % 4 for
// i = 0 .. 15.  The softmax over keys is a matter of a lane's own registers and of the lane 32 away.  The product with the values sums over keys in any order, so the
// registers 8 c .. 8 c + 7, as 16-bit numbers, are the operand of 16 keys as they stand, if V's operand takes the keys in the same order: two transposing
// reads of LDS, each of four neighbouring keys by 16 dims to 16 lanes.  The outputs come out as D[dim][query].
//
// Rows lie in LDS as in memory, in pieces of 16 bytes that are exchanged inside a row so that both ways of reading find all banks (swizzle()).
#ifndef SLKV_ATTEND_TILES_H
#define SLKV_ATTEND_TILES_H

#include "attend_rows.h"
#include "launch.h"
#include "tile_plan.h"

#include <algorithm>

namespace slkv {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

// Segment and tile of a workgroup; the same in all its lanes.
struct TileWork {
  const unsigned char *k, *v, *ks, *vs;   // first row of the segment
  const unsigned char* q;                 // query (token 0, head 0) of the segment
  unsigned char* out;
  float* lse;                             // may be NULL
  const uint64_t* sees;                   // [token]; NULL: causal
  int64_t q_tok, q_head, o_tok, o_head, lse_head;   // bytes; bytes; elements
  int64_t k_row, v_row;                   // bytes
  int rows, r0;                           // query rows of the segment; first one of the tile
  int hist;                               // token t sees the keys j <= hist + t, or j < hist and those of its bits
  int begin, end;                         // keys of this part of the tile's
  int part, parts;                        // parts that have keys, 1 at least
  int slot0, slot_step;                   // where the parts' results are
};

struct TileArgs {
  int32_t G, T;                           // heads of a segment; tokens (tree)
  int32_t blocks;                         // tiles and their parts
  float c_log2;                           // log2(e) / sqrt(d)
  float* part_o;                          // [slot][tile row][D], relative to the part's reference
  float* part_ml;                         // [slot][tile row][2]: reference (log2), sum
};

// 16 bytes per lane from base + off into LDS at lds (the same for the whole wave) + 16 * lane.  The caller waits for it (vmcnt); the compiler does not know of it.
// s_nop 4: a load into LDS needs a wait state behind a scalar write of m0, and its scalar address five behind a vector instruction that wrote it; inside a statement nobody else sees to either.
__device__ __forceinline__ void stage16(const unsigned char* base, uint32_t off, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(off), "s"(base), "s"(lds) : "memory", "m0");
}

template <class T>
__device__ __forceinline__ T lds_at(uint32_t at) { return *(const __attribute__((address_space(3))) T*)(uintptr_t)at; }
template <class T>
__device__ __forceinline__ void lds_put(uint32_t at, T v) { *(__attribute__((address_space(3))) T*)(uintptr_t)at = v; }

template <int KIND, int D, int WQ, int WK>
struct Tiles {
  typedef typename Kind<KIND>::wide wide;
  static constexpr bool kF32 = KIND == SLKV_F32;
  static constexpr bool kNarrow = Kind<KIND>::kBits < 16;
  static constexpr int kWaves = WQ * WK, kThreads = kWaves * kWave;
  static constexpr int kQueries = 32 * WQ;             // query rows of a workgroup
  static constexpr int kSub = WK == 1 ? 2 : 1;         // subtiles of 32 keys that a wave takes of a staged tile
  static constexpr int kKeys = 32 * kSub * WK;         // rows of a staged tile
  static constexpr int kRow = D * (int)sizeof(wide);   // bytes of a row in LDS
  static constexpr int kChunks = kRow / 16;
  static constexpr int kTileBytes = kKeys * kRow;      // of K; V the same behind it
  static constexpr int kSrcRow = D * Kind<KIND>::kBits / 8;
  static constexpr int kScales = D / kScaleBlock;
  static constexpr int kDT = D / 32;                   // tiles of 32 dims
  static constexpr int kOutRow = D + 4;                // floats of a row of sums in LDS
  // Narrow rows of four subtiles a step: one tile in LDS, the next one in registers, so that two workgroups share a CU.
  static constexpr bool kSingle = kNarrow && WK == 4 && WQ == 1;
  static constexpr int kTilesBytes = (kSingle ? 2 : 4) * kTileBytes;
  // Whether a workgroup takes tiles in turn: the ones that have a CU to themselves.  Where workgroups share one they fill each other's beginnings and ends, and the chip deals tiles out
  // more evenly (3 prompts of 1111 tokens in fp16, with one number a weight: in turn on 512 places 34 us, on 768 27, dealt out 25; with two 31).
  static constexpr bool kTurns = kWaves == 8;
  static constexpr int kOutBytes = WK == 1 ? 0 : kWaves * 32 * kOutRow * 4;
  static constexpr int kLds = kTilesBytes > kOutBytes ? kTilesBytes : kOutBytes;
  // waves of a SIMD, at least: what LDS and registers allow
  static constexpr int kPerSimd = D == 64 ? 2 : kF32 || (WQ == 1 && WK == 4 && !kSingle) ? 1 : 2;
  // Reference of fp16 weights: they reach 2^15, so that those down to 2^-26 of the largest keep all their bits.
  static constexpr float kBelow = KIND == SLKV_F16 ? 12.f : 0.f, kBelowPower = KIND == SLKV_F16 ? 0x1p-12f : 1.f;
  static constexpr float kAbove = KIND == SLKV_F16 ? 15.f : 8.f;   // a product this far above the reference moves it

  // Piece p of row r stands at p ^ swizzle(r).  Keys are read 32 rows at one piece, values 4 rows at 4 neighbouring pieces (fp32: 2 rows, 4 apart, at 8): with these
  // exchanges each finds all 64 banks.
  static __device__ __forceinline__ constexpr int swizzle(int r) {
    if constexpr (kF32) return (r & 3) | (r >> 3 & 1) << 2 | (r >> 2 & 1) << 3;
    else if constexpr (kChunks == 16) return (r & 3) << 2 | (r >> 2 & 3);
    else return (r >> 1 & 1) << 2 | (r >> 2 & 3);
  }

  // ---- staging of kKeys rows of K and V from row `first` on; rows from `end` on are the last one before it again

  static constexpr int kLoads = kKeys * kChunks / kThreads;   // 16-byte pieces of K a thread stages (not narrow)
  static __device__ __forceinline__ void stage(const TileWork& w, int first, int end, uint32_t lds) {
    constexpr int kRowsEach = kThreads / kChunks;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int r = tid / kChunks, p = tid % kChunks, last = end - 1 - first;
    const unsigned char* const kb = w.k + first * w.k_row;
    const unsigned char* const vb = w.v + first * w.v_row;
    const int ks = (int)w.k_row, vs = (int)w.v_row;
    if (last >= kKeys - 1) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int row = r + i * kRowsEach;
        stage16(kb, (uint32_t)(row * ks + (p ^ swizzle(row)) * 16), lds + (i * kThreads + wave * kWave) * 16);
      }
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int row = r + i * kRowsEach;
        stage16(vb, (uint32_t)(row * vs + (p ^ swizzle(row)) * 16), lds + kTileBytes + (i * kThreads + wave * kWave) * 16);
      }
    } else {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int row = r + i * kRowsEach, there = min(row, last);
        stage16(kb, (uint32_t)(there * ks + (p ^ swizzle(row)) * 16), lds + (i * kThreads + wave * kWave) * 16);
        stage16(vb, (uint32_t)(there * vs + (p ^ swizzle(row)) * 16), lds + kTileBytes + (i * kThreads + wave * kWave) * 16);
      }
    }
  }

  // narrow rows go through registers: pieces of 16 bytes are 16 or 32 elements
  static constexpr int kSrcChunks = kNarrow ? kSrcRow / 16 : 1;
  static constexpr int kUnits = kKeys * kSrcChunks, kFetch = (kUnits + kThreads - 1) / kThreads;
  struct Fetched { u32x4 k[kFetch], v[kFetch]; uint32_t ks[kFetch], vs[kFetch]; };
  // A wave takes whole rows, neighbouring lanes the same piece of neighbouring rows: what 16 of them write lies in 64 different banks.  (All the same 30 % (MXFP4) and 39 % (E4M3) of the LDS cycles
  // of narrow rows' kernels are conflicts, 10 and 13 % of all cycles; bf16 rows of 128 dims, which are read the same way and not written like this, have none.  The cause is not known.)
  static constexpr int kUnitRows = kWave / kSrcChunks;
  static __device__ __forceinline__ int row_of_unit(int u) { return u / kWave * kUnitRows + u % kUnitRows; }
  static __device__ __forceinline__ int chunk_of_unit(int u) { return u % kWave / kUnitRows; }
  static __device__ __forceinline__ void fetch(Fetched& f, const TileWork& w, int first, int end) {
#pragma unroll
    for (int i = 0; i < kFetch; ++i) {
      const int u = min((int)threadIdx.x + i * kThreads, kUnits - 1), c = chunk_of_unit(u);
      const int64_t row = min(first + row_of_unit(u), end - 1);
      f.k[i] = *(const u32x4*)(w.k + row * w.k_row + c * 16);
      f.v[i] = *(const u32x4*)(w.v + row * w.v_row + c * 16);
      if constexpr (KIND == SLKV_BF16_KV_MXFP4) {
        f.ks[i] = w.ks[row * kScales + c];
        f.vs[i] = w.vs[row * kScales + c];
      }
    }
  }
  static __device__ __forceinline__ void put(const Fetched& f, uint32_t lds) {
    auto one = [&](u32x4 x, uint32_t e, int row, int c, uint32_t base) __attribute__((always_inline)) {
      if constexpr (KIND == SLKV_BF16_KV_MXFP4) {
        const float s = scale_of(e);
#pragma unroll
        for (int j = 0; j < 4; ++j)
          lds_put(base + row * kRow + ((c * 4 + j) ^ swizzle(row)) * 16, u32x4{fp4_pair<0>(x[j], s), fp4_pair<1>(x[j], s), fp4_pair<2>(x[j], s), fp4_pair<3>(x[j], s)});
      } else {
#pragma unroll
        for (int j = 0; j < 2; ++j)
          lds_put(base + row * kRow + ((c * 2 + j) ^ swizzle(row)) * 16,
                  u32x4{fp8_pair<false>(x[j * 2]), fp8_pair<true>(x[j * 2]), fp8_pair<false>(x[j * 2 + 1]), fp8_pair<true>(x[j * 2 + 1])});
      }
    };
#pragma unroll
    for (int i = 0; i < kFetch; ++i) {
      const int u = (int)threadIdx.x + i * kThreads;
      if (kUnits % kThreads && u >= kUnits) break;
      one(f.k[i], f.ks[i], row_of_unit(u), chunk_of_unit(u), lds);
      one(f.v[i], f.vs[i], row_of_unit(u), chunk_of_unit(u), lds + kTileBytes);
    }
  }

  // ---- products

  static __device__ __forceinline__ f32x16 mfma(u32x4 x, u32x4 y, f32x16 c) {
    if constexpr (KIND == SLKV_F16)
      return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, x), __builtin_bit_cast(f16x8, y), c, 0, 0, 0);
    else
      return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, y), c, 0, 0, 0);
  }
  static __device__ __forceinline__ uint32_t pair(float x, float y) {
    if constexpr (KIND == SLKV_F16) return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{x, y}), f16x2));
    else return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{x, y}), bf16x2));
  }
  static __device__ __forceinline__ u32x2 read_turned(uint32_t at) {
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(uintptr_t)at));
  }
  // element of V of a staged row
  static __device__ __forceinline__ float value(uint32_t vt, int row, int dim) {
    const uint32_t at = vt + row * kRow + ((dim * (int)sizeof(wide) / 16) ^ swizzle(row)) * 16 + dim * (int)sizeof(wide) % 16;
    if constexpr (kF32) return lds_at<float>(at);
    else if constexpr (KIND == SLKV_F16) return (float)lds_at<_Float16>(at);
    else return __uint_as_float((uint32_t)lds_at<uint16_t>(at) << 16);
  }

  // queries of the lane: 16-bit: product u takes the dims 16 u + 8 g .. + 7 of lane group g = lane / 32; fp32: 8 u + 4 g + j
  struct Queries { u32x4 w[kF32 ? D / 8 : D / 16]; };

  // x[sub] of the wave's subtiles; kt: K in LDS, at the wave's first subtile
  static __device__ __forceinline__ void logits(f32x16 (&x)[kSub], const Queries& q, uint32_t kt, int l32, int g) {
    const uint32_t at = kt + l32 * kRow + (uint32_t)((g ^ swizzle(l32)) * 16);      // (chunk 2 u + g) ^ swizzle = (2 u) ^ (g ^ swizzle)
#pragma unroll
    for (int s = 0; s < kSub; ++s) {
      if constexpr (kF32) {
        // four sums side by side: one chain of D additions is what the result's error comes from
        f32x16 y[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) y[j] = f32x16{};
#pragma unroll
        for (int u = 0; u < D / 8; ++u) {
          const f32x4 ko = lds_at<f32x4>((at ^ (u * 32)) + s * 32 * kRow);
#pragma unroll
          for (int j = 0; j < 4; ++j) y[j] = __builtin_amdgcn_mfma_f32_32x32x2f32(ko[j], __uint_as_float(q.w[u][j]), y[j], 0, 0, 0);
        }
        x[s] = (y[0] + y[1]) + (y[2] + y[3]);
      } else {
        x[s] = f32x16{};
#pragma unroll
        for (int u = 0; u < D / 16; ++u) {
          const u32x4 ko = lds_at<u32x4>((at ^ (u * 32)) + s * 32 * kRow);
          x[s] = mfma(ko, q.w[u], x[s]);
        }
      }
    }
  }

  // Two weights >= 0 as a pair of 16-bit numbers, rounded towards 0, and the pair of what is left, which is above 0 wherever the first number is: an infinite value times the one and times the other
  // makes no NaN.  bf16: 2^-20 of the weight more than what is left; fp16: 2^-24 at least, 2^-36 of the query's largest weight.  (With what is left as it is, and NaN looked for in the outputs and mended
  // by a second turn, 2 to 40 % slower: registers.)
  static __device__ __forceinline__ void halves(float x, float y, uint32_t& hi, uint32_t& lo) {
    if constexpr (KIND == SLKV_F16) {
      typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
      const f16x2 h = __builtin_bit_cast(f16x2, __builtin_amdgcn_cvt_pkrtz(x, y));
      const u16x2 rest = __builtin_bit_cast(u16x2, __builtin_amdgcn_cvt_pkrtz(x - (float)h[0], y - (float)h[1]));
      uint32_t one = 0x00010001u;
      asm("" : "+s"(one));                             // (a minimum with a known 1 becomes four comparisons and selections)
      hi = __builtin_bit_cast(uint32_t, h);
      lo = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(rest, __builtin_elementwise_min(__builtin_bit_cast(u16x2, h), __builtin_bit_cast(u16x2, one))));
    } else {
      constexpr float kMore = 1.f + 0x1p-20f;
      const uint32_t xb = __float_as_uint(x), yb = __float_as_uint(y);
      hi = __builtin_amdgcn_perm(yb, xb, 0x07060302u);
      lo = pair(fmaf(x, kMore, -__uint_as_float(xb & 0xffff0000u)), fmaf(y, kMore, -__uint_as_float(yb & 0xffff0000u)));
    }
  }

  // acc += p V of one subtile; vt: V in LDS, at the subtile.  16-bit types: a weight enters as two numbers, which hold it to 2^-16 (fp16: 2^-21) of itself, as in slkv_attend_cache: one
  // (ONE, where the caller asks for it) would add as much error as the output's own rounding.  The second product is half of the call's matrix work more: a third of the time where that is what a call takes its time with (32 heads of
  // 128 in bf16: 32768 tokens 7.9 ms with one number, 10.6 with two; 512 queries behind 65024 keys 555, 715 us), 6 % where it is not (32 drafted tokens on 128 segments of 1024 rows 38.5, 40.8 us).
  template <bool ONE>
  static __device__ __forceinline__ void add_values(f32x16 (&acc)[kDT], const f32x16& p, uint32_t vt, int lane) {
    if constexpr (kF32) {
      const int g = lane >> 5, l32 = lane & 31;
      const uint32_t at = vt + 4 * g * kRow + (uint32_t)((l32 / 4) ^ (g << 3)) * 16 + l32 % 4 * 4;
      // The 32 keys are summed on their own and then added: a product adds two keys, and a sum that takes 16384 of these loses what the weights' sum keeps.
      f32x16 y[kDT];
#pragma unroll
      for (int dt = 0; dt < kDT; ++dt) y[dt] = f32x16{};
#pragma unroll
      for (int i = 0; i < 16; ++i)
#pragma unroll
        for (int dt = 0; dt < kDT; ++dt) {
          const float v = lds_at<float>((at ^ (uint32_t)((i & 3 | (i >> 2 & 1) << 2 | dt << 3) * 16)) + (i / 4 * 8 + i % 4) * kRow);
          y[dt] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, p[i], y[dt], 0, 0, 0);
        }
#pragma unroll
      for (int dt = 0; dt < kDT; ++dt) acc[dt] += y[dt];
    } else {
      // lane i of 16 reads the piece i % 4, of 8 bytes, of row i / 4: of the rows 4 g .. 4 g + 3 and, with j2, 8 rows on; 16 dims to 16 lanes
      const int g = lane >> 5, h = lane >> 4 & 1, i4 = lane >> 2 & 3, i1 = lane >> 1 & 1;
      const int row = 4 * g + i4;
      const uint32_t at = vt + row * kRow + (uint32_t)((2 * h + i1) ^ swizzle(row)) * 16 + (lane & 1) * 8;
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        u32x4 hi, lo, vo[kDT];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float x = p[c * 8 + j * 2], y = p[c * 8 + j * 2 + 1];
          if constexpr (ONE) {
            hi[j] = pair(x, y);
          } else {
            uint32_t h2, l2;
            halves(x, y, h2, l2);
            hi[j] = h2;
            lo[j] = l2;
          }
        }
#pragma unroll
        for (int dt = 0; dt < kDT; ++dt)
#pragma unroll
          for (int j2 = 0; j2 < 2; ++j2) {
            // 8 rows on: swizzle changes bit 1
            const u32x2 t = read_turned((at ^ (uint32_t)(dt * 64 ^ j2 * 32)) + (c * 16 + j2 * 8) * kRow);
            vo[dt][j2 * 2] = t[0];
            vo[dt][j2 * 2 + 1] = t[1];
          }
#pragma unroll
        for (int dt = 0; dt < kDT; ++dt) acc[dt] = mfma(vo[dt], hi, acc[dt]);
        if constexpr (!ONE) {
#pragma unroll
          for (int dt = 0; dt < kDT; ++dt) acc[dt] = mfma(vo[dt], lo, acc[dt]);
        }
      }
    }
  }

  // whether some value of the subtile's 32 rows is not finite
  static __device__ __forceinline__ bool any_not_finite(uint32_t vt, int lane) {
    // an exponent of all ones carries into the sign's place
    constexpr uint32_t kExp = kF32 ? 0x7f800000u : KIND == SLKV_F16 ? 0x7c007c00u : 0x7f807f80u, kOne = kF32 ? 0x00800000u : KIND == SLKV_F16 ? 0x04000400u : 0x00800080u;
    uint32_t carries = 0;
#pragma unroll
    for (int i = 0; i < 32 * kChunks / kWave; ++i) {
      const u32x4 x = lds_at<u32x4>(vt + (i * kWave + lane) * 16);
#pragma unroll
      for (int j = 0; j < 4; ++j) carries |= (x[j] & kExp) + kOne;
    }
    const bool bad = (carries & (kF32 ? 0x80000000u : 0x80008000u)) != 0;
    return __ballot(bad) != 0;
  }
};

// The drafted tokens that token t sees, a bit each; causal: none.
__device__ __forceinline__ uint64_t bits_of(const TileWork& w, int t, int T) {
  return w.sees ? w.sees[t] & (T < 64 ? (1ull << T) - 1 : ~0ull) : 0ull;
}
// Whether nothing is seen by token t.  (A tree's token that sees nothing of the draft sees what is before it.)
__device__ __forceinline__ bool sees_none(const TileWork& w, int t, uint64_t bits) {
  if (!w.sees) return w.hist + t < 0;
  // rows of the draft that are there: hist + u >= 0
  if (w.hist > 0) return false;
  return w.hist <= -64 || (bits >> -w.hist) == 0;
}

// The lowest n bits, for any n.
__device__ __forceinline__ uint32_t first_bits(int n) { return n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1u; }

// What a query gets of its reference and its sum: the log-sum-exp, and the outputs' factor.
template <class A>
__device__ __forceinline__ float tile_lse(float top, float total, bool none) {
  return none ? -INFINITY : total > 0.f ? ((top + A::kBelow) + __builtin_amdgcn_logf(total * A::kBelowPower)) * kLn2 : NAN;
}
__device__ __forceinline__ float total_scale(float total) { return total > 0.f ? 1.f / total : NAN; }

// A tile of queries, or a part of one's keys, a workgroup; workgroups of 8 waves take tiles in turn: as many of them as the chip has places go through the tiles back and forth, so that tiles that
// get smaller come out even, and the next tile's first rows and queries are on their way while the outputs are written.  (Without turns, and with outputs through LDS, a workgroup took 17 us beside
// its steps, of which 6 between two workgroups of a CU, 4 for the first rows, 6 for the outputs; with one number a weight 16 prompts of 1024 tokens went from 270 to 218 us, 4096 tokens
// from 147 to 137: with two they take 254 and 187.)
// Bound by the chip's power in long prompts (32768 tokens, 32 heads of 128 in bf16: 10.6 to 11.8 ms by box, 1.1 to 1.24 PFLOP/s of matrix work where the library's large product reaches 1.13; matrix units 64 %, vector units 54 %
// of the cycles busy at a clock of 1.82 GHz), by a workgroup's beginning and end in short ones, by memory and the join where queries are few.
template <int KIND, int D, int WQ, int WK, class TAB>
__global__ __launch_bounds__(WQ* WK* kWave, (Tiles<KIND, D, WQ, WK>::kPerSimd)) void attend_tiles_kernel(const TileArgs a, const TAB tab) {
  using A = Tiles<KIND, D, WQ, WK>;
  constexpr int kSub = A::kSub, kDT = A::kDT;
  __shared__ __align__(1024) unsigned char sh[A::kLds];
  constexpr int kRowsOut = WK > 1 ? 32 * WQ : 1;
  __shared__ float sh_m[WK][kRowsOut], sh_l[WK][kRowsOut], sh_scale[kRowsOut];
  __shared__ int64_t sh_at[kRowsOut];
  const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)sh;
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave));
  const int l32 = lane & 31, g = lane >> 5, wq = wave % WQ, wk = wave / WQ;
  const int first = wq * 32;                           // the wave's first row of a tile

  // The table goes through LDS: one round trip to the arguments, and none for the tiles after the first.
  __shared__ typename TAB::Words table;
  {
    constexpr int kWords = sizeof(typename TAB::Words) / 4;
    const uint32_t* const from = (const uint32_t*)&tab.words;
    for (int i = threadIdx.x; i < kWords; i += A::kThreads) ((uint32_t*)&table)[i] = from[i];
    __syncthreads();
  }
  int turn = 0;
  // the number of the workgroup's next tile, -1: there is none
  auto next_block = [&]() __attribute__((always_inline)) {
    while (A::kTurns || turn == 0) {
      if (turn * (int64_t)gridDim.x >= a.blocks) break;
      const int block = turn * (int)gridDim.x + (turn & 1 ? (int)gridDim.x - 1 - (int)blockIdx.x : (int)blockIdx.x);
      ++turn;
      if (block < a.blocks) return block;
    }
    return -1;
  };
  // the next tile whose part has keys, or outputs to write; false: there is none
  auto next_tile = [&](TileWork& w) __attribute__((always_inline)) {
    while (true) {
      const int block = next_block();
      if (block < 0) return false;
      w = tab.template describe<A::kQueries, A::kKeys, D, KIND>(a, table, tab.template locate<A::kQueries>(a, table, block));
      if (w.part < w.parts) return true;
    }
  };
  TileWork w;
  if (!next_tile(w)) return;

  typename A::Fetched raw;
  typename A::Queries q;
  int t_of, head_of;                                   // the lane's row: token and head
  uint64_t bits;
  auto load_rows = [&]() __attribute__((always_inline)) {
    if (w.begin < w.end) {
      if constexpr (A::kNarrow) A::fetch(raw, w, w.begin, w.end);
      else A::stage(w, w.begin, w.end, lds);
    }
  };
  auto load_queries = [&]() __attribute__((always_inline)) {
    const int t0 = w.r0 / a.G, rem0 = w.r0 - t0 * a.G;  // token and head of the tile's first row
    const int r = rem0 + max(min(first + l32, w.rows - 1 - w.r0), 0), dt = divide(r, a.G);
    t_of = t0 + dt;
    head_of = r - dt * a.G;
    const unsigned char* const at = w.q + t_of * w.q_tok + head_of * w.q_head;
#pragma unroll
    for (int u = 0; u < (A::kF32 ? D / 8 : D / 16); ++u) q.w[u] = *(const u32x4*)(at + u * 32 + g * 16);
    bits = bits_of(w, t_of, a.T);
  };
  load_rows();
  load_queries();

  while (true) {
    const bool busy = w.r0 + first < w.rows;           // (waves without queries only stage)
    float ref = -INFINITY, sum = 0.f;
    f32x16 acc[kDT];
#pragma unroll
    for (int dt = 0; dt < kDT; ++dt) acc[dt] = f32x16{};
    // keys that every query of the tile sees
    const int all = w.sees ? w.hist : w.hist + w.r0 / a.G + 1;
    // bit j: the lane's query sees the key key0 + j, which is there
    auto seen = [&](int key0) __attribute__((always_inline)) {
      uint32_t m = first_bits((w.sees ? w.hist : w.hist + t_of + 1) - key0);
      if (w.sees) {
        const int u = key0 - w.hist;                   // the draft's first row is bit -u
        m |= u >= 64 || u <= -32 ? 0u : u >= 0 ? (uint32_t)(bits >> u) : (uint32_t)bits << -u;
      }
      return m & first_bits(w.end - key0);
    };

    auto step = [&](auto tail_c, int key0, uint32_t buf) __attribute__((always_inline)) {
      constexpr bool tail = decltype(tail_c)::value;
      const uint32_t kt = buf + wk * 32 * kSub * A::kRow, vt = kt + A::kTileBytes;
      const int mine = key0 + wk * 32 * kSub;
      f32x16 x[kSub];
      A::logits(x, q, kt, l32, g);
      if constexpr (tail) {
#pragma unroll
        for (int s = 0; s < kSub; ++s) {
          const uint32_t m = seen(mine + s * 32) >> (4 * g);
#pragma unroll
          for (int i = 0; i < 16; ++i) x[s][i] = m & 1u << (i / 4 * 8 + i % 4) ? x[s][i] : -INFINITY;
        }
      }
      float top = -INFINITY;
#pragma unroll
      for (int s = 0; s < kSub; ++s)
#pragma unroll
        for (int i = 0; i < 16; ++i) top = fmaxf(top, x[s][i]);
      top *= a.c_log2;
      if (__ballot(top > ref + A::kAbove)) {
        top = fmaxf(top, __shfl_xor(top, 32));
        const float now = fmaxf(ref, top - A::kBelow);
        const float f = ref == -INFINITY ? 0.f : exp2_fast(ref - now);
        // (sums of a NaN stay one)
        sum *= f;
#pragma unroll
        for (int dt = 0; dt < kDT; ++dt) acc[dt] *= f;
        ref = now;
      }
      // (one rounding, of the difference: a large product's own would be an error of the weight)
      const float from = ref == -INFINITY ? 0.f : ref;
      // A step's weights are added to each other first, in four chains: the sum takes one addition for every 64 keys (WK = 4: 128).  (Added one by one, thousands of weights of 2^-24 of
      // it leave no trace: a lane's half of 32767 of them behind one large key was lost, 8.7e-4 of the log-sum-exp.)
      float part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < kSub; ++s)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          x[s][i] = exp2_fast(fmaf(x[s][i], a.c_log2, -from));
          part[i % 4] += x[s][i];
        }
      sum += (part[0] + part[1]) + (part[2] + part[3]);
#pragma unroll
      for (int s = 0; s < kSub; ++s) {
        const uint32_t vs = vt + s * 32 * A::kRow;
        if (tail && A::any_not_finite(vs, lane)) {
          // a row at a time, to the queries that see it: an infinity or NaN reaches no other through a weight of 0
          const uint32_t m = seen(mine + s * 32);
          for (int row = 0; row < 32; ++row) {
            float p = 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i)
              if (i == row / 8 * 4 + row % 4) p = x[s][i];
            p = __shfl(p, (row / 4 & 1) * 32 + l32);
            if (m >> row & 1) {
#pragma unroll
              for (int dt = 0; dt < kDT; ++dt)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[dt][i] += p * A::value(vs, row, dt * 32 + i / 4 * 8 + 4 * g + i % 4);
            }
          }
        } else {
          A::template add_values<TAB::kOneNumber>(acc, x[s], vs, lane);
        }
      }
    };

    // Tiles of keys that every query sees whole, then the others: the steps are two programs, so that the first has no branches for what the second has to look after (in one, with copies of
    // the sums where its ways met, 32768 tokens took 8.90 ms where 7.97 were left, with one number a weight).
    uint32_t buf = lds, other = lds + 2 * A::kTileBytes;
    int key0 = w.begin;
    const int whole_end = w.begin + max(min(all, w.end) - w.begin, 0) / A::kKeys * A::kKeys;
    if constexpr (A::kNarrow) {
      if (w.begin < w.end) A::put(raw, buf);
    }
    auto run = [&](auto tail_c, int until) __attribute__((always_inline)) {
      for (; key0 < until; key0 += A::kKeys) {
        const bool more = key0 + A::kKeys < w.end;
        if constexpr (A::kNarrow) {
          if (more) A::fetch(raw, w, key0 + A::kKeys, w.end);
          __syncthreads();
        } else {
          asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
          __syncthreads();
          if (more) A::stage(w, key0 + A::kKeys, w.end, other);
        }
        if (busy) step(tail_c, key0, buf);
        if constexpr (A::kSingle) {
          __syncthreads();
          if (more) A::put(raw, buf);
        } else {
          if constexpr (A::kNarrow) {
            if (more) A::put(raw, other);
          }
          const uint32_t t = buf;
          buf = other;
          other = t;
        }
      }
    };
    run(std::integral_constant<bool, false>{}, whole_end);
    run(std::integral_constant<bool, true>{}, w.end);

    const TileWork now = w;
    const int t_now = t_of, head_now = head_of;
    const uint64_t bits_now = bits;
    bool more = false;
    if constexpr (A::kTurns) more = next_tile(w);
    const bool whole = now.parts == 1;
    const int64_t row0 = (int64_t)(now.slot0 + now.part * now.slot_step) * A::kQueries;
    const float total = sum + __shfl_xor(sum, 32);
    __syncthreads();                                   // the last rows have been read
    if constexpr (WK == 1) {
      if (more) {
        load_rows();
        load_queries();
      }
      if (now.r0 + first + l32 < now.rows) {
        if (whole) {
          const bool none = sees_none(now, t_now, bits_now);
          const float scale = total_scale(total);
          unsigned char* const at = now.out + t_now * now.o_tok + head_now * now.o_head;
#pragma unroll
          for (int dt = 0; dt < kDT; ++dt) {
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[dt][i] = none ? 0.f : acc[dt][i] * scale;
            if constexpr (A::kF32) {
#pragma unroll
              for (int i = 0; i < 4; ++i)
                *(f32x4*)(at + (dt * 32 + i * 8 + 4 * g) * 4) = f32x4{acc[dt][i * 4], acc[dt][i * 4 + 1], acc[dt][i * 4 + 2], acc[dt][i * 4 + 3]};
            } else {
              // dims 8 i .. 8 i + 3 are in lane l, the next four in lane l + 32: of two neighbouring i each gets one whole
#pragma unroll
              for (int i = 0; i < 4; i += 2) {
                u32x4 o;
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                  const uint32_t x = A::pair(acc[dt][i * 4 + 2 * e], acc[dt][i * 4 + 2 * e + 1]), y = A::pair(acc[dt][i * 4 + 4 + 2 * e], acc[dt][i * 4 + 5 + 2 * e]);
                  const u32x2 t = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(x, y, false, false));
                  o[e] = t[0];
                  o[2 + e] = t[1];
                }
                *(u32x4*)(at + (dt * 32 + (i + g) * 8) * 2) = o;
              }
            }
          }
          if (now.lse && g == 0) now.lse[head_now * now.lse_head + t_now] = tile_lse<A>(ref, total, none);
        } else {
          const int64_t row = row0 + first + l32;
#pragma unroll
          for (int dt = 0; dt < kDT; ++dt)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              *(f32x4*)(a.part_o + row * D + dt * 32 + i * 8 + 4 * g) = f32x4{acc[dt][i * 4], acc[dt][i * 4 + 1], acc[dt][i * 4 + 2], acc[dt][i * 4 + 3]};
          if (g == 0) *(f32x2*)(a.part_ml + row * 2) = f32x2{ref, total};
        }
      }
    } else {
      // the waves that share queries are put together through LDS
      float* const sh_o = (float*)sh;
      if (g == 0) {
        sh_m[wk][first + l32] = ref;
        sh_l[wk][first + l32] = total;
      }
      __syncthreads();
      float top = -INFINITY;
#pragma unroll
      for (int i = 0; i < WK; ++i) top = fmaxf(top, sh_m[i][first + l32]);
      // (a wave that saw nothing has a sum of 0, or NaN where a product was NaN)
      const float mine = ref == -INFINITY ? 1.f : exp2_fast(ref - top);
#pragma unroll
      for (int dt = 0; dt < kDT; ++dt)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          *(f32x4*)&sh_o[((wk * WQ + wq) * 32 + l32) * A::kOutRow + dt * 32 + i * 8 + 4 * g] =
              f32x4{acc[dt][i * 4], acc[dt][i * 4 + 1], acc[dt][i * 4 + 2], acc[dt][i * 4 + 3]} * mine;
      if (wk == 0 && g == 0 && now.r0 + first + l32 < now.rows) {
        const int r = first + l32;
        float l = 0.f;
#pragma unroll
        for (int i = 0; i < WK; ++i) l += sh_l[i][r] * (sh_m[i][r] == -INFINITY ? 1.f : exp2_fast(sh_m[i][r] - top));
        if (whole) {
          const bool none = sees_none(now, t_now, bits_now);
          sh_scale[r] = none ? 0.f : total_scale(l);
          sh_at[r] = t_now * now.o_tok + head_now * now.o_head;
          if (now.lse) now.lse[head_now * now.lse_head + t_now] = tile_lse<A>(top, l, none);
        } else {
          *(f32x2*)(a.part_ml + (row0 + r) * 2) = f32x2{top, l};
        }
      }
      __syncthreads();
      constexpr int kLanes = D / 4;                    // threads of a row of outputs
      for (int idx = threadIdx.x; idx < 32 * WQ * kLanes; idx += A::kThreads) {
        const int r = idx / kLanes, d0 = idx % kLanes * 4;   // row of the tile, dims
        if (now.r0 + r >= now.rows) break;
        f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < WK; ++i) o += *(const f32x4*)&sh_o[(i * WQ * 32 + r) * A::kOutRow + d0];
        if (whole) store_out<KIND>(now.out + sh_at[r] + d0 * (int)sizeof(typename A::wide), o * sh_scale[r]);
        else *(f32x4*)(a.part_o + (row0 + r) * D + d0) = o;
      }
      if (more) {
        __syncthreads();
        load_rows();
        load_queries();
      }
    }
    if (!more) return;
  }
}

// The parts of a tile put together, in their order.  The workgroups of a part (join_slices() of them) take every so many'th group of rows.  Bound by latency: all references and sums of a row are asked for at once,
// by the lanes that share the row, and of the outputs eight parts at a time.
template <int KIND, int D, int WQ, int WK, class TAB>
__global__ __launch_bounds__(256) void join_tiles_kernel(const TileArgs a, const TAB tab) {
  using A = Tiles<KIND, D, WQ, WK>;
  const TileWork w = tab.template describe<A::kQueries, A::kKeys, D, KIND>(a, tab.words, tab.template locate<A::kQueries>(a, tab.words, (int)blockIdx.x));
  if (w.parts == 1 || w.part >= w.parts) return;
  constexpr int kLanes = D / 4, kRows = 256 / kLanes, kAtOnce = 8;
  const int t0 = w.r0 / a.G, rem0 = w.r0 % a.G, lane = threadIdx.x % kLanes, d0 = lane * 4;
  const int turn = w.parts * (int)gridDim.y * kRows;
  for (int r = (w.part * (int)gridDim.y + (int)blockIdx.y) * kRows + threadIdx.x / kLanes; r < A::kQueries && w.r0 + r < w.rows; r += turn) {
    auto at = [&](int p) __attribute__((always_inline)) { return (int64_t)(w.slot0 + p * w.slot_step) * A::kQueries + r; };
    f32x4 x[kAtOnce];
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) x[i] = *(const f32x4*)(a.part_o + at(min(i, w.parts - 1)) * D + d0);
    // the lane's parts: lane, lane + kLanes, ..
    f32x2 ml = f32x2{-INFINITY, 0.f};
    if (lane < w.parts) ml = *(const f32x2*)(a.part_ml + at(lane) * 2);
    float top = ml[0];
    for (int p = lane + kLanes; p < w.parts; p += kLanes) top = fmaxf(top, a.part_ml[at(p) * 2]);
    top = reduce_lanes(top, kLanes, [](float u, float v) { return fmaxf(u, v); });
    f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
    float l = 0.f;
    for (int p0 = 0; p0 < w.parts; p0 += kLanes) {     // (kLanes is a multiple of kAtOnce)
      if (p0 && p0 + lane < w.parts) ml = *(const f32x2*)(a.part_ml + at(p0 + lane) * 2);
      const float f = ml[0] == -INFINITY ? 1.f : exp2_fast(ml[0] - top);
      if (p0 + lane < w.parts) l += ml[1] * f;
      for (int q0 = p0; q0 < min(w.parts, p0 + kLanes); q0 += kAtOnce) {
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
          const float fi = __shfl(f, ((int)threadIdx.x & ~(kLanes - 1)) + q0 - p0 + i);
          if (q0 + i < w.parts) o += x[i] * fi;
        }
        if (q0 + kAtOnce < w.parts) {
#pragma unroll
          for (int i = 0; i < kAtOnce; ++i) x[i] = *(const f32x4*)(a.part_o + at(min(q0 + kAtOnce + i, w.parts - 1)) * D + d0);
        }
      }
    }
    l = reduce_lanes(l, kLanes, [](float u, float v) { return u + v; });
    const int dt = divide(rem0 + r, a.G), head = rem0 + r - dt * a.G, t = t0 + dt;
    const bool none = sees_none(w, t, bits_of(w, t, a.T));
    store_out<KIND>(w.out + t * w.o_tok + head * w.o_head + d0 * (int)sizeof(typename A::wide), none ? f32x4{0.f, 0.f, 0.f, 0.f} : o * total_scale(l));
    if (w.lse && d0 == 0) w.lse[head * w.lse_head + t] = tile_lse<A>(top, l, none);
  }
}

// ------------------------------------------------------------------ host

// Workgroups of a launch, at most: as many as the registers and LDS of the chip have places for.
template <class A>
constexpr unsigned tile_places() {
  if (!A::kTurns) return ~0u;
  const int waves = 4 * A::kPerSimd / A::kWaves, lds = 160 * 1024 / (A::kLds + 4096);
  return 256 * (unsigned)std::max(1, std::min(waves, lds));
}

// f with the waves of a shape as compile-time constants.
template <int KIND, int D, int S = 0, class F>
void with_shape(int shape, F f) {
  if constexpr (S < kTileShapeCount) {
    if constexpr (has_shape(KIND, D, S)) {
      if (shape == S) return f(std::integral_constant<int, kTileShapes[S].wq>{}, std::integral_constant<int, kTileShapes[S].wk>{});
    }
    with_shape<KIND, D, S + 1>(shape, f);
  }
}

}  // namespace slkv
#endif
