// Attention of tiles of queries over tiles of rows that are staged in LDS: what slkv_attend_prompt and slkv_attend_tree share.
//
// The G = Hq/Hkv heads that share a KV head's rows are put together: query row r of a segment (sequence, KV head) is token r / G, head r % G, so that a tile of
// 32 rows covers 32/G neighbouring tokens and the mask cuts few of its keys.  A workgroup is WQ x WK waves; a wave holds QT tiles of 32 query rows in
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

#include <cmath>

namespace slkv {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr int kTileWaves = 4;

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
  int n;                                  // keys of the segment
  int begin, end;                         // keys of this part of the tile's
  int part, parts;                        // parts that have keys, 1 at least
  int slot0, slot_step;                   // where the parts' results are
};

struct TileArgs {
  int32_t G, T;                           // heads of a segment; tokens (tree)
  float c_log2;                           // log2(e) / sqrt(d)
  float* part_o;                          // [slot][tile row][D], relative to the part's reference
  float* part_ml;                         // [slot][tile row][2]: reference (log2), sum
};

// 16 bytes per lane from base + off into LDS at lds (the same for the whole wave) + 16 * lane.  The caller waits for it (vmcnt); the compiler does not know of it.
__device__ __forceinline__ void stage16(const unsigned char* base, uint32_t off, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %2\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(off), "s"(base), "s"(lds) : "memory", "m0");
}

template <class T>
__device__ __forceinline__ T lds_at(uint32_t at) { return *(const __attribute__((address_space(3))) T*)(uintptr_t)at; }
template <class T>
__device__ __forceinline__ void lds_put(uint32_t at, T v) { *(__attribute__((address_space(3))) T*)(uintptr_t)at = v; }

template <int KIND, int D, int QT, int WQ, int WK>
struct Tiles {
  typedef typename Kind<KIND>::wide wide;
  static constexpr bool kF32 = KIND == SLKV_F32;
  static constexpr bool kNarrow = Kind<KIND>::kBits < 16;
  static constexpr int kThreads = WQ * WK * kWave;
  static constexpr int kQueries = 32 * QT * WQ;        // query rows of a workgroup
  static constexpr int kSub = WK == 1 ? 2 : 1;         // subtiles of 32 keys that a wave takes of a staged tile
  static constexpr int kKeys = 32 * kSub * WK;         // rows of a staged tile
  static constexpr int kRow = D * (int)sizeof(wide);   // bytes of a row in LDS
  static constexpr int kChunks = kRow / 16;
  static constexpr int kTileBytes = kKeys * kRow;      // of K; V the same behind it
  static constexpr int kSrcRow = D * Kind<KIND>::kBits / 8;
  static constexpr int kScales = D / kScaleBlock;
  static constexpr int kDT = D / 32;                   // tiles of 32 dims
  static constexpr int kOutRow = D + 4;                // floats of a row of sums in LDS
  static constexpr int kLds = 4 * kTileBytes > kTileWaves * 32 * kOutRow * 4 ? 4 * kTileBytes : kTileWaves * 32 * kOutRow * 4;
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
  static __device__ __forceinline__ void fetch(Fetched& f, const TileWork& w, int first, int end) {
#pragma unroll
    for (int i = 0; i < kFetch; ++i) {
      const int u = min((int)threadIdx.x + i * kThreads, kUnits - 1), c = u % kSrcChunks;
      const int64_t row = min(first + u / kSrcChunks, end - 1);
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
      one(f.k[i], f.ks[i], u / kSrcChunks, u % kSrcChunks, lds);
      one(f.v[i], f.vs[i], u / kSrcChunks, u % kSrcChunks, lds + kTileBytes);
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
  struct Queries { u32x4 w[QT][kF32 ? D / 8 : D / 16]; };

  // x[sub][qt] of the wave's subtiles; kt: K in LDS, at the wave's first subtile
  static __device__ __forceinline__ void logits(f32x16 (&x)[kSub][QT], const Queries& q, uint32_t kt, int l32, int g) {
    const uint32_t at = kt + l32 * kRow + (uint32_t)((g ^ swizzle(l32)) * 16);      // (chunk 2 u + g) ^ swizzle = (2 u) ^ (g ^ swizzle)
#pragma unroll
    for (int s = 0; s < kSub; ++s) {
      if constexpr (kF32) {
        // four sums side by side: one chain of D additions is what the result's error comes from
        f32x16 y[QT][4];
#pragma unroll
        for (int qt = 0; qt < QT; ++qt)
#pragma unroll
          for (int j = 0; j < 4; ++j) y[qt][j] = f32x16{};
#pragma unroll
        for (int u = 0; u < D / 8; ++u) {
          const f32x4 ko = lds_at<f32x4>((at ^ (u * 32)) + s * 32 * kRow);
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int qt = 0; qt < QT; ++qt)
              y[qt][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(ko[j], __uint_as_float(q.w[qt][u][j]), y[qt][j], 0, 0, 0);
        }
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) x[s][qt] = (y[qt][0] + y[qt][1]) + (y[qt][2] + y[qt][3]);
      } else {
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) x[s][qt] = f32x16{};
#pragma unroll
        for (int u = 0; u < D / 16; ++u) {
          const u32x4 ko = lds_at<u32x4>((at ^ (u * 32)) + s * 32 * kRow);
#pragma unroll
          for (int qt = 0; qt < QT; ++qt) x[s][qt] = mfma(ko, q.w[qt][u], x[s][qt]);
        }
      }
    }
  }

  // acc[qt] += p V of one subtile; vt: V in LDS, at the subtile
  static __device__ __forceinline__ void add_values(f32x16 (&acc)[QT][kDT], const f32x16 (&p)[QT], uint32_t vt, int lane) {
    if constexpr (kF32) {
      const int g = lane >> 5, l32 = lane & 31;
      const uint32_t at = vt + 4 * g * kRow + (uint32_t)((l32 / 4) ^ (g << 3)) * 16 + l32 % 4 * 4;
#pragma unroll
      for (int i = 0; i < 16; ++i)
#pragma unroll
        for (int dt = 0; dt < kDT; ++dt) {
          const float v = lds_at<float>((at ^ (uint32_t)((i & 3 | (i >> 2 & 1) << 2 | dt << 3) * 16)) + (i / 4 * 8 + i % 4) * kRow);
#pragma unroll
          for (int qt = 0; qt < QT; ++qt) acc[qt][dt] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, p[qt][i], acc[qt][dt], 0, 0, 0);
        }
    } else {
      // lane i of 16 reads the piece i % 4, of 8 bytes, of row i / 4: of the rows 4 g .. 4 g + 3 and, with j2, 8 rows on; 16 dims to 16 lanes
      const int g = lane >> 5, h = lane >> 4 & 1, i4 = lane >> 2 & 3, i1 = lane >> 1 & 1;
      const int row = 4 * g + i4;
      const uint32_t at = vt + row * kRow + (uint32_t)((2 * h + i1) ^ swizzle(row)) * 16 + (lane & 1) * 8;
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        u32x4 po[QT];
#pragma unroll
        for (int qt = 0; qt < QT; ++qt)
#pragma unroll
          for (int j = 0; j < 4; ++j) po[qt][j] = pair(p[qt][c * 8 + j * 2], p[qt][c * 8 + j * 2 + 1]);
#pragma unroll
        for (int dt = 0; dt < kDT; ++dt) {
          u32x4 vo;
#pragma unroll
          for (int j2 = 0; j2 < 2; ++j2) {
            // 8 rows on: swizzle changes bit 1
            const u32x2 t = read_turned((at ^ (uint32_t)(dt * 64 ^ j2 * 32)) + (c * 16 + j2 * 8) * kRow);
            vo[j2 * 2] = t[0];
            vo[j2 * 2 + 1] = t[1];
          }
#pragma unroll
          for (int qt = 0; qt < QT; ++qt) acc[qt][dt] = mfma(vo, po[qt], acc[qt][dt]);
        }
      }
    }
  }

  // whether some value of the subtile's 32 rows is not finite
  static __device__ __forceinline__ bool any_not_finite(uint32_t vt, int lane) {
    bool bad = false;
#pragma unroll
    for (int i = 0; i < 32 * kChunks / kWave; ++i) {
      const u32x4 x = lds_at<u32x4>(vt + (i * kWave + lane) * 16);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if constexpr (kF32) {
          bad |= (x[j] & 0x7f800000u) == 0x7f800000u;
        } else {
          constexpr uint32_t kExp = KIND == SLKV_F16 ? 0x7c00u : 0x7f80u;
          bad |= (x[j] & kExp) == kExp || (x[j] >> 16 & kExp) == kExp;
        }
      }
    }
    return __ballot(bad) != 0;
  }
};

// Whether nothing is seen by token t.  (A tree's token that sees nothing of the draft sees what is before it.)
__device__ __forceinline__ uint64_t bits_of(const TileWork& w, int t, int T) {
  return w.sees ? w.sees[t] & (T < 64 ? (1ull << T) - 1 : ~0ull) : 0ull;
}
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
__device__ __forceinline__ f32x4 tile_output(f32x4 o, float total, bool none) {
  const float inv = 1.f / total;
#pragma unroll
  for (int e = 0; e < 4; ++e) o[e] = none ? 0.f : total > 0.f ? o[e] * inv : NAN;
  return o;
}

template <int KIND, int D, int QT, int WQ, int WK, class TAB>
__global__ __launch_bounds__(WQ* WK* kWave, QT == 1 && WK < 4 && KIND != SLKV_F32 ? 2 : 1) void attend_tiles_kernel(const TileArgs a, const TAB tab) {
  using A = Tiles<KIND, D, QT, WQ, WK>;
  constexpr int kSub = A::kSub, kDT = A::kDT;
  __shared__ __align__(1024) unsigned char sh[A::kLds];
  __shared__ float sh_m[WK][32 * WQ], sh_l[WK][32 * WQ];
  const TileWork w = tab.template find<A::kQueries, A::kKeys, D, KIND>(a, (int)blockIdx.x);
  if (w.part >= w.parts) return;
  const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)sh;
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave));
  const int l32 = lane & 31, g = lane >> 5, wq = wave % WQ, wk = wave / WQ;
  const int t0 = w.r0 / a.G, rem0 = w.r0 % a.G;        // token and head of the tile's first row
  const int first = wq * 32 * QT;                      // the wave's first row of the tile
  const bool busy = w.r0 + first < w.rows;             // (waves without queries only stage)

  typename A::Queries q;
  int t_of[QT];
  uint64_t bits[QT];
#pragma unroll
  for (int qt = 0; qt < QT; ++qt) {
    const int r = min(first + qt * 32 + l32, w.rows - 1 - w.r0);
    const int dt = divide(rem0 + max(r, 0), a.G), head = rem0 + max(r, 0) - dt * a.G;
    t_of[qt] = t0 + dt;
    bits[qt] = bits_of(w, t_of[qt], a.T);
    const unsigned char* p = w.q + t_of[qt] * w.q_tok + head * w.q_head;
#pragma unroll
    for (int u = 0; u < (A::kF32 ? D / 8 : D / 16); ++u) q.w[qt][u] = *(const u32x4*)(p + u * 32 + g * 16);
  }

  float ref[QT], sum[QT];
  f32x16 acc[QT][kDT];
#pragma unroll
  for (int qt = 0; qt < QT; ++qt) {
    ref[qt] = -INFINITY;
    sum[qt] = 0.f;
#pragma unroll
    for (int dt = 0; dt < kDT; ++dt) acc[qt][dt] = f32x16{};
  }
  // keys that every query of the tile sees
  const int all = w.sees ? w.hist : w.hist + t0 + 1;
  // bit j: the lane's query sees the key key0 + j, which is there
  auto seen = [&](int qt, int key0) __attribute__((always_inline)) {
    uint32_t m = first_bits((w.sees ? w.hist : w.hist + t_of[qt] + 1) - key0);
    if (w.sees) {
      const int u = key0 - w.hist;                     // the draft's first row is bit -u
      m |= u >= 64 || u <= -32 ? 0u : u >= 0 ? (uint32_t)(bits[qt] >> u) : (uint32_t)bits[qt] << -u;
    }
    return m & first_bits(w.end - key0);
  };

  auto step = [&](int key0, uint32_t buf) __attribute__((always_inline)) {
    const uint32_t kt = buf + wk * 32 * kSub * A::kRow, vt = kt + A::kTileBytes;
    const int mine = key0 + wk * 32 * kSub;
    f32x16 x[kSub][QT];
    A::logits(x, q, kt, l32, g);
    const bool tail = key0 + A::kKeys > all;
    if (tail) {
#pragma unroll
      for (int s = 0; s < kSub; ++s)
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) {
          const uint32_t m = seen(qt, mine + s * 32) >> (4 * g);
#pragma unroll
          for (int i = 0; i < 16; ++i) x[s][qt][i] = m & 1u << (i / 4 * 8 + i % 4) ? x[s][qt][i] : -INFINITY;
        }
    }
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
      float top = -INFINITY;
#pragma unroll
      for (int s = 0; s < kSub; ++s)
#pragma unroll
        for (int i = 0; i < 16; ++i) top = fmaxf(top, x[s][qt][i]);
      top *= a.c_log2;
      if (__ballot(top > ref[qt] + A::kAbove)) {
        top = fmaxf(top, __shfl_xor(top, 32));
        const float now = fmaxf(ref[qt], top - A::kBelow);
        const float f = ref[qt] == -INFINITY ? 0.f : exp2_fast(ref[qt] - now);
        // (sums of a NaN stay one)
        sum[qt] *= f;
#pragma unroll
        for (int dt = 0; dt < kDT; ++dt) acc[qt][dt] *= f;
        ref[qt] = now;
      }
      // (one rounding, of the difference: a large product's own would be an error of the weight)
      const float from = ref[qt] == -INFINITY ? 0.f : ref[qt];
#pragma unroll
      for (int s = 0; s < kSub; ++s)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          x[s][qt][i] = exp2_fast(fmaf(x[s][qt][i], a.c_log2, -from));
          sum[qt] += x[s][qt][i];
        }
    }
#pragma unroll
    for (int s = 0; s < kSub; ++s) {
      const uint32_t vs = vt + s * 32 * A::kRow;
      if (tail && A::any_not_finite(vs, lane)) {
        // a row at a time, to the queries that see it: an infinity or NaN reaches no other through a weight of 0
        uint32_t m[QT];
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) m[qt] = seen(qt, mine + s * 32);
        for (int row = 0; row < 32; ++row) {
#pragma unroll
          for (int qt = 0; qt < QT; ++qt) {
            float p = 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i)
              if (i == row / 8 * 4 + row % 4) p = x[s][qt][i];
            p = __shfl(p, (row / 4 & 1) * 32 + l32);
            if (m[qt] >> row & 1) {
#pragma unroll
              for (int dt = 0; dt < kDT; ++dt)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[qt][dt][i] += p * A::value(vs, row, dt * 32 + i / 4 * 8 + 4 * g + i % 4);
            }
          }
        }
      } else {
        A::add_values(acc, x[s], vs, lane);
      }
    }
  };

  uint32_t buf = lds, other = lds + 2 * A::kTileBytes;
  if constexpr (A::kNarrow) {
    typename A::Fetched f;
    if (w.begin < w.end) {
      A::fetch(f, w, w.begin, w.end);
      A::put(f, buf);
    }
    for (int key0 = w.begin; key0 < w.end; key0 += A::kKeys) {
      const bool more = key0 + A::kKeys < w.end;
      if (more) A::fetch(f, w, key0 + A::kKeys, w.end);
      __syncthreads();
      if (busy) step(key0, buf);
      if (more) A::put(f, other);
      const uint32_t t = buf;
      buf = other;
      other = t;
    }
  } else {
    if (w.begin < w.end) A::stage(w, w.begin, w.end, buf);
    for (int key0 = w.begin; key0 < w.end; key0 += A::kKeys) {
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __syncthreads();
      if (key0 + A::kKeys < w.end) A::stage(w, key0 + A::kKeys, w.end, other);
      if (busy) step(key0, buf);
      const uint32_t t = buf;
      buf = other;
      other = t;
    }
  }

  // The waves that share queries are put together, and the outputs turned round, through LDS.
  const bool whole = w.parts == 1;
  const int slot = w.slot0 + w.part * w.slot_step;
  float* const sh_o = (float*)sh;
#pragma unroll
  for (int qt = 0; qt < QT; ++qt) {
    const float total = sum[qt] + __shfl_xor(sum[qt], 32);
    __syncthreads();                                   // (the last tile, or the tile of queries before, has been read)
    if (g == 0) {
      sh_m[wk][wq * 32 + l32] = ref[qt];
      sh_l[wk][wq * 32 + l32] = total;
    }
    if constexpr (WK > 1) __syncthreads();
    float f = 1.f;
    if constexpr (WK > 1) {
      float top = -INFINITY;
#pragma unroll
      for (int i = 0; i < WK; ++i) top = fmaxf(top, sh_m[i][wq * 32 + l32]);
      // (a wave that saw nothing has a sum of 0, or NaN where a product was NaN)
      f = ref[qt] == -INFINITY ? 1.f : exp2_fast(ref[qt] - top);
    }
#pragma unroll
    for (int dt = 0; dt < kDT; ++dt)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *(f32x4*)&sh_o[((wk * WQ + wq) * 32 + l32) * A::kOutRow + dt * 32 + i * 8 + 4 * g] =
            f32x4{acc[qt][dt][i * 4], acc[qt][dt][i * 4 + 1], acc[qt][dt][i * 4 + 2], acc[qt][dt][i * 4 + 3]} * f;
    __syncthreads();
    constexpr int kLanes = D / 4;                      // threads of a row of outputs
    for (int idx = threadIdx.x; idx < 32 * WQ * kLanes; idx += A::kThreads) {
      const int row = idx / kLanes, d0 = idx % kLanes * 4;
      const int r = row / 32 * 32 * QT + qt * 32 + row % 32;          // row of the tile
      if (w.r0 + r >= w.rows) continue;
      f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
      float top = -INFINITY, l = 0.f;
#pragma unroll
      for (int i = 0; i < WK; ++i) {
        o += *(const f32x4*)&sh_o[(i * WQ * 32 + row) * A::kOutRow + d0];
        top = fmaxf(top, sh_m[i][row]);
      }
#pragma unroll
      for (int i = 0; i < WK; ++i) l += sh_l[i][row] * (WK == 1 || sh_m[i][row] == -INFINITY ? 1.f : exp2_fast(sh_m[i][row] - top));
      if (whole) {
        const int dt = divide(rem0 + r, a.G), head = rem0 + r - dt * a.G, t = t0 + dt;
        const bool none = sees_none(w, t, bits_of(w, t, a.T));
        store_out<KIND>(w.out + t * w.o_tok + head * w.o_head + d0 * (int)sizeof(typename A::wide), tile_output(o, l, none));
        if (w.lse && d0 == 0) w.lse[head * w.lse_head + t] = tile_lse<A>(top, l, none);
      } else {
        *(f32x4*)(a.part_o + ((int64_t)slot * A::kQueries + r) * D + d0) = o;
        if (d0 == 0) *(f32x2*)(a.part_ml + ((int64_t)slot * A::kQueries + r) * 2) = f32x2{top, l};
      }
    }
  }
}

// The parts of a tile put together, in their order.  The workgroup of part p takes every parts'th group of rows.
template <int KIND, int D, int QT, int WQ, int WK, class TAB>
__global__ __launch_bounds__(256) void join_tiles_kernel(const TileArgs a, const TAB tab) {
  using A = Tiles<KIND, D, QT, WQ, WK>;
  const TileWork w = tab.template find<A::kQueries, A::kKeys, D, KIND>(a, (int)blockIdx.x);
  if (w.parts == 1 || w.part >= w.parts) return;
  constexpr int kLanes = D / 4, kRows = 256 / kLanes;
  const int t0 = w.r0 / a.G, rem0 = w.r0 % a.G, d0 = threadIdx.x % kLanes * 4;
  for (int r = w.part * kRows + threadIdx.x / kLanes; r < A::kQueries && w.r0 + r < w.rows; r += w.parts * kRows) {
    float top = -INFINITY, l = 0.f;
    f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int p = 0; p < w.parts; ++p) top = fmaxf(top, a.part_ml[((int64_t)(w.slot0 + p * w.slot_step) * A::kQueries + r) * 2]);
    for (int p = 0; p < w.parts; ++p) {
      const int64_t at = (int64_t)(w.slot0 + p * w.slot_step) * A::kQueries + r;
      const f32x2 ml = *(const f32x2*)(a.part_ml + at * 2);
      const float f = ml[0] == -INFINITY ? 1.f : exp2_fast(ml[0] - top);
      l += ml[1] * f;
      o += *(const f32x4*)(a.part_o + at * D + d0) * f;
    }
    const int dt = divide(rem0 + r, a.G), head = rem0 + r - dt * a.G, t = t0 + dt;
    const bool none = sees_none(w, t, bits_of(w, t, a.T));
    store_out<KIND>(w.out + t * w.o_tok + head * w.o_head + d0 * (int)sizeof(typename A::wide), tile_output(o, l, none));
    if (w.lse && d0 == 0) w.lse[head * w.lse_head + t] = tile_lse<A>(top, l, none);
  }
}

}  // namespace slkv
#endif
