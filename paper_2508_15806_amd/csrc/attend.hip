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

#include <cmath>

namespace slkv {

constexpr int kAttendThreads = 256;  // of the joining kernel
constexpr int kTileRows = 32;        // rows of a tile of stored logits, and what parts of a segment are a multiple of
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

constexpr int kJoinPairs = 4096;     // (part, query) pairs of a segment, at most: the joining kernel holds a number of each

// Segments of a launch: first row of their rooms.  A table of more than 64 says in which order the segments' parts are launched, and how many parts come before every
// 16th segment of that order.
template <int N>
struct AttendTab {
  static constexpr int kSegs = N;
  static constexpr int kGroup = 16;
  static constexpr bool kOrdered = N > 64;
  int32_t nseg, seg0, ordered;       // ordered 0: as they stand
  int32_t start[N + 1];
  int32_t before[kOrdered ? (N + kGroup - 1) / kGroup : 1];
  uint16_t order[kOrdered ? N : 1];
};
constexpr int kAttendSegs = 600;

struct AttendArgs {
  const unsigned char *k, *v, *k_scale, *v_scale, *q;
  unsigned char* out;
  const int32_t* lengths;
  float* lse;
  const float* w_in;
  float* w_out;
  float* part_o;                     // [part][R][D] sums of a part, relative to its reference
  float* part_ml;                    // [part][R][2] reference (log2), sum
  float* logits;                     // q . k: tiles of [R][32 rows]
  int32_t T, R;
  int32_t tiles_each;                // room of a part in tiles of 32 rows
  int32_t row0;                      // first row of the call's rooms; logits of segment s, row j: tile (start - row0) / 32 + s + j / 32
  float c_log2;                      // log2(e) / sqrt(d)
};

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// x / y for 0 <= x < 2^21, y > 0: (x + 1/2) / y is at least 1 / (2 y) from a whole number, and what reciprocal and product are off by, 2^-22 of it, is less.
__device__ __forceinline__ int divide(int x, int y) { return (int)(((float)x + 0.5f) * __builtin_amdgcn_rcpf((float)y)); }
// ceil(n / 32), at most 2^20: rooms have at most 2^25 rows.
__device__ __forceinline__ int tiles_of(int n) { return (n + kTileRows - 1) / kTileRows; }

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
  static __device__ __forceinline__ Rows rows_of(const AttendArgs& a, int64_t first, int rows) {
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

// A query's log-sum-exp in log2 units, +infinity where it sees no row (its weights come out 0), and what the caller gets.  The logarithm is taken of the sum without the
// 2^12 that fp16 weights carry: a number twice as large rounds twice as far (root mean square for 3000 rows: 14 to 17 times 2^-24 with them, 7 without).
template <class A>
__device__ __forceinline__ float lse_of(float top, float total, bool none) {
  return none ? INFINITY : total > 0.f ? (top + A::kBelow) + __builtin_amdgcn_logf(total * A::kBelowPower) : NAN;
}
__device__ __forceinline__ float lse_out(float lse2, bool none) { return none ? -INFINITY : lse2 * kLn2; }
__device__ __forceinline__ f32x4 output_of(f32x4 o, float total, bool none) {
  const float inv = 1.f / total;
#pragma unroll
  for (int e = 0; e < 4; ++e) o[e] = none ? 0.f : total > 0.f ? o[e] * inv : NAN;
  return o;
}

// Weights of rows j0 .. j1 - 1 of a segment (j0 a multiple of 32) from its logits, four rows a thread; SHARED: where rows are few and queries many, 1 << bits threads
// share the R queries (48 segments, 15 queries: the join 6.7 us -> 6.4; 8 segments, 64 queries: 14.2 -> 11.9).  lse: of the queries, in LDS.  The first numbers can
// be asked for before the log-sum-exp is known.  Logits of rows that a query does not see are -infinity and add 0, unless the query's log-sum-exp is NaN: sums that
// come out NaN where not every query sees the row are taken again from the queries that do.
constexpr int kAheadQueries = 4;
struct WeightsAhead { f32x4 x[kAheadQueries], w; };
template <int NT, bool SHARED>
struct Weights {
  const AttendArgs& a;
  const int64_t start;
  const int tile, j1, all;                             // the segment's first tile, end, rows that every query sees
  int bits = 0, sp = 0, first;                         // the thread's queries sp, sp + (1 << bits), .., its first row
  __device__ __forceinline__ Weights(const AttendArgs& args, int64_t start_row, int first_tile, int n, int j0, int end)
      : a(args), start(start_row), tile(first_tile), j1(end), all(n - args.T + 1) {
    if constexpr (SHARED) {
      while (bits < 4 && 4 * (NT >> (bits + 1)) >= j1 - j0 && (kAheadQueries << bits) < a.R) ++bits;
      sp = (int)threadIdx.x / (NT >> bits);
    }
    first = j0 + 4 * ((int)threadIdx.x & ((NT >> bits) - 1));
  }
  __device__ __forceinline__ const float* logits_of(int j) const { return a.logits + (int64_t)(tile + j / kTileRows) * a.R * kTileRows + j % kTileRows; }
  __device__ __forceinline__ void load(WeightsAhead& h, int j) const {
    if (j >= j1) return;
    const float* l = logits_of(j);
#pragma unroll
    for (int e = 0; e < 4; ++e) h.w[e] = sp == 0 && a.w_in && j + e < j1 ? a.w_in[start + j + e] : 0.f;
#pragma unroll
    for (int i = 0; i < kAheadQueries; ++i)
      if (sp + (i << bits) < a.R) h.x[i] = *(const f32x4*)(l + (sp + (i << bits)) * kTileRows);
  }
  __device__ __forceinline__ f32x4 sum(const WeightsAhead& h, int j, const float* lse) const {
    f32x4 s = f32x4{0.f, 0.f, 0.f, 0.f};
    auto one = [&](f32x4 x, float l) __attribute__((always_inline)) {
#pragma unroll
      for (int e = 0; e < 4; ++e) s[e] += exp2_fast(fmaf(x[e], a.c_log2, -l));
    };
#pragma unroll
    for (int i = 0; i < kAheadQueries; ++i)
      if (sp + (i << bits) < a.R) one(h.x[i], lse[sp + (i << bits)]);
    const float* l = logits_of(j);
#pragma unroll 8
    for (int r = sp + (kAheadQueries << bits); r < a.R; r += 1 << bits) one(*(const f32x4*)(l + r * kTileRows), lse[r]);
    const float any = (s[0] + s[1]) + (s[2] + s[3]);
    if (a.T > 1 && j + 3 >= all && any != any) {
      s = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
      for (int r = sp; r < a.R; r += 1 << bits) {
        const f32x4 x = *(const f32x4*)(l + r * kTileRows);
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (j + e < all + r % a.T) s[e] += exp2_fast(fmaf(x[e], a.c_log2, -lse[r]));
      }
    }
    return s + h.w;
  }
  __device__ __forceinline__ void store(f32x4 s, int j) const {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (j + e < j1) a.w_out[start + j + e] = s[e];
  }
  // h: loaded at `first`; shared: NT places
  __device__ __forceinline__ void add(WeightsAhead& h, const float* lse, f32x4* shared) const {
    if (!SHARED || bits == 0) {
      for (int j = first; j < j1; j += 4 * NT) {
        const f32x4 s = sum(h, j, lse);
        load(h, j + 4 * NT);
        store(s, j);
      }
      return;
    }
    f32x4 s = f32x4{0.f, 0.f, 0.f, 0.f};
    if (first < j1) shared[threadIdx.x] = s = sum(h, first, lse);
    __syncthreads();
    if (sp == 0 && first < j1) {
      for (int v = 1; v < 1 << bits; ++v) s += shared[v * (NT >> bits) + (int)threadIdx.x];
      store(s, first);
    }
  }
};

// The segment of a workgroup, which is a part of one: segments have max(1, ceil(room / rows_each)) parts.  One wave looks it up and reads the length for all: the
// table is read from the kernel's arguments, where a workgroup that goes through 3 KB of it with every wave waits up to 20 us behind the others (768 workgroups; this way 1 to 2).
struct Where { int seg, start, part, first, n, tile, each, active; };   // rows of a part; parts that have any: the rows in use are spread over the parts of the room
template <class TAB>
__device__ __forceinline__ Where find_part(const AttendArgs& a, const TAB& tab, Where& shared) {
  if (threadIdx.x < kWave) {
    const int lane = threadIdx.x, part_id = blockIdx.x;
    int s = lane, first0 = 0;
    bool in = lane < tab.nseg;
    if constexpr (TAB::kOrdered) {
      const int groups = (tab.nseg + TAB::kGroup - 1) / TAB::kGroup;
      const int b = tab.before[min(lane, groups - 1)];
      const int g = __popcll(__ballot(lane < groups && b <= part_id)) - 1;
      first0 = __builtin_amdgcn_readlane(b, g);
      in = lane < TAB::kGroup && g * TAB::kGroup + lane < tab.nseg;
      s = min(g * TAB::kGroup + lane, tab.nseg - 1);
      if (tab.ordered) s = tab.order[s];
    }
    s = min(s, tab.nseg - 1);
    const int in_use = a.lengths ? a.lengths[tab.seg0 + s] : 0, at = tab.start[s], room = tab.start[s + 1] - at;
    const int parts = in ? max(1, divide(tiles_of(room) + a.tiles_each - 1, a.tiles_each)) : 0;
    const int first = first0 + (int)wave_incl_scan((uint32_t)parts) - parts;
    if (parts && first <= part_id && part_id < first + parts) {
      Where w;
      w.seg = tab.seg0 + s;
      w.start = at;
      w.part = part_id - first;
      w.first = first;
      w.n = a.lengths ? min(max(in_use, 0), room) : room;
      w.tile = (at - a.row0) / kTileRows + w.seg;
      const int tiles = tiles_of(w.n), each = divide(tiles + parts - 1, parts);
      w.each = each * kTileRows;
      w.active = each ? divide(tiles + each - 1, each) : 0;
      shared = w;
    }
  }
  __syncthreads();
  Where w;
  w.seg = __builtin_amdgcn_readfirstlane(shared.seg);
  w.start = __builtin_amdgcn_readfirstlane(shared.start);
  w.part = __builtin_amdgcn_readfirstlane(shared.part);
  w.each = __builtin_amdgcn_readfirstlane(shared.each);
  w.active = __builtin_amdgcn_readfirstlane(shared.active);
  w.first = __builtin_amdgcn_readfirstlane(shared.first);
  w.n = __builtin_amdgcn_readfirstlane(shared.n);
  w.tile = __builtin_amdgcn_readfirstlane(shared.tile);
  return w;
}

// RT: tiles of 16 queries.
constexpr int attend_waves_per_cu(int rt) { return rt == 4 ? 4 : 8; }
template <int KIND, int D, int RT, int W, class TAB>
__global__ __launch_bounds__(W * kWave, attend_waves_per_cu(RT) / W) void attend_kernel(const AttendArgs a, const TAB tab) {
  using A = Attend<KIND, D>;
  constexpr int kProducts = A::kF32 ? D / 4 : D / 32, kVD = A::kVD, kEach = A::kEach;
  // The next step's rows are on their way during a step.  More tiles of queries leave no registers for them beside the careful step, the second copy of the step in
  // this kernel, which decides how many it takes: with D = 128 two tiles take 197 to 248 of 256 without rows ahead (168 to 244 if the careful step is compiled out, with rows
  // ahead 213 to 253, fp32 in scratch), and four tiles put 84 to 444 bytes a lane into scratch (none if it is).
  constexpr bool kAhead = RT * D <= 128;
  __shared__ __align__(16) float sh_o[W][16][D + 4];
  __shared__ float sh_m[W][16 * RT], sh_l[W][16 * RT];
  __shared__ float sh_lse[16 * RT], sh_total[16 * RT];
  __shared__ Where sh_at;
  const Where at = find_part(a, tab, sh_at);
  const int seg = at.seg, start = at.start, part = at.part, n = at.n;
  const int begin = part * at.each, end = min(n, begin + at.each);
  if (begin >= end && part > 0) return;
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave)), lane = threadIdx.x % kWave;
  const int rq = lane & 15, g = lane >> 4, R = a.R, T = a.T;
  const int64_t base = start;

  const typename A::Rows rows = A::rows_of(a, base + begin, end - begin);
  typename A::KRegs kr0, kr1;
  typename A::VRegs vr0, vr1;
  typename A::Place place = A::place_of(wave, lane);
  A::load_k(kr0, rows, place);
  A::load_v(vr0, rows, place);

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
  // Logits go through a buffer as well, of no bytes where nobody asks for weights, and at places beyond its end for queries that are not there, so that a step has no
  // branch for them.  (256 segments of 536 to 5994 E4M3 rows: 34.5 us with the logits, 29.1 without, of which the stores are 2.5 to 3, whole segments' weights 2.)
  const __amdgpu_buffer_rsrc_t logits = __builtin_amdgcn_make_buffer_rsrc(
      (void*)(a.logits ? a.logits + (int64_t)(at.tile + begin / kTileRows) * R * kTileRows : nullptr), 0, a.logits ? tiles_of(end - begin) * kTileRows * R * 4 : 0, 0x00027000);
  uint32_t logit_at[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) logit_at[rt] = rt * 16 + rq < R ? (rt * 16 + rq) * kTileRows * 4 + g * kEach * 4 : 0x80000000u;

  float ref[RT], sum[RT];
  f32x4 acc[RT][kVD];
  // The weights go into the products with the values as two 16-bit numbers each, which leaves 2^-16 of a weight (fp16: 2^-22, or 2^-25 of the reference; one number: 2^-9 of each, as much again as
  // the rounding of the output).  An infinite value would make NaN of the second one's zero, and values of rows that a query does not see would reach it through
  // a weight of zero: sums that come out not finite are taken again, with such values kept out of the second number's products and, where not every query
  // sees the row, out of both.
  auto step = [&](auto careful_c, const typename A::KRegs& kr, const typename A::VRegs& vr, const int key0) __attribute__((always_inline)) {
    constexpr bool careful = decltype(careful_c)::value;
    f32x4 x[RT][A::kTiles];
    if constexpr (A::kF32) {
      // several sums side by side: one chain of D/4 additions is what the result's error comes from
      constexpr int kChains = RT == 4 ? 2 : 4;
      f32x4 s[RT][kChains];
#pragma unroll
      for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int i = 0; i < kChains; ++i) s[rt][i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int u = 0; u < kProducts; ++u)
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
          s[rt][u % kChains] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kr.w[0][u]), qf[rt][u], s[rt][u % kChains], 0, 0, 0);
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        x[rt][0] = s[rt][0] + s[rt][1];
        if constexpr (kChains == 4) x[rt][0] += s[rt][2] + s[rt][3];
      }
    } else {
#pragma unroll
      for (int t = 0; t < A::kTiles; ++t) {
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) x[rt][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int u = 0; u < kProducts; ++u) {
          const u32x4 ko = A::k_operand(kr, t, u);
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) x[rt][t] = A::mfma(ko, q[rt][u], x[rt][t]);
        }
      }
    }
    const int mine = key0 + g * kEach;                 // the lane's rows: mine .. mine + kEach - 1
    const uint32_t logit_step = ((key0 - begin) / kTileRows * R * kTileRows + key0 % kTileRows) * 4;
    const bool tail = key0 + A::kStep > min(end, n - T + 1);
    float p[RT][kEach];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
#pragma unroll
      for (int j = 0; j < kEach; ++j) p[rt][j] = x[rt][j / 4][j % 4];
      if (tail) {
#pragma unroll
        for (int j = 0; j < kEach; ++j)
          if (mine + j >= sees[rt]) p[rt][j] = -INFINITY;
      }
      float top = -INFINITY;
#pragma unroll
      for (int j = 0; j < kEach; ++j) top = fmaxf(top, p[rt][j]);
      top *= a.c_log2;
#pragma unroll
      for (int j = 0; j < kEach; j += 4) {
        const f32x4 l = f32x4{p[rt][j], p[rt][j + 1], p[rt][j + 2], p[rt][j + 3]};
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, l), logits, logit_at[rt] + logit_step + j * 4, 0, 0);
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
      // (one rounding, of the difference: a large product's own would be an error of the weight)
      const float from = ref[rt] == -INFINITY ? 0.f : ref[rt];
#pragma unroll
      for (int j = 0; j < kEach; ++j) {
        p[rt][j] = exp2_fast(fmaf(p[rt][j], a.c_log2, -from));
        sum[rt] += p[rt][j];
      }
    }
    uint32_t hold = ~0u;                               // bit j: the lane's row j takes part in the products
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
      hold = mine >= from ? 0u : mine + kEach <= from ? ~0u : (1u << (from - mine)) - 1u;
    }
    if constexpr (A::kF32) {
#pragma unroll
      for (int m = 0; m < kVD; ++m)
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
          const float v = !careful || hold >> j & 1 ? __uint_as_float(vr.w[j][m]) : 0.f;
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) acc[rt][m] = __builtin_amdgcn_mfma_f32_16x16x4f32(v, p[rt][j], acc[rt][m], 0, 0, 0);
        }
    } else {
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
      auto product = [&](auto u_c) __attribute__((always_inline)) {
        constexpr int u = decltype(u_c)::value;
        uint32_t pair[kEach];
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
          pair[j] = A::template v_pair<u>(vr, j);
          if constexpr (careful) pair[j] = hold >> j & 1 ? pair[j] : 0u;
        }
#pragma unroll
        for (int m = 2 * u; m < 2 * u + 2; ++m) {
          u32x4 vo;
#pragma unroll
          for (int j = 0; j < 4; ++j) vo[j] = __builtin_amdgcn_perm(pair[2 * j + 1], pair[2 * j], m % 2 ? 0x07060302u : 0x05040100u);
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) acc[rt][m] = A::mfma(vo, hi[rt], acc[rt][m]);
          if constexpr (careful) vo = A::finite(vo);
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) acc[rt][m] = A::mfma(vo, lo[rt], acc[rt][m]);
        }
      };
      product(std::integral_constant<int, 0>{});
      product(std::integral_constant<int, 1>{});
      if constexpr (kVD == 8) {
        product(std::integral_constant<int, 2>{});
        product(std::integral_constant<int, 3>{});
      }
    }
  };
  auto clear = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      ref[rt] = -INFINITY;
      sum[rt] = 0.f;
#pragma unroll
      for (int m = 0; m < kVD; ++m) acc[rt][m] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
  };
  using std::integral_constant;
  constexpr int kStride = W * A::kStep;
  clear();
  if constexpr (kAhead) {
    for (int key0 = begin + wave * A::kStep; key0 < end; key0 += kStride) {
      A::advance(place, W);                 // (beyond the end nothing is fetched)
      A::load_k(kr1, rows, place);
      A::load_v(vr1, rows, place);
      step(integral_constant<bool, false>{}, kr0, vr0, key0);
      key0 += kStride;
      if (key0 >= end) break;
      A::advance(place, W);
      A::load_k(kr0, rows, place);
      A::load_v(vr0, rows, place);
      step(integral_constant<bool, false>{}, kr1, vr1, key0);
    }
  } else {
    for (int key0 = begin + wave * A::kStep; key0 < end; key0 += kStride) {
      step(integral_constant<bool, false>{}, kr0, vr0, key0);
      A::advance(place, W);
      A::load_k(kr0, rows, place);
      A::load_v(vr0, rows, place);
    }
  }
  float zero[4] = {0.f, 0.f, 0.f, 0.f};                // NaN where a sum is not finite
#pragma unroll
  for (int rt = 0; rt < RT; ++rt)
#pragma unroll
    for (int m = 0; m < kVD; ++m)
#pragma unroll
      for (int e = 0; e < 4; ++e) zero[e] = fmaf(acc[rt][m][e], 0.f, zero[e]);
  if (__ballot((zero[0] + zero[1]) + (zero[2] + zero[3]) != 0.f)) {
    clear();
    place = A::place_of(wave, lane);
    for (int key0 = begin + wave * A::kStep; key0 < end; key0 += kStride) {
      A::load_k(kr0, rows, place);
      A::load_v(vr0, rows, place);
      step(integral_constant<bool, true>{}, kr0, vr0, key0);
      A::advance(place, W);
    }
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
  const bool whole = at.active <= 1;
  float* const ml = a.part_ml + (int64_t)blockIdx.x * 2 * R;
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    float top = -INFINITY, total = 0.f, mine = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w) top = fmaxf(top, sh_m[w][rt * 16 + rq]);
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const float m = sh_m[w][rt * 16 + rq], l = sh_l[w][rt * 16 + rq];
      // (a wave that saw nothing has a sum of 0, or NaN where a product was NaN)
      const float f = m == -INFINITY ? 1.f : exp2_fast(m - top);
      total += l * f;
      if (w == wave) mine = f;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int m = 0; m < kVD; m += 4)
        *(f32x4*)&sh_o[wave][rq][(g * 4 + e) * kVD + m] = f32x4{acc[rt][m][e], acc[rt][m + 1][e], acc[rt][m + 2][e], acc[rt][m + 3][e]} * mine;
    const int r = rt * 16 + rq;
    if (wave == 0 && g == 0 && r < R) {
      const bool none = n - T + 1 + r % T <= 0;
      sh_total[r] = total;
      if (whole) {
        const float lse2 = lse_of<A>(top, total, none);
        sh_lse[r] = lse2;
        if (a.lse) a.lse[(int64_t)seg * R + r] = lse_out(lse2, none);
      } else {
        *(f32x2*)(ml + 2 * r) = f32x2{top, total};
      }
    }
    __syncthreads();
    for (int idx = threadIdx.x; idx < 16 * D / 4; idx += (W * kWave)) {
      const int r16 = idx / (D / 4), d0 = idx % (D / 4) * 4, row = rt * 16 + r16;
      if (row >= R) continue;
      f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < W; ++w) o += *(const f32x4*)&sh_o[w][r16][d0];
      if (whole) {
        store_out<KIND>(a.out + (((int64_t)seg * R + row) * D + d0) * (int)sizeof(typename A::wide), output_of(o, sh_total[row], n - T + 1 + row % T <= 0));
      } else {
        *(f32x4*)(a.part_o + ((int64_t)blockIdx.x * R + row) * D + d0) = o;
      }
    }
    __syncthreads();
  }
  if (!whole || !a.w_out) return;
  __threadfence_block();
  __syncthreads();
  const Weights<W * kWave, false> weights(a, base, at.tile, n, 0, n);
  WeightsAhead h;
  weights.load(h, weights.first);
  weights.add(h, sh_lse, nullptr);
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

// Segments of more than one part: the parts put together, in their order.  The workgroup of part p of a segment adds up the references and sums of its R queries over
// all parts, 256 / R lanes a query, 4 to 64, and finishes every active'th group of 64 to 512 outputs and the weights of the part's rows.  What it reads is asked for at once: behind
// the table and the length there is one round trip.  Bound by latency, of the instructions too.  (Two other ways were measured.  The workgroups of a segment waiting for
// each other in the launch above: 40 us instead of 34 for one long history, whose memory traffic their meeting competes with, nothing gained elsewhere; the last one to
// arrive joining the segment alone: 25 to 40 % slower.)
template <int KIND, int D, int UNITS, class TAB>
__global__ __launch_bounds__(kAttendThreads) void attend_join_kernel(const AttendArgs a, const TAB tab) {
  __shared__ Where sh_at;
  __shared__ float sh_lse[64], sh_total[64], sh_factor[kJoinPairs], sh_sum[kJoinPairs];   // [part][query] (sh_factor: references at first)
  __shared__ f32x4 sh_o[UNITS][kAttendThreads / kWave][16], sh_w[kAttendThreads];
  const Where w = find_part(a, tab, sh_at);
  const int n = w.n, part = w.part, active = w.active;
  if (active <= 1 || part >= active) return;
  const int R = a.R, T = a.T, tid = threadIdx.x;
  const float* ml = a.part_ml + (int64_t)w.first * 2 * R;
  const float* po = a.part_o + (int64_t)w.first * R * D;
  // the queries: 1 << bits lanes each, a lane per part
  const int bits = R <= 4 ? 6 : R <= 8 ? 5 : R <= 16 ? 4 : R <= 32 ? 3 : 2, share = 1 << bits;
  const int r = tid >> bits, lane = tid & (share - 1);
  // (more parts than lanes: through LDS, so that all are asked for at once; the same case 15.5 us -> 14.7)
  const bool staged = active > share;
  f32x2 pair = f32x2{-INFINITY, 0.f};
  if (staged) {
    for (int i0 = tid; i0 < active * R; i0 += 8 * kAttendThreads) {
      f32x2 t[8];
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i0 + i * kAttendThreads < active * R) t[i] = *(const f32x2*)(ml + 2 * (i0 + i * kAttendThreads));
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i0 + i * kAttendThreads < active * R) sh_factor[i0 + i * kAttendThreads] = t[i][0], sh_sum[i0 + i * kAttendThreads] = t[i][1];
    }
  } else if (r < R && lane < active) {
    pair = *(const f32x2*)(ml + 2 * (lane * R + r));
  }
  // the outputs, in units of 64: 16 threads take four each, `groups` of these the parts, 2 to 16, and what is left other units, UNITS of them at a time
  // (64 queries, 32 segments of 4000 rows on average, 128 units a segment: 12.4 us with four; 16.5 with one; 14.7 with 16, whose code has to be fetched too)
  const int groups = active <= 2 ? 2 : active <= 4 ? 4 : active <= 8 ? 8 : 16, grp_bits = active <= 2 ? 1 : active <= 4 ? 2 : active <= 8 ? 3 : 4;
  const int units = R * (D / 64), f = tid & 15, grp = (tid >> 4) & (groups - 1), at_once = 16 >> grp_bits, sub = tid >> (4 + grp_bits);
  f32x4 x[UNITS];
  int first = part * at_once;
  auto unit_of = [&](int i) __attribute__((always_inline)) { return first + i * active * at_once + sub; };
  auto load_units = [&](int p) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < UNITS; ++i)
      if (unit_of(i) < units && p < active) x[i] = *(const f32x4*)(po + (int64_t)p * R * D + unit_of(i) * 64 + f * 4);
  };
  load_units(grp);
  const int end = min(n, (part + 1) * w.each);
  const Weights<kAttendThreads, true> weights(a, w.start, w.tile, n, part * w.each, end);
  WeightsAhead h;
  if (a.w_out) weights.load(h, weights.first);

  auto factor_of = [](float m, float top) __attribute__((always_inline)) { return m == -INFINITY ? 1.f : exp2_fast(m - top); };
  float top = pair[0], total = 0.f;
  if (staged) {
    __syncthreads();
    if (r < R)
      for (int p = lane; p < active; p += share) top = fmaxf(top, sh_factor[p * R + r]);
  }
  top = reduce_lanes(top, share, [](float u, float v) { return fmaxf(u, v); });
  if (r < R)
    for (int p = lane; p < active; p += share) {
      if (staged) pair = f32x2{sh_factor[p * R + r], sh_sum[p * R + r]};
      const float s = factor_of(pair[0], top);
      sh_factor[p * R + r] = s;
      total += pair[1] * s;
    }
  total = reduce_lanes(total, share, [](float u, float v) { return u + v; });
  if (r < R && lane == 0) {
    const bool none = n - T + 1 + r % T <= 0;
    const float lse2 = lse_of<Attend<KIND, D>>(top, total, none);
    sh_total[r] = total;
    sh_lse[r] = lse2;
    if (part == 0 && a.lse) a.lse[(int64_t)w.seg * R + r] = lse_out(lse2, none);
  }
  __syncthreads();
  while (true) {
    f32x4 o[UNITS];
#pragma unroll
    for (int i = 0; i < UNITS; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int p = grp; p < active; p += groups) {
#pragma unroll
      for (int i = 0; i < UNITS; ++i)
        if (unit_of(i) < units) o[i] += x[i] * sh_factor[p * R + unit_of(i) / (D / 64)];
      load_units(p + groups);
    }
#pragma unroll
    for (int i = 0; i < UNITS; ++i) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        o[i][e] += __shfl_xor(o[i][e], 16);
        if (groups > 2) o[i][e] += __shfl_xor(o[i][e], 32);
      }
      if (groups > 4 && (tid & (kWave - 1)) < 16) sh_o[i][tid / kWave][f] = o[i];
    }
    if (groups > 4) __syncthreads();
#pragma unroll
    for (int i = 0; i < UNITS; ++i) {
      if (grp != 0 || unit_of(i) >= units) continue;
      if (groups > 4)
        for (int v = 1; v < groups / 4; ++v) o[i] += sh_o[i][tid / kWave + v][f];
      const int row = unit_of(i) / (D / 64);
      store_out<KIND>(a.out + ((int64_t)w.seg * R * D + unit_of(i) * 64 + f * 4) * (int)sizeof(typename Kind<KIND>::wide),
                      output_of(o[i], sh_total[row], n - T + 1 + row % T <= 0));
    }
    first += UNITS * active * at_once;
    if (first >= units) break;
    __syncthreads();
    load_units(grp);
  }
  if (a.w_out) weights.add(h, sh_lse, sh_w);
}

// ------------------------------------------------------------------ host

struct AttendPlan {
  int64_t rows_each;                 // room rows of a part, at most: a multiple of 32
  int64_t parts;                     // of a launch, the most
  bool split;                        // some segment has more than one part
  int waves;                         // of a workgroup
  size_t off_ml, off_o, off_logits, bytes;
};

static int64_t parts_of(const slkv_cache_desc* d, int64_t s, int64_t rows_each) {
  const uint32_t room = (uint32_t)(d->h_offsets[s + 1] - d->h_offsets[s]);
  return std::max<uint32_t>(1u, (room + (uint32_t)rows_each - 1) / (uint32_t)rows_each);
}

static AttendPlan plan_attend(const slkv_cache_desc* d, int T, bool weights) {
  AttendPlan p;
  const int64_t S = (int64_t)d->B * d->Hkv, rows = d->h_offsets[S] - d->h_offsets[0];
  const int64_t R = (int64_t)(d->Hq / d->Hkv) * T;
  constexpr int64_t kMost = 1 << 21;                   // a part's bytes are a 32-bit number
  auto round = [](int64_t n) { return (n + kTileRows - 1) / kTileRows * kTileRows; };
  const double row_bytes = d->d * kind_bits(d->dtype) / 4;
  const int rt = R <= 16 ? 1 : R <= 32 ? 2 : 4;
  int64_t most = 0;
  for (int64_t s = 0; s < S; ++s) most = std::max(most, d->h_offsets[s + 1] - d->h_offsets[s]);
  // Eight waves a workgroup where segments are few and long: half as many parts to join (8 segments of 4224 rows 14.3 us, of 32 K 32.2; four waves 15.4, 32.3).  Four
  // otherwise: two workgroups on a CU fill each other's beginnings and ends (128 segments of 270 to 3012 rows 22.9 us, 256 of E4M3 43.8; eight waves 23.5, 50.6).
  p.waves = rt == 1 && S <= 64 && rows >= 32768 ? 8 : 4;
  const int64_t places = 256 * attend_waves_per_cu(rt) / p.waves;
  // Whole segments while the longest is done, beside the others, before parts and the second launch that joins them would be.  One workgroup: 10.2 ns a row of 512
  // bytes, 4.9 of MXFP4 (128 bytes, which leave its exponents out, as all of this rule's do), and 0.4 of the time that the chip takes for all rows at 5 TB/s, which it shares with the others; the second launch: 5 us.  (Whole, from 65 segments on the longest first, and in parts, which are launched as they stand, us: 8 segments of 96 to
  // 440 rows 10.2, 12.8; 8 of 1016 rows of 512 bytes 15.3, 12.5; 512 of 280 to 2189 rows of MXFP4 23.5, 32.7; 256 of up to 3140 rows of 512 bytes 54.0, 40.4; 512 of up to 3140 of
  // 256 bytes 45.0, 46.6; 256 of up to 3140 of MXFP4 25.6, 20.9.)
  const double whole_us = most * (0.0035 * rt + row_bytes / 75e3), split_us = rows * row_bytes / 5e6 * 0.6 + 5;
  if (most <= kMost && whole_us <= split_us) {
    p.rows_each = std::max<int64_t>(kTileRows, round(most));
  } else {
    // The workgroups that are on the chip at once share the rows.  Segments end inside a part, so a part is made larger until all are on the chip.
    const int64_t least = std::max<int64_t>(p.waves * 32, round(most / (kJoinPairs / R) + 1));
    p.rows_each = std::min(kMost, std::max<int64_t>(least, round((rows + places - 1) / places)));
    for (int tries = 0; tries < 4 && S <= places / 4 * 3 && p.rows_each < kMost; ++tries) {
      int64_t parts = 0;
      for (int64_t s = 0; s < S; ++s) parts += parts_of(d, s, p.rows_each);
      if (parts <= places) break;
      p.rows_each = std::min(kMost, std::max(p.rows_each + kTileRows, round(p.rows_each * parts / (places + S / 4))));
    }
  }
  p.parts = 0;
  p.split = most > p.rows_each;
  for (int64_t s0 = 0; s0 < S; s0 += kAttendSegs) {
    int64_t here = 0;
    for (int64_t s = s0; s < std::min<int64_t>(S, s0 + kAttendSegs); ++s) here += parts_of(d, s, p.rows_each);
    p.parts = std::max(p.parts, here);
  }
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

// The order in which a launch's whole segments begin: the longest first, by sixteenths of the longest.  Heads of unequal capacity come at the same places in every
// sequence, so that in their own order long ones meet on a CU: 64 sequences of 8 heads with 270 to 2061 rows 31.0 us, sorted 25.0; 128 of shorter ones 130 and 87.
template <class TAB>
static void order_segments(TAB& tab, const AttendPlan& p) {
  constexpr int kSteps = 16;
  int from[kSteps + 1] = {};
  uint8_t key[TAB::kSegs];
  for (int i = 0; i < tab.nseg; ++i) {
    key[i] = (uint8_t)(kSteps - 1 - (tab.start[i + 1] - tab.start[i]) * (int64_t)(kSteps - 1) / p.rows_each);
    ++from[key[i] + 1];
  }
  for (int k = 0; k < kSteps; ++k) from[k + 1] += from[k];
  for (int i = 0; i < tab.nseg; ++i) tab.order[from[key[i]]++] = (uint16_t)i;
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

  a.tiles_each = (int32_t)(p.rows_each / kTileRows);
  auto launch = [&](auto tab, int64_t s0, int64_t ns) {
    using TAB = decltype(tab);
    tab.nseg = (int32_t)ns;
    tab.seg0 = (int32_t)s0;
    for (int64_t i = 0; i <= ns; ++i) tab.start[i] = (int32_t)desc->h_offsets[s0 + i];
    int64_t parts = 0;
    if constexpr (TAB::kOrdered) {
      tab.ordered = !p.split;
      if (tab.ordered) order_segments(tab, p);
      for (int64_t i = 0; i < ns; ++i) {
        if (i % TAB::kGroup == 0) tab.before[i / TAB::kGroup] = (int32_t)parts;
        parts += p.split ? parts_of(desc, s0 + i, p.rows_each) : 1;
      }
    } else {
      for (int64_t i = 0; i < ns; ++i) parts += parts_of(desc, s0 + i, p.rows_each);
    }
    const dim3 grid((unsigned)parts);
    with_kind(desc->dtype, [&](auto kind) {
      auto with_dim = [&](auto dim) {
        constexpr int kKind = decltype(kind)::value, kDim = decltype(dim)::value;
        {
          ScopedKernelTimer timer(SLKV_K_ATTEND);
          if (a.R <= 16 && p.waves == 8) SLKV_LAUNCH((attend_kernel<kKind, kDim, 1, 8, TAB>), grid, dim3(8 * kWave), 0, stream, a, tab);
          else if (a.R <= 16) SLKV_LAUNCH((attend_kernel<kKind, kDim, 1, 4, TAB>), grid, dim3(4 * kWave), 0, stream, a, tab);
          else if (a.R <= 32) SLKV_LAUNCH((attend_kernel<kKind, kDim, 2, 4, TAB>), grid, dim3(4 * kWave), 0, stream, a, tab);
          else SLKV_LAUNCH((attend_kernel<kKind, kDim, 4, 4, TAB>), grid, dim3(4 * kWave), 0, stream, a, tab);
        }
        if (p.split) {
          ScopedKernelTimer timer(SLKV_K_ATTEND_JOIN);
          // a workgroup has R d / 64 units of outputs, divided by 9 to 17 (or the parts, if they are more)
          if (a.R * (kDim / 64) <= 9) SLKV_LAUNCH((attend_join_kernel<kKind, kDim, 1, TAB>), grid, dim3(kAttendThreads), 0, stream, a, tab);
          else SLKV_LAUNCH((attend_join_kernel<kKind, kDim, 4, TAB>), grid, dim3(kAttendThreads), 0, stream, a, tab);
        }
      };
      if (desc->d == 64) with_dim(std::integral_constant<int, 64>{});
      else with_dim(std::integral_constant<int, 128>{});
    });
  };
  if (S <= kFewSegs) launch(AttendTab<kFewSegs>{}, 0, S);
  else
    for (int64_t s0 = 0; s0 < S; s0 += kAttendSegs) launch(AttendTab<kAttendSegs>{}, s0, std::min<int64_t>(kAttendSegs, S - s0));
  return launch_status("attend");
}
