// Rows into and out of a cache (slkv_fill_cache, slkv_append_cache, slkv_cache_rows) and eviction by accumulated attention weight (slkv_evict_cache).
#include "cache.h"
#include "device_utils.h"
#include "launch.h"

namespace slkv {

struct CacheArrays {
  unsigned char *k, *v, *k_scale, *v_scale;
  int32_t* lengths;
  int32_t* pos;
  float* weight;
};

static CacheArrays arrays_of(const slkv_cache* c) {
  CacheArrays a;
  a.k = (unsigned char*)c->d_k;
  a.v = (unsigned char*)c->d_v;
  a.k_scale = (unsigned char*)c->d_k_scale;
  a.v_scale = (unsigned char*)c->d_v_scale;
  a.lengths = c->d_lengths;
  a.pos = c->d_pos;
  a.weight = c->d_weight;
  return a;
}

// ------------------------------------------------------------------ conversions, a unit of 8 elements a lane

struct Unit { u32x4 lo, hi; };       // 8 wide elements: 16 bytes in lo, or 32 (fp32)

// Rows that are read once and in whole lines are loaded past the caches' order of use: 131072 rows of bf16 into a cache 30.7 -> 25.1 us, eviction from 16
// conversations 37.0 -> 31.6; loads of 4 bytes (rows of MXFP4) are slower this way, 17.4 -> 22.0, and stores gain 3 % or nothing.

template <int KIND>
__device__ __forceinline__ Unit load_unit(const unsigned char* row, int unit) {
  Unit u;
  constexpr int kBytes = 8 * (int)sizeof(typename Kind<KIND>::wide);
  u.lo = __builtin_nontemporal_load((const u32x4*)(row + unit * kBytes));
  if constexpr (kBytes == 32) u.hi = __builtin_nontemporal_load((const u32x4*)(row + unit * kBytes + 16));
  return u;
}

// Largest of four neighbouring lanes.
__device__ __forceinline__ uint32_t quad_max(uint32_t v) {
  v = max(v, dpp_move<0xb1>(0u, v));     // quad_perm 1, 0, 3, 2
  return max(v, dpp_move<0x4e>(0u, v));  // quad_perm 2, 3, 0, 1
}

// One unit of a row into the cache.  All four lanes of a quad hold neighbouring units of the same row (or none does).
template <int KIND, int D>
__device__ __forceinline__ void store_unit(unsigned char* __restrict__ dst, unsigned char* __restrict__ scales, int64_t row, int unit, const Unit& u) {
  if constexpr (KIND == SLKV_BF16_KV_FP8) {
    uint32_t out[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      uint32_t o = 0;
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        const uint32_t w = u.lo[h * 2 + p];
        float x[2] = {__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)};
        bool nan[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          nan[i] = (__float_as_uint(x[i]) & 0x7f800000u) == 0x7f800000u;
          x[i] = fminf(fmaxf(x[i], -448.f), 448.f);      // the converter's own answer beyond 448 depends on a mode bit
        }
        uint32_t two = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false) & 0xffffu;
        if (nan[0]) two |= 0x7fu;
        if (nan[1]) two |= 0x7f00u;
        o |= two << (16 * p);
      }
      out[h] = o;
    }
    *(u32x2*)(dst + row * D + unit * 8) = u32x2{out[0], out[1]};
  } else if constexpr (KIND == SLKV_BF16_KV_MXFP4) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) top = max(top, max((u.lo[i] << 16) & 0x7fffffffu, u.lo[i] & 0x7fff0000u));
    top = quad_max(top);
    // top = m 2^x with m in [1, 2): at most 7 2^e = 1.75 2^(e+2), so e = x - 2, or x - 1 for m > 1.75; not below -127
    const int field = (int)(top >> 23);
    const int e = top >= 0x7f800000u ? 255 : max(field - 2 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0), 0);
    const float scale = scale_of((uint32_t)(e == 255 ? 127 : e));
    const uint32_t w0 = u.lo[0], w1 = u.lo[1], w2 = u.lo[2], w3 = u.lo[3];   // (bit casts of a vector's elements take its first)
    uint32_t o = 0;
    o = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(o, __builtin_bit_cast(bf16x2, w0), scale, 0);
    o = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(o, __builtin_bit_cast(bf16x2, w1), scale, 1);
    o = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(o, __builtin_bit_cast(bf16x2, w2), scale, 2);
    o = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(o, __builtin_bit_cast(bf16x2, w3), scale, 3);
    *(uint32_t*)(dst + row * (D / 2) + unit * 4) = o;
    if (unit % 4 == 0) scales[row * (D / kScaleBlock) + unit / 4] = (unsigned char)e;
  } else {
    constexpr int kBytes = 8 * (int)sizeof(typename Kind<KIND>::wide);
    *(u32x4*)(dst + row * (D / 8 * kBytes) + unit * kBytes) = u.lo;
    if constexpr (kBytes == 32) *(u32x4*)(dst + row * (D / 8 * kBytes) + unit * kBytes + 16) = u.hi;
  }
}

// One unit of a cache row, widened.
template <int KIND, int D>
__device__ __forceinline__ Unit widen_unit(const unsigned char* __restrict__ src, const unsigned char* __restrict__ scales, int64_t row, int unit) {
  Unit u;
  if constexpr (KIND == SLKV_BF16_KV_FP8) {
    const u32x2 c = *(const u32x2*)(src + row * D + unit * 8);
    u.lo = u32x4{fp8_pair<false>(c[0]), fp8_pair<true>(c[0]), fp8_pair<false>(c[1]), fp8_pair<true>(c[1])};
  } else if constexpr (KIND == SLKV_BF16_KV_MXFP4) {
    const uint32_t c = *(const uint32_t*)(src + row * (D / 2) + unit * 4);
    const float s = scale_of(scales[row * (D / kScaleBlock) + unit / 4]);
    u.lo = u32x4{fp4_pair<0>(c, s), fp4_pair<1>(c, s), fp4_pair<2>(c, s), fp4_pair<3>(c, s)};
  } else {
    u = load_unit<KIND>(src + row * (D * (int)sizeof(typename Kind<KIND>::wide)), unit);
  }
  return u;
}

// ------------------------------------------------------------------ fill

constexpr int kBlockRows = 32;        // rows of a workgroup of fill and of rows
constexpr int kThreads = 256;
template <int N>
using RowsTab = SegWords<N, 3>;       // w[0] room of the segment (first row), w[1] its rows outside the cache, w[2] workgroups before it
// The same for more segments, whose rooms and rows outside are below 2^16: a launch for each 290 segments took 512 of them 4 us longer, and the host 4.
struct RowsTabShort {
  static constexpr int kSegs = 800, kGroup = 16;
  int32_t nseg, seg0, least;          // least: workgroups of a segment without rows
  int32_t w[3][kSegs / kGroup];       // as above, of every 16th segment
  uint16_t room[kSegs], count[kSegs];
};

// The segment of a workgroup.  One wave looks it up for all: the table stands in the kernel's arguments, which thousands of workgroups read past the caches.
struct RowsAt { int seg, first, start, room, other, count; };
template <class TAB>
__device__ __forceinline__ RowsAt find_rows(const TAB& tab, RowsAt& shared) {
  if (threadIdx.x < kWave) {
    const int block = blockIdx.x, lane = threadIdx.x;
    if constexpr (std::is_same_v<TAB, RowsTabShort>) {
      const int groups = (tab.nseg + TAB::kGroup - 1) / TAB::kGroup;
      const int g = __popcll(__ballot(lane < groups && tab.w[2][min(lane, groups - 1)] <= block)) - 1, i = g * TAB::kGroup + lane;
      const bool in = lane < TAB::kGroup && i < tab.nseg;
      RowsAt r;
      r.room = in ? tab.room[i] : 0;
      r.count = in ? tab.count[i] : 0;
      const int blocks = in ? max(tab.least, (min(r.room, r.count) + kBlockRows - 1) / kBlockRows) : 0;
      const int first = tab.w[2][g] + (int)row_incl_scan((uint32_t)blocks) - blocks;
      r.start = tab.w[0][g] + (int)row_incl_scan((uint32_t)r.room) - r.room;
      r.other = tab.w[1][g] + (int)row_incl_scan((uint32_t)r.count) - r.count;
      r.seg = tab.seg0 + i;
      r.first = (block - first) * kBlockRows;
      if (blocks && first <= block && block < first + blocks) shared = r;
    } else {
      const int i = find_segment_wave(tab.nseg, block, [&](int s) { return tab.w[2][s]; });
      if (lane == 0) {
        RowsAt r;
        r.seg = tab.seg0 + i;
        r.first = (block - tab.w[2][i]) * kBlockRows;
        r.start = tab.w[0][i];
        r.room = tab.w[0][i + 1] - r.start;
        r.other = tab.w[1][i];
        r.count = tab.w[1][i + 1] - r.other;
        shared = r;
      }
    }
  }
  __syncthreads();
  return shared;
}

// Bound by memory: 4 d bytes read and 2 (d/2 + d/32) written a row for MXFP4.  A lane takes 8 elements of a row, so
// that a wave's loads and stores are whole lines and a block's magnitude is a maximum over four lanes.
template <int KIND, int D, class TAB>
__global__ __launch_bounds__(kThreads) void fill_kernel(const CacheArrays c, const unsigned char* __restrict__ k_src,
                                                        const unsigned char* __restrict__ v_src, const int32_t* __restrict__ pos_src, const TAB tab) {
  __shared__ RowsAt sh_at;
  const RowsAt at = find_rows(tab, sh_at);
  const int first = at.first, src0 = at.other, count = at.count, dst0 = at.start;
  if (first == 0 && threadIdx.x == 0) c.lengths[at.seg] = count;
  const int rows = min(count - first, kBlockRows);       // 0 in the one workgroup of a segment without rows
  constexpr int kUnits = D / 8, kRowsAtOnce = kThreads / (2 * kUnits);
  constexpr int kWideRow = D * (int)sizeof(typename Kind<KIND>::wide);
  const int unit = threadIdx.x % kUnits, isv = threadIdx.x / kUnits % 2;
  const unsigned char* src = isv ? v_src : k_src;
  unsigned char* dst = isv ? c.v : c.k;
  unsigned char* scales = isv ? c.v_scale : c.k_scale;
  Unit u[kBlockRows / kRowsAtOnce];
#pragma unroll
  for (int i = 0; i < kBlockRows / kRowsAtOnce; ++i) {
    const int r = threadIdx.x / (2 * kUnits) + i * kRowsAtOnce;
    if (r < rows) u[i] = load_unit<KIND>(src + (int64_t)(src0 + first + r) * kWideRow, unit);
  }
#pragma unroll
  for (int i = 0; i < kBlockRows / kRowsAtOnce; ++i) {
    const int r = threadIdx.x / (2 * kUnits) + i * kRowsAtOnce;
    if (r < rows) store_unit<KIND, D>(dst, scales, dst0 + first + r, unit, u[i]);
  }
  if ((int)threadIdx.x < rows) {
    const int64_t row = dst0 + first + (int)threadIdx.x;
    if (pos_src) c.pos[row] = pos_src[src0 + first + (int)threadIdx.x];
    if (c.weight) c.weight[row] = 0.f;
  }
}

// ------------------------------------------------------------------ append

constexpr int kAppendSegs = 880;
template <int N>
using RoomTab = SegWords<N, 1>;       // w[0] first row of the segment's room
struct AppendArgs {
  CacheArrays c;
  const unsigned char *k_src, *v_src;
  int64_t kb, kh, kt, vb, vh, vt;     // strides in bytes
  const int32_t* pos_src;
  const int32_t* at;
  int32_t T, hkv;
};

// A wave per segment: nobody else reads or writes the segment's length, so the lengths may be read and written in one launch, in place.  Bound by latency:
// one round trip for the length, beside that of the rows.
template <int KIND, int D, class TAB>
__global__ __launch_bounds__(kThreads) void append_kernel(const AppendArgs a, const TAB tab) {
  const int i = blockIdx.x * (kThreads / kWave) + __builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave));
  if (i >= tab.nseg) return;
  const int seg = tab.seg0 + i, b = seg / a.hkv, h = seg % a.hkv, lane = threadIdx.x % kWave;
  const int start = tab.w[0][i], room = tab.w[0][i + 1] - start;
  const int n = rows_in_use(a.at ? a.at : a.c.lengths, seg, room);
  const int T = a.T, fit = min(T, room - n);
  constexpr int kUnits = D / 8;
  const int unit = lane % kUnits, isv = lane / kUnits % 2;
  const unsigned char* src = isv ? a.v_src + b * a.vb + h * a.vh : a.k_src + b * a.kb + h * a.kh;
  const int64_t stride = isv ? a.vt : a.kt;
  unsigned char* dst = isv ? a.c.v : a.c.k;
  unsigned char* scales = isv ? a.c.v_scale : a.c.k_scale;
  constexpr int kRowsAtOnce = kWave / (2 * kUnits);
  for (int t0 = 0; t0 < T; t0 += 4 * kRowsAtOnce) {
    Unit u[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int t = t0 + j * kRowsAtOnce + lane / (2 * kUnits);
      if (t < T) u[j] = load_unit<KIND>(src + t * stride, unit);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int t = t0 + j * kRowsAtOnce + lane / (2 * kUnits);
      if (t < fit) store_unit<KIND, D>(dst, scales, (int64_t)start + n + t, unit, u[j]);
    }
  }
  if (lane < fit) {
    if (a.pos_src) a.c.pos[(int64_t)start + n + lane] = a.pos_src[(int64_t)b * T + lane];
    if (a.c.weight) a.c.weight[(int64_t)start + n + lane] = 0.f;
  }
  if (lane == 0) a.c.lengths[seg] = n + fit;
}

// ------------------------------------------------------------------ rows

// Bound by memory, as fill.
template <int KIND, int D, class TAB>
__global__ __launch_bounds__(kThreads) void rows_kernel(const CacheArrays c, unsigned char* __restrict__ k_dst, unsigned char* __restrict__ v_dst,
                                                        int32_t* __restrict__ pos_dst, const TAB tab) {
  __shared__ RowsAt sh_at;
  const RowsAt at = find_rows(tab, sh_at);
  const int first = at.first, dst0 = at.other, start = at.start;
  const int n = rows_in_use(c.lengths, at.seg, at.room);
  const int take = min(n, at.count);
  const int rows = min(take - first, kBlockRows);
  if (rows <= 0) return;
  const int64_t src0 = (int64_t)start + n - take + first;
  constexpr int kUnits = D / 8, kRowsAtOnce = kThreads / (2 * kUnits);
  constexpr int kWideRow = D * (int)sizeof(typename Kind<KIND>::wide);
  const int unit = threadIdx.x % kUnits, isv = threadIdx.x / kUnits % 2;
  Unit u[kBlockRows / kRowsAtOnce];
#pragma unroll
  for (int i = 0; i < kBlockRows / kRowsAtOnce; ++i) {
    const int r = threadIdx.x / (2 * kUnits) + i * kRowsAtOnce;
    if (r < rows) u[i] = widen_unit<KIND, D>(isv ? c.v : c.k, isv ? c.v_scale : c.k_scale, src0 + r, unit);
  }
  unsigned char* dst = isv ? v_dst : k_dst;
#pragma unroll
  for (int i = 0; i < kBlockRows / kRowsAtOnce; ++i) {
    const int r = threadIdx.x / (2 * kUnits) + i * kRowsAtOnce;
    if (r >= rows) continue;
    unsigned char* const p = dst + (int64_t)(dst0 + first + r) * kWideRow + unit * (kWideRow / kUnits);
    *(u32x4*)p = u[i].lo;
    if constexpr (sizeof(typename Kind<KIND>::wide) == 4) *(u32x4*)(p + 16) = u[i].hi;
  }
  if (pos_dst && (int)threadIdx.x < rows) pos_dst[dst0 + first + (int)threadIdx.x] = c.pos[src0 + (int)threadIdx.x];
}

// ------------------------------------------------------------------ eviction

constexpr int kEvictThreads = 1024, kEvictWaves = kEvictThreads / kWave;
constexpr int kEvictHeld = 12288, kEvictHeldLong = 36864;   // keys that stay in LDS: with two workgroups on a CU, with one
constexpr int kEvictRank = 256;       // keys that are ranked against each other
constexpr int kEvictSlice = 512;      // rows that a workgroup copies, at most (512 segments of 512 rows: 69 us; 79 with 1024)
constexpr int kEvictSegs = 240;
template <int N>
using EvictTab = SegWords<N, 4>;      // w[0] room of the segment, w[1] its room in the other cache, w[2] workgroups before it, w[3] max(C_h, w)
// The same for more than kEvictSegs segments, whose rooms are below 2^16: one launch (512 segments of up to 1634 rows to 512: 79 us at 1024 rows a slice;
// 113 in three launches).
struct EvictTabShort {
  static constexpr int kSegs = 560, kGroup = 16;
  int32_t nseg, seg0;
  int32_t w[3][kSegs / kGroup];       // as above, of every 16th segment
  uint16_t room[kSegs], other[kSegs], cap[kSegs];
};

__device__ __forceinline__ uint32_t weight_key(float v) { return v != v ? 0xffffffffu : float_key(v); }

template <int HELD>
struct EvictLds {
  uint32_t held[HELD], hist[kHistBins], scan[16], res[2], near_key[kEvictRank];
  uint32_t ends[2][kEvictWaves];      // a wave's smallest and largest key: written before a barrier, read behind it and never written again, since no other barrier follows where all keys are equal
  uint32_t votes[2][kEvictWaves];     // a wave's keys above the smallest kept one, and equal to it, while others may still be reading `ends`
  int32_t near_row[kEvictRank], near_count, from[kEvictSlice * (HELD == kEvictHeld ? 1 : 2)];
};

// The `want` largest of m keys, 0 < want < m: the smallest kept key and how many of the rows that have it stay, the lower ones.  A wave looks after neighbouring rows i0 ..
// i1 - 1, lane by lane.  The key is found by digits of 11 bits of the keys' distance from the smallest, the first one as fine as their range allows (weights lie within some
// octaves, so fixed digits would pile up in a few counters); when no more than kEvictRank keys share the digit of the last one, these are ranked against each other.  The first
// HELD keys stay in LDS, others are read again from memory.  Bound by latency, of the instructions too: loops are not unrolled far.
template <int HELD>
__device__ __forceinline__ uint32_t evict_key(const EvictLds<HELD>& l, const float* __restrict__ keys, int i) {
  if constexpr (HELD == kEvictHeld) return l.held[i];
  else return i < HELD ? l.held[i] : weight_key(keys[i]);
}
template <int HELD>
__device__ __forceinline__ void evict_threshold(EvictLds<HELD>& l, const float* __restrict__ keys, int m, uint32_t want, int i0, int i1, uint32_t& least, uint32_t& count) {
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  auto key_of = [&](int i) __attribute__((always_inline)) { return evict_key<HELD>(l, keys, i); };
  uint32_t lo = ~0u, hi = 0u;
#pragma unroll 8
  for (int i = i0; i < i1; i += kWave) {
    const uint32_t x = weight_key(keys[i]);
    if (HELD == kEvictHeld || i < HELD) l.held[i] = x;
    lo = min(lo, x);
    hi = max(hi, x);
  }
  auto smaller = [](uint32_t x, uint32_t y) { return min(x, y); };
  auto larger = [](uint32_t x, uint32_t y) { return max(x, y); };
  lo = wave_reduce_to_last(lo, smaller);
  hi = wave_reduce_to_last(hi, larger);
  if (lane == kWave - 1) l.ends[0][wave] = lo, l.ends[1][wave] = hi;
  for (int i = tid; i < kHistBins; i += kEvictThreads) l.hist[i] = 0;
  if (tid == 0) l.near_count = 0;
  __syncthreads();
  lo = (uint32_t)__builtin_amdgcn_readlane((int)wave_reduce_to_last(l.ends[0][lane % kEvictWaves], smaller), kWave - 1);
  hi = (uint32_t)__builtin_amdgcn_readlane((int)wave_reduce_to_last(l.ends[1][lane % kEvictWaves], larger), kWave - 1);
  // the keys from `lo` on, of which `bits` bits are undecided; the k-th largest of these is looked for
  int bits = hi == lo ? 0 : 32 - __clz(hi - lo);
  uint32_t k = want;
  while (bits > 0) {
    const int shift = max(bits - 11, 0);
#pragma unroll 4
    for (int i = i0; i < i1; i += kWave) {
      const uint32_t x = key_of(i), d = x - lo;
      if (x >= lo && (d >> shift) < (1u << (bits - shift))) atomicAdd(&l.hist[d >> shift], 1u);   // (a last digit may have fewer bits)
    }
    __syncthreads();
    select_bin<kEvictThreads>(l.hist, k, l.scan, l.res);
    const uint32_t digit = l.res[0], share = l.hist[digit];
    k = l.res[1];
    lo += digit << shift;
    bits = shift;
    __syncthreads();
    if (bits == 0) break;
    if (share <= (uint32_t)kEvictRank) {
#pragma unroll 4
      for (int i = i0; i < i1; i += kWave) {
        const uint32_t x = key_of(i);
        if (x >= lo && (x - lo) >> bits == 0) {
          const int at = atomicAdd(&l.near_count, 1);
          l.near_key[at] = x;
          l.near_row[at] = i;
        }
      }
      __syncthreads();
      // four lanes a key: how many are larger, how many equal ones come before it
      const int c = tid / 4;
      uint32_t above = 0, before = 0;
      if (c < (int)share) {
        const uint32_t x = l.near_key[c];
        const int row = l.near_row[c];
        for (uint32_t i = tid % 4; i < share; i += 4) {
          above += l.near_key[i] > x;
          before += l.near_key[i] == x && l.near_row[i] < row;
        }
      }
      above += dpp_move<0xb1>(0u, above);
      above += dpp_move<0x4e>(0u, above);
      before += dpp_move<0xb1>(0u, before);
      before += dpp_move<0x4e>(0u, before);
      if (c < (int)share && tid % 4 == 0 && above + before == k - 1) l.res[0] = l.near_key[c], l.res[1] = before + 1;
      __syncthreads();
      lo = l.res[0];
      k = l.res[1];
      break;
    }
    for (int i = tid; i < kHistBins; i += kEvictThreads) l.hist[i] = 0;
    __syncthreads();
  }
  least = lo;
  count = k;
}

// A workgroup copies a slice of a segment's kept rows, `slice` of them, UNITS of 16 bytes a row of K; which rows these are every workgroup of the segment finds by
// itself, so that nothing waits for a selection that is not its own: 128 segments of up to 3345 rows, nearly all of them kept, 31 us (137 MB), with a launch that selects
// (10 us, by the longest segment) and one that copies 40.  Of 16 segments of up to 10047 rows down to 1024 on average (MXFP4) the selection is 11 of 19 us.  The copy is bound by memory: 16 rows of every wave are on their way at once.
template <int UNITS, int SCALES, int HELD, class TAB>
__global__ __launch_bounds__(kEvictThreads) void evict_kernel(const CacheArrays in, const CacheArrays out, int32_t* __restrict__ kept_idx, int w, int slice, const TAB tab) {
  __shared__ EvictLds<HELD> l;
  __shared__ int32_t sh_at[6];                         // segment, its slice, first row of the room, rows in use, first row of the other room, max(C_h, w)
  const int tid = threadIdx.x, lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  if (tid < kWave) {
    const int block = blockIdx.x;
    if constexpr (std::is_same_v<TAB, EvictTabShort>) {
      const int groups = (tab.nseg + TAB::kGroup - 1) / TAB::kGroup;
      const int g = __popcll(__ballot(lane < groups && tab.w[2][min(lane, groups - 1)] <= block)) - 1, i = g * TAB::kGroup + lane;
      const bool here = lane < TAB::kGroup && i < tab.nseg;
      const int room = here ? tab.room[i] : 0, other = here ? tab.other[i] : 0, cap = here ? tab.cap[i] : 0;
      const int blocks = here ? max(1, (min(room, cap) + slice - 1) / slice) : 0;
      const int before = tab.w[2][g] + (int)row_incl_scan((uint32_t)blocks) - blocks;
      const int start = tab.w[0][g] + (int)row_incl_scan((uint32_t)room) - room, to = tab.w[1][g] + (int)row_incl_scan((uint32_t)other) - other;
      if (blocks && before <= block && block < before + blocks) {
        sh_at[0] = tab.seg0 + i;
        sh_at[1] = block - before;
        sh_at[2] = start;
        sh_at[3] = rows_in_use(in.lengths, tab.seg0 + i, room);
        sh_at[4] = to;
        sh_at[5] = cap;
      }
    } else {
      const int i = find_segment_wave(tab.nseg, block, [&](int s) { return tab.w[2][s]; });
      if (tid == 0) {
        sh_at[0] = tab.seg0 + i;
        sh_at[1] = block - tab.w[2][i];
        sh_at[2] = tab.w[0][i];
        sh_at[3] = rows_in_use(in.lengths, tab.seg0 + i, tab.w[0][i + 1] - tab.w[0][i]);
        sh_at[4] = tab.w[1][i];
        sh_at[5] = tab.w[3][i];
      }
    }
  }
  __syncthreads();
  const int seg = sh_at[0], first = sh_at[1] * slice, start = sh_at[2], n = sh_at[3], cap = sh_at[5];
  const int kept = min(n, cap), rows = min(kept - first, slice);
  if (first == 0 && tid == 0) out.lengths[seg] = kept;
  if (rows <= 0) return;
  const int m = n - w, want = cap - w;
  if (n <= cap) {
    for (int r = tid; r < rows; r += kEvictThreads) l.from[r] = first + r;
  } else {
    for (int r = max(want - first, 0) + tid; r < rows; r += kEvictThreads) l.from[r] = m + first + r - want;   // of the latest w
    if (first < want) {
      const float* keys = in.weight + start;
      const int rows_each = (m + kEvictThreads - 1) / kEvictThreads * kWave;     // of a wave
      const int b0 = wave * rows_each, i0 = b0 + lane, i1 = min(m, b0 + rows_each);
      uint32_t least, k;
      evict_threshold(l, keys, m, (uint32_t)want, i0, i1, least, k);
      auto key_of = [&](int i) __attribute__((always_inline)) { return evict_key<HELD>(l, keys, i); };
      // a wave counts its kept rows by votes, then emits them at the places that the waves before it leave
      uint32_t gt = 0, eq = 0;
      for (int b = b0; b < i1; b += 4 * kWave) {
        uint32_t x[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) x[t] = b + t * kWave + lane < i1 ? key_of(b + t * kWave + lane) : 0u;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const bool in = b + t * kWave + lane < i1;
          gt += (uint32_t)__popcll(__ballot(in && x[t] > least));
          eq += (uint32_t)__popcll(__ballot(in && x[t] == least));
        }
      }
      if (lane == 0) l.votes[0][wave] = gt, l.votes[1][wave] = eq;
      __syncthreads();
      uint32_t at = 0, e = 0;                         // kept rows, and rows of the smallest kept key, in the waves before
      for (int v = 0; v < wave; ++v) {
        at += l.votes[0][v];
        e += l.votes[1][v];
      }
      at += min(e, k);
      const uint64_t below = (1ull << lane) - 1;
      const bool mine = (int)(at + gt + eq) > first && (int)at < first + rows;   // some of the wave's rows may be in the slice
      for (int b = mine ? b0 : i1; b < i1; b += kWave) {
        const int i = b + lane;
        const uint32_t x = i < i1 ? key_of(i) : 0u;
        const bool is_eq = i < i1 && x == least;
        const uint64_t eqs = __ballot(is_eq);
        const bool stays = (i < i1 && x > least) || (is_eq && e + (uint32_t)__popcll(eqs & below) < k);
        const uint64_t all = __ballot(stays);
        const int r = (int)(at + (uint32_t)__popcll(all & below)) - first;
        if (stays && r >= 0 && r < rows) l.from[r] = i;
        at += (uint32_t)__popcll(all);
        e += (uint32_t)__popcll(eqs);
      }
    }
  }
  __syncthreads();
  const int64_t to0 = (int64_t)sh_at[4] + first, src0 = start;
  constexpr int kRowsAtOnce = kEvictThreads / UNITS, kTimes = 4;
  const int u = tid % UNITS, r0 = tid / UNITS;
  for (int r1 = r0; r1 < rows; r1 += kTimes * kRowsAtOnce) {
    u32x4 k[kTimes], v[kTimes];
#pragma unroll
    for (int t = 0; t < kTimes; ++t) {
      const int r = r1 + t * kRowsAtOnce;
      if (r < rows) {
        const int64_t s = (src0 + l.from[r]) * UNITS + u;
        k[t] = __builtin_nontemporal_load((const u32x4*)in.k + s);
        v[t] = __builtin_nontemporal_load((const u32x4*)in.v + s);
      }
    }
#pragma unroll
    for (int t = 0; t < kTimes; ++t) {
      const int r = r1 + t * kRowsAtOnce;
      if (r < rows) {
        const int64_t d = (to0 + r) * UNITS + u;
        ((u32x4*)out.k)[d] = k[t];
        ((u32x4*)out.v)[d] = v[t];
      }
    }
  }
  if constexpr (SCALES > 0) {
    typedef std::conditional_t<SCALES == 4, uint32_t, uint16_t> word;          // a row's exponents
    for (int r = tid; r < rows; r += kEvictThreads) {
      const int64_t s = src0 + l.from[r];
      ((word*)out.k_scale)[to0 + r] = ((const word*)in.k_scale)[s];
      ((word*)out.v_scale)[to0 + r] = ((const word*)in.v_scale)[s];
    }
  }
  for (int r = tid; r < rows; r += kEvictThreads) {
    const int64_t s = src0 + l.from[r], t = to0 + r;
    if (in.pos && out.pos) out.pos[t] = in.pos[s];
    if (in.weight && out.weight) out.weight[t] = in.weight[s];
    if (kept_idx) kept_idx[t] = l.from[r];
  }
}

// ------------------------------------------------------------------ launches

// Calls f(tab, blocks) for groups of segments that one table holds; word(s, row of the table) gives the table's words, s up to S inclusive; the
// words of row PREFIX are the workgroups before a segment, blocks_of(s) of them each.
template <template <int> class TABLE, int MANY, int PREFIX, class WORD, class BLOCKS, class F>
static void for_tables(int64_t S, WORD word, BLOCKS blocks_of, F f) {
  auto one = [&](auto tab, int64_t s0, int64_t ns) {
    constexpr int kWords = sizeof(tab.w) / sizeof(tab.w[0]);
    tab.nseg = (int32_t)ns;
    tab.seg0 = (int32_t)s0;
    int64_t blocks = 0;
    for (int64_t i = 0; i <= ns; ++i) {
      for (int r = 0; r < kWords; ++r) tab.w[r][i] = r == PREFIX ? (int32_t)blocks : word(s0 + i, r);
      if (i < ns) blocks += blocks_of(s0 + i);
    }
    if (blocks) f(tab, (int)blocks);
  };
  if (S <= kFewSegs) return one(TABLE<kFewSegs>{}, 0, S);
  for (int64_t s0 = 0; s0 < S; s0 += MANY) one(TABLE<MANY>{}, s0, std::min<int64_t>(MANY, S - s0));
}

// The launches of fill and rows: room offsets, offsets outside, workgroups of a segment without rows.
template <class F>
static void for_rows(int64_t S, const int64_t* room, const int64_t* other, int least, F f) {
  auto blocks_of = [&](int64_t s) { return std::max<int64_t>(least, (std::min(other[s + 1] - other[s], room[s + 1] - room[s]) + kBlockRows - 1) / kBlockRows); };
  bool is_short = S > kFewSegs;
  for (int64_t s = 0; is_short && s < S; ++s) is_short = room[s + 1] - room[s] < 65536 && other[s + 1] - other[s] < 65536;
  if (!is_short) return for_tables<RowsTab, kManySegs3, 2>(S, [&](int64_t s, int r) { return (int32_t)(r == 0 ? room[s] : other[s]); }, blocks_of, f);
  for (int64_t s0 = 0; s0 < S; s0 += RowsTabShort::kSegs) {
    RowsTabShort tab;
    tab.nseg = (int32_t)std::min<int64_t>(RowsTabShort::kSegs, S - s0);
    tab.seg0 = (int32_t)s0;
    tab.least = least;
    int64_t blocks = 0;
    for (int i = 0; i < tab.nseg; ++i) {
      if (i % RowsTabShort::kGroup == 0) {
        tab.w[0][i / RowsTabShort::kGroup] = (int32_t)room[s0 + i];
        tab.w[1][i / RowsTabShort::kGroup] = (int32_t)other[s0 + i];
        tab.w[2][i / RowsTabShort::kGroup] = (int32_t)blocks;
      }
      tab.room[i] = (uint16_t)(room[s0 + i + 1] - room[s0 + i]);
      tab.count[i] = (uint16_t)(other[s0 + i + 1] - other[s0 + i]);
      blocks += blocks_of(s0 + i);
    }
    if (blocks) f(tab, (int)blocks);
  }
}

template <class F>
static void with_dim(int d, F f) {
  if (d == 64) f(std::integral_constant<int, 64>{});
  else f(std::integral_constant<int, 128>{});
}

static int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

static bool overlap(const void* a, const void* b, int64_t bytes_a, int64_t bytes_b) {
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  return a && b && x < y + (uintptr_t)bytes_b && y < x + (uintptr_t)bytes_a;
}

static slkv_status evict_checks(const slkv_cache_desc* desc, const slkv_cache_desc* od, int32_t w, const int32_t* h_budgets) {
  slkv_status st = validate_cache_desc(desc);
  if (st != SLKV_OK) return st;
  if ((st = validate_cache_desc(od, "out_desc")) != SLKV_OK) return st;
  if (od->dtype != desc->dtype || od->B != desc->B || od->Hq != desc->Hq || od->Hkv != desc->Hkv || od->d != desc->d)
    return fail(SLKV_ERR_BAD_ARG, "out_desc differs from desc in dtype, B, Hq, Hkv or d");
  if (w < 0) return fail(SLKV_ERR_BAD_ARG, "w < 0");
  if (!h_budgets) return fail(SLKV_ERR_NULL, "h_budgets is NULL");
  for (int h = 0; h < desc->Hkv; ++h)
    if (h_budgets[h] < 0) return fail(SLKV_ERR_BAD_ARG, "budget[%d] < 0", h);
  return SLKV_OK;
}

}  // namespace slkv

using namespace slkv;

extern "C" slkv_status slkv_fill_cache(const slkv_cache_desc* desc, const slkv_cache* cache, const int64_t* h_src_offsets,
                                       const void* d_k_rows, const void* d_v_rows, const int32_t* d_pos_rows, void* hip_stream) {
  clear_error();
  slkv_status st = validate_cache_desc(desc);
  if (st != SLKV_OK) return st;
  if ((st = validate_cache(desc, cache)) != SLKV_OK) return st;
  const int64_t S = (int64_t)desc->B * desc->Hkv;
  if ((st = validate_offsets(h_src_offsets, S, "h_src_offsets")) != SLKV_OK) return st;
  if (!cache->d_lengths) return fail(SLKV_ERR_NULL, "cache: d_lengths is NULL");
  if (h_src_offsets[S] > h_src_offsets[0] && (!d_k_rows || !d_v_rows)) return fail(SLKV_ERR_NULL, "a required device pointer is NULL");
  if (d_pos_rows && !cache->d_pos) return fail(SLKV_ERR_NULL, "cache: d_pos is NULL");
  const void* ptrs[] = {d_k_rows, d_v_rows, d_pos_rows};
  for (const void* ptr : ptrs)
    if ((uintptr_t)ptr % 16) return fail(SLKV_ERR_BAD_ARG, "device pointer %p not 16-byte aligned", ptr);
  for (int64_t s = 0; s < S; ++s)
    if (h_src_offsets[s + 1] - h_src_offsets[s] > desc->h_offsets[s + 1] - desc->h_offsets[s])
      return fail(SLKV_ERR_CAPACITY, "segment %lld: %lld rows into a room of %lld", (long long)s, (long long)(h_src_offsets[s + 1] - h_src_offsets[s]),
                  (long long)(desc->h_offsets[s + 1] - desc->h_offsets[s]));
  ScopedKernelTimer timer(SLKV_K_CACHE_STORE);
  with_kind(desc->dtype, [&](auto kind) {
    with_dim(desc->d, [&](auto dim) {
      for_rows(S, desc->h_offsets, h_src_offsets, 1, [&](const auto& tab, int blocks) {
        SLKV_LAUNCH((fill_kernel<decltype(kind)::value, decltype(dim)::value, std::decay_t<decltype(tab)>>), dim3(blocks), dim3(kThreads), 0,
                    (hipStream_t)hip_stream, arrays_of(cache), (const unsigned char*)d_k_rows, (const unsigned char*)d_v_rows, d_pos_rows, tab);
      });
    });
  });
  return launch_status("fill");
}

extern "C" slkv_status slkv_append_cache(const slkv_cache_desc* desc, const slkv_cache* cache, int32_t T, const void* d_k, const void* d_v,
                                         const int64_t k_stride[3], const int64_t v_stride[3], const int32_t* d_pos, const int32_t* d_at,
                                         void* hip_stream) {
  clear_error();
  slkv_status st = validate_cache_desc(desc);
  if (st != SLKV_OK) return st;
  if ((st = validate_cache(desc, cache)) != SLKV_OK) return st;
  if (!cache->d_lengths) return fail(SLKV_ERR_NULL, "cache: d_lengths is NULL");
  if (T < 1) return fail(SLKV_ERR_BAD_ARG, "T must be >= 1");
  if (T > 64) return fail(SLKV_ERR_UNSUPPORTED, "T = %d > 64", T);
  if (!d_k || !d_v || !k_stride || !v_stride) return fail(SLKV_ERR_NULL, "a required pointer is NULL");
  if (d_pos && !cache->d_pos) return fail(SLKV_ERR_NULL, "cache: d_pos is NULL");
  const void* ptrs[] = {d_k, d_v, d_pos, d_at};
  for (const void* ptr : ptrs)
    if ((uintptr_t)ptr % 16) return fail(SLKV_ERR_BAD_ARG, "device pointer %p not 16-byte aligned", ptr);
  const int elt = wide_bytes(desc->dtype);
  for (int i = 0; i < 3; ++i)
    if (k_stride[i] < 0 || v_stride[i] < 0 || k_stride[i] * elt % 16 || v_stride[i] * elt % 16)
      return fail(SLKV_ERR_BAD_ARG, "stride %d not a non-negative multiple of 16 bytes", i);
  AppendArgs a;
  a.c = arrays_of(cache);
  a.k_src = (const unsigned char*)d_k;
  a.v_src = (const unsigned char*)d_v;
  a.kb = k_stride[0] * elt, a.kh = k_stride[1] * elt, a.kt = k_stride[2] * elt;
  a.vb = v_stride[0] * elt, a.vh = v_stride[1] * elt, a.vt = v_stride[2] * elt;
  a.pos_src = d_pos;
  a.at = d_at;
  a.T = T;
  a.hkv = desc->Hkv;
  ScopedKernelTimer timer(SLKV_K_CACHE_STORE);
  const int64_t S = (int64_t)desc->B * desc->Hkv;
  with_kind(desc->dtype, [&](auto kind) {
    with_dim(desc->d, [&](auto dim) {
      for_tables<RoomTab, kAppendSegs, -1>(
          S, [&](int64_t s, int) { return (int32_t)desc->h_offsets[s]; }, [&](int64_t) { return 1; },
          [&](const auto& tab, int segs) {
            SLKV_LAUNCH((append_kernel<decltype(kind)::value, decltype(dim)::value, std::decay_t<decltype(tab)>>),
                        dim3((unsigned)ceil_div(segs, kThreads / kWave)), dim3(kThreads), 0, (hipStream_t)hip_stream, a, tab);
          });
    });
  });
  return launch_status("append");
}

extern "C" slkv_status slkv_cache_rows(const slkv_cache_desc* desc, const slkv_cache* cache, const int64_t* h_out_offsets,
                                       void* d_k_rows, void* d_v_rows, int32_t* d_pos_rows, void* hip_stream) {
  clear_error();
  slkv_status st = validate_cache_desc(desc);
  if (st != SLKV_OK) return st;
  if ((st = validate_cache(desc, cache)) != SLKV_OK) return st;
  const int64_t S = (int64_t)desc->B * desc->Hkv;
  if ((st = validate_offsets(h_out_offsets, S, "h_out_offsets")) != SLKV_OK) return st;
  if (h_out_offsets[S] > h_out_offsets[0] && (!d_k_rows || !d_v_rows)) return fail(SLKV_ERR_NULL, "a required device pointer is NULL");
  if (d_pos_rows && !cache->d_pos) return fail(SLKV_ERR_NULL, "cache: d_pos is NULL");
  const void* ptrs[] = {d_k_rows, d_v_rows, d_pos_rows};
  for (const void* ptr : ptrs)
    if ((uintptr_t)ptr % 16) return fail(SLKV_ERR_BAD_ARG, "device pointer %p not 16-byte aligned", ptr);
  ScopedKernelTimer timer(SLKV_K_CACHE_ROWS);
  with_kind(desc->dtype, [&](auto kind) {
    with_dim(desc->d, [&](auto dim) {
      for_rows(S, desc->h_offsets, h_out_offsets, 0, [&](const auto& tab, int blocks) {
        SLKV_LAUNCH((rows_kernel<decltype(kind)::value, decltype(dim)::value, std::decay_t<decltype(tab)>>), dim3(blocks), dim3(kThreads), 0,
                    (hipStream_t)hip_stream, arrays_of(cache), (unsigned char*)d_k_rows, (unsigned char*)d_v_rows, d_pos_rows, tab);
      });
    });
  });
  return launch_status("rows");
}

extern "C" slkv_status slkv_evict_cache(const slkv_cache_desc* desc, const slkv_cache* cache, const slkv_cache_desc* out_desc, const slkv_cache* out,
                                        int32_t w, const int32_t* h_budgets, int32_t* d_kept_idx, void* hip_stream) {
  clear_error();
  slkv_status st = evict_checks(desc, out_desc, w, h_budgets);
  if (st != SLKV_OK) return st;
  if ((st = validate_cache(desc, cache)) != SLKV_OK) return st;
  if ((st = validate_cache(out_desc, out, "out")) != SLKV_OK) return st;
  const int64_t S = (int64_t)desc->B * desc->Hkv, rows_in = desc->h_offsets[S], rows_out = out_desc->h_offsets[S];
  if (!out->d_lengths) return fail(SLKV_ERR_NULL, "out: d_lengths is NULL");
  if (rows_in > desc->h_offsets[0] && !cache->d_weight) return fail(SLKV_ERR_NULL, "cache: d_weight is NULL");
  if ((uintptr_t)d_kept_idx % 16) return fail(SLKV_ERR_BAD_ARG, "device pointer %p not 16-byte aligned", (void*)d_kept_idx);
  const int64_t row_bytes = (int64_t)desc->d * kind_bits(desc->dtype) / 8, scale_bytes = desc->dtype == SLKV_BF16_KV_MXFP4 ? desc->d / kScaleBlock : 0;
  // (a segment with a shorter room never holds cap rows)
  auto cap_of = [&](int64_t s) { return std::max(h_budgets[s % desc->Hkv], w); };
  auto most_of = [&](int64_t s) { return std::min<int64_t>(desc->h_offsets[s + 1] - desc->h_offsets[s], cap_of(s)); };
  int64_t most = 0, longest = 0;
  for (int64_t s = 0; s < S; ++s) {
    const int64_t rows = most_of(s), room = out_desc->h_offsets[s + 1] - out_desc->h_offsets[s];
    if (room < rows) return fail(SLKV_ERR_CAPACITY, "segment %lld: up to %lld rows into a room of %lld", (long long)s, (long long)rows, (long long)room);
    most += rows;
    longest = std::max(longest, desc->h_offsets[s + 1] - desc->h_offsets[s]);
  }
  const void* ins[] = {cache->d_k, cache->d_v, cache->d_k_scale, cache->d_v_scale, cache->d_pos, cache->d_weight, cache->d_lengths};
  const void* outs[] = {out->d_k, out->d_v, out->d_k_scale, out->d_v_scale, out->d_pos, out->d_weight, out->d_lengths, d_kept_idx};
  const int64_t each[] = {row_bytes, row_bytes, scale_bytes, scale_bytes, 4, 4, 0, 4};
  for (int i = 0; i < 7; ++i)
    for (int j = 0; j < 8; ++j)
      if (overlap(ins[i], outs[j], i == 6 ? 4 * S : rows_in * each[i], j == 6 ? 4 * S : rows_out * each[j]))
        return fail(SLKV_ERR_BAD_ARG, "arrays of cache and out overlap");
  // Rooms of up to kEvictHeld rows: two workgroups a CU and all keys in LDS.  Longer ones: one workgroup a CU, with three times the keys in LDS and slices of twice the rows (8
  // segments of up to 34 K rows to 1024 54.7 -> 40.4 us, 64 of them in 4 bits 73.3 -> 44.6, 16 of up to 37 K to 16 K 94.5 -> 90.4).
  const bool held_all = longest <= kEvictHeld;
  // slices: as many workgroups, if the rows are enough for that; a segment's last one is half empty on average
  const int64_t places = held_all ? 512 : 256;
  const int slice = (int)std::min<int64_t>(held_all ? kEvictSlice : 2 * kEvictSlice, std::max<int64_t>(64, ceil_div(most, std::max(places - S / 2, places / 2))));
  ScopedKernelTimer timer(SLKV_K_EVICT);
  auto blocks_of = [&](int64_t s) { return std::max<int64_t>(1, (most_of(s) + slice - 1) / slice); };
  auto launch = [&](const auto& tab, int blocks) {
    using TAB = std::decay_t<decltype(tab)>;
    auto go = [&](auto units, auto scales) {
      auto with = [&](auto held) {
        SLKV_LAUNCH((evict_kernel<decltype(units)::value, decltype(scales)::value, decltype(held)::value, TAB>), dim3(blocks), dim3(kEvictThreads), 0,
                    (hipStream_t)hip_stream, arrays_of(cache), arrays_of(out), d_kept_idx, w, slice, tab);
      };
      if (held_all) with(std::integral_constant<int, kEvictHeld>{});
      else with(std::integral_constant<int, kEvictHeldLong>{});
    };
    using std::integral_constant;
    const integral_constant<int, 0> none{};
    if (scale_bytes == 4) go(integral_constant<int, 4>{}, integral_constant<int, 4>{});
    else if (scale_bytes == 2) go(integral_constant<int, 2>{}, integral_constant<int, 2>{});
    else if (row_bytes == 64) go(integral_constant<int, 4>{}, none);
    else if (row_bytes == 128) go(integral_constant<int, 8>{}, none);
    else if (row_bytes == 256) go(integral_constant<int, 16>{}, none);
    else go(integral_constant<int, 32>{}, none);
  };
  const int64_t* const from = desc->h_offsets;
  const int64_t* const to = out_desc->h_offsets;
  bool is_short = S > kEvictSegs;
  for (int64_t s = 0; is_short && s < S; ++s) is_short = from[s + 1] - from[s] < 65536 && to[s + 1] - to[s] < 65536;
  if (!is_short) {
    for_tables<EvictTab, kEvictSegs, 2>(
        S, [&](int64_t s, int r) { return r == 0 ? (int32_t)from[s] : r == 1 ? (int32_t)to[s] : s < S ? cap_of(s) : 0; }, blocks_of, launch);
    return launch_status("evict");
  }
  for (int64_t s0 = 0; s0 < S; s0 += EvictTabShort::kSegs) {
    EvictTabShort tab;
    tab.nseg = (int32_t)std::min<int64_t>(EvictTabShort::kSegs, S - s0);
    tab.seg0 = (int32_t)s0;
    int64_t blocks = 0;
    for (int i = 0; i < tab.nseg; ++i) {
      const int64_t s = s0 + i;
      if (i % EvictTabShort::kGroup == 0) {
        tab.w[0][i / EvictTabShort::kGroup] = (int32_t)from[s];
        tab.w[1][i / EvictTabShort::kGroup] = (int32_t)to[s];
        tab.w[2][i / EvictTabShort::kGroup] = (int32_t)blocks;
      }
      tab.room[i] = (uint16_t)(from[s + 1] - from[s]);
      tab.other[i] = (uint16_t)(to[s + 1] - to[s]);
      tab.cap[i] = (uint16_t)std::min(cap_of(s), 65535);        // (above every room)
      blocks += blocks_of(s);
    }
    launch(tab, (int)blocks);
  }
  return launch_status("evict");
}
