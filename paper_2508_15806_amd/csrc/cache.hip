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

template <int KIND>
__device__ __forceinline__ Unit load_unit(const unsigned char* row, int unit) {
  Unit u;
  constexpr int kBytes = 8 * (int)sizeof(typename Kind<KIND>::wide);
  u.lo = *(const u32x4*)(row + unit * kBytes);
  if constexpr (kBytes == 32) u.hi = *(const u32x4*)(row + unit * kBytes + 16);
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

// Bound by memory: 4 d bytes read and 2 (d/2 + d/32) written a row for MXFP4.  A lane takes 8 elements of a row, so
// that a wave's loads and stores are whole lines and a block's magnitude is a maximum over four lanes.
template <int KIND, int D, class TAB>
__global__ __launch_bounds__(kThreads) void fill_kernel(const CacheArrays c, const unsigned char* __restrict__ k_src,
                                                        const unsigned char* __restrict__ v_src, const int32_t* __restrict__ pos_src, const TAB tab) {
  const int block = blockIdx.x;
  const int seg = find_segment_wave(tab.nseg, block, [&](int s) { return tab.w[2][s]; });
  const int first = (block - tab.w[2][seg]) * kBlockRows;
  const int src0 = tab.w[1][seg], count = tab.w[1][seg + 1] - src0, dst0 = tab.w[0][seg];
  if (first == 0 && threadIdx.x == 0) c.lengths[tab.seg0 + seg] = count;
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
    if (c.pos && pos_src) c.pos[row] = pos_src[src0 + first + (int)threadIdx.x];
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
    if (a.c.pos && a.pos_src) a.c.pos[(int64_t)start + n + lane] = a.pos_src[(int64_t)b * T + lane];
    if (a.c.weight) a.c.weight[(int64_t)start + n + lane] = 0.f;
  }
  if (lane == 0) a.c.lengths[seg] = n + fit;
}

// ------------------------------------------------------------------ rows

// Bound by memory, as fill.
template <int KIND, int D, class TAB>
__global__ __launch_bounds__(kThreads) void rows_kernel(const CacheArrays c, unsigned char* __restrict__ k_dst, unsigned char* __restrict__ v_dst,
                                                        int32_t* __restrict__ pos_dst, const TAB tab) {
  const int block = blockIdx.x;
  const int seg = find_segment_wave(tab.nseg, block, [&](int s) { return tab.w[2][s]; });
  const int first = (block - tab.w[2][seg]) * kBlockRows;
  const int dst0 = tab.w[1][seg], start = tab.w[0][seg];
  const int n = rows_in_use(c.lengths, tab.seg0 + seg, tab.w[0][seg + 1] - start);
  const int take = min(n, tab.w[1][seg + 1] - dst0);
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

constexpr int kEvictThreads = 1024, kEvictEach = 4;
template <int N>
using EvictTab = SegWords<N, 3>;      // w[0] room of the segment, w[1] its room in the other cache, w[2] max(C_h, w)

__device__ __forceinline__ uint32_t weight_key(float v) { return v != v ? 0xffffffffu : float_key(v); }

// Rows that stay, as row numbers inside the segment, ascending.  A workgroup per segment: the cap - w largest keys by three digits of 11, 11 and 10
// bits, from the largest; then the kept ones in order, a tile of rows at a time.
template <class TAB>
__global__ __launch_bounds__(kEvictThreads) void evict_select_kernel(const float* __restrict__ weight, const int32_t* lengths, int32_t* lengths_out, int w,
                                                                     int32_t* __restrict__ list, const TAB tab) {
  __shared__ uint32_t hist[kHistBins], scan[16], res[2];
  const int seg = blockIdx.x, tid = threadIdx.x;
  const int start = tab.w[0][seg], cap = tab.w[2][seg];
  const int n = rows_in_use(lengths, tab.seg0 + seg, tab.w[0][seg + 1] - start);
  list += tab.w[1][seg];
  const int kept = min(n, cap);
  __syncthreads();                                    // every thread has read the length: it may be the same word
  if (tid == 0) lengths_out[tab.seg0 + seg] = kept;
  if (n <= cap) {
    for (int i = tid; i < n; i += kEvictThreads) list[i] = i;
    return;
  }
  const int m = n - w, want = cap - w;
  for (int i = tid; i < w; i += kEvictThreads) list[want + i] = m + i;
  if (want == 0) return;
  const float* keys = weight + start;
  uint32_t prefix = 0, k = (uint32_t)want;
#pragma unroll
  for (int level = 0; level < 3; ++level) {
    const int shift = level == 0 ? 21 : level == 1 ? 10 : 0, bits = level == 2 ? 10 : 11;
    for (int i = tid; i < kHistBins; i += kEvictThreads) hist[i] = 0;
    __syncthreads();
    for (int i = tid; i < m; i += kEvictThreads) {
      const uint32_t key = weight_key(keys[i]);
      if (level == 0 || key >> (shift + bits) == prefix) atomicAdd(&hist[key >> shift & ((1u << bits) - 1u)], 1u);
    }
    __syncthreads();
    select_bin<kEvictThreads>(hist, k, scan, res);
    prefix = prefix << bits | res[0];
    k = res[1];
    __syncthreads();
  }
  // prefix: the smallest kept key, of which the first k stay
  uint32_t equal = 0, out = 0;
  for (int base = 0; base < m; base += kEvictThreads * kEvictEach) {
    uint32_t key[kEvictEach], gt = 0, eq = 0;
#pragma unroll
    for (int j = 0; j < kEvictEach; ++j) {
      const int i = base + tid * kEvictEach + j;
      key[j] = i < m ? weight_key(keys[i]) : 0u;
      const bool in = i < m;
      gt += in && key[j] > prefix;
      eq += in && key[j] == prefix;
    }
    const uint32_t incl = block_incl_scan<kEvictThreads>(gt | eq << 16, scan);
    uint32_t e = equal + (incl >> 16) - eq, g = (incl & 0xffffu) - gt;
    // kept before this thread's rows: the larger ones, and of the equal ones the first k
    uint32_t at = out + g + (min(e, k) - min(equal, k));
#pragma unroll
    for (int j = 0; j < kEvictEach; ++j) {
      const int i = base + tid * kEvictEach + j;
      if (i >= m) continue;
      if (key[j] > prefix || (key[j] == prefix && e < k)) list[at++] = i;
      e += key[j] == prefix;
    }
    if (tid == kEvictThreads - 1) {
      res[0] = incl & 0xffffu;
      res[1] = incl >> 16;
    }
    __syncthreads();
    out += res[0] + (min(equal + res[1], k) - min(equal, k));
    equal += res[1];
    __syncthreads();
  }
}

// The kept rows' bytes.  Bound by memory.
template <class TAB>
__global__ __launch_bounds__(kThreads) void evict_copy_kernel(const CacheArrays in, const CacheArrays out, const int32_t* __restrict__ list, int32_t* __restrict__ kept_idx,
                                                              int row_bytes, int scale_bytes, const TAB tab) {
  const int block = blockIdx.x;
  const int seg = find_segment_wave(tab.nseg, block, [&](int s) { return tab.w[2][s]; });
  const int first = (block - tab.w[2][seg]) * kBlockRows;
  const int start = tab.w[0][seg], dst0 = tab.w[1][seg];
  const int rows = min(rows_in_use(out.lengths, tab.seg0 + seg, tab.w[1][seg + 1] - dst0) - first, kBlockRows);
  if (rows <= 0) return;
  __shared__ int32_t from[kBlockRows];
  if ((int)threadIdx.x < rows) from[threadIdx.x] = list[dst0 + first + (int)threadIdx.x];
  __syncthreads();
  const int64_t to0 = (int64_t)dst0 + first;
  const int units = row_bytes / 16;
  for (int i = threadIdx.x; i < rows * units * 2; i += kThreads) {
    const int u = i % units, r = i / units % rows, isv = i / (units * rows);
    const int64_t s = (int64_t)start + from[r];
    const unsigned char* src = isv ? in.v : in.k;
    unsigned char* dst = isv ? out.v : out.k;
    *(u32x4*)(dst + (to0 + r) * row_bytes + u * 16) = *(const u32x4*)(src + s * row_bytes + u * 16);
  }
  if (scale_bytes)
    for (int i = threadIdx.x; i < rows * scale_bytes * 2; i += kThreads) {
      const int u = i % scale_bytes, r = i / scale_bytes % rows, isv = i / (scale_bytes * rows);
      const unsigned char* src = isv ? in.v_scale : in.k_scale;
      unsigned char* dst = isv ? out.v_scale : out.k_scale;
      dst[(to0 + r) * scale_bytes + u] = src[((int64_t)start + from[r]) * scale_bytes + u];
    }
  if ((int)threadIdx.x < rows) {
    const int64_t s = (int64_t)start + from[threadIdx.x], t = to0 + (int)threadIdx.x;
    if (in.pos && out.pos) out.pos[t] = in.pos[s];
    if (out.weight) out.weight[t] = in.weight[s];
    if (kept_idx) kept_idx[t] = from[threadIdx.x];
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
      for_tables<RowsTab, kManySegs3, 2>(
          S, [&](int64_t s, int r) { return (int32_t)(r == 0 ? desc->h_offsets[s] : h_src_offsets[s]); },
          [&](int64_t s) { return std::max<int64_t>(1, ceil_div(h_src_offsets[s + 1] - h_src_offsets[s], kBlockRows)); },
          [&](const auto& tab, int blocks) {
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
      for_tables<RowsTab, kManySegs3, 2>(
          S, [&](int64_t s, int r) { return (int32_t)(r == 0 ? desc->h_offsets[s] : h_out_offsets[s]); },
          [&](int64_t s) { return ceil_div(std::min(h_out_offsets[s + 1] - h_out_offsets[s], desc->h_offsets[s + 1] - desc->h_offsets[s]), kBlockRows); },
          [&](const auto& tab, int blocks) {
            SLKV_LAUNCH((rows_kernel<decltype(kind)::value, decltype(dim)::value, std::decay_t<decltype(tab)>>), dim3(blocks), dim3(kThreads), 0,
                        (hipStream_t)hip_stream, arrays_of(cache), (unsigned char*)d_k_rows, (unsigned char*)d_v_rows, d_pos_rows, tab);
          });
    });
  });
  return launch_status("rows");
}

extern "C" slkv_status slkv_evict_workspace_bytes(const slkv_cache_desc* desc, const slkv_cache_desc* out_desc, int32_t w, const int32_t* h_budgets, size_t* bytes) {
  clear_error();
  if (!bytes) return fail(SLKV_ERR_NULL, "bytes is NULL");
  slkv_status st = evict_checks(desc, out_desc, w, h_budgets);
  if (st != SLKV_OK) return st;
  *bytes = std::max<size_t>(16, (size_t)out_desc->h_offsets[(int64_t)desc->B * desc->Hkv] * sizeof(int32_t));
  return SLKV_OK;
}

extern "C" slkv_status slkv_evict_cache(const slkv_cache_desc* desc, const slkv_cache* cache, const slkv_cache_desc* out_desc, const slkv_cache* out,
                                        int32_t w, const int32_t* h_budgets, int32_t* d_kept_idx,
                                        void* d_workspace, size_t workspace_bytes, void* hip_stream) {
  clear_error();
  slkv_status st = evict_checks(desc, out_desc, w, h_budgets);
  if (st != SLKV_OK) return st;
  if ((st = validate_cache(desc, cache)) != SLKV_OK) return st;
  if ((st = validate_cache(out_desc, out, "out")) != SLKV_OK) return st;
  const int64_t S = (int64_t)desc->B * desc->Hkv, rows_in = desc->h_offsets[S], rows_out = out_desc->h_offsets[S];
  if (!out->d_lengths) return fail(SLKV_ERR_NULL, "out: d_lengths is NULL");
  if (rows_in > desc->h_offsets[0] && !cache->d_weight) return fail(SLKV_ERR_NULL, "cache: d_weight is NULL");
  if (!d_workspace) return fail(SLKV_ERR_NULL, "d_workspace is NULL");
  if ((uintptr_t)d_kept_idx % 16 || (uintptr_t)d_workspace % 16) return fail(SLKV_ERR_BAD_ARG, "device pointer not 16-byte aligned");
  const int64_t row_bytes = (int64_t)desc->d * kind_bits(desc->dtype) / 8, scale_bytes = desc->dtype == SLKV_BF16_KV_MXFP4 ? desc->d / kScaleBlock : 0;
  // a segment's shorter room may never hold cap rows
  auto cap_of = [&](int64_t s) { return std::max(h_budgets[s % desc->Hkv], w); };
  auto most_of = [&](int64_t s) { return std::min<int64_t>(desc->h_offsets[s + 1] - desc->h_offsets[s], cap_of(s)); };
  for (int64_t s = 0; s < S; ++s)
    if (out_desc->h_offsets[s + 1] - out_desc->h_offsets[s] < most_of(s))
      return fail(SLKV_ERR_CAPACITY, "segment %lld: up to %lld rows into a room of %lld", (long long)s, (long long)most_of(s),
                  (long long)(out_desc->h_offsets[s + 1] - out_desc->h_offsets[s]));
  const void* ins[] = {cache->d_k, cache->d_v, cache->d_k_scale, cache->d_v_scale, cache->d_pos, cache->d_weight, cache->d_lengths};
  const void* outs[] = {out->d_k, out->d_v, out->d_k_scale, out->d_v_scale, out->d_pos, out->d_weight, out->d_lengths};
  const int64_t each[] = {row_bytes, row_bytes, scale_bytes, scale_bytes, 4, 4, 0};
  for (int i = 0; i < 7; ++i)
    for (int j = 0; j < 7; ++j)
      if (!(i == 6 && j == 6 && ins[i] == outs[j]) &&
          overlap(ins[i], outs[j], i == 6 ? 4 * S : rows_in * each[i], j == 6 ? 4 * S : rows_out * each[j]))
        return fail(SLKV_ERR_BAD_ARG, "arrays of cache and out overlap");
  size_t need = 0;
  if ((st = slkv_evict_workspace_bytes(desc, out_desc, w, h_budgets, &need)) != SLKV_OK) return st;
  if (workspace_bytes < need) return fail(SLKV_ERR_WORKSPACE, "workspace %zu < %zu bytes", workspace_bytes, need);
  ScopedKernelTimer timer(SLKV_K_EVICT);
  hipStream_t const stream = (hipStream_t)hip_stream;
  int32_t* const list = (int32_t*)d_workspace;
  for_tables<EvictTab, kManySegs3, -1>(
      S, [&](int64_t s, int r) { return r == 0 ? (int32_t)desc->h_offsets[s] : r == 1 ? (int32_t)out_desc->h_offsets[s] : s < S ? cap_of(s) : 0; },
      [&](int64_t) { return 1; },
      [&](const auto& tab, int segs) {
        SLKV_LAUNCH((evict_select_kernel<std::decay_t<decltype(tab)>>), dim3(segs), dim3(kEvictThreads), 0, stream, cache->d_weight, cache->d_lengths,
                    out->d_lengths, w, list, tab);
      });
  for_tables<RowsTab, kManySegs3, 2>(
      S, [&](int64_t s, int r) { return (int32_t)(r == 0 ? desc->h_offsets[s] : out_desc->h_offsets[s]); },
      [&](int64_t s) { return ceil_div(most_of(s), kBlockRows); },
      [&](const auto& tab, int blocks) {
        SLKV_LAUNCH((evict_copy_kernel<std::decay_t<decltype(tab)>>), dim3(blocks), dim3(kThreads), 0, stream, arrays_of(cache), arrays_of(out), list,
                    d_kept_idx, (int)row_bytes, (int)scale_bytes, tab);
      });
  return launch_status("evict");
}
