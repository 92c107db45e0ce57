// What becomes of a draft (slkv_accept_cache): the rows of the accepted tokens move together, behind those before the draft, and the weights of the accepted tokens'
// attention are added up.
//
// A segment's workgroups: one for the rows of the draft, which alone reads and writes them, and one for every kWeighRows rows of its room, for the weights of the rows
// before the draft, which every accepted token sees.  The workgroup of the draft sets the length, unless the others read it (drafts behind the rows in use, and weights): a
// launch of its own does so then.
#include "attend_rows.h"
#include "launch.h"

#include <algorithm>
#include <cmath>

namespace slkv {

constexpr int kAcceptThreads = 256, kAcceptWaves = kAcceptThreads / kWave;
constexpr int kWeighEach = 64, kWeighRows = kWeighEach * kAcceptWaves;   // rows of a wave, of a workgroup
constexpr int kMostDraft = 64;

struct AcceptArgs {
  unsigned char *k, *v, *k_scale, *v_scale;
  int32_t *lengths, *pos;
  float* weight;
  const int32_t *path, *at;
  const unsigned char* q;
  const float* lse;                  // NULL: no weights
  float* w_out;
  int32_t T, A, G, hkv;
  int32_t lengths_later;             // a launch of their own sets the lengths
  float c_log2;                      // log2(e) / sqrt(d)
};

// Segments of a launch: first rows of their rooms, and workgroups before every 16th of them.
template <int N>
struct AcceptTab {
  static constexpr int kSegs = N, kGroup = 16, kGroups = (N + kGroup - 1) / kGroup;
  static_assert(kGroups <= kWave, "a lane for every group");
  int32_t nseg, seg0, weights;
  int32_t start[N + 1], before[kGroups];
  struct Place { int seg, block, start, room; };
  __host__ __device__ int blocks_of(int room) const { return 1 + (weights ? (room + kWeighRows - 1) / kWeighRows : 0); }
  // two round trips to the arguments
  __device__ __forceinline__ Place find(int block) const {
    const int lane = threadIdx.x % kWave, groups = (nseg + kGroup - 1) / kGroup;
    const int b0 = before[min(lane, groups - 1)];
    const int grp = __popcll(__ballot(lane < groups && b0 <= block)) - 1, i = min(grp * kGroup + min(lane, kGroup - 1), nseg - 1);
    const int at = start[i], room = start[i + 1] - at, mine = lane < kGroup && grp * kGroup + lane < nseg ? blocks_of(room) : 0;
    const int first = __builtin_amdgcn_readlane(b0, grp) + (int)wave_incl_scan((uint32_t)mine) - mine;
    const int which = __popcll(__ballot(mine && first <= block)) - 1;
    return Place{seg0 + grp * kGroup + which, block - __builtin_amdgcn_readlane(first, which), __builtin_amdgcn_readlane(at, which), __builtin_amdgcn_readlane(room, which)};
  }
};
constexpr int kAcceptSegs = 880;

// The accepted tokens of a segment whose rows are there: lane i has the i-th one's number; the row of token 0, which may be below 0; how many.
struct Accepted { int token, base, count; };
__device__ __forceinline__ Accepted accepted_of(const AcceptArgs& a, int seg, int room, int lane) {
  Accepted r;
  r.base = __builtin_amdgcn_readfirstlane(a.at ? min(max(a.at[seg], 0), room) : rows_in_use(a.lengths, seg, room) - a.T);
  const int p = lane < a.A ? a.path[(int64_t)(seg / a.hkv) * a.A + lane] : -1;
  const uint64_t ends = __ballot(p < 0 || p >= a.T);
  const int length = ends ? __builtin_ctzll(ends) : kWave;             // the path ends at the first number that is none
  const bool there = lane < length && r.base + p >= 0 && r.base + p < room;
  const uint64_t all = __ballot(there);
  const int found = __popcll(all);
  r.count = min(found, room - max(r.base, 0));                         // (a number that comes twice is a row twice: there may not be room for all)
  // (nearly always all of the path)
  int from = lane;
  if (found != length) {
    uint64_t left = all;
    for (int i = 0; i < lane && left; ++i) left &= left - 1;
    from = left ? __builtin_ctzll(left) : 0;
  }
  r.token = __shfl(p, from);
  return r;
}

// Weights of kWeighEach rows from row j0 of a segment on, up to `end`, one wave; those of the draft, from row `drafted` on, are seen by the tokens that were accepted with or
// after them.  tokens: the accepted ones, in LDS.  Bound by latency and by memory: the rows' keys, what they have so far and the first queries are asked for at once, but only behind the path's
// round trips (table, length, path) and a barrier; the next queries a tile ahead.  (256 segments of 2048 E4M3 rows, 8 tokens: 27 us, 3.2 TB/s.  A wave that goes through several times as many rows, the next ones on their way in registers: 31 to 44.)
template <int KIND, int D>
struct Weigh {
  using A = Attend<KIND, D>;
  static constexpr int kSteps = kWeighEach / A::kStep, kProducts = A::kF32 ? D / 4 : D / 32, kEach = A::kEach, kWords = A::kF32 ? kProducts / 4 : kProducts;
  struct Rows { typename A::KRegs k[kSteps]; float had[kSteps]; };      // had: what the rows have so far; lane rq of 16 has its row rq of every step
  struct Query { u32x4 w[kWords]; float lse; int sees; };               // sees: the last row that it sees

  static __device__ __forceinline__ void load(Rows& r, const AcceptArgs& a, int64_t start, int j0, int end) {
    const int lane = threadIdx.x % kWave, rq = lane & 15, g = lane >> 4;
    typename A::Rows rows;
    rows.k = A::buffer(a.k, start + j0, end - j0, A::kRowBytes);
    if constexpr (KIND == SLKV_BF16_KV_MXFP4) rows.ks = A::buffer(a.k_scale, start + j0, end - j0, A::kScales);
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      const typename A::Place place = A::place_of(s, lane);
      A::load_k(r.k[s], rows, place);
    }
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      const int row = j0 + s * A::kStep + g * kEach + rq;
      r.had[s] = a.weight && rq < kEach && row < end ? a.weight[start + row] : 0.f;
    }
  }

  static __device__ __forceinline__ void add(const Rows& rows, const AcceptArgs& a, int seg, int64_t start, int j0, int end, int drafted, int count, const int* tokens) {
    const int lane = threadIdx.x % kWave, rq = lane & 15, g = lane >> 4, R = count * a.G;
    float w[kSteps][kEach];
#pragma unroll
    for (int s = 0; s < kSteps; ++s)
#pragma unroll
      for (int j = 0; j < kEach; ++j) w[s][j] = 0.f;
    const bool tail = j0 + kWeighEach > drafted;
    Query ahead;
    auto load_queries = [&](int r0) __attribute__((always_inline)) {
      const int r = min(r0 + rq, R - 1), i = divide(r, a.G);
      const int64_t query = ((int64_t)seg * a.G + (r - i * a.G)) * a.T + tokens[i];
      const unsigned char* p = a.q + query * (D * (int)sizeof(typename A::wide));
#pragma unroll
      for (int u = 0; u < kWords; ++u) ahead.w[u] = *(const u32x4*)(p + (A::kF32 ? A::dim_of(u * 4, g) * 4 : A::dim_of(u, g) * 2));
      ahead.lse = a.lse[query];
      ahead.sees = drafted + i;
    };
    if (R > 0) load_queries(0);
    for (int r0 = 0; r0 < R; r0 += 16) {
      const Query now = ahead;
      if (r0 + 16 < R) load_queries(r0 + 16);
      // a query that saw nothing has no weights, whatever its products are; nor has one that is not there
      const float l2 = now.lse * kLog2e;
      const int sees = now.lse == -INFINITY || r0 + rq >= R ? -1 : tail ? now.sees : INT32_MAX;
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        f32x4 x[A::kTiles];
        if constexpr (A::kF32) {
          // several sums side by side: one chain of D/4 additions is what the result's error comes from
          f32x4 y[4];
#pragma unroll
          for (int c = 0; c < 4; ++c) y[c] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int u = 0; u < kProducts; ++u)
            y[u % 4] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(rows.k[s].w[0][u]), __uint_as_float(now.w[u / 4][u % 4]), y[u % 4], 0, 0, 0);
          x[0] = (y[0] + y[1]) + (y[2] + y[3]);
        } else {
#pragma unroll
          for (int t = 0; t < A::kTiles; ++t) {
            x[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int u = 0; u < kProducts; ++u) x[t] = A::mfma(A::k_operand(rows.k[s], t, u), now.w[u], x[t]);
          }
        }
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
          const float e = exp2_fast(fmaf(x[j / 4][j % 4], a.c_log2, -l2));
          w[s][j] += j0 + s * A::kStep + g * kEach + j <= sees ? e : 0.f;
        }
      }
    }
    // over the 16 queries of a row of lanes; lane rq of it gets its row rq
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      float mine = 0.f;
#pragma unroll
      for (int j = 0; j < kEach; ++j) {
        const float sum = reduce_lanes(w[s][j], 16, [](float x, float y) { return x + y; });
        if (j == rq) mine = sum;
      }
      const int row = j0 + s * A::kStep + g * kEach + rq;
      if (rq < kEach && row < end) a.w_out[start + row] = rows.had[s] + mine;
    }
  }

  static __device__ __forceinline__ void run(const AcceptArgs& a, int seg, int64_t start, int j0, int end, int drafted, int count, const int* tokens) {
    if (j0 >= end) return;
    Rows rows;
    load(rows, a, start, j0, end);
    add(rows, a, seg, start, j0, end, drafted, count, tokens);
  }
};

template <int KIND, int D, class TAB>
__global__ __launch_bounds__(kAcceptThreads) void accept_kernel(const AcceptArgs a, const TAB tab) {
  constexpr int kRow = D * Kind<KIND>::kBits / 8, kUnits = kRow / 16, kScales = D / kScaleBlock;
  constexpr int kMoves = (kMostDraft * kUnits + kAcceptThreads - 1) / kAcceptThreads;   // 16-byte units of K a thread moves
  __shared__ int sh_token[kMostDraft], sh_base, sh_count;
  const typename TAB::Place place = tab.find((int)blockIdx.x);
  const int seg = place.seg, block = place.block, start = place.start, room = place.room;
  const int tid = threadIdx.x, lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  if (tid < kWave) {
    const Accepted r = accepted_of(a, seg, room, lane);
    sh_token[lane] = r.token;
    if (lane == 0) sh_base = r.base, sh_count = r.count;
  }
  __syncthreads();
  const int base = __builtin_amdgcn_readfirstlane(sh_base), count = __builtin_amdgcn_readfirstlane(sh_count), to = max(base, 0);
  if (block > 0) {                                     // rows before the draft
    const int j0 = (block - 1) * kWeighRows + wave * kWeighEach;
    Weigh<KIND, D>::run(a, seg, start, j0, min(to, j0 + kWeighEach), to, count, sh_token);
    return;
  }
  // All rows are read before one is written: the path may go through the rows in any order, and more than once through one.
  const int64_t from0 = (int64_t)start + base, to0 = (int64_t)start + to;
  u32x4 k[kMoves], v[kMoves];
  uint32_t scales[2][kScales];
  int32_t pos = 0;
  float weight = 0.f;
#pragma unroll
  for (int i = 0; i < kMoves; ++i) {
    const int u = tid + i * kAcceptThreads, row = u / kUnits;
    if (row < count) {
      const int64_t at = (from0 + sh_token[row]) * kRow + u % kUnits * 16;
      k[i] = *(const u32x4*)(a.k + at);
      v[i] = *(const u32x4*)(a.v + at);
    }
  }
  if (tid < count) {
    const int64_t row = from0 + sh_token[tid];
    if constexpr (KIND == SLKV_BF16_KV_MXFP4) {
#pragma unroll
      for (int c = 0; c < kScales; ++c) scales[0][c] = a.k_scale[row * kScales + c], scales[1][c] = a.v_scale[row * kScales + c];
    }
    if (a.pos) pos = a.pos[row];
    if (a.weight) weight = a.weight[row];
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kMoves; ++i) {
    const int u = tid + i * kAcceptThreads, row = u / kUnits;
    if (row < count) {
      const int64_t at = (to0 + row) * kRow + u % kUnits * 16;
      *(u32x4*)(a.k + at) = k[i];
      *(u32x4*)(a.v + at) = v[i];
    }
  }
  if (tid < count) {
    const int64_t row = to0 + tid;
    if constexpr (KIND == SLKV_BF16_KV_MXFP4) {
#pragma unroll
      for (int c = 0; c < kScales; ++c) a.k_scale[row * kScales + c] = (uint8_t)scales[0][c], a.v_scale[row * kScales + c] = (uint8_t)scales[1][c];
    }
    if (a.pos) a.pos[row] = pos;
    if (a.weight) a.weight[row] = weight;
  }
  if (!a.lengths_later && tid == 0) a.lengths[seg] = to + count;
  if (!a.lse) return;
  __threadfence_block();
  __syncthreads();
  if (wave == 0) Weigh<KIND, D>::run(a, seg, start, to, to + count, to, count, sh_token);
}

template <class TAB>
__global__ __launch_bounds__(kAcceptThreads) void lengths_kernel(const AcceptArgs a, const TAB tab) {
  const int i = blockIdx.x * kAcceptWaves + __builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave));
  if (i >= tab.nseg) return;
  const int seg = tab.seg0 + i, lane = threadIdx.x % kWave;
  const Accepted r = accepted_of(a, seg, tab.start[i + 1] - tab.start[i], lane);
  if (lane == 0) a.lengths[seg] = max(r.base, 0) + r.count;
}

}  // namespace slkv

using namespace slkv;

extern "C" slkv_status slkv_accept_cache(const slkv_cache_desc* desc, const slkv_cache* cache, int32_t T, int32_t A, const int32_t* d_path, const int32_t* d_at,
                                         const void* d_q, const float* d_lse, float* d_weight_out, void* hip_stream) {
  clear_error();
  slkv_status st = validate_cache_desc(desc);
  if (st != SLKV_OK) return st;
  if ((st = validate_cache(desc, cache)) != SLKV_OK) return st;
  if (!cache->d_lengths) return fail(SLKV_ERR_NULL, "cache: d_lengths is NULL");
  if (T < 1 || A < 1) return fail(SLKV_ERR_BAD_ARG, "T and A must be >= 1");
  if (T > kMostDraft || A > kMostDraft) return fail(SLKV_ERR_UNSUPPORTED, "T = %d or A = %d > %d", T, A, kMostDraft);
  if (desc->Hq / desc->Hkv > (1 << 14)) return fail(SLKV_ERR_UNSUPPORTED, "Hq/Hkv = %d > 2^14", desc->Hq / desc->Hkv);
  if (!d_path) return fail(SLKV_ERR_NULL, "d_path is NULL");
  if ((d_q == nullptr) != (d_lse == nullptr) || (d_q == nullptr) != (d_weight_out == nullptr))
    return fail(SLKV_ERR_NULL, "d_q, d_lse and d_weight_out are given together");
  const void* ptrs[] = {d_path, d_at, d_q, d_lse, d_weight_out};
  for (const void* ptr : ptrs)
    if ((uintptr_t)ptr % 16) return fail(SLKV_ERR_BAD_ARG, "device pointer %p not 16-byte aligned", ptr);
  AcceptArgs a;
  a.k = (unsigned char*)cache->d_k, a.v = (unsigned char*)cache->d_v;
  a.k_scale = (unsigned char*)cache->d_k_scale, a.v_scale = (unsigned char*)cache->d_v_scale;
  a.lengths = cache->d_lengths, a.pos = cache->d_pos, a.weight = cache->d_weight;
  a.path = d_path, a.at = d_at;
  a.q = (const unsigned char*)d_q, a.lse = d_lse, a.w_out = d_weight_out;
  a.T = T, a.A = A, a.G = desc->Hq / desc->Hkv, a.hkv = desc->Hkv;
  a.c_log2 = kLog2e / std::sqrt((float)desc->d);
  hipStream_t const stream = (hipStream_t)hip_stream;
  const int64_t S = (int64_t)desc->B * desc->Hkv;
  // (a workgroup reads its own segment's number alone before it sets the length)
  if (d_at && d_at != cache->d_lengths && d_at < cache->d_lengths + S && cache->d_lengths < d_at + S)
    return fail(SLKV_ERR_BAD_ARG, "d_at overlaps d_lengths and is not d_lengths itself");
  // (a row's weight is read and written by the same thread; rows of a segment in no order)
  const int64_t rows = desc->h_offsets[S] - desc->h_offsets[0];
  if (d_weight_out && cache->d_weight && d_weight_out != cache->d_weight && d_weight_out < cache->d_weight + rows && cache->d_weight < d_weight_out + rows)
    return fail(SLKV_ERR_BAD_ARG, "d_weight_out overlaps the cache's weights and is not these themselves");
  a.lengths_later = d_q && (!d_at || d_at == cache->d_lengths);
  auto launch = [&](auto tab, int64_t s0, int64_t ns) {
    using TAB = decltype(tab);
    tab.nseg = (int32_t)ns, tab.seg0 = (int32_t)s0, tab.weights = d_q != nullptr;
    int64_t blocks = 0;
    for (int64_t i = 0; i <= ns; ++i) tab.start[i] = (int32_t)desc->h_offsets[s0 + i];
    for (int64_t i = 0; i < ns; ++i) {
      if (i % TAB::kGroup == 0) tab.before[i / TAB::kGroup] = (int32_t)blocks;
      blocks += tab.blocks_of(tab.start[i + 1] - tab.start[i]);
    }
    with_kind(desc->dtype, [&](auto kind) {
      auto with_dim = [&](auto dim) {
        ScopedKernelTimer timer(SLKV_K_ACCEPT);
        SLKV_LAUNCH((accept_kernel<decltype(kind)::value, decltype(dim)::value, TAB>), dim3((unsigned)blocks), dim3(kAcceptThreads), 0, stream, a, tab);
      };
      if (desc->d == 64) with_dim(std::integral_constant<int, 64>{});
      else with_dim(std::integral_constant<int, 128>{});
    });
    if (a.lengths_later) {
      ScopedKernelTimer timer(SLKV_K_ACCEPT);
      SLKV_LAUNCH((lengths_kernel<TAB>), dim3((unsigned)((ns + kAcceptWaves - 1) / kAcceptWaves)), dim3(kAcceptThreads), 0, stream, a, tab);
    }
  };
  if (S <= kFewSegs) launch(AcceptTab<kFewSegs>{}, 0, S);
  else
    for (int64_t s0 = 0; s0 < S; s0 += kAcceptSegs) launch(AcceptTab<kAcceptSegs>{}, s0, std::min<int64_t>(kAcceptSegs, S - s0));
  return launch_status("accept");
}
