// Attention of a tree of drafted tokens over a cache (slkv_attend_tree).
#include "attend_tiles.h"

#include <algorithm>

namespace slkv {

// ------------------------------------------------------------------ attention

// Segments of a launch: first rows of their rooms, the order in which they are launched, and how many parts come before every 16th of it; a segment has
// max(1, ceil(room / each)).  Workgroups: parts, in each of them the tiles of queries.
template <int N>
struct TreeTab {
  static constexpr bool kOneNumber = false;            // of the queries' type a weight
  static constexpr int kSegs = N, kGroup = 16, kGroups = (N + kGroup - 1) / kGroup;
  static_assert(kGroups <= kWave, "a lane for every group");
  const unsigned char *k, *v, *k_scale, *v_scale, *q;
  unsigned char* out;
  float* lse;
  const uint64_t* sees;
  const int32_t* lengths;
  int32_t nseg, seg0, hkv, each;
  struct Words {
    int32_t start[N + 1], before[kGroups];
    uint16_t order[N];
  } words;

  // segment, tile of queries, part; of the segment: first row and room, parts, parts of others before its own
  struct Place { int s, tile, part, at, room, parts, first; };
  template <int QUERIES>
  __device__ __forceinline__ Place locate(const TileArgs& a, const Words& t, int block) const {
    const int tiles = (a.G * a.T + QUERIES - 1) / QUERIES, part_id = block / tiles, lane = threadIdx.x % kWave;
    const int groups = (nseg + kGroup - 1) / kGroup;
    const int b0 = t.before[min(lane, groups - 1)];
    const int grp = __popcll(__ballot(lane < groups && b0 <= part_id)) - 1;
    const int in_group = t.order[min(grp * kGroup + min(lane, kGroup - 1), nseg - 1)];
    const int at_lane = t.start[in_group], room_lane = t.start[in_group + 1] - at_lane;
    const bool in = lane < kGroup && grp * kGroup + lane < nseg;
    const int parts_lane = in ? max(1, (room_lane + each - 1) / each) : 0;
    const int first_lane = __builtin_amdgcn_readlane(b0, grp) + (int)wave_incl_scan((uint32_t)parts_lane) - parts_lane;
    const int which = __popcll(__ballot(in && first_lane <= part_id)) - 1;
    const int first = __builtin_amdgcn_readlane(first_lane, which);
    return Place{__builtin_amdgcn_readlane(in_group, which), block - part_id * tiles, part_id - first, __builtin_amdgcn_readlane(at_lane, which),
                 __builtin_amdgcn_readlane(room_lane, which), __builtin_amdgcn_readlane(parts_lane, which), first};
  }

  template <int QUERIES, int KEYS, int D, int KIND>
  __device__ __forceinline__ TileWork describe(const TileArgs& a, const Words&, const Place& p) const {
    const int seg = seg0 + p.s, b = seg / hkv, h = seg % hkv, at = p.at, room = p.room, parts = p.parts;
    const int tiles = (a.G * a.T + QUERIES - 1) / QUERIES;
    constexpr int kRow = D * Kind<KIND>::kBits / 8, kWide = D * (int)sizeof(typename Kind<KIND>::wide), kScales = D / kScaleBlock;
    TileWork w;
    w.part = p.part;
    w.rows = a.G * a.T;
    w.r0 = p.tile * QUERIES;
    const int n = __builtin_amdgcn_readfirstlane(rows_in_use(lengths, seg, room));
    w.hist = n - a.T;
    // the rows in use are spread over the parts of the room
    const int steps = (n + KEYS - 1) / KEYS, each = (steps + parts - 1) / parts * KEYS;
    w.parts = each ? (n + each - 1) / each : 1;
    w.begin = w.part * each;
    w.end = min(n, w.begin + each);
    w.k = k + (int64_t)at * kRow;
    w.v = v + (int64_t)at * kRow;
    w.ks = KIND == SLKV_BF16_KV_MXFP4 ? k_scale + (int64_t)at * kScales : nullptr;
    w.vs = KIND == SLKV_BF16_KV_MXFP4 ? v_scale + (int64_t)at * kScales : nullptr;
    const int64_t head = ((int64_t)b * hkv + h) * a.G;
    w.q = q + head * a.T * kWide;
    w.out = out + head * a.T * kWide;
    w.lse = lse ? lse + head * a.T : nullptr;
    w.sees = sees + (int64_t)b * a.T;
    w.q_tok = w.o_tok = kWide;
    w.q_head = w.o_head = (int64_t)a.T * kWide;
    w.lse_head = a.T;
    w.k_row = w.v_row = kRow;
    w.slot0 = p.first * tiles + p.tile;
    w.slot_step = tiles;
    return w;
  }
};
// The segments with the longest parts first, by sixteenths of the longest.
template <class TAB>
static void order_segments(TAB& t) {
  constexpr int kSteps = 16;
  int from[kSteps + 1] = {};
  uint8_t key[TAB::kSegs];
  auto length = [&](int i) {
    const int64_t room = t.words.start[i + 1] - t.words.start[i], parts = std::max<int64_t>(1, (room + t.each - 1) / t.each);
    return (room + parts - 1) / parts;
  };
  int64_t most = 1;
  for (int i = 0; i < t.nseg; ++i) most = std::max(most, length(i));
  for (int i = 0; i < t.nseg; ++i) ++from[(key[i] = (uint8_t)(kSteps - 1 - length(i) * (kSteps - 1) / most)) + 1];
  for (int k = 0; k < kSteps; ++k) from[k + 1] += from[k];
  for (int i = 0; i < t.nseg; ++i) t.words.order[from[key[i]]++] = (uint16_t)i;
}

static slkv_status tree_checks(const slkv_cache_desc* desc, int32_t T, TreePlan& plan) {
  slkv_status st = validate_cache_desc(desc);
  if (st != SLKV_OK) return st;
  if (T < 1) return fail(SLKV_ERR_BAD_ARG, "T must be >= 1");
  if (T > 64) return fail(SLKV_ERR_UNSUPPORTED, "T = %d > 64", T);
  plan = plan_tree(desc, T);
  if (plan.slots >= (1 << 24)) return fail(SLKV_ERR_UNSUPPORTED, "more than 2^24 workgroups");
  return SLKV_OK;
}

}  // namespace slkv

using namespace slkv;

extern "C" slkv_status slkv_tree_workspace_bytes(const slkv_cache_desc* desc, int32_t T, size_t* bytes) {
  clear_error();
  if (!bytes) return fail(SLKV_ERR_NULL, "bytes is NULL");
  TreePlan p;
  const slkv_status st = tree_checks(desc, T, p);
  if (st != SLKV_OK) return st;
  *bytes = p.bytes;
  return SLKV_OK;
}

extern "C" slkv_status slkv_attend_tree(const slkv_cache_desc* desc, const slkv_cache* cache, int32_t T, const void* d_q, const uint64_t* d_sees, void* d_out,
                                        float* d_lse, void* d_workspace, size_t workspace_bytes, void* hip_stream) {
  clear_error();
  TreePlan p;
  slkv_status st = tree_checks(desc, T, p);
  if (st != SLKV_OK) return st;
  if ((st = validate_cache(desc, cache)) != SLKV_OK) return st;
  if (!d_q || !d_sees || !d_out || !d_workspace) return fail(SLKV_ERR_NULL, "a required device pointer is NULL");
  const void* ptrs[] = {d_q, d_sees, d_out, d_lse, d_workspace};
  for (const void* ptr : ptrs)
    if ((uintptr_t)ptr % 16) return fail(SLKV_ERR_BAD_ARG, "device pointer %p not 16-byte aligned", ptr);
  if (workspace_bytes < p.bytes) return fail(SLKV_ERR_WORKSPACE, "workspace %zu < %zu bytes", workspace_bytes, p.bytes);
  const int64_t S = (int64_t)desc->B * desc->Hkv;
  TileArgs a;
  a.G = desc->Hq / desc->Hkv;
  a.T = T;
  a.c_log2 = kLog2e / std::sqrt((float)desc->d);
  a.part_o = (float*)d_workspace;
  a.part_ml = (float*)((unsigned char*)d_workspace + p.off_ml);
  hipStream_t const stream = (hipStream_t)hip_stream;
  const int64_t tiles = ((int64_t)a.G * T + p.queries - 1) / p.queries;
  auto launch_table = [&](auto t, int64_t s0, int64_t ns) {
    using TAB = decltype(t);
    t.k = (const unsigned char*)cache->d_k, t.v = (const unsigned char*)cache->d_v;
    t.k_scale = (const unsigned char*)cache->d_k_scale, t.v_scale = (const unsigned char*)cache->d_v_scale;
    t.q = (const unsigned char*)d_q, t.out = (unsigned char*)d_out;
    t.lse = d_lse, t.sees = d_sees, t.lengths = cache->d_lengths;
    t.nseg = (int32_t)ns, t.seg0 = (int32_t)s0, t.hkv = desc->Hkv;
    int64_t blocks = 0;
    t.each = (int32_t)p.each;
    for (int64_t i = 0; i <= ns; ++i) t.words.start[i] = (int32_t)desc->h_offsets[s0 + i];
    order_segments(t);
    for (int64_t i = 0; i < ns; ++i) {
      if (i % TAB::kGroup == 0) t.words.before[i / TAB::kGroup] = (int32_t)blocks;
      blocks += tree_parts(desc, s0 + t.words.order[i], p.each);
    }
    blocks *= tiles;
    a.blocks = (int32_t)blocks;
    auto launch = [&](auto kind, auto dim) {
      constexpr int kKind = decltype(kind)::value, kDim = decltype(dim)::value;
      with_shape<kKind, kDim>(p.shape, [&](auto wq, auto wk) {
        constexpr int kWQ = decltype(wq)::value, kWK = decltype(wk)::value;
        {
          ScopedKernelTimer timer(SLKV_K_TREE);
          SLKV_LAUNCH((attend_tiles_kernel<kKind, kDim, kWQ, kWK, TAB>), dim3(std::min((unsigned)blocks, tile_places<Tiles<kKind, kDim, kWQ, kWK>>())), dim3(kWQ * kWK * kWave), 0, stream, a, t);
        }
        if (p.split) {
          ScopedKernelTimer timer(SLKV_K_TILES_JOIN);
          SLKV_LAUNCH((join_tiles_kernel<kKind, kDim, kWQ, kWK, TAB>), dim3((unsigned)blocks, join_slices(p.queries)), dim3(256), 0, stream, a, t);
        }
      });
    };
    with_kind(desc->dtype, [&](auto kind) {
      if (desc->d == 64) launch(kind, std::integral_constant<int, 64>{});
      else launch(kind, std::integral_constant<int, 128>{});
    });
  };
  if (S <= kFewSegs) launch_table(TreeTab<kFewSegs>{}, 0, S);
  else
    for (int64_t s0 = 0; s0 < S; s0 += kTreeSegs) launch_table(TreeTab<kTreeSegs>{}, s0, std::min<int64_t>(kTreeSegs, S - s0));
  return launch_status("attend_tree");
}
