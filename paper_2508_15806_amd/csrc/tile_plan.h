// Which workgroups a call of slkv_attend_prompt or slkv_attend_tree gets: host arithmetic alone, without HIP, so that a host compiler builds it by itself.
#ifndef SLKV_TILE_PLAN_H
#define SLKV_TILE_PLAN_H

#include <algorithm>
#include <cmath>
#include <cstddef>

#include "slkv_internal.h"

namespace slkv {

// Waves of a workgroup: along the queries, along the keys of a staged tile.
struct TileShape { int wq, wk; };
constexpr TileShape kTileShapes[] = {{1, 4}, {2, 2}, {4, 1}, {4, 2}, {8, 1}};
constexpr int kTileShapeCount = 5;
inline int tile_queries(int shape) { return 32 * kTileShapes[shape].wq; }
// fp32 has two shapes: others do not fit LDS or registers.  d = 64 has no use for the last one (8192 tokens in fp16: 402 us, 348 in shape 2).
constexpr bool has_shape(int dtype, int d, int shape) { return dtype == SLKV_F32 ? shape == 1 || shape == 2 : d != 64 || shape != 4; }

// What a call consists of in a shape: workgroups without parts, keys of all and of the longest.
struct TileLoad { double tiles, keys, longest; };
struct TileChoice { int shape; int64_t each; };        // each: keys of a part, at most

// The shape and the parts that should be done first.  A workgroup takes kBegin us and, for every 64 keys (128: shape 0), alone[shape] us on a CU that it has to itself, loaded[shape] where all places are
// taken; longer where nobody else reads the same rows.  The keys and values of all segments (bytes) come at 4.8 TB/s at best; parts cost a second launch, and their sums are written and read.
// (The figures are those of one 16-bit number a weight.  With two, full chips take 1.36 times as long in shapes 2 and 4, 1.2 in 1 and 3, 1.1 in 0, and with figures to match the rule chose worse: 4096 tokens in shape 2.
// us, bf16, d = 128, 32 heads, 8 KV heads: 32768 tokens in shape 4 10600, in 2 10600, in 3 11920, in 1 12140; 4096: 180, 192, in shape 1 222; 1024: 30 in shape 2, 26 in shape 1, 47 in shape 0; 130: 9.0, 8.6, 8.1;
// 128 queries a segment on 128 segments of 1056 rows: 34 in shape 3, 36 in shape 2, in two parts 33 and 35, in four 46 and 40; 64 on 512 segments of 1040 MXFP4 rows: 39 in shape 1 whole, 58 in two parts.)
template <class LOAD>
TileChoice choose_tiles(int dtype, int d, int64_t rows, int64_t segments, double bytes, LOAD load) {
  constexpr double kBegin = 5.5, kJoin = 6;
  constexpr double kShared[] = {1.45, 0.85, 1.25, 1.2, 1.9}, kStreaming[] = {1.8, 1.5, 1.9, 1.4, 2.1}, kLoaded[] = {1.45, 1.24, 1.94, 1.2, 1.9};
  constexpr int kKeys[] = {128, 64, 64, 64, 64}, kPlaces[] = {1, 2, 2, 1, 1};
  const bool f32 = dtype == SLKV_F32, narrow = kind_bits(dtype) < 16;
  TileChoice best{2, 1};
  double least = 1e300;
  for (int s = 0; s < kTileShapeCount; ++s) {
    if (!has_shape(dtype, d, s)) continue;
    if (s > 0 && rows <= tile_queries(s) / 2 && !(f32 && s == 1)) continue;   // (no more waves than queries)
    const TileLoad l = load(tile_queries(s));
    const double scale = (f32 ? (d == 64 ? 4 : 8) * (s == 1 ? 0.78 : 1) : d == 64 ? 0.55 : 1) * (narrow ? 1.2 : 1);
    const double alone = (l.tiles < 4.0 * segments && !f32 ? kStreaming[s] : kShared[s]) * scale, loaded = f32 ? alone : std::max(kLoaded[s] * scale, alone) * (narrow && s == 0 ? 2 : 1);
    const double places = 256.0 * (f32 ? 1 : narrow && s == 0 ? 2 : kPlaces[s]);
    const bool even = l.keys > 0.95 * l.longest * l.tiles;
    for (int parts = 1; parts <= 256; parts += parts < 4 ? 1 : parts / 2) {
      const double each = std::ceil(std::ceil(l.longest / parts) / kKeys[s]) * kKeys[s];
      const double groups = l.tiles * (parts == 1 ? 1 : even ? std::ceil(l.longest / each) : std::max(1.0, l.keys / l.tiles / each + 0.4));
      const double steps = l.keys / kKeys[s] + 1.2 * groups, mean = std::min(1.0, steps / groups / (each / kKeys[s]));
      const double one = each / kKeys[s] * (groups <= 256 ? alone : alone + (loaded - alone) * mean);
      // (more workgroups than places: the last ones begin late; parts are about equal, whole tiles the longest first)
      const double all = steps * loaded / places + (groups <= places ? 0 : parts > 1 ? 0.5 * one : 0.1 * one);
      double us = kBegin + std::max(std::max(one, all), bytes / 4.8e6 + (parts > 1 || l.tiles < places ? 0.2 * one : 0));
      if (parts > 1) us += kJoin + groups * tile_queries(s) * d * 8 / 6e6;
      if (us < least) least = us, best = TileChoice{s, (int64_t)std::max(each, 1.0)};
      if (each <= kKeys[s]) break;
    }
  }
  return best;
}

// Workgroups of a part that join tiles.
inline unsigned join_slices(int queries) { return (unsigned)std::max(1, queries / 32); }

constexpr int kPromptSeqs = 64;      // sequences of a launch
constexpr int kTreeSegs = 600;       // segments of a launch

struct PromptPlan {
  int shape;                         // waves and tiles of a workgroup
  int queries;                       // rows of a workgroup's tile
  int64_t each;                      // keys of a part, about
  int64_t slots;                     // workgroups of a launch, the most
  bool split;
  size_t off_ml, bytes;
};

inline int64_t seq_tiles(const slkv_prompt_desc* d, int64_t b, int queries) {
  return ((d->h_cu_q[b + 1] - d->h_cu_q[b]) * (d->Hq / d->Hkv) + queries - 1) / queries;
}
inline const int64_t* cu_k_of(const slkv_prompt_desc* d) { return d->h_cu_k ? d->h_cu_k : d->h_cu_q; }
inline int64_t seq_parts(const slkv_prompt_desc* d, int64_t b, int64_t each) {
  return std::max<int64_t>(1, (cu_k_of(d)[b + 1] - cu_k_of(d)[b] + each - 1) / each);
}

inline PromptPlan plan_prompt(const slkv_prompt_desc* d) {
  PromptPlan p;
  const int64_t G = d->Hq / d->Hkv;
  const int64_t* ck = cu_k_of(d);
  int64_t rows = 0, kv = 0;
  for (int64_t b = 0; b < d->B; ++b) rows = std::max(rows, (d->h_cu_q[b + 1] - d->h_cu_q[b]) * G), kv += ck[b + 1] - ck[b];
  const TileChoice c = choose_tiles(d->dtype, d->d, rows, (int64_t)d->B * d->Hkv, (double)kv * d->Hkv * d->d * kind_bits(d->dtype) / 4, [&](int queries) {
    TileLoad l{0, 0, 1};
    for (int64_t b = 0; b < d->B; ++b) {
      const int64_t t = seq_tiles(d, b, queries) * d->Hkv, n = d->h_cu_q[b + 1] - d->h_cu_q[b], m = ck[b + 1] - ck[b];
      if (!t) continue;
      l.tiles += t;
      l.keys += (double)t * std::max<int64_t>(1, m - n / 2);
      l.longest = std::max(l.longest, (double)m);
    }
    l.tiles = std::max(l.tiles, 1.0);
    return l;
  });
  p.shape = c.shape;
  p.each = c.each;
  p.queries = tile_queries(p.shape);
  p.split = false;
  for (int64_t b = 0; b < d->B; ++b) p.split |= seq_tiles(d, b, p.queries) && seq_parts(d, b, p.each) > 1;
  p.slots = 0;
  for (int64_t b0 = 0; b0 < d->B; b0 += kPromptSeqs) {
    int64_t here = 0;
    for (int64_t b = b0; b < std::min<int64_t>(d->B, b0 + kPromptSeqs); ++b) here += seq_tiles(d, b, p.queries) * d->Hkv * seq_parts(d, b, p.each);
    p.slots = std::max(p.slots, here);
  }
  const size_t o = p.split ? (size_t)p.slots * p.queries * d->d * sizeof(float) : 0;
  p.off_ml = o;
  p.bytes = std::max<size_t>(16, o + (p.split ? (size_t)p.slots * p.queries * 2 * sizeof(float) : 0));
  return p;
}

// Whether the tiles of the launch from sequence b0 on come sequence by sequence, not in the order of their keys.
inline bool prompt_in_order(const slkv_prompt_desc* d, const PromptPlan& p, int64_t b0) {
  const int64_t end = std::min<int64_t>(d->B, b0 + kPromptSeqs), *cq = d->h_cu_q, *ck = cu_k_of(d);
  bool even = true;
  int64_t blocks = 0;
  for (int64_t b = b0; b < end; ++b) {
    even &= cq[b + 1] - cq[b] == cq[b0 + 1] - cq[b0] && ck[b + 1] - ck[b] == ck[b0 + 1] - ck[b0];
    blocks += seq_tiles(d, b, p.queries) * d->Hkv * seq_parts(d, b, p.each);
  }
  return p.split || even || blocks <= 512;             // (looking a tile up in the other order takes 1.5 us)
}

struct TreePlan {
  int shape, queries;
  int64_t each;                      // room rows of a part, at most
  int64_t slots;
  bool split;
  size_t off_ml, bytes;
};

inline int64_t tree_parts(const slkv_cache_desc* d, int64_t s, int64_t each) {
  return std::max<int64_t>(1, (d->h_offsets[s + 1] - d->h_offsets[s] + each - 1) / each);
}

inline TreePlan plan_tree(const slkv_cache_desc* d, int T) {
  TreePlan p;
  const int64_t S = (int64_t)d->B * d->Hkv, R = (int64_t)(d->Hq / d->Hkv) * T, rows = d->h_offsets[S] - d->h_offsets[0];
  int64_t most = 1;
  for (int64_t s = 0; s < S; ++s) most = std::max(most, d->h_offsets[s + 1] - d->h_offsets[s]);
  const TileChoice c = choose_tiles(d->dtype, d->d, R, S, (double)rows * d->d * kind_bits(d->dtype) / 4, [&](int queries) {
    const double tiles = (double)((R + queries - 1) / queries);
    return TileLoad{S * tiles, std::max<double>(1, (double)rows) * tiles, (double)most};
  });
  p.shape = c.shape;
  p.each = std::min(most, c.each);
  p.queries = tile_queries(p.shape);
  const int64_t tiles = (R + p.queries - 1) / p.queries;
  p.split = most > p.each;
  p.slots = 0;
  for (int64_t s0 = 0; s0 < S; s0 += kTreeSegs) {
    int64_t here = 0;
    for (int64_t s = s0; s < std::min<int64_t>(S, s0 + kTreeSegs); ++s) here += tree_parts(d, s, p.each) * tiles;
    p.slots = std::max(p.slots, here);
  }
  const size_t o = p.split ? (size_t)p.slots * p.queries * d->d * sizeof(float) : 0;
  p.off_ml = o;
  p.bytes = std::max<size_t>(16, o + (p.split ? (size_t)p.slots * p.queries * 2 * sizeof(float) : 0));
  return p;
}

}  // namespace slkv
#endif
