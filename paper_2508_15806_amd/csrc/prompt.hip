// Causal attention of packed prompts (slkv_attend_prompt): the prefill whose keys and values slkv_compress_layer chooses from.
#include "attend_tiles.h"

#include <algorithm>

namespace slkv {

// Sequences of a launch, those with the most keys first.  Tiles of queries come in the order of their keys, the most first, whatever sequence they are of, and for each of them the KV heads, so
// that with 8 of these a head stays on an XCD and its L2.  In order (where there are parts, and for sequences of one length, whose keys and values stay in the caches this way: 64 of 256 tokens 130 us, else
// 140): sequence, tiles from the last one down, parts of the keys, KV heads.  (8 sequences of 110 to 4000 tokens: 590 us in order, else 542.)
struct PromptTab {
  static constexpr int kSeqs = kPromptSeqs;
  static constexpr bool kOneNumber = false;            // of the queries' type a weight
  const unsigned char *k, *v, *q;
  unsigned char* out;
  float* lse;
  int64_t q_tok, q_head, o_tok, o_head, k_row, v_row, k_head, v_head, lse_head;   // bytes; lse_head: elements
  int32_t nseq, hkv, in_order, shift;                  // 2^shift: tokens of a tile, about
  struct Words { int32_t first[kSeqs + 1], q0[kSeqs], nq[kSeqs], k0[kSeqs], nk[kSeqs], parts[kSeqs]; } words;

  // sequence; of it, tiles from the last one down and their parts; KV head
  struct Place { int s, rest, h; };
  template <int QUERIES>
  __device__ __forceinline__ Place locate(const TileArgs& a, const Words& t, int block) const {
    int s = 0, rest, h;
    if (in_order) {
      if (nseq > 1) s = find_segment_wave(nseq, block, [&](int i) { return t.first[i]; });
      const int i = block - __builtin_amdgcn_readfirstlane(t.first[s]);
      rest = i / hkv;
      h = i - rest * hkv;
    } else {
      // The i-th tile from the end of sequence b has the level nk[b] / 2^shift - i; lane b counts its tiles of a level and above.  Of the tiles down to the level wanted `rank`
      // come before.
      const int rank = block / hkv, lane = threadIdx.x % kWave;
      h = block - rank * hkv;
      const int mine = lane < nseq ? (a.G * t.nq[min(lane, nseq - 1)] + QUERIES - 1) / QUERIES : 0, top = lane < nseq ? t.nk[min(lane, nseq - 1)] >> shift : 0;
      auto count = [&](int level) __attribute__((always_inline)) {
        const uint32_t all = wave_incl_scan((uint32_t)min(max(top - level + 1, 0), mine));
        return (int)__builtin_amdgcn_readlane((int)all, kWave - 1);
      };
      int lo = -(1 << 30), hi = __builtin_amdgcn_readfirstlane(top) + 1;     // count(lo) > rank >= count(hi)
      // (the levels end where the last tiles of all sequences do)
      const uint32_t least = wave_reduce_to_last((uint32_t)(mine ? top - mine + 1 : hi) ^ 0x80000000u, [](uint32_t x, uint32_t y) { return min(x, y); });
      lo = (int)((uint32_t)__builtin_amdgcn_readlane((int)least, kWave - 1) ^ 0x80000000u);
      while (hi - lo > 1) {
        const int mid = lo + (hi - lo) / 2;
        if (count(mid) > rank) lo = mid;
        else hi = mid;
      }
      uint64_t there = __ballot(mine && top >= lo && top - lo < mine);
      for (int skip = rank - count(lo + 1); skip > 0; --skip) there &= there - 1;
      s = __builtin_ctzll(there);
      rest = __builtin_amdgcn_readlane(top, s) - lo;
    }
    return Place{s, rest, h};
  }

  template <int QUERIES, int KEYS, int D, int KIND>
  __device__ __forceinline__ TileWork describe(const TileArgs& a, const Words& t, const Place& at) const {
    auto uniform = [](int x) __attribute__((always_inline)) { return __builtin_amdgcn_readfirstlane(x); };
    const int s = at.s, h = at.h, rest = at.rest;
    const int parts_here = in_order ? uniform(t.parts[s]) : 1, new_tokens = uniform(t.nq[s]), keys = uniform(t.nk[s]), rows = a.G * new_tokens;
    const int64_t key0 = uniform(t.k0[s]), query0 = uniform(t.q0[s]);
    const int tiles = (rows + QUERIES - 1) / QUERIES, tile = tiles - 1 - rest / parts_here;
    TileWork w;
    w.part = rest % parts_here;
    w.rows = rows;
    w.r0 = tile * QUERIES;
    w.hist = keys - new_tokens;
    const int last = (min(w.r0 + QUERIES, rows) - 1) / a.G, end = min(max(w.hist + last + 1, 0), keys);
    const int steps = (end + KEYS - 1) / KEYS, each = (steps + parts_here - 1) / parts_here * KEYS;
    w.parts = each ? (end + each - 1) / each : 1;
    w.begin = w.part * each;
    w.end = min(end, w.begin + each);
    w.k = k + h * k_head + key0 * k_row;
    w.v = v + h * v_head + key0 * v_row;
    w.ks = w.vs = nullptr;
    w.q = q + (int64_t)h * a.G * q_head + query0 * q_tok;
    w.out = out + (int64_t)h * a.G * o_head + query0 * o_tok;
    w.lse = lse ? lse + (int64_t)h * a.G * lse_head + query0 : nullptr;
    w.sees = nullptr;
    w.q_tok = q_tok, w.q_head = q_head, w.o_tok = o_tok, w.o_head = o_head, w.lse_head = lse_head;
    w.k_row = k_row, w.v_row = v_row;
    w.slot0 = in_order ? uniform(t.first[s]) + rest / parts_here * parts_here * hkv + h : 0;
    w.slot_step = hkv;
    return w;
  }
};

struct PromptTabOne : PromptTab {
  static constexpr bool kOneNumber = true;
};

// Everything that can be checked without the arrays; the plan of a descriptor that passes.
static slkv_status prompt_checks(const slkv_prompt_desc* d, PromptPlan& plan) {
  if (!d) return fail(SLKV_ERR_NULL, "desc is NULL");
  if (d->struct_size != sizeof(slkv_prompt_desc)) return fail(SLKV_ERR_BAD_ARG, "desc.struct_size %u != %zu", d->struct_size, sizeof(slkv_prompt_desc));
  if (d->dtype < SLKV_F32 || d->dtype > SLKV_BF16_KV_MXFP4) return fail(SLKV_ERR_BAD_ARG, "unknown dtype %d", d->dtype);
  if (d->dtype == SLKV_BF16_KV_MXFP4) return fail(SLKV_ERR_UNSUPPORTED, "prompts have no MXFP4 keys and values");
  if (d->B < 1 || d->Hq < 1 || d->Hkv < 1) return fail(SLKV_ERR_BAD_ARG, "B, Hq, Hkv must be >= 1");
  if (d->B > (1 << 20) || d->Hkv > (1 << 16) || d->Hq > (1 << 16)) return fail(SLKV_ERR_BAD_ARG, "B, Hq or Hkv too large");
  if (d->Hq % d->Hkv) return fail(SLKV_ERR_BAD_ARG, "Hq %% Hkv != 0");
  if (d->d != 64 && d->d != 128) return fail(SLKV_ERR_UNSUPPORTED, "head_dim %d (supported: 64, 128)", d->d);
  if (d->options & ~SLKV_PROMPT_SHORT_WEIGHTS) return fail(SLKV_ERR_BAD_ARG, "desc.options: unknown bits %d", d->options);
  if (d->reserved) return fail(SLKV_ERR_BAD_ARG, "desc.reserved must be 0");
  slkv_status st = validate_offsets(d->h_cu_q, d->B, "h_cu_q");
  if (st != SLKV_OK) return st;
  if (d->h_cu_k && (st = validate_offsets(d->h_cu_k, d->B, "h_cu_k")) != SLKV_OK) return st;
  const int wide = wide_bytes(d->dtype), narrow = d->dtype == SLKV_BF16_KV_FP8 ? 1 : wide;
  const int64_t strides[] = {d->q_stride_tok, d->q_stride_head, d->out_stride_tok, d->out_stride_head, d->k_stride_tok, d->k_stride_head, d->v_stride_tok, d->v_stride_head};
  for (int i = 0; i < 8; ++i) {
    const int elt = i < 4 ? wide : narrow;
    if (strides[i] < 0 || strides[i] > (int64_t(1) << 40) || strides[i] * elt % 16) return fail(SLKV_ERR_BAD_ARG, "stride %lld not a non-negative multiple of 16 bytes", (long long)strides[i]);
    if ((i == 4 || i == 6) && strides[i] * elt >= (1 << 24)) return fail(SLKV_ERR_UNSUPPORTED, "token stride %lld of keys or values: 2^24 bytes and more", (long long)strides[i]);
  }
  const int64_t G = d->Hq / d->Hkv;
  for (int64_t b = 0; b < d->B; ++b)
    if (cu_k_of(d)[b + 1] - cu_k_of(d)[b] > (int64_t(1) << 30)) return fail(SLKV_ERR_UNSUPPORTED, "sequence %lld: more than 2^30 tokens", (long long)b);
  for (int64_t b = 0; b < d->B; ++b)
    if ((d->h_cu_q[b + 1] - d->h_cu_q[b]) * G >= (int64_t(1) << 31) - 512) return fail(SLKV_ERR_UNSUPPORTED, "sequence %lld: 2^31 - 512 query rows of a KV head and more", (long long)b);
  const int64_t n = d->h_cu_q[d->B] - d->h_cu_q[0];
  // (element numbers stay below 2^40)
  const int64_t tokens = cu_k_of(d)[d->B];
  for (int i = 0; i < 8; i += 2)
    if ((double)(i < 4 ? d->h_cu_q[d->B] : tokens) * strides[i] + (double)(i < 4 ? d->Hq : d->Hkv) * strides[i + 1] > 0x1p40)
      return fail(SLKV_ERR_BAD_ARG, "strides %lld, %lld reach beyond 2^40 elements", (long long)strides[i], (long long)strides[i + 1]);
  const bool by_head = (n < 2 || d->out_stride_tok >= d->d) && (d->Hq < 2 || d->out_stride_head >= (n - 1) * d->out_stride_tok + d->d);
  const bool by_token = (d->Hq < 2 || d->out_stride_head >= d->d) && (n < 2 || d->out_stride_tok >= (d->Hq - 1) * d->out_stride_head + d->d);
  if (n && !by_head && !by_token) return fail(SLKV_ERR_BAD_ARG, "out: rows overlap");
  plan = plan_prompt(d);
  if (plan.slots >= (1 << 24)) return fail(SLKV_ERR_UNSUPPORTED, "more than 2^24 workgroups");
  return SLKV_OK;
}

}  // namespace slkv

using namespace slkv;

extern "C" slkv_status slkv_prompt_workspace_bytes(const slkv_prompt_desc* desc, size_t* bytes) {
  clear_error();
  if (!bytes) return fail(SLKV_ERR_NULL, "bytes is NULL");
  PromptPlan p;
  const slkv_status st = prompt_checks(desc, p);
  if (st != SLKV_OK) return st;
  *bytes = p.bytes;
  return SLKV_OK;
}

extern "C" slkv_status slkv_attend_prompt(const slkv_prompt_desc* desc, const void* d_q, const void* d_k, const void* d_v, void* d_out, float* d_lse,
                                          void* d_workspace, size_t workspace_bytes, void* hip_stream) {
  clear_error();
  PromptPlan p;
  const slkv_status st = prompt_checks(desc, p);
  if (st != SLKV_OK) return st;
  const int64_t* ck = cu_k_of(desc);
  const int64_t queries = desc->h_cu_q[desc->B] - desc->h_cu_q[0], keys = ck[desc->B] - ck[0];
  if (!d_workspace || (queries && (!d_q || !d_out)) || (keys && (!d_k || !d_v))) return fail(SLKV_ERR_NULL, "a required device pointer is NULL");
  const void* ptrs[] = {d_q, d_k, d_v, d_out, d_lse, d_workspace};
  for (const void* ptr : ptrs)
    if ((uintptr_t)ptr % 16) return fail(SLKV_ERR_BAD_ARG, "device pointer %p not 16-byte aligned", ptr);
  if (workspace_bytes < p.bytes) return fail(SLKV_ERR_WORKSPACE, "workspace %zu < %zu bytes", workspace_bytes, p.bytes);
  const int wide = wide_bytes(desc->dtype), narrow = desc->dtype == SLKV_BF16_KV_FP8 ? 1 : wide;
  TileArgs a;
  a.G = desc->Hq / desc->Hkv;
  a.T = 0;
  a.c_log2 = kLog2e / std::sqrt((float)desc->d);
  a.part_o = (float*)d_workspace;
  a.part_ml = (float*)((unsigned char*)d_workspace + p.off_ml);
  hipStream_t const stream = (hipStream_t)hip_stream;
  for (int64_t b0 = 0; b0 < desc->B; b0 += PromptTab::kSeqs) {
    PromptTab t;
    t.k = (const unsigned char*)d_k, t.v = (const unsigned char*)d_v, t.q = (const unsigned char*)d_q;
    t.out = (unsigned char*)d_out;
    t.lse = d_lse;
    t.q_tok = desc->q_stride_tok * wide, t.q_head = desc->q_stride_head * wide;
    t.o_tok = desc->out_stride_tok * wide, t.o_head = desc->out_stride_head * wide;
    t.k_row = desc->k_stride_tok * narrow, t.k_head = desc->k_stride_head * narrow;
    t.v_row = desc->v_stride_tok * narrow, t.v_head = desc->v_stride_head * narrow;
    t.lse_head = desc->h_cu_q[desc->B];
    t.hkv = desc->Hkv;
    t.shift = 0;
    while (2 << t.shift <= p.queries / a.G) ++t.shift;
    t.nseq = (int32_t)std::min<int64_t>(PromptTab::kSeqs, desc->B - b0);
    auto length = [&](int i, const int64_t* cu) { return cu[b0 + i + 1] - cu[b0 + i]; };
    int order[PromptTab::kSeqs];
    for (int i = 0; i < t.nseq; ++i) order[i] = i;
    std::sort(order, order + t.nseq, [&](int x, int y) {
      const int64_t kx = length(x, ck), ky = length(y, ck);
      return kx != ky ? kx > ky : x < y;
    });
    int64_t blocks = 0;
    for (int i = 0; i < t.nseq; ++i) {
      const int64_t b = b0 + order[i];
      PromptTab::Words& x = t.words;
      x.first[i] = (int32_t)blocks;
      x.q0[i] = (int32_t)desc->h_cu_q[b], x.nq[i] = (int32_t)(desc->h_cu_q[b + 1] - desc->h_cu_q[b]);
      x.k0[i] = (int32_t)ck[b], x.nk[i] = (int32_t)(ck[b + 1] - ck[b]);
      x.parts[i] = (int32_t)seq_parts(desc, b, p.each);
      blocks += seq_tiles(desc, b, p.queries) * desc->Hkv * x.parts[i];
    }
    t.words.first[t.nseq] = (int32_t)blocks;
    t.in_order = prompt_in_order(desc, p, b0);
    if (!blocks) continue;
    a.blocks = (int32_t)blocks;
    auto launch = [&](auto kind, auto dim) {
      constexpr int kKind = decltype(kind)::value, kDim = decltype(dim)::value;
      with_shape<kKind, kDim>(p.shape, [&](auto wq, auto wk) {
        constexpr int kWQ = decltype(wq)::value, kWK = decltype(wk)::value;
        {
          ScopedKernelTimer timer(SLKV_K_PROMPT);
          const dim3 grid(std::min((unsigned)blocks, tile_places<Tiles<kKind, kDim, kWQ, kWK>>())), block(kWQ * kWK * kWave);
          if (kKind == SLKV_F32 || !(desc->options & SLKV_PROMPT_SHORT_WEIGHTS)) {
            SLKV_LAUNCH((attend_tiles_kernel<kKind, kDim, kWQ, kWK, PromptTab>), grid, block, 0, stream, a, t);
          } else if constexpr (kKind != SLKV_F32) {
            SLKV_LAUNCH((attend_tiles_kernel<kKind, kDim, kWQ, kWK, PromptTabOne>), grid, block, 0, stream, a, PromptTabOne{t});
          }
        }
        if (p.split) {
          ScopedKernelTimer timer(SLKV_K_TILES_JOIN);
          SLKV_LAUNCH((join_tiles_kernel<kKind, kDim, kWQ, kWK, PromptTab>), dim3((unsigned)blocks, join_slices(p.queries)), dim3(256), 0, stream, a, t);
        }
      });
    };
    auto with_dim = [&](auto kind) {
      if (desc->d == 64) launch(kind, std::integral_constant<int, 64>{});
      else launch(kind, std::integral_constant<int, 128>{});
    };
    switch (desc->dtype) {
      case SLKV_F32: with_dim(std::integral_constant<int, SLKV_F32>{}); break;
      case SLKV_BF16: with_dim(std::integral_constant<int, SLKV_BF16>{}); break;
      case SLKV_F16: with_dim(std::integral_constant<int, SLKV_F16>{}); break;
      default: with_dim(std::integral_constant<int, SLKV_BF16_KV_FP8>{});
    }
  }
  return launch_status("attend_prompt");
}
