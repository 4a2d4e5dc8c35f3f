// What the two attention kernels of the paged cache share (cache_attn.hip, cache_chunk.hip).
#pragma once

#include "cache.h"

namespace spade {

// What the join of a tile's splits has to know, written by the first split.
struct JoinHead {
  int splits;                // 0: no such tile, 1: its result is written
  int t0, nq, head0, heads;  // first token, tokens, first query head, query heads
};

struct AttnArgs {
  DevCache c;
  DevBatch b;
  const __bf16* q;
  const int* counts;
  const int* indices;
  int topk, Hq, G;
  int QT, RT;               // tokens a tile; row tiles a K/V head (G larger than a tile)
  float scale2;             // logit scale * log2(e)
  int causal;
  __bf16* o;
  float* lse;
  JoinHead* join;
  float* part;              // partial results (splits > 1)
  int64_t items;            // tiles of all sequences, at most
  int splits;               // most workgroups that share a tile's walk
  int wgs;                  // workgroups a call is split into, about
  uint32_t first;           // workgroup of the launch
};

// Many queries a sequence: tiles of 128 rows, four waves of 32, that share staged keys
// (cache_chunk.hip). A wave holds kChunkRows / G tokens.
constexpr int kChunkRows = 32, kChunkWaves = 4;
constexpr int kChunkUnits = 32;  // units of 32 keys a split of such a tile is worth, at least
hipError_t launch_chunk_attn(const AttnArgs& a, int d, hipStream_t s);

#ifdef __HIPCC__
constexpr float kLn2f = 0.69314718055994530942f;
constexpr float kNegInf = -__builtin_huge_valf();

// Visible tokens of a sequence's new tokens: token i of n sees first + i * step, clamped.
struct Seen {
  int first, step, len;
  __device__ __forceinline__ int of(int i) const { return min(max(first + i * step, 0), len); }
};
__device__ __forceinline__ Seen seen_of(const AttnArgs& a, const SeqItem& it) {
  const int64_t raw = it.len;
  Seen s;
  s.len = int(min(max(raw, int64_t(0)), int64_t(a.b.max_pages) * a.c.page));
  s.step = a.causal;
  // a context of fewer tokens than are new leaves the first ones nothing to see
  s.first = a.causal ? int(max(raw - it.n + 1, int64_t(-(1 << 30)))) : s.len;
  return s;
}
#endif

}  // namespace spade
