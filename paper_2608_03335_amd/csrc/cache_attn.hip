// Attention of single queries over the paged cache (gfx950).
//
// A work item is a tile of up to 16 query rows that share one K/V head: the G query heads
// of one token, or of the 16 / G neighbouring tokens of one sequence when G < 16. It walks
// the union of its tokens' page lists (all visible pages without lists) in units of 32
// keys; its four waves take every fourth unit, and the launch may split the walk over
// several workgroups, joined by a second kernel in fixed order.
//
// One unit of a wave: S^T (32 keys x 16 rows) = K Q^T, two 16-key tiles of mfma 16x16x32;
// softmax with a running maximum; O^T += V^T P^T with the same instruction. The pages hold
// both operands as the instruction reads them (cache.h), so a fragment is one contiguous
// load straight into registers: no LDS, no shuffle, no transpose on the way.
//
// Scores, the running maximum and sum, and O are fp32. P is rounded to bf16 for the
// product with V (as in the block-sparse attention). 4-bit keys become bf16 exactly
// (e2m1 times a power of two); for V the power of two is moved into P, whose bf16
// rounding it commutes with.
//
// Masked places: keys beyond the tile's last visible token are cleared in V as well as in
// P (their memory may hold anything, NaN among it). A key that some rows of the tile see
// and others do not can hold a NaN or infinity in V that 0 * x would carry into the rows
// that must not see it: a wave whose result has a NaN repeats its walk token by token,
// clearing V for each (`careful`).
#include "cache.h"

namespace spade {
namespace {

constexpr int kWaves = 4;
constexpr int kThreads = 64 * kWaves;
constexpr int kMaxSplits = 64;
constexpr float kLn2f = 0.69314718055994530942f;
constexpr float kNegInf = -__builtin_huge_valf();

struct AttnArgs {
  DevCache c;
  DevBatch b;
  const __bf16* q;
  const int* counts;
  const int* indices;
  int topk, Hq, G, QT, RT;  // QT: tokens a tile; RT: row tiles a K/V head (G > 16)
  float scale2;             // logit scale * log2(e)
  int causal;
  __bf16* o;
  float* lse;
  float* part;              // partial results (splits > 1)
  int splits;
};

// What a work item covers; the same in the attention and in the join.
struct Tile {
  int b, t0, nq;       // sequence, first token, tokens
  int h, head0, heads; // K/V head, first query head, query heads of the tile
  int first_seen;      // visible tokens of the tile's first token
  int step;            // by how much the next token sees more (causal: 1)
  int len;             // no token sees more than this
  int pages;           // pages its last token sees
  int splits;          // workgroups that share its walk
  __device__ __forceinline__ int seen(int i) const {
    return min(max(first_seen + i * step, 0), len);
  }
};

__device__ __forceinline__ bool find_tile(const AttnArgs& a, Tile* t) {
  const SeqItem it = find_item(a.b, blockIdx.x, a.QT, a.QT > 1, kThreads);
  if (it.b < 0) return false;
  const int skip = it.first * a.QT;
  if (skip >= it.n) return false;
  t->b = it.b;
  t->t0 = it.t0 + skip;
  t->nq = min(a.QT, it.n - skip);
  t->h = blockIdx.y / a.RT;
  const int r0 = (blockIdx.y - t->h * a.RT) * 16;
  t->head0 = t->h * a.G + r0;
  t->heads = min(a.G - r0, 16);
  const int P = a.c.page;
  const int64_t raw = a.b.lens[it.b];
  t->len = int(min(max(raw, int64_t(0)), int64_t(a.b.max_pages) * P));
  t->step = a.causal;
  // a context of fewer tokens than are new leaves the first ones nothing to see
  t->first_seen = a.causal ? int(max(raw - it.n + skip + 1, int64_t(-(1 << 30)))) : t->len;
  const int most = t->seen(t->nq - 1);
  t->pages = (most + P - 1) / P;
  int walk = t->pages;
  if (a.topk) {  // an upper bound of the union of the lists
    int64_t sum = 0;
    for (int i = 0; i < t->nq; ++i) {
      const int n = a.counts[int64_t(t->t0 + i) * a.c.H + t->h];
      sum += min(max(n, 0), a.topk);
    }
    walk = int(min(sum, int64_t(walk)));
  }
  const int units = walk * (P >> 5);
  t->splits = min(max((units + 4 * kWaves - 1) / (4 * kWaves), 1), a.splits);
  return true;
}

__device__ __forceinline__ float max16(float v) {  // over the lanes of one row
  v = fmaxf(v, __shfl_xor(v, 16));
  return fmaxf(v, __shfl_xor(v, 32));
}
__device__ __forceinline__ float sum16(float v) {
  v += __shfl_xor(v, 16);
  return v + __shfl_xor(v, 32);
}

// Factor that takes a partial result with maximum m to maximum `top`. A part without a key
// (m = -inf) holds zeros, or the NaN of scores that are none: passed on as it is.
__device__ __forceinline__ float lift(float m, float top) {
  return m == kNegInf ? 1.0f : __builtin_amdgcn_exp2f(m - top);
}

template <int D, bool FP4>
struct UnitLoad {
  static constexpr int KK = D / 32;  // K steps
  static constexpr int CT = D / 16;  // V column tiles
  cu32x4 k[FP4 ? D / 64 : 2 * KK];   // 4 bit: two tiles of D / 32 dwords
  cu32x4 v[FP4 ? D / 64 : CT];
  uint32_t ks[2];
  cu32x2 vs[FP4 ? D / 32 : 1];
};

template <int D, bool FP4>
__device__ __forceinline__ void load_unit(const DevCache& c, int64_t base, int kb, int lane,
                                          UnitLoad<D, FP4>& u) {
  using L = UnitLoad<D, FP4>;
  if constexpr (!FP4) {
    const cu32x4* kp = (const cu32x4*)((const __bf16*)c.k + base + kb * 32 * D) + lane;
    const cu32x4* vp = (const cu32x4*)((const __bf16*)c.v + base + kb * 32 * D) + lane;
#pragma unroll
    for (int i = 0; i < 2 * L::KK; ++i) u.k[i] = kp[i * 64];
#pragma unroll
    for (int i = 0; i < L::CT; ++i) u.v[i] = vp[i * 64];
  } else {
    const uint8_t* kp = (const uint8_t*)c.k + (base >> 1) + kb * 16 * D;
    const uint8_t* vp = (const uint8_t*)c.v + (base >> 1) + kb * 16 * D;
    const uint8_t* ks = c.ks + (base >> 5) + kb * D;
    const uint8_t* vs = c.vs + (base >> 5) + kb * D;
    const int g = lane >> 4, m = lane & 15;
    if constexpr (D == 128) {
      u.k[0] = ((const cu32x4*)kp)[lane];
      u.k[1] = ((const cu32x4*)kp)[64 + lane];
      u.v[0] = ((const cu32x4*)vp)[lane];
      u.v[1] = ((const cu32x4*)vp)[64 + lane];
    } else {
      const cu32x2 x = ((const cu32x2*)kp)[lane], y = ((const cu32x2*)kp)[64 + lane];
      u.k[0] = cu32x4{x[0], x[1], y[0], y[1]};
      u.v[0] = ((const cu32x4*)vp)[lane];
    }
    const int gr = D == 128 ? g : g >> 1;
    u.ks[0] = ks[gr * 16 + m];
    u.ks[1] = ks[D / 2 + gr * 16 + m];
#pragma unroll
    for (int i = 0; i < D / 32; ++i) u.vs[i] = ((const cu32x2*)vs)[g * (D / 32) + i];
  }
}

template <int D, bool FP4>
struct Wave {
  static constexpr int KK = D / 32, CT = D / 16;
  cbf16x8 q[KK];
  cf32x4 o[CT];
  float m, l;  // running maximum (base-2 logits) and this lane's share of the sum
};

// The rows' query fragments: the K product's channel order (contiguous pieces of d / 4
// channels a lane group for 4 bits).
template <int D, bool FP4>
__device__ __forceinline__ void load_q(const AttnArgs& a, const Tile& t, int lane, Wave<D, FP4>& w) {
  const int r = lane & 15, g = lane >> 4;
  const int qi = r / t.heads, gh = r - qi * t.heads;
  const bool live = qi < t.nq;
  const __bf16* src = a.q + (int64_t(t.t0 + qi) * a.Hq + t.head0 + gh) * D;
#pragma unroll
  for (int s = 0; s < D / 32; ++s) {
    const int ch = FP4 ? g * (D / 4) + s * 8 : s * 32 + g * 8;
    w.q[s] = live ? *(const cbf16x8*)(src + ch) : cbf16x8{};
  }
}

// One unit: keys at..at+31 of the sequence. full: every row sees every key. V is cleared from
// key v_seen on; the rows of lanes without `take` keep what they had.
template <int D, bool FP4>
__device__ __forceinline__ void step_unit(const UnitLoad<D, FP4>& u, Wave<D, FP4>& w, int lane,
                                          float scale2, int at, int row_seen, bool row_in,
                                          int v_seen, bool full, bool take) {
  constexpr int KK = D / 32, CT = D / 16;
  const int g = lane >> 4;
  cf32x4 s[2] = {};
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int k = 0; k < KK; ++k) {
      cbf16x8 f;
      if constexpr (FP4) f = fp4_eight(u.k[(i * KK + k) >> 2][(i * KK + k) & 3], scale_of(u.ks[i]));
      else f = __builtin_bit_cast(cbf16x8, u.k[i * KK + k]);
      s[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, w.q[k], s[i], 0, 0, 0);
    }
  float p[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int key = at + (i >> 2) * 16 + g * 4 + (i & 3);
    p[i] = s[i >> 2][i & 3] * scale2;
    if (!full) p[i] = row_in && key < row_seen ? p[i] : kNegInf;
  }
  float top = p[0];
#pragma unroll
  for (int i = 1; i < 8; ++i) top = fmaxf(top, p[i]);
  top = max16(top);
  const float m = fmaxf(w.m, top);
  const float base = m == kNegInf ? 0.0f : m;  // no key yet: every p is 2^-inf = 0
  const float alpha = __builtin_amdgcn_exp2f(w.m - base);
  float sum = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    p[i] = __builtin_amdgcn_exp2f(p[i] - base);
    sum += p[i];
  }
  // V^T operands, cleared beyond v_seen
  const bool edge = at + 32 > v_seen;
  if constexpr (!FP4) {
    cbf16x8 pf;
#pragma unroll
    for (int i = 0; i < 8; ++i) pf[i] = (__bf16)p[i];
#pragma unroll
    for (int c = 0; c < CT; ++c) {
      cbf16x8 f = __builtin_bit_cast(cbf16x8, u.v[c]);
      if (edge)
#pragma unroll
        for (int i = 0; i < 8; ++i)
          f[i] = at + (i >> 2) * 16 + g * 4 + (i & 3) < v_seen ? f[i] : (__bf16)0.0f;
      const cf32x4 x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, pf, w.o[c] * alpha, 0, 0, 0);
      w.o[c] = take ? x : w.o[c];
    }
  } else {
    float two[8];
#pragma unroll
    for (int gr = 0; gr < D / 32; ++gr) {
      cbf16x8 pf;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        two[i] = scale_of((u.vs[gr][i >> 2] >> (8 * (i & 3))) & 255u);
        if (edge) two[i] = at + (i >> 2) * 16 + g * 4 + (i & 3) < v_seen ? two[i] : 0.0f;
        pf[i] = (__bf16)(p[i] * two[i]);
      }
#pragma unroll
      for (int cc = 0; cc < 2; ++cc) {
        const int c = gr * 2 + cc;
        const cf32x4 x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
            fp4_eight(u.v[c >> 2][c & 3], 1.0f), pf, w.o[c] * alpha, 0, 0, 0);
        w.o[c] = take ? x : w.o[c];
      }
    }
  }
  if (take) {
    w.l = w.l * alpha + sum;
    w.m = m;
  }
}

template <int D, bool FP4>
__global__ void __launch_bounds__(kThreads) cache_attn_kernel(AttnArgs a) {
  constexpr int CT = D / 16;
  constexpr int OROW = D + 4;  // fp32 row of the waves' merge in LDS
  extern __shared__ __attribute__((aligned(16))) char lds[];
  __shared__ float ml[kWaves][16][2];
  __shared__ int s_len;
  Tile t;
  if (!find_tile(a, &t)) return;
  const int split = blockIdx.z;
  if (split >= t.splits) return;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int P = a.c.page, upp = P >> 5;
  uint32_t* list = (uint32_t*)lds;  // entries: page << 16 | tokens of the tile that keep it
  int entries = t.pages;
  if (a.topk) {
    for (int j = tid; j < t.pages; j += kThreads) list[j] = 0;
    __syncthreads();
    for (int i = 0; i < t.nq; ++i) {
      const int64_t row = int64_t(t.t0 + i) * a.c.H + t.h;
      const int n = min(max(a.counts[row], 0), a.topk);
      const int vis = (t.seen(i) + P - 1) / P;
      for (int k = tid; k < n; k += kThreads) {
        const int j = a.indices[row * a.topk + k];
        if (j >= 0 && j < vis) atomicOr(&list[j], 1u << i);
      }
    }
    __syncthreads();
    if (wave == 0) {  // compaction in place: entry e comes from a page >= e
      int n = 0;
      for (int j0 = 0; j0 < t.pages; j0 += 64) {
        const int j = j0 + lane;
        const uint32_t x = j < t.pages ? list[j] : 0;
        const uint64_t bits = __ballot(x != 0);
        const int at = n + __popcll(bits & ((uint64_t(1) << lane) - 1));
        if (x) list[at] = uint32_t(j) << 16 | x;
        n += __popcll(bits);
      }
      if (lane == 0) s_len = n;
    }
    __syncthreads();
    entries = s_len;
  }
  const int units = entries * upp;
  const int u0 = int(int64_t(units) * split / t.splits), u1 = int(int64_t(units) * (split + 1) / t.splits);

  Wave<D, FP4> w;
  load_q(a, t, lane, w);
  const int qi = (lane & 15) / t.heads;  // the row's token inside the tile
  const int row_seen = qi < t.nq ? t.seen(qi) : 0;
  const int least = t.seen(0), most = t.seen(t.nq - 1);
  const uint32_t all = (1u << t.nq) - 1;
  const int* table = a.b.table + int64_t(t.b) * a.b.max_pages;

  for (int pass = 0; pass < 2; ++pass) {
    w.m = kNegInf;
    w.l = 0.0f;
#pragma unroll
    for (int c = 0; c < CT; ++c) w.o[c] = cf32x4{};
    for (int u = u0 + wave; u < u1; u += kWaves) {
      const int e = u / upp, kb = u - e * upp;
      const uint32_t x = a.topk ? list[e] : uint32_t(e);
      const int j = a.topk ? int(x >> 16) : e;
      const uint32_t who = a.topk ? x & 0xffffu : all;
      const int at = j * P + kb * 32;
      if (at >= most) continue;
      const int phys = table[j];
      if (phys < 0 || phys >= a.c.n_pages) continue;
      UnitLoad<D, FP4> ld;
      load_unit<D, FP4>(a.c, (int64_t(phys) * a.c.H + t.h) * P * D, kb, lane, ld);
      const bool full = who == all && at + 32 <= least;
      const bool row_in = qi < t.nq && (who >> qi & 1);
      if (pass == 0) {
        step_unit<D, FP4>(ld, w, lane, a.scale2, at, row_seen, row_in, most, full, true);
      } else {
        for (int i = 0; i < t.nq; ++i)
          step_unit<D, FP4>(ld, w, lane, a.scale2, at, row_seen, row_in,
                            (who >> i & 1) ? t.seen(i) : 0, full, qi == i);
      }
    }
    if (pass == 0) {
      bool bad = false;
#pragma unroll
      for (int c = 0; c < CT; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) bad |= !(w.o[c][i] == w.o[c][i]);
      if (t.nq == 1 || !__any(bad)) break;
    }
  }
  w.l = sum16(w.l);

  // the waves' results, joined in wave order
  float* osum = (float*)lds;
  __syncthreads();  // the list is no longer read
  const int r = lane & 15, g = lane >> 4;
  if (g == 0) {
    ml[wave][r][0] = w.m;
    ml[wave][r][1] = w.l;
  }
  __syncthreads();
  float M = kNegInf;
#pragma unroll
  for (int i = 0; i < kWaves; ++i) M = fmaxf(M, ml[i][r][0]);
  const float f = lift(w.m, M);
#pragma unroll
  for (int c = 0; c < CT; ++c)
    *(cf32x4*)(osum + (wave * 16 + r) * OROW + c * 16 + g * 4) = w.o[c] * f;
  __syncthreads();
  const int64_t slot = (int64_t(blockIdx.x) * gridDim.y + blockIdx.y) * a.splits + split;
  float* po = a.part + slot * (16 * D + 32);
  for (int i = tid; i < 16 * (D / 4); i += kThreads) {
    const int row = i / (D / 4), c4 = i % (D / 4);
    const int rq = row / t.heads, gh = row - rq * t.heads;
    if (rq >= t.nq) continue;
    cf32x4 x{};
    float top = kNegInf, sum = 0.0f;
#pragma unroll
    for (int v = 0; v < kWaves; ++v) {
      x += *(cf32x4*)(osum + (v * 16 + row) * OROW + c4 * 4);
      top = fmaxf(top, ml[v][row][0]);
    }
#pragma unroll
    for (int v = 0; v < kWaves; ++v)
      sum += ml[v][row][1] * lift(ml[v][row][0], top);
    if (t.splits > 1) {
      *(cf32x4*)(po + row * D + c4 * 4) = x;
      if (c4 == 0) {
        po[16 * D + row * 2] = top;
        po[16 * D + row * 2 + 1] = sum;
      }
    } else {
      const float inv = top == kNegInf ? 0.0f : 1.0f / sum;
      const int64_t orow = int64_t(t.t0 + rq) * a.Hq + t.head0 + gh;
      cu32x2 y;
      y[0] = __builtin_bit_cast(uint32_t, __builtin_convertvector(cf32x2{x[0] * inv, x[1] * inv}, cbf16x2));
      y[1] = __builtin_bit_cast(uint32_t, __builtin_convertvector(cf32x2{x[2] * inv, x[3] * inv}, cbf16x2));
      *(cu32x2*)(a.o + orow * D + c4 * 4) = y;
      if (a.lse && c4 == 0) a.lse[orow] = (top + log2f(sum)) * kLn2f;
    }
  }
}

// Joins the splits of one tile, in split order.
template <int D>
__global__ void __launch_bounds__(kThreads) cache_join_kernel(AttnArgs a) {
  Tile t;
  if (!find_tile(a, &t) || t.splits <= 1) return;
  const int64_t slot = (int64_t(blockIdx.x) * gridDim.y + blockIdx.y) * a.splits;
  const float* po = a.part + slot * (16 * D + 32);
  for (int i = threadIdx.x; i < 16 * (D / 4); i += kThreads) {
    const int row = i / (D / 4), c4 = i % (D / 4);
    const int rq = row / t.heads, gh = row - rq * t.heads;
    if (rq >= t.nq) continue;
    float top = kNegInf;
    for (int s = 0; s < t.splits; ++s) top = fmaxf(top, po[int64_t(s) * (16 * D + 32) + 16 * D + row * 2]);
    cf32x4 x{};
    float sum = 0.0f;
    for (int s = 0; s < t.splits; ++s) {
      const float* p = po + int64_t(s) * (16 * D + 32);
      const float m = p[16 * D + row * 2];
      const float f = lift(m, top);
      x += *(const cf32x4*)(p + row * D + c4 * 4) * f;
      sum += p[16 * D + row * 2 + 1] * f;
    }
    const float inv = top == kNegInf ? 0.0f : 1.0f / sum;
    const int64_t orow = int64_t(t.t0 + rq) * a.Hq + t.head0 + gh;
    cu32x2 y;
    y[0] = __builtin_bit_cast(uint32_t, __builtin_convertvector(cf32x2{x[0] * inv, x[1] * inv}, cbf16x2));
    y[1] = __builtin_bit_cast(uint32_t, __builtin_convertvector(cf32x2{x[2] * inv, x[3] * inv}, cbf16x2));
    *(cu32x2*)(a.o + orow * D + c4 * 4) = y;
    if (a.lse && c4 == 0) a.lse[orow] = (top + log2f(sum)) * kLn2f;
  }
}

struct Plan {
  int G, QT, RT, splits;
  int64_t items;
  int lds;
};

Plan plan(const DevCache& c, const DevBatch& b, int d, int Hq, int topk) {
  Plan p;
  p.G = Hq / c.H;
  p.QT = p.G < 16 ? 16 / p.G : 1;
  p.RT = (p.G + 15) / 16;
  p.items = p.QT > 1 ? item_base(b.n_tokens, b.B, p.QT, 1) : b.n_tokens;
  // workgroups without splits: tiles that hold tokens (at most), heads, row tiles
  const int64_t tiles = p.QT > 1 ? b.n_tokens / p.QT + (b.B < b.n_tokens ? b.B : b.n_tokens) : b.n_tokens;
  const int64_t wgs = tiles * c.H * p.RT;
  int64_t walk = b.max_pages;
  if (topk && int64_t(topk) * p.QT < walk) walk = int64_t(topk) * p.QT;
  const int64_t units = walk * (c.page / 32);
  int64_t s = (1024 + wgs - 1) / (wgs > 0 ? wgs : 1);
  const int64_t most = (units + 4 * kWaves - 1) / (4 * kWaves);
  s = s < most ? s : most;
  s = s < kMaxSplits ? s : kMaxSplits;
  p.splits = int(s < 1 ? 1 : s);
  const int merge = kWaves * 16 * (d + 4) * 4;
  const int list = topk ? b.max_pages * 4 : 0;
  p.lds = merge > list ? merge : list;
  return p;
}

template <int D, bool FP4>
hipError_t run(const AttnArgs& a, const Plan& p, hipStream_t s) {
  if (p.lds > 48 * 1024) {
    const hipError_t e = ensure_dynamic_lds((const void*)cache_attn_kernel<D, FP4>, kCacheMaxPages * 4);
    if (e != hipSuccess) return e;
  }
  const unsigned ny = unsigned(a.c.H * p.RT);
  cache_attn_kernel<D, FP4><<<dim3(unsigned(p.items), ny, p.splits), kThreads, p.lds, s>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.splits == 1) return e;
  cache_join_kernel<D><<<dim3(unsigned(p.items), ny), kThreads, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

size_t cache_attn_workspace_bytes(const DevCache& c, const DevBatch& b, int d, int Hq, int topk) {
  const Plan p = plan(c, b, d, Hq, topk);
  if (p.splits == 1) return 0;
  return size_t(p.items) * c.H * p.RT * p.splits * (16 * d + 32) * 4;
}

hipError_t launch_cache_attn(const DevCache& c, const DevBatch& b, int d, const CacheAttn& x,
                             void* ws, hipStream_t s) {
  const Plan p = plan(c, b, d, x.Hq, x.topk);
  AttnArgs a;
  a.c = c;
  a.b = b;
  a.q = (const __bf16*)x.q;
  a.counts = x.counts;
  a.indices = x.indices;
  a.topk = x.topk;
  a.Hq = x.Hq;
  a.G = p.G;
  a.QT = p.QT;
  a.RT = p.RT;
  a.scale2 = x.scale * 1.44269504088896340736f;
  a.causal = x.causal;
  a.o = (__bf16*)x.o;
  a.lse = x.lse;
  a.part = (float*)ws;
  a.splits = p.splits;
  if (d == 128) return c.fp4 ? run<128, true>(a, p, s) : run<128, false>(a, p, s);
  return c.fp4 ? run<64, true>(a, p, s) : run<64, false>(a, p, s);
}

}  // namespace spade
