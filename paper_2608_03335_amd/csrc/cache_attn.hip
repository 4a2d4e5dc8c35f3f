// Attention over the paged cache in tiles of 16 query rows (gfx950): single tokens, short
// chunks, chunks under lists in few heads, and groups of more than 32 query heads.
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
// A row's reference m is set 2^8 above its maximum and raised only when that passes it, so
// weights are 1 at most: sums of them times V stay finite while keys x |V| < 2^127.
//
// Scores, the reference, the sum, and O are fp32. P is rounded to bf16 for the
// product with V (as in the block-sparse attention). 4-bit keys become bf16 exactly
// (e2m1 times a power of two); for V the power of two is moved into P, whose bf16
// rounding it commutes with.
//
// Masked places: keys beyond the tile's last visible token are cleared in V as well as in
// P (their memory may hold anything, NaN among it). A key that some rows of the tile see
// and others do not can hold a NaN or infinity in V that 0 * x would carry into the rows
// that must not see it: a workgroup whose result has a NaN repeats its walk for each token
// alone, clearing V beyond what that token sees.
//
// Bound by HBM where contexts are long: two of 131072 tokens, 32 x 4 heads of 128 in bf16, 493 MB
// in 90 us (5.5 TB/s) and 6 for the join. In 4 bits by the chain of a unit (load, widen, product,
// maximum, exponent, product) with too few waves to hide it: 64 contexts of up to 16384 tokens,
// 32 x 8 heads of 128, 605 MB in 168 us (3.6 TB/s), vector instructions in 34% of the SIMDs'
// cycles, 1.6 waves a SIMD on average where three fit, since the contexts differ in length.
// Bound by the latency of one walk where they are short: one token over 16 pages of 64, 10 us
// and 4 for the join.
#include "cache_attn.h"

namespace spade {
namespace {

constexpr int kWaves = 4;
constexpr int kThreads = 64 * kWaves;
constexpr int kMaxSplits = 64;
constexpr int kCUs = 256;
constexpr int64_t kMaxIdle = 65536;  // workgroups of a split call, tiles without tokens among them
constexpr int kMaxShared = 4096;   // sequences of a split call
constexpr int kMinUnits = 16;      // units a split is worth: its start and join cost as much
// Workgroups that are on the card at once (256 CUs, by registers): a call is split into about
// as many. On 64 4-bit contexts of up to 16384 tokens: 384 186 us, 512 183, 768 175, 1024 177,
// 2048 200; two of 131072 in bf16: 384 108, 512 106, 768 and more 117.
template <int D, bool FP4>
constexpr int target_wgs() { return kCUs * (D == 128 && !FP4 ? 2 : 3); }
constexpr float kLazy = 8.0f;      // a row's reference lies up to 2^8 above its largest score

// What a work item covers.
struct Tile {
  int b, t0, nq;        // sequence, first token, tokens
  int h, head0, heads;  // K/V head, first query head, query heads of the tile
  Seen seen;            // of the tile's tokens
  int pages;            // pages its last token sees
  int splits;           // workgroups that share its walk
};

__device__ __forceinline__ int tile_walk(const AttnArgs& a, int pages) {  // pages, at most
  return a.topk ? int(min(int64_t(a.topk) * a.QT, int64_t(pages))) : pages;
}

// Workgroups are numbered with the heads running fastest, then the tiles, then the splits:
// the XCDs, which take them in turn, get equal shares of every sequence.
__device__ __forceinline__ bool find_tile(const AttnArgs& a, int tile, int y, Tile* t) {
  // all units of the call, for the splits' size
  __shared__ unsigned long long total;
  if (threadIdx.x == 0) total = 0;
  const int P = a.c.page;
  if (a.splits > 1) {
    __syncthreads();
    unsigned long long mine = 0;
    for (int b = threadIdx.x; b < a.b.B; b += kThreads) {
      const int64_t n = int64_t(a.b.cu[b + 1]) - a.b.cu[b];
      const int64_t len = min(max(int64_t(a.b.lens[b]), int64_t(0)), int64_t(a.b.max_pages) * P);
      if (n > 0) mine += int64_t((n + a.QT - 1) / a.QT) * tile_walk(a, int((len + P - 1) / P));
    }
    if (mine) atomicAdd(&total, mine);
  }
  const SeqItem it = find_item(a.b, tile, a.QT, a.QT > 1);
  if (it.b < 0) return false;
  const int skip = it.first * a.QT;
  if (skip >= it.n) return false;
  t->b = it.b;
  t->t0 = it.t0 + skip;
  t->nq = min(a.QT, it.n - skip);
  t->h = y / a.RT;
  const int r0 = (y - t->h * a.RT) * 16;
  t->head0 = t->h * a.G + r0;
  t->heads = min(a.G - r0, 16);
  t->seen = seen_of(a, it);
  t->seen.first += skip * t->seen.step;
  t->pages = (t->seen.of(t->nq - 1) + P - 1) / P;
  t->splits = 1;
  if (a.splits > 1) {
    const int64_t upp = P >> 5, units = tile_walk(a, t->pages) * upp;
    const uint64_t all = total;
    const int64_t sum = int64_t(uint64_t(__builtin_amdgcn_readfirstlane(uint32_t(all >> 32))) << 32 |
                                __builtin_amdgcn_readfirstlane(uint32_t(all)));
    const int64_t even = (sum * upp * (a.c.H * a.RT) + a.wgs - 1) / a.wgs;
    const int64_t size = max(even, int64_t(kMinUnits));
    t->splits = int(min(max((units + size - 1) / size, int64_t(1)), int64_t(a.splits)));
  }
  return true;
}

__device__ __forceinline__ float max16(float v) {  // over the four lanes of a row
  const auto x = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1]));
  const auto y = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(y[0]), __uint_as_float(y[1]));
}
__device__ __forceinline__ float sum16(float v) {
  v += __shfl_xor(v, 16);
  return v + __shfl_xor(v, 32);
}

// Factor that takes a partial result with reference m to reference `top`. A part without a key
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
  float m, l;  // reference (base-2 logits) and this lane's share of the sum
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

// One unit: keys at..at+31 of the sequence. row_in: the lane's row keeps the page. edge (the
// same for all lanes): a row sees the keys below row_seen, and V is cleared from key v_seen on.
template <int D, bool FP4>
__device__ __forceinline__ void step_unit(UnitLoad<D, FP4>& u, Wave<D, FP4>& w, int lane,
                                          float scale2, int at, bool edge, int row_seen,
                                          bool row_in, int v_seen) {
  constexpr int KK = D / 32, CT = D / 16;
  const int g = lane >> 4;
  const int key0 = at + g * 4;  // the lane's keys: key0 + {0..3, 16..19}
  cf32x4 s[2] = {};
#pragma unroll
  for (int k = 0; k < KK; ++k)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      cbf16x8 f;
      if constexpr (FP4) f = fp4_eight(u.k[(i * KK + k) >> 2][(i * KK + k) & 3], scale_of(u.ks[i]));
      else f = __builtin_bit_cast(cbf16x8, u.k[i * KK + k]);
      s[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, w.q[k], s[i], 0, 0, 0);
    }
  float p[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) p[i] = s[i >> 2][i & 3];
  if (edge)
#pragma unroll
    for (int i = 0; i < 8; ++i) p[i] = key0 + (i >> 2) * 16 + (i & 3) < row_seen ? p[i] : kNegInf;
  float top = fmaxf(p[0], p[1]);
#pragma unroll
  for (int i = 2; i < 8; i += 2) top = fmaxf(fmaxf(top, p[i]), p[i + 1]);
  top = max16(top) * scale2;
  top = row_in ? top : kNegInf;
  float m = w.m;
  if (__any(top > m)) {
    m = top > m ? top + kLazy : m;
    const float alpha = w.m == kNegInf ? 0.0f : __builtin_amdgcn_exp2f(w.m - m);
#pragma unroll
    for (int c = 0; c < CT; ++c) w.o[c] *= alpha;
    w.l *= alpha;
    w.m = m;
  }
  // rows that do not keep the page, or have no key yet: 2^(s - inf) = 0
  const float bias = row_in && m != kNegInf ? -m : kNegInf;
  float sum = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    p[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(p[i], scale2, bias));
    sum += p[i];
  }
  w.l += sum;
  if constexpr (!FP4) {
    if (edge) {
      uint32_t keep[4];  // halves of a V fragment's dwords
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int key = key0 + (i >> 1) * 16 + (i & 1) * 2;
        keep[i] = (key < v_seen ? 0xffffu : 0u) | (key + 1 < v_seen ? 0xffff0000u : 0u);
      }
#pragma unroll
      for (int c = 0; c < CT; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) u.v[c][i] &= keep[i];
    }
    cbf16x8 pf;
#pragma unroll
    for (int i = 0; i < 8; ++i) pf[i] = (__bf16)p[i];
#pragma unroll
    for (int c = 0; c < CT; ++c)
      w.o[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(cbf16x8, u.v[c]), pf, w.o[c], 0, 0, 0);
  } else {
    if (edge) {  // scale 2^-127 becomes 0 for a key nobody sees: p is 0, its V code is finite
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        uint32_t keep = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) keep |= key0 + i * 16 + j < v_seen ? 255u << (8 * j) : 0u;
#pragma unroll
        for (int gr = 0; gr < D / 32; ++gr) u.vs[gr][i] &= keep;
      }
    }
#pragma unroll
    for (int gr = 0; gr < D / 32; ++gr) {
      float two[8];
#pragma unroll
      for (int i = 0; i < 2; ++i) scales_of(u.vs[gr][i], two + 4 * i);
      cbf16x8 pf;
#pragma unroll
      for (int i = 0; i < 8; ++i) pf[i] = (__bf16)(p[i] * two[i]);
#pragma unroll
      for (int cc = 0; cc < 2; ++cc) {
        const int c = gr * 2 + cc;
        w.o[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fp4_eight(u.v[c >> 2][c & 3], 1.0f), pf, w.o[c], 0, 0, 0);
      }
    }
  }
}

// The pages the tile walks, ascending, in LDS; their number.
__device__ __forceinline__ int build_list(const AttnArgs& a, const Tile& t, uint32_t* list) {
  __shared__ int s_len;
  const int tid = threadIdx.x, lane = tid & 63, P = a.c.page;
  const int64_t row0 = int64_t(t.t0) * a.c.H + t.h;
  if (t.nq == 1) {  // one token's list, as selections write it, is the walk already
    const int n = min(max(a.counts[row0], 0), a.topk);
    bool good = true;
    // (as many entries as the table has pages fit; a longer list cannot ascend)
    for (int k = tid; k < min(n, a.b.max_pages); k += kThreads) {
      const int j = a.indices[row0 * a.topk + k];
      const int before = k ? a.indices[row0 * a.topk + k - 1] : -1;
      good &= j > before && j < t.pages;
      list[k] = uint32_t(j) << 16 | 1u;
    }
    if (__syncthreads_and(good && n <= a.b.max_pages)) return n;
  }
  for (int j = tid; j < t.pages; j += kThreads) list[j] = 0;
  __syncthreads();
  for (int i = 0; i < t.nq; ++i) {
    const int64_t row = row0 + int64_t(i) * a.c.H;
    const int n = min(max(a.counts[row], 0), a.topk);
    const int vis = (t.seen.of(i) + P - 1) / P;
    for (int k = tid; k < n; k += kThreads) {
      const int j = a.indices[row * a.topk + k];
      if (j >= 0 && j < vis) atomicOr(&list[j], 1u << i);
    }
  }
  __syncthreads();
  if (tid < 64) {  // compaction in place: entry e comes from a page >= e
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
  return s_len;
}

// Four channels of a finished row.
template <int D>
__device__ __forceinline__ void write_row(const AttnArgs& a, int64_t orow, int c4, cf32x4 x, float top,
                                          float sum) {
  const float inv = top == kNegInf ? 0.0f : 1.0f / sum;
  cu32x2 y;
  y[0] = __builtin_bit_cast(uint32_t, __builtin_convertvector(cf32x2{x[0] * inv, x[1] * inv}, cbf16x2));
  y[1] = __builtin_bit_cast(uint32_t, __builtin_convertvector(cf32x2{x[2] * inv, x[3] * inv}, cbf16x2));
  *(cu32x2*)(a.o + orow * D + c4 * 4) = y;
  if (a.lse && c4 == 0) a.lse[orow] = (top + log2f(sum)) * kLn2f;
}

template <int D, bool FP4>
__global__ void __launch_bounds__(kThreads, FP4 ? 3 : 2) cache_attn_kernel(AttnArgs a) {
  constexpr int CT = D / 16;
  constexpr int OROW = D + 4;  // fp32 row of the waves' merge in LDS
  extern __shared__ __attribute__((aligned(16))) char lds[];
  __shared__ float ml[kWaves][16][2];
  const int ny = a.c.H * a.RT;
  const uint32_t wg = a.first + blockIdx.x;
  const int per = int(a.items), y = wg % ny;
  const int split = wg / ny / per, tile = wg / ny % per;
  Tile t;
  const bool any = find_tile(a, tile, y, &t);
  if (a.splits > 1 && split == 0 && threadIdx.x == 0)
    a.join[int64_t(tile) * ny + y] =
        any ? JoinHead{t.splits, t.t0, t.nq, t.head0, t.heads} : JoinHead{0, 0, 0, 0, 0};
  if (!any || split >= t.splits) return;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int P = a.c.page, upp = P >> 5;
  Wave<D, FP4> w;
  load_q(a, t, lane, w);
  uint32_t* list = (uint32_t*)lds;  // entries: page << 16 | tokens of the tile that keep it
  int entries = t.pages;
  if (a.topk) entries = __builtin_amdgcn_readfirstlane(build_list(a, t, list));
  const int units = entries * upp;
  const int u0 = int(int64_t(units) * split / t.splits), u1 = int(int64_t(units) * (split + 1) / t.splits);

  const int qi = (lane & 15) / t.heads;  // the row's token inside the tile
  const int row_seen = qi < t.nq ? t.seen.of(qi) : 0;
  const uint32_t all = (1u << t.nq) - 1;
  const int* table = a.b.table + int64_t(t.b) * a.b.max_pages;

  // The wave's units, every fourth of the split's. Lane i knows entry 64 win + i of the walk,
  // so the address of a unit to load needs no memory access but every 64 pages.
  int win = -1, w_entry = 0, w_phys = -1;
  uint32_t w_who = 0;
  auto look = [&](int first) {
    win = first;
    const int i = first * 64 + lane;
    const uint32_t x = i >= entries ? 0u : a.topk ? list[i] : all;
    w_entry = i >= entries ? 0 : a.topk ? int(x >> 16) : i;
    w_phys = i >= entries ? -1 : table[w_entry];
    w_who = x & 0xffffu;
    asm volatile("" : "+v"(w_phys));  // waited for here, not at every use
  };
  struct Unit {
    int at;        // first key
    uint32_t who;  // tokens of the tile that keep its page; 0: nothing to compute
  };
  constexpr int NB = 2;  // units in flight
  float* osum = (float*)(lds + (a.topk ? (a.b.max_pages * 4 + 15) / 16 * 16 : 0));
  // only < 0: all tokens at once; else the tile's tokens one by one (see the head of the file)
  for (int only = -1; only < t.nq; ++only) {
    const int least = t.seen.of(max(only, 0)), most = only < 0 ? t.seen.of(t.nq - 1) : least;
    const uint32_t ours = only < 0 ? all : 1u << only;
    w.m = kNegInf;
    w.l = 0.0f;
#pragma unroll
    for (int c = 0; c < CT; ++c) w.o[c] = cf32x4{};
    UnitLoad<D, FP4> ld[NB];
    Unit un[NB];
    int u = u0 + wave;
    // A unit that holds nothing for the tile (a page outside the pool, past the walk's end)
    // still loads, from page 0: the loads in flight are then the same on every path, and no
    // wait has to assume the worst.
    auto next = [&](Unit& x, UnitLoad<D, FP4>& to) {
      const int e = u / upp, kb = u - e * upp;
      if (u < u1 && e >> 6 != win) look(e >> 6);
      const int phys = __builtin_amdgcn_readlane(w_phys, e & 63);
      const bool ok = u < u1 && phys >= 0 && phys < a.c.n_pages;
      x.at = __builtin_amdgcn_readlane(w_entry, e & 63) * P + kb * 32;
      x.who = ok && x.at < most ? __builtin_amdgcn_readlane(w_who, e & 63) & ours : 0u;
      load_unit<D, FP4>(a.c, (int64_t(x.who ? phys : 0) * a.c.H + t.h) * P * D, kb, lane, to);
      u += kWaves;
    };
#pragma unroll
    for (int i = 0; i < NB; ++i) next(un[i], ld[i]);
    int mine = (u1 - u0 - wave + kWaves - 1) / kWaves;
    while (mine > 0) {
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        const uint32_t who = un[i].who;
        const bool row_in = qi < t.nq && (who >> qi & 1);
        step_unit<D, FP4>(ld[i], w, lane, a.scale2, un[i].at, who == 0 || un[i].at + 32 > least,
                          who ? row_seen : 0, row_in, who ? most : 0);
        if (--mine <= 0) break;
        next(un[i], ld[i]);
      }
    }
    if (only < 0 && t.nq > 1) {
      bool bad = false;
#pragma unroll
      for (int c = 0; c < CT; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) bad |= !(w.o[c][i] == w.o[c][i]);
      if (__syncthreads_or(bad)) continue;
    }
    w.l = sum16(w.l);

    // the waves' results, joined in wave order
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
    const int64_t slot = (int64_t(tile) * ny + y) * a.splits + split;
    float* po = a.part + slot * (16 * D + 32);
    for (int i = tid; i < 16 * (D / 4); i += kThreads) {
      const int row = i / (D / 4), c4 = i % (D / 4);
      const int rq = row / t.heads, gh = row - rq * t.heads;
      if (rq >= t.nq || (only >= 0 && rq != only)) continue;
      cf32x4 x{};
      float top = kNegInf, sum = 0.0f;
#pragma unroll
      for (int v = 0; v < kWaves; ++v) {
        x += *(cf32x4*)(osum + (v * 16 + row) * OROW + c4 * 4);
        top = fmaxf(top, ml[v][row][0]);
      }
#pragma unroll
      for (int v = 0; v < kWaves; ++v) sum += ml[v][row][1] * lift(ml[v][row][0], top);
      if (t.splits > 1) {
        *(cf32x4*)(po + row * D + c4 * 4) = x;
        if (c4 == 0) {
          po[16 * D + row * 2] = top;
          po[16 * D + row * 2 + 1] = sum;
        }
      } else {
        write_row<D>(a, int64_t(t.t0 + rq) * a.Hq + t.head0 + gh, c4, x, top, sum);
      }
    }
    if (only < 0) break;
    __syncthreads();
  }
}

// Joins the splits of one tile of ROWS rows, in split order: a wave takes one row. Rows lie in
// groups of GROUP (a wave's), a group's tokens one after the other with their heads.
template <int D, int ROWS, int GROUP>
__global__ void __launch_bounds__(kThreads) cache_join_kernel(AttnArgs a) {
  constexpr int PIECES = D / 4, RUNS = 64 / PIECES, AHEAD = 8;
  constexpr int64_t STRIDE = ROWS * (D + 2);
  const uint32_t tile = a.first + blockIdx.x;
  const JoinHead t = a.join[tile];
  if (t.splits <= 1) return;
  const int lane = threadIdx.x & 63, c4 = lane % PIECES, run = lane / PIECES;
  const int row = blockIdx.y * kWaves + (threadIdx.x >> 6);
  const int in_group = row % GROUP, q = in_group / t.heads, gh = in_group - q * t.heads;
  const int per_group = GROUP / t.heads, rq = row / GROUP * per_group + q;
  if (q >= per_group || rq >= t.nq) return;
  const float* po = a.part + int64_t(tile) * a.splits * STRIDE;
  // loads of the partial results a batch ahead of their use, the first ahead of the statistics
  cf32x4 next[AHEAD];
  auto fetch = [&](int s0) {
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
      next[i] = *(const cf32x4*)(po + min(s0 + i * RUNS + run, t.splits - 1) * STRIDE + row * D + c4 * 4);
    __builtin_amdgcn_sched_barrier(0);
  };
  fetch(0);
  static_assert(kMaxSplits <= 64, "a lane holds one split's statistics");
  const bool in = lane < t.splits;
  const float m = in ? po[lane * STRIDE + ROWS * D + row * 2] : kNegInf;
  const float l = in ? po[lane * STRIDE + ROWS * D + row * 2 + 1] : 0.0f;
  float top = m;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
  const float f = in ? lift(m, top) : 0.0f;
  float sum = in ? l * f : 0.0f;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
  cf32x4 x{};
  for (int s0 = 0; s0 < t.splits; s0 += AHEAD * RUNS) {
    cf32x4 y[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) y[i] = next[i];
    if (s0 + AHEAD * RUNS < t.splits) fetch(s0 + AHEAD * RUNS);
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      const int s = s0 + i * RUNS + run;
      const float fs = __shfl(f, min(s, t.splits - 1));
      if (s < t.splits) x += y[i] * fs;
    }
  }
#pragma unroll
  for (int o = PIECES; o < 64; o <<= 1)
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] += __shfl_xor(x[i], o);
  if (run == 0) write_row<D>(a, int64_t(t.t0 + rq) * a.Hq + t.head0 + gh, c4, x, top, sum);
}

struct Plan {
  bool chunk;
  int G, QT, RT, splits, wgs;
  int64_t items;
  int lds;
};

// Splits for a launch of `wgs` workgroups that should be about `want`, of walks of `pages`.
int splits_of(int64_t want, int64_t wgs, int64_t pages, int page, int least_units) {
  const int64_t most = (pages * (page / 32) + least_units - 1) / least_units;
  int64_t s = want / (wgs < 1 ? 1 : wgs);
  s = s < most ? s : most;
  s = s < kMaxSplits ? s : kMaxSplits;
  return int(s < 1 ? 1 : s);
}

Plan plan(const DevCache& c, const DevBatch& b, int d, int Hq, int topk) {
  Plan p;
  p.G = Hq / c.H;
  p.wgs = d == 128 ? (c.fp4 ? target_wgs<128, true>() : target_wgs<128, false>())
                   : (c.fp4 ? target_wgs<64, true>() : target_wgs<64, false>());
  const int64_t each = (int64_t(b.n_tokens) + b.B - 1) / b.B;  // tokens a sequence, on average
  const int64_t holders = b.B < b.n_tokens ? b.B : b.n_tokens;  // sequences with tokens, at most
  auto walk = [&](int64_t tokens) {                             // pages a tile walks, at most
    return topk && topk * tokens < b.max_pages ? topk * tokens : int64_t(b.max_pages);
  };
  // Many rows a sequence: tiles of 128 rows share their keys, where they fill half the card. Calls
  // that read all tokens split the keys of such tiles to fill it twice. Measured, in us, this side
  // and tiles of 16 rows (bf16, width 128, one sequence; Hq x H, context, new tokens):
  //   all tokens   16 x 4, 8192, 500: 61, 102    32 x 8, 16384, 200: 90, 154   64: 53, 55   24: 39, 37
  //                12 x 12, 16384, 1200: 170, 323, and 398 without splits; 32 x 8, 4-bit, 200: 112, 165
  //   listed pages 32 x 8, 16384, 200, 32 pages: 78, 62    16 x 4, width 64, 4-bit, 400, 24: 49, 36
  // Lists leave a tile's rows little in common, so what fills the card is more and smaller tiles.
  const int64_t rows = int64_t(b.n_tokens) * p.G;
  p.chunk = false;
  if (p.G <= kChunkRows && rows >= int64_t(b.B) * 64) {
    p.QT = kChunkRows / p.G * kChunkWaves;
    p.RT = 1;
    p.items = item_base(b.n_tokens, b.B, p.QT, 1);
    p.lds = 0;
    p.splits = 1;
    if (!topk && rows >= int64_t(b.B) * 128) {
      const int64_t wgs = (b.n_tokens / p.QT + holders) * c.H;
      p.splits = splits_of(2 * kCUs, wgs, b.max_pages, c.page, kChunkUnits);
      p.chunk = wgs * p.splits >= kCUs / 2;
    }
    p.chunk = p.chunk || rows / 128 * c.H >= kCUs / 2;
    if (p.chunk) return p;
  }
  p.QT = p.G < 16 ? 16 / p.G : 1;
  p.RT = (p.G + 15) / 16;
  p.items = p.QT > 1 ? item_base(b.n_tokens, b.B, p.QT, 1) : b.n_tokens;
  // workgroups without splits: tiles that hold tokens (at most), heads, row tiles
  const int64_t wgs = (p.QT > 1 ? b.n_tokens / p.QT + holders : b.n_tokens) * c.H * p.RT;
  p.splits = splits_of(2 * p.wgs + wgs - 1, wgs, walk(each < p.QT ? each : p.QT), c.page, kMinUnits);
  // tiles of sequences without tokens are as many for each split, and a split call's workgroups
  // add up all sequences
  const int64_t idle = kMaxIdle / (p.items * c.H * p.RT);
  p.splits = b.B > kMaxShared || idle < 1 ? 1 : int(p.splits < idle ? p.splits : idle);
  p.lds = kWaves * 16 * (d + 4) * 4 + (topk ? (b.max_pages * 4 + 15) / 16 * 16 : 0);
  return p;
}

size_t join_bytes(size_t tiles) { return (tiles * sizeof(JoinHead) + 255) / 256 * 256; }

template <int D, bool FP4>
hipError_t run(const AttnArgs& a, const Plan& p, hipStream_t s) {
  if (p.lds > 48 * 1024) {
    const hipError_t e = ensure_dynamic_lds((const void*)cache_attn_kernel<D, FP4>,
                                            kCacheMaxPages * 4 + kWaves * 16 * (D + 4) * 4);
    if (e != hipSuccess) return e;
  }
  return launch_parts(cache_attn_kernel<D, FP4>, a, p.items * a.c.H * p.RT * p.splits, 1, kThreads, p.lds, s);
}

template <int D>
hipError_t join(const AttnArgs& a, const Plan& p, hipStream_t s) {
  const int64_t tiles = p.items * a.c.H * p.RT;
  if (p.chunk)
    return launch_parts(cache_join_kernel<D, kChunkRows * kChunkWaves, kChunkRows>, a, tiles,
                        kChunkRows * kChunkWaves / kWaves, kThreads, 0, s);
  const int rows = p.QT * (p.G < 16 ? p.G : 16);
  return launch_parts(cache_join_kernel<D, 16, 16>, a, tiles, (rows + kWaves - 1) / kWaves, kThreads, 0, s);
}

}  // namespace

bool cache_attn_fits(const DevCache& c, const DevBatch& b, int d, int Hq, int topk) {
  const Plan p = plan(c, b, d, Hq, topk);
  return p.items * c.H * p.RT * p.splits + 8 <= 0x7fffffff;
}

size_t cache_attn_workspace_bytes(const DevCache& c, const DevBatch& b, int d, int Hq, int topk) {
  const Plan p = plan(c, b, d, Hq, topk);
  if (p.splits == 1) return 0;
  const size_t tiles = size_t(p.items) * c.H * p.RT, rows = p.chunk ? kChunkRows * kChunkWaves : 16;
  return join_bytes(tiles) + tiles * p.splits * rows * (d + 2) * 4;
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
  a.join = (JoinHead*)ws;
  a.part = (float*)((char*)ws + join_bytes(size_t(p.items) * c.H * p.RT));
  a.splits = p.splits;
  a.items = p.items;
  a.wgs = p.wgs;
  hipError_t e;
  if (p.chunk) e = launch_chunk_attn(a, d, s);
  else if (d == 128) e = c.fp4 ? run<128, true>(a, p, s) : run<128, false>(a, p, s);
  else e = c.fp4 ? run<64, true>(a, p, s) : run<64, false>(a, p, s);
  if (e != hipSuccess || p.splits == 1) return e;
  return d == 128 ? join<128>(a, p, s) : join<64>(a, p, s);
}

}  // namespace spade
