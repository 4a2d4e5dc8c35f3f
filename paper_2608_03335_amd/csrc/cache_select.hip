// Page selection (gfx950): Top-K pages for every query and K/V head.
//
// score(t, h, j) = sum_c (sum_g q[t, h G + g, c]) mean[j, h, c]: the mean estimate of the
// block selection with the query side summed over the heads that share a K/V head. Every
// (query, head) keeps min(topk, visible) pages: the first `sink` and last `local` ones,
// then by (score descending, index ascending), a NaN after every number.
//
// The result is that of fp64 scores: the heads in order, then 16 runs of d / 16 channels,
// added pairwise, the same for every page. (Terms that span fewer than some 23 bits sum exactly;
// wider ones are off by (G + d) 2^-53 of their sizes' sum at most, and only pages closer than that
// depend on the order.) Nearly every page is decided by far less. Two kernels:
//   scores  s~ on the matrix unit: tiles of 16 queries x 128 pages, the summed query split
//           into two bf16 terms. |s~ - s| <= E = 2^-13 |A|_1 M, with A = sum_g |q| and M the
//           largest |mean| of the walk: 2^-16 A for the third term left out, G 2^-24 A for
//           the sum over g, 2 d 2^-23 A for fp32 accumulation, each times M, and as much
//           again to spare; and 2^-118 (A + M + 1) for what underflows.
//   top-k   the k-th largest s~, T, by bits of its order-preserving integer; pages above
//           T + 2 E are in, below T - 2 E out (the k-th largest s is within E of T). Only
//           where more pages lie between than places are left are their scores computed in
//           fp64 (usually two or three pages in a row out of three), and ranked the same way.
// A row with an infinity or NaN in sight is ranked in fp64 as a whole.
//
// Scores are bound by the means' bytes (d bf16 a page and head), in short launches by the
// latency of one chain: offsets, table, means, product. The search makes about 20 passes over
// a row's scores, which a wave holds in registers, each waiting for the last. Measured: 16
// sequences of up to 1024 pages, 8 heads of 128, one query each: scores 13 us (18 MB), search
// 11; 3890 queries, 2 heads of 64, 513 pages: 20 and 31.
#include "cache.h"

namespace spade {
namespace {

constexpr int kThreads = 256;
constexpr int kTileQ = 16;       // queries a score tile
constexpr int kTileP = 128;      // pages a score tile
constexpr int kMaxVals = 16;     // scores a lane holds, at most
constexpr int kFew = 64;         // pages in doubt that are ranked by comparing all pairs
constexpr int64_t kSlab = int64_t(1) << 26;  // scores kept at once

struct SelectArgs {
  DevCache c;
  DevBatch b;
  const __bf16* q;
  int Hq, G, topk, sink, local;
  int causal;
  int* counts;
  int* indices;
  // scratch of a slab: tokens t0..t1-1
  int t0, t1, stride, chunks, chunk_tiles;
  float* score;   // [tokens, H, stride]
  float* a1;      // [tokens, H]: |A|_1
  float* m;       // [items, H, chunks]: largest |mean|
};

// Visible pages of token i of a sequence's n.
__device__ __forceinline__ int visible(const SelectArgs& a, int64_t raw, int n, int i) {
  const int64_t P = a.c.page;
  const int64_t len = min(max(raw, int64_t(0)), int64_t(a.b.max_pages) * P);
  const int64_t seen = a.causal ? min(max(raw - n + i + 1, int64_t(0)), len) : len;
  return int((seen + P - 1) / P);
}

template <int D>
__global__ void __launch_bounds__(kThreads) cache_score_kernel(SelectArgs a) {
  constexpr int KK = D / 32;
  __shared__ uint32_t top;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, g = lane >> 4;
  const int item = blockIdx.x, h = blockIdx.y, chunk = blockIdx.z;
  if (tid == 0) top = 0;
  const SeqItem it = find_item(a.b, item, kTileQ, 1, a.t0, a.t1);
  if (it.b < 0) return;
  const int b = it.b, t = it.t0 + it.first * kTileQ, nq = min(kTileQ, it.t0 + it.n - t);
  if (nq <= 0) return;
  const int pages = visible(a, it.len, it.all, t + nq - 1 - it.start);
  const int first = chunk * a.chunk_tiles * kTileP;
  if (first >= pages) return;
  const int end = min(pages, first + a.chunk_tiles * kTileP);

  const int* table = a.b.table + int64_t(b) * a.b.max_pages;
  // means of this wave's 2 x 16 pages of a tile: the A operand
  cu32x4 f[2][KK];
  auto load = [&](int c0) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int j = c0 + (wave * 2 + i) * 16 + (lane & 15);
      const int phys = j < end ? table[j] : 0;
      const bool ok = phys >= 0 && phys < a.c.n_pages;
      const __bf16* src = (const __bf16*)a.c.mean + (int64_t(ok ? phys : 0) * a.c.H + h) * D + g * 8;
#pragma unroll
      for (int k = 0; k < KK; ++k) {
        const cu32x4 x = *(const cu32x4*)(src + k * 32);
        const cu32x4 bad = {0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u};
        f[i][k] = ok ? x : bad;
      }
    }
  };
  load(first);  // on its way while the queries are summed
  // summed queries in two terms: the B operand
  const bool live = (lane & 15) < nq;
  const __bf16* q = a.q + (int64_t(t + (live ? lane & 15 : 0)) * a.Hq + int64_t(h) * a.G) * D + g * 8;
  float sum[KK][8] = {}, mag = 0.0f;
#pragma unroll 4
  for (int i = 0; i < a.G; ++i) {
#pragma unroll
    for (int k = 0; k < KK; ++k) {
      const cbf16x8 x = *(const cbf16x8*)(q + i * D + k * 32);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float v = float(x[e]);
        sum[k][e] += v;
        mag += fabsf(v);
      }
    }
  }
  cbf16x8 hi[KK], lo[KK];
#pragma unroll
  for (int k = 0; k < KK; ++k)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      hi[k][e] = (__bf16)sum[k][e];
      lo[k][e] = (__bf16)(sum[k][e] - float(hi[k][e]));
    }
  const int64_t row = int64_t(t - a.t0 + (lane & 15)) * a.c.H + h;
  uint32_t m = 0;  // the largest |mean|, as its bits
  for (int c0 = first; c0 < end; c0 += kTileP) {
    if (c0 > first) load(c0);
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (c0 + (wave * 2 + i) * 16 + (lane & 15) < end)
#pragma unroll
        for (int k = 0; k < KK; ++k)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t y = f[i][k][e];
            m = max(m, max(y & 0x7fff0000u, (y << 16) & 0x7fff0000u));
          }
    cf32x4 acc[2] = {};
#pragma unroll
    for (int k = 0; k < KK; ++k)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const cbf16x8 x = __builtin_bit_cast(cbf16x8, f[i][k]);
        acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, hi[k], acc[i], 0, 0, 0);
        acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, lo[k], acc[i], 0, 0, 0);
      }
    if (live) {
      float* dst = a.score + row * a.stride + c0 + wave * 32 + g * 4;
      *(cf32x4*)dst = acc[0];
      *(cf32x4*)(dst + 16) = acc[1];
    }
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) m = max(m, __shfl_xor(m, o));
  if (lane == 0) atomicMax(&top, m);
  mag += __shfl_xor(mag, 16);
  mag += __shfl_xor(mag, 32);
  if (chunk == 0 && wave == 0 && g == 0 && live)
    a.a1[int64_t(t - a.t0 + lane) * a.c.H + h] = mag;
  __syncthreads();
  if (tid == 0) a.m[(int64_t(item) * a.c.H + h) * a.chunks + chunk] = __uint_as_float(top);
}

// Order-preserving integers: larger score, larger key; NaN lowest, -0 as +0.
__device__ __forceinline__ uint32_t key32(float x) {
  if (!(x == x)) return 0;
  const uint32_t u = __float_as_uint(x + 0.0f);
  return u >> 31 ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float key32_value(uint32_t k) {
  return __uint_as_float(k >> 31 ? k & 0x7fffffffu : ~k);
}
__device__ __forceinline__ uint64_t key64(double x) {
  if (!(x == x)) return 0;
  const uint64_t u = __builtin_bit_cast(uint64_t, x + 0.0);
  return u >> 63 ? ~u : u | (uint64_t(1) << 63);
}

// The W waves of a row.
template <int W>
struct Team {
  int* slots;  // LDS, 2 x W
  int wave, turn;
  __device__ __forceinline__ int sum(int wave_count) {
    if constexpr (W == 1) return wave_count;
    int* s = slots + (turn & 1) * W;
    ++turn;
    if ((threadIdx.x & 63) == 0) s[wave] = wave_count;
    __syncthreads();
    int all = 0;
#pragma unroll
    for (int i = 0; i < W; ++i) all += s[i];
    return all;
  }
  __device__ __forceinline__ float most(float x) {  // W > 1
    int* s = slots + (turn & 1) * W;
    ++turn;
    if ((threadIdx.x & 63) == 0) s[wave] = __float_as_int(x);
    __syncthreads();
    float y = __int_as_float(s[0]);
#pragma unroll
    for (int i = 1; i < W; ++i) y = fmaxf(y, __int_as_float(s[i]));
    return y;
  }
};

// The largest t that at least k of the lanes' keys reach (0 where fewer are above 0: keys that
// do not compete are 0). Stops as soon as exactly k do: then t lies between the k-th largest
// key and the next.
template <int W, int VALS, typename K>
__device__ __forceinline__ K kth_largest(const K* key, int k, Team<W>& team) {
  K t = 0;
  for (int bit = sizeof(K) * 8 - 1; bit >= 0; --bit) {
    const K cand = t | K(1) << bit;
    int n = 0;
#pragma unroll
    for (int v = 0; v < VALS; ++v) n += __popcll(__ballot(key[v] >= cand));
    n = team.sum(n);
    if (n >= k) t = cand;
    if (n == k) break;
  }
  return t;
}

// W waves of VALS scores a lane rank one row; kThreads / 64 / W rows a workgroup (W <= 4), 16
// waves for the longest.
// The k-th largest of the row's scores (NaN: no score), all within [low, top] of the lane. One
// wave halves the interval, which isolates the k largest in about eleven steps; scores too
// close for that are told apart by the bits of their keys. Several waves go by the bits at
// once: a step costs them a barrier, and the interval's ends four more.
template <int W, int VALS>
__device__ __forceinline__ float kth_score(const float* x, int nv, int k, float low, float top,
                                           Team<W>& team) {
  bool found = false;
  float cut = 0.0f;
  if constexpr (W == 1) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      top = fmaxf(top, __shfl_xor(top, o));
      low = fminf(low, __shfl_xor(low, o));
    }
    for (int i = 0; i < 16 && !found; ++i) {
      cut = low + 0.5f * (top - low);
      int mine = 0, n = 0;  // of this lane, at most 16: summed over the lanes bit by bit
#pragma unroll
      for (int v = 0; v < VALS; ++v) {
        if (v >= nv) break;
        mine += x[v] >= cut;
      }
#pragma unroll
      for (int j = 0; (1 << j) <= VALS; ++j) n += __popcll(__ballot(mine >> j & 1)) << j;
      found = n == k;
      if (n > k) low = cut; else top = cut;
    }
  }
  if (!found) {
    uint32_t key[VALS];
#pragma unroll
    for (int v = 0; v < VALS; ++v) key[v] = v < nv ? key32(x[v]) : 0;
    cut = key32_value(kth_largest<W, VALS>(key, k, team));
  }
  // the least score that reaches the cut
  float least = __builtin_huge_valf();
#pragma unroll
  for (int v = 0; v < VALS; ++v) {
    if (v >= nv) break;
    if (x[v] >= cut) least = fminf(least, x[v]);
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) least = fminf(least, __shfl_xor(least, o));
  if constexpr (W > 1) least = -team.most(-least);
  return least;
}

template <int D, int W, int VALS>
__global__ void __launch_bounds__(W == 16 ? 1024 : kThreads) cache_topk_kernel(SelectArgs a) {
  constexpr int ROWS = W == 16 ? 1 : kThreads / 64 / W;
  __shared__ int slots[W == 1 ? 1 : 2 * W], before[VALS][W];
  __shared__ int few_page[ROWS][kFew];
  __shared__ uint64_t few_key[ROWS][kFew];
  const int lane = threadIdx.x & 63;
  const int wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t r = int64_t(blockIdx.x) * ROWS + wid / W;
  const int64_t rows = int64_t(a.t1 - a.t0) * a.c.H;
  if (r >= rows) return;  // W > 1: one row a workgroup, all waves leave
  const int t = a.t0 + int(r / a.c.H), h = int(r % a.c.H);
  // the row's sequence: a lane looks at every 64th (of many: at every 64th of those that are left)
  int b = -1, lo = 0, vis = 0;
  int first_b = 0, n_b = a.b.B;  // one of first_b..first_b+n_b-1: the last that begins before t
  while (n_b > kScan / 4) {
    const int step = (n_b + 63) / 64, at = lane * step;
    const bool before = at < n_b && min(max(a.b.cu[first_b + at], 0), a.b.n_tokens) <= t;
    const int skip = max(__popcll(__ballot(before)) - 1, 0) * step;
    first_b += skip;
    n_b = min(n_b - skip, step);
  }
  for (int b0 = first_b; b0 < first_b + n_b && b < 0; b0 += 64) {
    const int i = b0 + lane;
    int start = 0, end = 0, len = 0;
    if (i < first_b + n_b) {
      start = min(max(a.b.cu[i], 0), a.b.n_tokens);
      end = min(max(a.b.cu[i + 1], 0), a.b.n_tokens);
      len = a.b.lens[i];
    }
    const uint64_t hits = __ballot(start <= t && t < end);
    if (hits) {
      const int l = __builtin_ctzll(hits);
      b = b0 + l;
      start = __builtin_amdgcn_readlane(start, l);
      lo = max(start, a.t0);
      vis = visible(a, __builtin_amdgcn_readlane(len, l), __builtin_amdgcn_readlane(end, l) - start, t - start);
    }
  }
  if (b < 0) return;
  const int keep = min(a.topk, vis);
  const int64_t out = int64_t(t) * a.c.H + h;
  Team<W> team{slots, wid % W, 0};
  if (team.wave == 0 && lane == 0) a.counts[out] = keep;
  if (keep == 0) return;
  // pages first..last-1 compete for `places`
  const int first = min(a.sink, vis), last = max(vis - a.local, first);
  const int places = keep - (vis - (last - first));
  const bool ranked = places < last - first;

  // this lane's pages: v * 64 W + 64 wave + lane
  const int p0 = team.wave * 64 + lane;
  const int nv = __builtin_amdgcn_readfirstlane((vis + 64 * W - 1) / (64 * W));
  float x[VALS];
  uint32_t in = 0, kept = 0;
#pragma unroll
  for (int v = 0; v < VALS; ++v) {
    if (v >= nv) break;
    const int j = v * 64 * W + p0;
    if (j >= first && j < last) in |= 1u << v;
    else if (j < vis) kept |= 1u << v;
  }
  if (!ranked) {
    kept |= in;
  } else if (places > 0) {
    // the summed query in fp64, 16 lanes sharing its channels. Few rows: at once, since nearly
    // every row asks for it and waits; many rows: those that need it
    constexpr int C = D / 16;
    const int c0 = (lane & 15) * C;
    double qs[C] = {};
    auto sum_query = [&] {
      const __bf16* q = a.q + (int64_t(t) * a.Hq + int64_t(h) * a.G) * D + c0;
#pragma unroll 4
      for (int i = 0; i < a.G; ++i)
#pragma unroll
        for (int e = 0; e < C; ++e) qs[e] += double(float(q[i * D + e]));
    };
    if constexpr (W > 1) sum_query();
    const float* s = a.score + (int64_t(t - a.t0) * a.c.H + h) * a.stride;
    bool odd = false;
    float top = -__builtin_huge_valf(), low = __builtin_huge_valf();
#pragma unroll
    for (int v = 0; v < VALS; ++v) {
      if (v >= nv) break;
      const bool c = in >> v & 1;
      x[v] = c ? s[v * 64 * W + p0] : __builtin_nanf("");  // a NaN reaches no threshold
      odd |= c && !(fabsf(x[v]) <= 3.0e37f);
      top = fmaxf(top, x[v]);
      low = fminf(low, x[v]);
    }
    // E; a row that holds what is not finite is ranked in fp64
    const int item = item_base(lo - a.t0, b, kTileQ, 1) + (t - lo) / kTileQ;
    const float* m = a.m + (int64_t(item) * a.c.H + h) * a.chunks;
    uint32_t big = 0;
    for (int i = lane; i * a.chunk_tiles * kTileP < vis; i += 64) big = max(big, __float_as_uint(m[i]));
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) big = max(big, __shfl_xor(big, o));
    const float A = a.a1[int64_t(t - a.t0) * a.c.H + h], M = __uint_as_float(big);
    const float E = A * M * 0x1p-13f + (A + M + 1.0f) * 0x1p-118f;
    odd |= !(E <= 1.0e37f);
    const bool exact_all = team.sum(__popcll(__ballot(odd))) > 0;
    uint32_t open = in;  // pages to rank in fp64
    int need = places, n_open = last - first;
    if (!exact_all) {
      const float T = kth_score<W, VALS>(x, nv, places, low, top, team);
      const float hi = T + 2.0f * E, lo = T - 2.0f * E;
      open = 0;
      int n_in = 0;
      n_open = 0;
#pragma unroll
      for (int v = 0; v < VALS; ++v) {
        if (v >= nv) break;
        const bool sure = x[v] > hi, maybe = !sure && x[v] >= lo;
        if (sure) kept |= 1u << v;
        if (maybe) open |= 1u << v;
        n_in += __popcll(__ballot(sure));
        n_open += __popcll(__ballot(maybe));
      }
      n_in = team.sum(n_in);
      n_open = team.sum(n_open);
      need = places - n_in;
      if (n_open == need) {
        kept |= open;
        open = 0;
        need = 0;
      }
    }
    if (need > 0) {
      if constexpr (W == 1) sum_query();
      // key of the page this lane's 16 lanes were given (-1: none)
      auto page_key = [&](int page) {
        double x = 0.0;
        bool ok = false;
        if (page >= 0) {
          const int phys = a.b.table[int64_t(b) * a.b.max_pages + page];
          ok = phys >= 0 && phys < a.c.n_pages;
          if (ok) {
            const __bf16* mean = (const __bf16*)a.c.mean + (int64_t(phys) * a.c.H + h) * D + c0;
#pragma unroll
            for (int e = 0; e < C; ++e) x += qs[e] * double(float(mean[e]));
          }
        }
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) x += __shfl_xor(x, o);
        return ok ? key64(x) : uint64_t(0);
      };
      if (n_open <= kFew) {
        // gather them; every pair is compared
        int* pages = few_page[wid / W];
        uint64_t* keys = few_key[wid / W];
        int at = 0;
        if constexpr (W > 1) {
          __syncthreads();
#pragma unroll
          for (int v = 0; v < VALS; ++v) {
            const int n = __popcll(__ballot(open >> v & 1));
            if (lane == 0) before[v][team.wave] = n;
          }
          __syncthreads();
        }
#pragma unroll
        for (int v = 0; v < VALS; ++v) {
          if (v >= nv) break;
          const uint64_t bits = __ballot(open >> v & 1);
          int mine = at + __popcll(bits & ((uint64_t(1) << lane) - 1));
          if constexpr (W > 1) {
#pragma unroll
            for (int i = 0; i < W; ++i) {
              mine += i < team.wave ? before[v][i] : 0;
              at += before[v][i];
            }
          } else {
            at += __popcll(bits);
          }
          if (open >> v & 1) pages[mine] = v * 64 * W + p0;
        }
        if constexpr (W > 1) __syncthreads();
        for (int i = team.wave * 4; i < n_open; i += 4 * W) {
          const int mine = i + (lane >> 4);
          const uint64_t x = page_key(mine < n_open ? pages[mine] : -1);
          if ((lane & 15) == 0 && mine < n_open) keys[mine] = x;
        }
        if constexpr (W > 1) __syncthreads();
        // pages ascend in the list: an equal key before this one wins
        const uint64_t my_key = lane < n_open ? keys[lane] : 0;
        const int my_page = lane < n_open ? pages[lane] : 0;
        int rank = 0;
        for (int i = 0; i < n_open; ++i) {
          const uint64_t x = keys[i];
          rank += x > my_key || (x == my_key && i < lane);
        }
        uint64_t won = __ballot(lane < n_open && rank < need);
        while (won) {
          const int page = __builtin_amdgcn_readlane(my_page, __builtin_ctzll(won));
          won &= won - 1;
          if ((page & 63) == lane && (page >> 6) % W == team.wave) kept |= 1u << (page / (64 * W));
        }
      } else {
        uint64_t wide[VALS];
#pragma unroll
        for (int v = 0; v < VALS; ++v) {
          wide[v] = 0;
          uint64_t todo = __ballot(open >> v & 1);
          while (todo) {
            int who[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              who[i] = todo ? __builtin_ctzll(todo) : -1;
              todo &= todo - 1;
            }
            const int mine = lane < 16 ? who[0] : lane < 32 ? who[1] : lane < 48 ? who[2] : who[3];
            const uint64_t x = page_key(mine < 0 ? -1 : v * 64 * W + team.wave * 64 + mine);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const uint64_t got = __shfl(x, i * 16);
              if (lane == who[i]) wide[v] = got;
            }
          }
        }
        const uint64_t tk = kth_largest<W, VALS>(wide, need, team);
        // above the threshold all; at it the first ones, unless the search found just enough
        int above = 0, at = 0;
#pragma unroll
        for (int v = 0; v < VALS; ++v) {
          above += __popcll(__ballot((open >> v & 1) && wide[v] > tk));
          at += __popcll(__ballot((open >> v & 1) && wide[v] >= tk));
        }
        above = team.sum(above);
        at = team.sum(at);
        if (at == need) {
#pragma unroll
          for (int v = 0; v < VALS; ++v)
            if ((open >> v & 1) && wide[v] >= tk) kept |= 1u << v;
        } else {
          int left = need - above, seen = 0;
#pragma unroll
          for (int v = 0; v < VALS; ++v) {
            const bool eq = (open >> v & 1) && wide[v] == tk;
            const uint64_t bits = __ballot(eq);
            int mine = seen;
            if constexpr (W > 1) {
              __syncthreads();
              if (lane == 0) before[v][team.wave] = __popcll(bits);
              __syncthreads();
#pragma unroll
              for (int i = 0; i < W; ++i) {
                mine += i < team.wave ? before[v][i] : 0;
                seen += before[v][i];
              }
            } else {
              seen += __popcll(bits);
            }
            mine += __popcll(bits & ((uint64_t(1) << lane) - 1));
            if (((open >> v & 1) && wide[v] > tk) || (eq && mine < left)) kept |= 1u << v;
          }
        }
      }
    }
  }

  // the kept pages, ascending
  int* dst = a.indices + out * a.topk;
  if constexpr (W > 1) {
    __syncthreads();
#pragma unroll
    for (int v = 0; v < VALS; ++v) {
      const int n = __popcll(__ballot(kept >> v & 1));
      if (lane == 0) before[v][team.wave] = n;
    }
    __syncthreads();
  }
  int at = 0;
#pragma unroll
  for (int v = 0; v < VALS; ++v) {
    if (v >= nv) break;
    const uint64_t bits = __ballot(kept >> v & 1);
    int mine = at + __popcll(bits & ((uint64_t(1) << lane) - 1));
    if constexpr (W > 1) {
#pragma unroll
      for (int i = 0; i < W; ++i) {
        mine += i < team.wave ? before[v][i] : 0;
        at += before[v][i];
      }
    } else {
      at += __popcll(bits);
    }
    if (kept >> v & 1) dst[mine] = v * 64 * W + p0;
  }
}

struct Plan {
  int stride, chunks, chunk_tiles, tokens;  // of a slab
  size_t score, a1, m;         // bytes
};

Plan plan(const DevCache& c, const DevBatch& b) {
  Plan p;
  const int tiles = (b.max_pages + kTileP - 1) / kTileP;
  p.stride = tiles * kTileP;
  const int64_t tokens = kSlab / (int64_t(c.H) * p.stride);
  p.tokens = int(tokens < 1 ? 1 : tokens < b.n_tokens ? tokens : b.n_tokens);
  // a workgroup walks several page tiles (its start costs as much as five) where the card is
  // full without more of them
  const int64_t items = int64_t(item_base(p.tokens, b.B, kTileQ, 1)) * c.H;
  const int64_t want = (1024 + items - 1) / items;
  p.chunk_tiles = int(want >= tiles ? 1 : (tiles + want - 1) / want);
  p.chunks = (tiles + p.chunk_tiles - 1) / p.chunk_tiles;
  auto up = [](size_t x) { return (x + 255) / 256 * 256; };
  p.score = up(size_t(p.tokens) * c.H * p.stride * 4);
  p.a1 = up(size_t(p.tokens) * c.H * 4);
  p.m = up(size_t(item_base(p.tokens, b.B, kTileQ, 1)) * c.H * p.chunks * 4);
  return p;
}

template <int D>
hipError_t run(SelectArgs& a, const Plan& p, hipStream_t s) {
  for (int t0 = 0; t0 < a.b.n_tokens; t0 += p.tokens) {
    a.t0 = t0;
    a.t1 = t0 + p.tokens < a.b.n_tokens ? t0 + p.tokens : a.b.n_tokens;
    const int n = a.t1 - a.t0;
    cache_score_kernel<D><<<dim3(unsigned(item_base(n, a.b.B, kTileQ, 1)), a.c.H, p.chunks), kThreads, 0, s>>>(a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int64_t rows = int64_t(n) * a.c.H;
    // four waves a row where rows are few (128 rows of 1024 pages: 11.6 us, one wave 24), one
    // where they fill the card
    if (a.b.max_pages <= 256)
      cache_topk_kernel<D, 1, 4><<<dim3(unsigned((rows + 3) / 4)), kThreads, 0, s>>>(a);
    else if (a.b.max_pages <= 1024 && rows < 2048)
      cache_topk_kernel<D, 4, 4><<<dim3(unsigned(rows)), kThreads, 0, s>>>(a);
    else if (a.b.max_pages <= 1024)
      cache_topk_kernel<D, 1, 16><<<dim3(unsigned((rows + 3) / 4)), kThreads, 0, s>>>(a);
    else if (a.b.max_pages <= 4096)
      cache_topk_kernel<D, 4, 16><<<dim3(unsigned(rows)), kThreads, 0, s>>>(a);
    else
      cache_topk_kernel<D, 16, 16><<<dim3(unsigned(rows)), 1024, 0, s>>>(a);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

static_assert(kCacheMaxPages <= 1024 * kMaxVals, "sixteen waves hold the longest row");

}  // namespace

bool cache_select_fits(const DevCache& c, const DevBatch& b) {
  const Plan p = plan(c, b);
  return int64_t(item_base(p.tokens, b.B, kTileQ, 1)) * c.H * p.chunks <= 0x7fffffff;
}

size_t cache_select_workspace_bytes(const DevCache& c, const DevBatch& b, int, int, int) {
  const Plan p = plan(c, b);
  return p.score + p.a1 + p.m;
}

hipError_t launch_cache_select(const DevCache& c, const DevBatch& b, int d, const CacheSelect& x,
                               void* ws, hipStream_t s) {
  const Plan p = plan(c, b);
  SelectArgs a;
  a.c = c;
  a.b = b;
  a.q = (const __bf16*)x.q;
  a.Hq = x.Hq;
  a.G = x.Hq / c.H;
  a.topk = x.topk;
  a.sink = x.sink;
  a.local = x.local;
  a.causal = x.causal;
  a.counts = x.counts;
  a.indices = x.indices;
  a.stride = p.stride;
  a.chunks = p.chunks;
  a.chunk_tiles = p.chunk_tiles;
  a.score = (float*)ws;
  a.a1 = (float*)((char*)ws + p.score);
  a.m = (float*)((char*)ws + p.score + p.a1);
  return d == 128 ? run<128>(a, p, s) : run<64>(a, p, s);
}

}  // namespace spade
