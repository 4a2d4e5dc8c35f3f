// Page selection for single queries (gfx950).
//
// score(t, h, j) = sum_c (sum_g q[t, h G + g, c]) mean[j, h, c]: the mean estimate of the
// block selection with the query side summed over the heads that share a K/V head. Every
// (query, head) keeps min(topk, visible) pages: the first `sink` and last `local` ones,
// then by (score descending, index ascending), a NaN after every number.
//
// Scores are fp64: a page's rank must not depend on the order of a sum.
#include "cache.h"

namespace spade {
namespace {

constexpr int kThreads = 256;

struct SelectArgs {
  DevCache c;
  DevBatch b;
  const __bf16* q;
  int Hq, topk, sink, local;
  int causal;
  int* counts;
  int* indices;
};

// Order-preserving map of a score: larger score, larger key; NaN lowest.
__device__ __forceinline__ uint64_t score_key(double x) {
  if (!(x == x)) return 0;
  x += 0.0;  // -0 ranks as +0
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  return u >> 63 ? ~u : u | (uint64_t(1) << 63);
}

// Sum of v over the block's threads before this one; *total: over all.
__device__ __forceinline__ int block_scan(int v, int* total) {
  __shared__ int wave_sum[kThreads / 64];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  int x = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(x, o);
    if (lane >= o) x += y;
  }
  __syncthreads();
  if (lane == 63) wave_sum[w] = x;
  __syncthreads();
  int before = 0, all = 0;
#pragma unroll
  for (int i = 0; i < kThreads / 64; ++i) {
    before += i < w ? wave_sum[i] : 0;
    all += wave_sum[i];
  }
  *total = all;
  return before + x - v;
}

// One workgroup a (query, K/V head).
template <int D>
__global__ void __launch_bounds__(kThreads) cache_select_kernel(SelectArgs a) {
  constexpr int LP = D / 8;  // lanes a page, 8 channels each
  extern __shared__ __attribute__((aligned(16))) char lds[];
  uint64_t* key = (uint64_t*)lds;
  __shared__ double qs[D];
  __shared__ int hist[256];
  __shared__ int pick[2];
  const int tid = threadIdx.x;
  const int t = blockIdx.x, h = blockIdx.y;
  const SeqItem it = find_item(a.b, t, 1, 0, kThreads);
  if (it.b < 0) return;
  const int P = a.c.page, G = a.Hq / a.c.H;
  const int64_t cap = int64_t(a.b.max_pages) * P;
  const int64_t len = min(max(int64_t(a.b.lens[it.b]), int64_t(0)), cap);
  int64_t seen = a.causal ? int64_t(a.b.lens[it.b]) - it.n + it.first + 1 : len;
  seen = min(max(seen, int64_t(0)), len);
  const int vis = int((seen + P - 1) / P);
  const int64_t row = int64_t(t) * a.c.H + h;
  const int keep = min(a.topk, vis);
  if (tid == 0) a.counts[row] = keep;
  if (keep == 0) return;

  if (tid < D) {
    const __bf16* q = a.q + (int64_t(t) * a.Hq + int64_t(h) * G) * D + tid;
    double s = 0.0;
    for (int g = 0; g < G; ++g) s += double(float(q[g * D]));
    qs[tid] = s;
  }
  __syncthreads();
  const int lane = tid % LP;
  const int* table = a.b.table + int64_t(it.b) * a.b.max_pages;
  for (int j0 = 0; j0 < vis; j0 += kThreads / LP) {
    const int j = j0 + tid / LP;
    double s = 0.0;
    bool have = false;
    if (j < vis) {
      const int phys = table[j];
      have = phys >= 0 && phys < a.c.n_pages;
      if (have) {
        const cbf16x8 m = *(const cbf16x8*)((const __bf16*)a.c.mean +
                                           (int64_t(phys) * a.c.H + h) * D + lane * 8);
#pragma unroll
        for (int i = 0; i < 8; ++i) s += qs[lane * 8 + i] * double(float(m[i]));
      }
    }
#pragma unroll
    for (int o = LP / 2; o > 0; o >>= 1) s += __shfl_xor(s, o);
    if (j < vis && lane == 0) {
      const bool forced = j < a.sink || j >= vis - a.local;
      key[j] = forced ? ~uint64_t(0) : have ? score_key(s) : 0;
    }
  }
  __syncthreads();

  // the keep-th largest key, digit by digit from the top
  uint64_t prefix = 0;
  int need = keep;  // how many of the keys that match the prefix so far
  for (int shift = 56; shift >= 0; shift -= 8) {
    hist[tid] = 0;
    __syncthreads();
    for (int j = tid; j < vis; j += kThreads) {
      const uint64_t k = key[j];
      if (shift == 56 || (k >> (shift + 8)) == prefix) atomicAdd(&hist[(k >> shift) & 255], 1);
    }
    __syncthreads();
    int all;
    // digits from the top: thread i holds digit 255 - i
    const int n = hist[255 - tid];
    const int before = block_scan(n, &all);
    if (before < need && need <= before + n) {
      pick[0] = 255 - tid;
      pick[1] = need - before;
    }
    __syncthreads();
    prefix = prefix << 8 | uint64_t(pick[0]);
    need = pick[1];
    __syncthreads();
  }
  // larger keys, and the first `need` of the equal ones, in page order
  int out = 0, equal = 0;
  int* dst = a.indices + row * a.topk;
  for (int j0 = 0; j0 < vis; j0 += kThreads) {
    const int j = j0 + tid;
    const uint64_t k = j < vis ? key[j] : 0;
    const bool eq = j < vis && k == prefix;
    int n_eq, n_take;
    const int e = equal + block_scan(eq, &n_eq);
    const bool take = j < vis && (k > prefix || (eq && e < need));
    const int at = out + block_scan(take, &n_take);
    if (take) dst[at] = j;
    equal += n_eq;
    out += n_take;
  }
}

}  // namespace

size_t cache_select_workspace_bytes(const DevCache&, const DevBatch&, int, int, int) { return 0; }

hipError_t launch_cache_select(const DevCache& c, const DevBatch& b, int d, const CacheSelect& p,
                               void*, hipStream_t s) {
  SelectArgs a;
  a.c = c;
  a.b = b;
  a.q = (const __bf16*)p.q;
  a.Hq = p.Hq;
  a.topk = p.topk;
  a.sink = p.sink;
  a.local = p.local;
  a.causal = p.causal;
  a.counts = p.counts;
  a.indices = p.indices;
  const void* fn = d == 128 ? (const void*)cache_select_kernel<128> : (const void*)cache_select_kernel<64>;
  const int bytes = b.max_pages * 8;
  if (bytes > 48 * 1024) {
    const hipError_t e = ensure_dynamic_lds(fn, kCacheMaxPages * 8);
    if (e != hipSuccess) return e;
  }
  const dim3 grid(b.n_tokens, c.H);
  if (d == 128) cache_select_kernel<128><<<grid, kThreads, bytes, s>>>(a);
  else cache_select_kernel<64><<<grid, kThreads, bytes, s>>>(a);
  return hipGetLastError();
}

}  // namespace spade
