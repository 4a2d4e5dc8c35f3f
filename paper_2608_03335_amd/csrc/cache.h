// Paged key/value cache (gfx950): the page layout and what its kernels share.
//
// A page holds P tokens of every K/V head (P a multiple of 32), laid out as the matrix
// instructions read it, so that every wave load of the attention is one contiguous piece
// and needs no transpose:
//   K, bf16: [tile of 16 tokens][d / 32][g: 4][m: 16][8 channels], the A operand of
//            mfma 16x16x32: token 16 tile + m, channel 32 s + 8 g + j; 1 KB a load.
//   V, bf16: [block of 32 tokens][d / 16][g: 4][m: 16][8 tokens], the A operand of
//            O^T = V^T P^T: channel 16 ct + m, tokens 4 g + {0..3} and 16 + 4 g + {0..3}:
//            those whose scores the lane holds after the K product, so P needs no shuffle.
//   4 bits:  e2m1 values (0, .5, 1, 1.5, 2, 3, 4, 6 with sign), one power of two for each
//            32 channels of a token, stored as its exponent + 127.
//   K, 4 bit: [tile][g][m][d / 4 channels], channel (d / 4) g + i: at d = 128 a lane's 16
//            bytes are one scale group. Scales [tile][d / 32][m].
//   V, 4 bit: [block][d / 64][g][m][4 column tiles][8 tokens]. Scales [block][g][d / 32][8
//            tokens], the lane's eight in one piece.
//   mean:    bf16 [page][H][d], the mean of the page's stored keys.
#pragma once

#include "spade_internal.h"

namespace spade {

struct DevCache {
  int H, page, n_pages;
  bool fp4;
  void* k;
  void* v;
  uint8_t* ks;
  uint8_t* vs;
  void* mean;
};

struct DevBatch {
  int B, max_pages, n_tokens;
  const int* table;
  const int* lens;
  const int* cu;
};

struct DevRope {
  const float* cos;
  const float* sin;
  const int* pos;
  int n_pos, rot, interleaved;
};

bool cache_append_fits(const DevCache& c, const DevBatch& b, int d, int Hq);  // its grid
hipError_t launch_cache_append(const DevCache& c, const DevBatch& b, int d, const DevRope& r,
                               const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                               const void* q, int64_t q_stride, int Hq, void* q_out,
                               hipStream_t s);
// Pages of a sequence that N tokens take.
inline int cache_read_pages(const DevCache& c, const DevBatch& b, int64_t N) {
  const int64_t pages = (N + c.page - 1) / c.page;
  return int(pages < b.max_pages ? pages : b.max_pages);
}
hipError_t launch_cache_read(const DevCache& c, const DevBatch& b, int d, int64_t N, void* k,
                             void* v, hipStream_t s);

struct CacheSelect {
  const void* q;
  int Hq, topk, sink, local;
  bool causal;
  int* counts;
  int* indices;
};
bool cache_select_fits(const DevCache& c, const DevBatch& b);  // its grid
size_t cache_select_workspace_bytes(const DevCache& c, const DevBatch& b, int d, int Hq, int topk);
hipError_t launch_cache_select(const DevCache& c, const DevBatch& b, int d, const CacheSelect& p,
                               void* ws, hipStream_t s);

struct CacheAttn {
  const void* q;
  int Hq, topk;         // topk 0: no lists, every visible token
  const int* counts;
  const int* indices;
  float scale;
  bool causal;
  void* o;
  float* lse;
};
bool cache_attn_fits(const DevCache& c, const DevBatch& b, int d, int Hq, int topk);  // its grid
size_t cache_attn_workspace_bytes(const DevCache& c, const DevBatch& b, int d, int Hq, int topk);
hipError_t launch_cache_attn(const DevCache& c, const DevBatch& b, int d, const CacheAttn& p,
                             void* ws, hipStream_t s);

constexpr int kCacheMaxPages = 16384;  // pages of a sequence that lists can name (LDS)
constexpr int kCacheMaxGroup = 128;    // query heads per K/V head

#ifdef __HIPCC__
typedef __bf16 cbf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 cbf16x8 __attribute__((ext_vector_type(8)));
typedef float cf32x4 __attribute__((ext_vector_type(4)));
typedef float cf32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t cu32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t cu32x2 __attribute__((ext_vector_type(2)));

// Launches workgroups 0..wgs-1 (fewer than 2^31) of a kernel whose arguments have a member
// `first`. A launch counts its threads in 32 bits: larger ones go in parts, each told its first
// workgroup.
template <typename Args>
hipError_t launch_parts(void (*kernel)(Args), Args a, int64_t wgs, int rows, int threads, int lds,
                        hipStream_t s) {
  const int64_t most = (int64_t(1) << 32) / threads - 8;  // a multiple of 8: XCDs keep their turns
  for (int64_t first = 0; first < wgs; first += most) {
    const int64_t n = wgs - first < most ? wgs - first : most;
    a.first = uint32_t(first);
    kernel<<<dim3(unsigned(n), unsigned(rows)), threads, lds, s>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// Work items cut from a batch: sequence b's new tokens cu[b]..cu[b+1]-1 fill at most
// floor(cu[b+1] / unit) - floor(cu[b] / unit) + extra items, a sum that telescopes, so
// item ranges need no scan over the sequences and the host knows their total.
struct SeqItem {
  int b;         // -1: no such item
  int first;     // index of the item inside the sequence
  int t0, n;     // the sequence's new tokens (inside from..to)
  int start, all;  // its first new token and their number, whatever from and to
  int64_t len;   // tokens in its cache, as given
};

// (at most 2^28 tokens and 2^20 sequences: 32 bits hold it)
__host__ __device__ inline int item_base(int tokens, int b, int unit, int extra) {
  return tokens / unit + extra * b;
}

// Finds the sequence of a work item among the tokens from..to-1: every thread of the block
// looks at some sequences, so the search and the sequence's length cost one load latency; of
// more than kScan sequences, a load latency more for each factor of the block's threads. All
// threads of the block must call. Offsets that do not ascend cannot lead out of the batch's
// arrays: an item then belongs to one of the sequences that claim it, or to none.
constexpr int kScan = 1024;
__device__ __forceinline__ SeqItem find_item(const DevBatch& bt, int item, int unit, int extra,
                                             int from, int to) {
  __shared__ int hit, info[5];
  if (threadIdx.x == 0) hit = -1;
  __syncthreads();
  SeqItem r;
  r.b = -1;
  r.len = 0;
  r.start = r.all = r.t0 = r.n = 0;
  int b0 = 0, n = bt.B;  // the item's sequence is one of b0..b0+n-1: the last that begins before it
  while (n > kScan) {
    const int step = (n + blockDim.x - 1) / blockDim.x, at = int(threadIdx.x) * step;
    bool before = false;
    if (at < n) {
      const int start = min(max(bt.cu[b0 + at], 0), bt.n_tokens);
      before = item_base(min(max(start, from), to) - from, b0 + at, unit, extra) <= item;
    }
    const int skip = max(__syncthreads_count(before) - 1, 0) * step;
    b0 += skip;
    n = min(n - skip, step);
  }
  for (int b = b0 + threadIdx.x; b < b0 + n; b += blockDim.x) {
    const int start = min(max(bt.cu[b], 0), bt.n_tokens), end = min(max(bt.cu[b + 1], 0), bt.n_tokens);
    const int len = bt.lens[b];
    const int lo = min(max(start, from), to), hi = min(max(end, from), to);
    if (hi > lo && item_base(lo - from, b, unit, extra) <= item &&
        item < item_base(hi - from, b + 1, unit, extra)) {
      r.b = b;
      r.t0 = lo;
      r.n = hi - lo;
      r.start = start;
      r.all = end - start;
      r.len = len;
      atomicMax(&hit, b);
    }
  }
  __syncthreads();
  const int found = __builtin_amdgcn_readfirstlane(hit);
  if (found >= 0 && r.b == found) {
    info[0] = r.t0;
    info[1] = r.n;
    info[2] = r.start;
    info[3] = r.all;
    info[4] = int(r.len);
  }
  __syncthreads();
  r.b = found;
  // (without a hit `info` is not set, and nobody reads what follows)
  // the same in every lane: kept in scalar registers, and so is what follows from them
  r.t0 = __builtin_amdgcn_readfirstlane(info[0]);
  r.n = __builtin_amdgcn_readfirstlane(info[1]);
  r.start = __builtin_amdgcn_readfirstlane(info[2]);
  r.all = __builtin_amdgcn_readfirstlane(info[3]);
  r.len = __builtin_amdgcn_readfirstlane(info[4]);
  r.first = item - item_base(r.t0 - from, r.b, unit, extra);
  return r;
}
__device__ __forceinline__ SeqItem find_item(const DevBatch& bt, int item, int unit, int extra) {
  return find_item(bt, item, unit, extra, 0, bt.n_tokens);
}

// 2^(code - 127); code 255, the mark of a group that held a NaN or an infinity, gives an
// infinity, and the group's values are stored as 0: 0 * inf is NaN wherever it is used.
__device__ __forceinline__ float scale_of(uint32_t code) { return __uint_as_float(code << 23); }

// The scales of a dword's four codes, one instruction each.
__device__ __forceinline__ void scales_of(uint32_t w, float* s) {
  uint32_t r;
  const uint32_t n = 23;
  asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:BYTE_0"
      : "=v"(r) : "v"(n), "v"(w));
  s[0] = __uint_as_float(r);
  asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:BYTE_1"
      : "=v"(r) : "v"(n), "v"(w));
  s[1] = __uint_as_float(r);
  asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:BYTE_2"
      : "=v"(r) : "v"(n), "v"(w));
  s[2] = __uint_as_float(r);
  asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:BYTE_3"
      : "=v"(r) : "v"(n), "v"(w));
  s[3] = __uint_as_float(r);
}

// bf16 pair from byte BYTE of x, times scale (a power of two: exact)
template <int BYTE>
__device__ __forceinline__ cbf16x2 fp4_pair(uint32_t x, float scale) {
  return __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, scale, BYTE);
}

// the eight values of a dword
__device__ __forceinline__ cbf16x8 fp4_eight(uint32_t x, float scale) {
  const cbf16x2 a = fp4_pair<0>(x, scale), b = fp4_pair<1>(x, scale), c = fp4_pair<2>(x, scale),
                d = fp4_pair<3>(x, scale);
  return cbf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
#endif

}  // namespace spade
