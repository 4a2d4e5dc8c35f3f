// Append to the paged cache with the position rotation, and read-back (gfx950).
//
// Append. A workgroup owns one page of one K/V head and one side (K or V): it stages the
// page's tokens as rows in LDS, rotates and rounds the new ones on the way, and writes
// them out in the page's fragment order, so global reads are whole rows and global writes
// whole fragments wherever a fragment is all new. Only one workgroup touches a page's
// bytes, so 4-bit dwords shared with older tokens are merged without atomics. The K side
// also reads the page's older keys and writes the page's mean key: from the stored values,
// in fp64, so it is the same however the tokens arrived (one by one, in chunks, rewritten
// after a rewind). The remaining workgroups of the launch rotate the queries.
//
// Rotation: a' = a cos - b sin, b' = a sin + b cos in fp32, every product and sum rounded
// once (no fused multiply-add: the same bits as the elementary operations), then one
// rounding to bf16, the type keys are kept and multiplied in.
//
// 4 bits: e is the least exponent in [-126, 126] with max|x| <= 7 2^e over 32 channels, so
// that no element is off by more than half a step of its place in {0,.5,1,1.5,2,3,4,6} 2^e
// (7 is half way between 6 and the next step, 8); nearest, ties to even. At e = 126 the
// grid ends at 3 2^126, the last value bf16 can hold.
#include "cache.h"

namespace spade {
namespace {

constexpr int kThreads = 256;

// Rows of a page in LDS: 8 elements of padding keep rows 16-byte aligned and spread the
// column reads of the V side over the banks.
template <int D>
constexpr int lds_row() { return D + 8; }

__device__ __forceinline__ float lo_f(uint32_t x) { return __uint_as_float(x << 16); }
__device__ __forceinline__ float hi_f(uint32_t x) { return __uint_as_float(x & 0xffff0000u); }
__device__ __forceinline__ uint32_t pack(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(cf32x2{a, b}, cbf16x2));
}

struct Chunk2 {
  cu32x4 a, b;  // two pieces of 8 channels
};

// Channels of unit u (16 of a row's channels): a pair of 8-channel pieces. Units below
// rot / 16 are rotated: pieces i and i + rot/2 (halves) or one run of pairs (interleaved).
struct UnitPlace {
  int a, b;
  bool turn;
};
__device__ __forceinline__ UnitPlace unit_place(const DevRope& r, int u) {
  UnitPlace p;
  p.turn = u < (r.rot >> 4);
  p.a = p.turn && !r.interleaved ? u * 8 : u * 16;
  p.b = p.turn && !r.interleaved ? u * 8 + (r.rot >> 1) : u * 16 + 8;
  return p;
}

__device__ __forceinline__ Chunk2 rotate_unit(const DevRope& r, Chunk2 x, int u, int pos) {
#pragma clang fp contract(off)
  const int64_t at = int64_t(pos) * (r.rot >> 1) + u * 8;
  float c[8], s[8], v[16];
  *(cf32x4*)(c) = *(const cf32x4*)(r.cos + at);
  *(cf32x4*)(c + 4) = *(const cf32x4*)(r.cos + at + 4);
  *(cf32x4*)(s) = *(const cf32x4*)(r.sin + at);
  *(cf32x4*)(s + 4) = *(const cf32x4*)(r.sin + at + 4);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = lo_f(x.a[i]);
    v[2 * i + 1] = hi_f(x.a[i]);
    v[8 + 2 * i] = lo_f(x.b[i]);
    v[9 + 2 * i] = hi_f(x.b[i]);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float a = r.interleaved ? v[2 * i] : v[i], b = r.interleaved ? v[2 * i + 1] : v[i + 8];
    const float ac = a * c[i], bs = b * s[i], as = a * s[i], bc = b * c[i];
    if (r.interleaved) {
      v[2 * i] = ac - bs;
      v[2 * i + 1] = as + bc;
    } else {
      v[i] = ac - bs;
      v[i + 8] = as + bc;
    }
  }
  Chunk2 y;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    y.a[i] = pack(v[2 * i], v[2 * i + 1]);
    y.b[i] = pack(v[8 + 2 * i], v[9 + 2 * i]);
  }
  return y;
}

// The table row of new token t at place `place`, or -1: outside the tables.
__device__ __forceinline__ int rope_row(const DevRope& r, int t, int64_t place) {
  if (r.rot == 0) return 0;
  const int64_t p = r.pos ? int64_t(r.pos[t]) : place;
  return p >= 0 && p < r.n_pos ? int(p) : -1;
}

// Shift of a group with largest magnitude `top` (finite): see the head of the file.
__device__ __forceinline__ int group_exponent(float top) {
  const int e = int(__float_as_uint(top) >> 23) - 127 - 2;  // top in [4, 8) 2^e when normal
  int x = e < -126 ? -126 : e;
  if (top > 7.0f * __uint_as_float(uint32_t(x + 127) << 23)) ++x;
  return x;
}

// Code of value x = y 2^e; inv = 2^-e.
__device__ __forceinline__ uint32_t e2m1(float y, float inv, uint32_t most) {
  const float a = fabsf(y) * inv;
  uint32_t c = uint32_t(a > 0.25f) + uint32_t(a >= 0.75f) + uint32_t(a > 1.25f) +
               uint32_t(a >= 1.75f) + uint32_t(a > 2.5f) + uint32_t(a >= 3.5f) +
               uint32_t(a > 5.0f);
  c = min(c, most);
  return c | (c != 0 && y < 0.0f ? 8u : 0u);
}

// Quantises 32 channels (16 dwords of bf16 pairs) to 4 dwords of codes; returns the scale byte.
__device__ __forceinline__ uint32_t quantise32(const cu32x4 x[4], uint32_t code[4]) {
  float top = 0.0f;
  bool bad = false;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float a = fabsf(lo_f(x[i][j])), b = fabsf(hi_f(x[i][j]));
      bad |= !(a <= 3.4e38f) | !(b <= 3.4e38f);
      top = fmaxf(top, fmaxf(a, b));
    }
  if (bad) {
#pragma unroll
    for (int i = 0; i < 4; ++i) code[i] = 0;
    return 255;
  }
  const int e = group_exponent(top);
  const float inv = __uint_as_float(uint32_t(127 - e) << 23);  // e in [-126, 126]
  const uint32_t most = e == 126 ? 5u : 7u;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t c = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      c |= (e2m1(lo_f(x[i][j]), inv, most) | e2m1(hi_f(x[i][j]), inv, most) << 4) << (8 * j);
    code[i] = c;
  }
  return uint32_t(e + 127);
}

template <int D>
__device__ __forceinline__ int64_t page_elem(const DevCache& c, int phys, int h) {
  return (int64_t(phys) * c.H + h) * c.page * D;
}

// Tokens [0, n) of a page's K side as rows in LDS (n <= page; whole tiles are read).
template <int D, bool FP4>
__device__ __forceinline__ void stage_k(const DevCache& c, int phys, int h, int n, __bf16* rows) {
  constexpr int R = lds_row<D>();
  const int tiles = (n + 15) >> 4;
  const int64_t base = page_elem<D>(c, phys, h);
  if constexpr (!FP4) {
    const cu32x4* src = (const cu32x4*)((const __bf16*)c.k + base);
    for (int i = threadIdx.x; i < tiles * 16 * (D / 8); i += kThreads) {
      const int m = i & 15, sg = (i >> 4) % (D / 8), tile = i / (2 * D);
      const int r = tile * 16 + m;
      if (r < n) *(cu32x4*)(rows + r * R + sg * 8) = src[i];
    }
  } else {
    const uint8_t* src = (const uint8_t*)c.k + base / 2;
    const uint8_t* sc = c.ks + base / 32;
    for (int i = threadIdx.x; i < tiles * 16 * (D / 8); i += kThreads) {
      // one dword: 8 channels of token (tile, m), lane group g
      const int w = i % (D / 32), gm = i / (D / 32) % 64, tile = i / (2 * D);
      const int g = gm >> 4, m = gm & 15, r = tile * 16 + m;
      const int ch = g * (D / 4) + w * 8;
      const uint32_t x = *(const uint32_t*)(src + int64_t(i) * 4);
      const float s = scale_of(sc[tile * (D / 2) + (ch >> 5) * 16 + m]);
      if (r < n) *(cbf16x8*)(rows + r * R + ch) = fp4_eight(x, s);
    }
  }
}

// The same for the V side.
template <int D, bool FP4>
__device__ __forceinline__ void stage_v(const DevCache& c, int phys, int h, int n, __bf16* rows) {
  constexpr int R = lds_row<D>();
  const int blocks = (n + 31) >> 5;
  const int64_t base = page_elem<D>(c, phys, h);
  for (int i = threadIdx.x; i < blocks * 4 * D; i += kThreads) {
    const int kb = i / (4 * D);
    cbf16x8 x;
    int ch, g;
    if constexpr (!FP4) {  // i = (kb, ct, g, m)
      const int m = i & 15, ct = (i >> 6) % (D / 16);
      g = (i >> 4) & 3;
      ch = ct * 16 + m;
      x = *(const cbf16x8*)((const __bf16*)c.v + base + int64_t(i) * 8);
    } else {  // i = (kb, half, g, m, ct)
      const int ct = i & 3, m = (i >> 2) & 15, half = (i >> 8) % (D / 64);
      g = (i >> 6) & 3;
      ch = (half * 4 + ct) * 16 + m;
      const uint32_t w = *(const uint32_t*)((const uint8_t*)c.v + base / 2 + int64_t(i) * 4);
      const uint8_t* sc = c.vs + base / 32 + kb * D + (g * (D / 32) + (ch >> 5)) * 8;
      const cbf16x8 y = fp4_eight(w, 1.0f);
      // a power of two times an e2m1 value: exact in bf16
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = (__bf16)(float(y[j]) * scale_of(sc[j]));
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int r = kb * 32 + (j >> 2) * 16 + g * 4 + (j & 3);
      if (r < n) rows[r * R + ch] = x[j];
    }
  }
}

struct AppendArgs {
  DevCache c;
  DevBatch b;
  DevRope r;
  const __bf16* k;
  const __bf16* v;
  const __bf16* q;
  __bf16* q_out;
  int64_t k_stride, v_stride, q_stride;
  int Hq;
  int64_t page_wgs;  // the first workgroups: 2 per (page item, head)
};

template <int D, bool FP4>
__global__ void __launch_bounds__(kThreads) cache_append_kernel(AppendArgs a) {
  constexpr int R = lds_row<D>();
  constexpr int U = D / 16;
  extern __shared__ __attribute__((aligned(16))) char lds[];
  __bf16* rows = (__bf16*)lds;
  const int64_t wg = blockIdx.x;
  const int tid = threadIdx.x;

  if (wg >= a.page_wgs) {  // queries
    const int64_t i = (wg - a.page_wgs) * kThreads + tid;
    const int64_t row = i / U;
    const int u = int(i % U);
    const int64_t t = row / a.Hq;
    if (t >= a.b.n_tokens) return;
    const int hq = int(row - t * a.Hq);
    // the token's place: only needed where the caller gives no positions
    int64_t place = 0;
    bool live = true;
    {
      int lo = 0, hi = a.b.B;  // last b with cu[b] <= t
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (a.b.cu[mid] <= t) lo = mid; else hi = mid;
      }
      const int c0 = a.b.cu[lo], c1 = a.b.cu[lo + 1];
      live = c0 <= t && t < c1;
      place = int64_t(a.b.lens[lo]) - c1 + t;
    }
    if (!live) return;  // behind the last sequence: left as it was
    const int pos = rope_row(a.r, int(t), place);
    const UnitPlace p = unit_place(a.r, u);
    const __bf16* src = a.q + t * a.q_stride + int64_t(hq) * D;
    Chunk2 x{*(const cu32x4*)(src + p.a), *(const cu32x4*)(src + p.b)};
    if (p.turn && pos >= 0) x = rotate_unit(a.r, x, u, pos);
    __bf16* dst = a.q_out + row * D;
    *(cu32x4*)(dst + p.a) = x.a;
    *(cu32x4*)(dst + p.b) = x.b;
    return;
  }

  const bool vside = wg & 1;
  const int64_t ih = wg >> 1;
  const int h = int(ih % a.c.H);
  const int P = a.c.page;
  const SeqItem it = find_item(a.b, int(ih / a.c.H), P, 2);
  if (it.b < 0) return;
  const int64_t len = it.len;
  const int64_t start = len - it.n;  // place of the first new token
  const int64_t from = max(start, int64_t(0));
  const int64_t to = min(len, int64_t(a.b.max_pages) * P);
  const int64_t j = from / P + it.first;
  if (from >= to || j > (to - 1) / P) return;
  const int phys = a.b.table[int64_t(it.b) * a.b.max_pages + j];
  if (phys < 0 || phys >= a.c.n_pages) return;
  const int lo = int(max(from - j * P, int64_t(0)));
  const int hi = int(min(to - j * P, int64_t(P)));
  const int64_t tok0 = it.t0 + (j * P - start);  // new token at row r: tok0 + r
  const int64_t base = page_elem<D>(a.c, phys, h);

  // new tokens to LDS
  if (!vside) {
    stage_k<D, FP4>(a.c, phys, h, lo, rows);
    for (int i = tid; i < (hi - lo) * U; i += kThreads) {
      const int r = lo + i / U, u = i % U;
      const int64_t t = tok0 + r;
      const UnitPlace p = unit_place(a.r, u);
      const __bf16* src = a.k + t * a.k_stride + int64_t(h) * D;
      Chunk2 x{*(const cu32x4*)(src + p.a), *(const cu32x4*)(src + p.b)};
      if (p.turn) {
        const int pos = rope_row(a.r, int(t), j * P + r);
        if (pos >= 0) x = rotate_unit(a.r, x, u, pos);
      }
      *(cu32x4*)(rows + r * R + p.a) = x.a;
      *(cu32x4*)(rows + r * R + p.b) = x.b;
    }
  } else {
    for (int i = tid; i < (hi - lo) * (D / 8); i += kThreads) {
      const int r = lo + i / (D / 8), x = i % (D / 8);
      const __bf16* src = a.v + (tok0 + r) * a.v_stride + int64_t(h) * D;
      *(cu32x4*)(rows + r * R + x * 8) = *(const cu32x4*)(src + x * 8);
    }
  }
  __syncthreads();

  if constexpr (FP4) {  // codes out (K) or kept in the row's place (V)
    for (int i = tid; i < (hi - lo) * (D / 32); i += kThreads) {
      const int r = lo + i / (D / 32), gr = i % (D / 32);
      cu32x4* row = (cu32x4*)(rows + r * R + gr * 32);
      cu32x4 x[4];
#pragma unroll
      for (int w = 0; w < 4; ++w) x[w] = row[w];
      uint32_t code[4];
      const uint32_t sc = quantise32(x, code);
      if (!vside) {
        const int tile = r >> 4, m = r & 15;
        uint8_t* kp = (uint8_t*)a.c.k + base / 2 + tile * 8 * D;
        if constexpr (D == 128) {
          *(cu32x4*)(kp + (gr * 16 + m) * 16) = cu32x4{code[0], code[1], code[2], code[3]};
        } else {
          *(cu32x2*)(kp + ((2 * gr) * 16 + m) * 8) = cu32x2{code[0], code[1]};
          *(cu32x2*)(kp + ((2 * gr + 1) * 16 + m) * 8) = cu32x2{code[2], code[3]};
        }
        a.c.ks[base / 32 + tile * (D / 2) + gr * 16 + m] = uint8_t(sc);
        const float s = scale_of(sc);
#pragma unroll
        for (int w = 0; w < 4; ++w)  // the stored values, for the mean
          row[w] = __builtin_bit_cast(cu32x4, fp4_eight(code[w], s));
      } else {
        const int kb = r >> 5, g = (r & 15) >> 2, jj = ((r >> 4) & 1) * 4 + (r & 3);
        a.c.vs[base / 32 + kb * D + (g * (D / 32) + gr) * 8 + jj] = uint8_t(sc);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          cu32x4 y;  // one code in each 16-bit place
#pragma unroll
          for (int z = 0; z < 4; ++z)
            y[z] = ((code[w] >> (8 * z)) & 15u) | ((code[w] >> (8 * z + 4)) & 15u) << 16;
          row[w] = y;
        }
      }
    }
    __syncthreads();
  }

  if (!vside) {
    if constexpr (!FP4) {
      const int t0 = lo >> 4, t1 = (hi + 15) >> 4;
      cu32x4* dst = (cu32x4*)((__bf16*)a.c.k + base);
      for (int i = t0 * 2 * D + tid; i < t1 * 2 * D; i += kThreads) {
        const int m = i & 15, sg = (i >> 4) % (D / 8), r = i / (2 * D) * 16 + m;
        if (r >= lo && r < hi) dst[i] = *(cu32x4*)(rows + r * R + sg * 8);
      }
    }
    // mean key of the page's tokens [0, hi)
    constexpr int PAIRS = D / 2, SEGS = kThreads / PAIRS;
    __shared__ double part[SEGS][D];
    const int cp = tid % PAIRS, seg = tid / PAIRS;
    double s0 = 0.0, s1 = 0.0;
    for (int r = seg; r < hi; r += SEGS) {
      const uint32_t x = *(const uint32_t*)(rows + r * R + cp * 2);
      s0 += double(lo_f(x));
      s1 += double(hi_f(x));
    }
    part[seg][cp * 2] = s0;
    part[seg][cp * 2 + 1] = s1;
    __syncthreads();
    if (tid < PAIRS) {
      s0 = s1 = 0.0;
#pragma unroll
      for (int s = 0; s < SEGS; ++s) {
        s0 += part[s][tid * 2];
        s1 += part[s][tid * 2 + 1];
      }
      // bf16 means halve what a selection reads; it ranks pages by them, no more
      ((uint32_t*)a.c.mean)[((int64_t(phys) * a.c.H + h) * D >> 1) + tid] =
          pack(float(s0 / hi), float(s1 / hi));
    }
  } else {
    const uint16_t* codes = (const uint16_t*)rows;
    const int b0 = lo >> 5, b1 = (hi + 31) >> 5;
    for (int i = b0 * 4 * D + tid; i < b1 * 4 * D; i += kThreads) {
      const int kb = i / (4 * D);
      int ch, g;
      if constexpr (!FP4) {
        ch = ((i >> 6) % (D / 16)) * 16 + (i & 15);
        g = (i >> 4) & 3;
      } else {
        ch = (((i >> 8) % (D / 64)) * 4 + (i & 3)) * 16 + ((i >> 2) & 15);
        g = (i >> 6) & 3;
      }
      uint16_t x[8];
      uint32_t mask = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int r = kb * 32 + (e >> 2) * 16 + g * 4 + (e & 3);
        const bool is_new = r >= lo && r < hi;
        mask |= uint32_t(is_new) << e;
        x[e] = is_new ? codes[r * R + ch] : uint16_t(0);
      }
      if (mask == 0) continue;
      if constexpr (!FP4) {
        uint16_t* dst = (uint16_t*)a.c.v + base + int64_t(i) * 8;
        if (mask == 255) {
          cu32x4 y;
#pragma unroll
          for (int e = 0; e < 4; ++e) y[e] = uint32_t(x[2 * e]) | uint32_t(x[2 * e + 1]) << 16;
          *(cu32x4*)dst = y;
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (mask >> e & 1) dst[e] = x[e];
        }
      } else {
        uint32_t* dst = (uint32_t*)((uint8_t*)a.c.v + base / 2) + i;
        uint32_t y = 0, keep = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          y |= uint32_t(x[e]) << (4 * e);
          keep |= (mask >> e & 1) ? 0u : 15u << (4 * e);
        }
        if (keep) y |= *dst & keep;
        *dst = y;
      }
    }
  }
}

struct ReadArgs {
  DevCache c;
  DevBatch b;
  __bf16* k;
  __bf16* v;
  int64_t N;
};

// A workgroup copies one page of one head and side: fragments to LDS rows to raster rows.
template <int D, bool FP4>
__global__ void __launch_bounds__(kThreads) cache_read_kernel(ReadArgs a) {
  constexpr int R = lds_row<D>();
  extern __shared__ __attribute__((aligned(16))) char lds[];
  __bf16* rows = (__bf16*)lds;
  const int64_t wg = blockIdx.x;
  const bool vside = wg & 1;
  const int64_t bj = (wg >> 1) / a.c.H;
  const int h = int((wg >> 1) - bj * a.c.H);
  const int b = int(bj / a.b.max_pages), j = int(bj - int64_t(b) * a.b.max_pages);
  const int P = a.c.page;
  const int64_t to = min(int64_t(a.b.lens[b]), a.N);
  const int n = int(min(to - int64_t(j) * P, int64_t(P)));
  if (n <= 0) return;
  const int phys = a.b.table[bj];
  if (phys < 0 || phys >= a.c.n_pages) return;
  if (vside) stage_v<D, FP4>(a.c, phys, h, n, rows);
  else stage_k<D, FP4>(a.c, phys, h, n, rows);
  __syncthreads();
  __bf16* dst = (vside ? a.v : a.k) + ((int64_t(b) * a.c.H + h) * a.N + int64_t(j) * P) * D;
  for (int i = threadIdx.x; i < n * (D / 8); i += kThreads) {
    const int r = i / (D / 8), x = i % (D / 8);
    *(cu32x4*)(dst + int64_t(i) * 8) = *(cu32x4*)(rows + r * R + x * 8);
  }
}

template <int D, bool FP4>
hipError_t append(const AppendArgs& a, int64_t wgs, hipStream_t s) {
  const int bytes = a.c.page * lds_row<D>() * 2;
  const void* fn = (const void*)cache_append_kernel<D, FP4>;
  if (bytes > 48 * 1024) {
    const hipError_t e = ensure_dynamic_lds(fn, 256 * lds_row<D>() * 2);
    if (e != hipSuccess) return e;
  }
  cache_append_kernel<D, FP4><<<dim3(unsigned(wgs)), kThreads, bytes, s>>>(a);
  return hipGetLastError();
}

template <int D, bool FP4>
hipError_t read(const ReadArgs& a, hipStream_t s) {
  const int bytes = a.c.page * lds_row<D>() * 2;
  if (bytes > 48 * 1024) {
    const hipError_t e = ensure_dynamic_lds((const void*)cache_read_kernel<D, FP4>, 256 * lds_row<D>() * 2);
    if (e != hipSuccess) return e;
  }
  const int64_t wgs = int64_t(a.b.B) * a.b.max_pages * a.c.H * 2;
  cache_read_kernel<D, FP4><<<dim3(unsigned(wgs)), kThreads, bytes, s>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_cache_append(const DevCache& c, const DevBatch& b, int d, const DevRope& r,
                               const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                               const void* q, int64_t q_stride, int Hq, void* q_out,
                               hipStream_t s) {
  AppendArgs a;
  a.c = c;
  a.b = b;
  a.r = r;
  a.k = (const __bf16*)k;
  a.v = (const __bf16*)v;
  a.q = (const __bf16*)q;
  a.q_out = (__bf16*)q_out;
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  a.q_stride = q_stride;
  a.Hq = Hq;
  a.page_wgs = int64_t(item_base(b.n_tokens, b.B, c.page, 2)) * c.H * 2;
  const int64_t units = q ? int64_t(b.n_tokens) * Hq * (d / 16) : 0;
  const int64_t wgs = a.page_wgs + (units + kThreads - 1) / kThreads;
  if (d == 128) return c.fp4 ? append<128, true>(a, wgs, s) : append<128, false>(a, wgs, s);
  return c.fp4 ? append<64, true>(a, wgs, s) : append<64, false>(a, wgs, s);
}

hipError_t launch_cache_read(const DevCache& c, const DevBatch& b, int d, int64_t N, void* k,
                             void* v, hipStream_t s) {
  ReadArgs a;
  a.c = c;
  a.b = b;
  a.k = (__bf16*)k;
  a.v = (__bf16*)v;
  a.N = N;
  if (d == 128) return c.fp4 ? read<128, true>(a, s) : read<128, false>(a, s);
  return c.fp4 ? read<64, true>(a, s) : read<64, false>(a, s);
}

}  // namespace spade
