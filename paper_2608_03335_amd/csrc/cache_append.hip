// Append to the paged cache with the position rotation, and read-back (gfx950).
//
// Append. A workgroup owns the K of one page and head, or 64 tokens of its V: it stages tokens
// as rows in LDS, rotates and rounds the new ones on the way, and writes them out in the
// page's fragment order, so global reads are whole rows and global writes whole fragments
// wherever a fragment is all new. Only one workgroup touches a page's bytes, so 4-bit dwords
// shared with older tokens are merged without atomics. The K side also reads the page's older
// keys and writes the page's mean key: from the stored values, in fp64, so it is the same
// however the tokens arrived (one by one, in chunks, rewritten after a rewind). The remaining
// workgroups of the launch rotate the queries, two heads a thread.
//
// Rotation: a' = a cos - b sin, b' = a sin + b cos in fp32, every product and sum rounded
// once (no fused multiply-add: the same bits as the elementary operations), then one
// rounding to bf16, the type keys are kept and multiplied in.
//
// 4 bits: e is the least exponent in [-126, 126] with max|x| <= 7 2^e over 32 channels, so
// that no element is off by more than half a step of its place in {0,.5,1,1.5,2,3,4,6} 2^e
// (7 is half way between 6 and the next step, 8); nearest, ties to even. At e = 126 the
// grid ends at 3 2^126, the last value bf16 can hold.
//
// Bound by HBM for many tokens, by the launch for few. Pieces of 64 tokens keep four
// workgroups a CU under way (whole pages of 128: 143 us where they take 126). Measured: 4680
// new tokens of 12 heads of 128, bf16, 89 MB with the queries 18.6 us (4.8 TB/s); 27673 tokens
// of 32 query and 8 K/V heads in 4 bits, 597 MB, 126 us (4.7 TB/s); one token of 32 sequences
// 7.7 us.
#include "cache.h"

namespace spade {
namespace {

constexpr int kThreads = 256;
constexpr int kHeads = 2;      // heads a thread turns with one load of the tables (4: 1 to 3 us more)
constexpr int kCuLds = 1024;   // sequences whose offsets a query workgroup keeps in LDS
constexpr int kPiece = 64;     // tokens of a page in LDS at once

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

// A unit's eight cosines and sines.
struct Turn {
  cf32x4 c[2], s[2];
};
__device__ __forceinline__ void load_turn(const DevRope& r, int u, int pos, Turn& f) {
  const int64_t at = int64_t(pos) * (r.rot >> 1) + u * 8;
  f.c[0] = *(const cf32x4*)(r.cos + at);
  f.c[1] = *(const cf32x4*)(r.cos + at + 4);
  f.s[0] = *(const cf32x4*)(r.sin + at);
  f.s[1] = *(const cf32x4*)(r.sin + at + 4);
}

__device__ __forceinline__ Chunk2 rotate_unit(const DevRope& r, Chunk2 x, const Turn& f) {
#pragma clang fp contract(off)
  float v[16];
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
    const float c = f.c[i >> 2][i & 3], s = f.s[i >> 2][i & 3];
    const float ac = a * c, bs = b * s, as = a * s, bc = b * c;
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

// Quantises 32 channels (16 dwords of bf16 pairs) to 4 dwords of codes; returns the scale byte.
// The conversion instruction rounds to nearest, ties to even, and saturates.
__device__ __forceinline__ uint32_t quantise32(const cu32x4 x[4], uint32_t code[4]) {
  typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
  u16x2 most = {0, 0};
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, x[i][j] & 0x7fff7fffu));
  const float top = __uint_as_float(uint32_t(max(most[0], most[1])) << 16);
  if (!(top <= 3.4e38f)) {
#pragma unroll
    for (int i = 0; i < 4; ++i) code[i] = 0;
    return 255;
  }
  const int e = group_exponent(top);
  const float two = __uint_as_float(uint32_t(127 + e) << 23);  // e in [-126, 126]
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    // (copies: a bit cast of a vector's element reads its first one)
    const uint32_t w0 = x[i][0], w1 = x[i][1], w2 = x[i][2], w3 = x[i][3];
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(cbf16x2, w0), two, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(cbf16x2, w1), two, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(cbf16x2, w2), two, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(cbf16x2, w3), two, 3);
    if (e == 126) {  // 4 2^126 is beyond bf16: codes 6 and 7 become 5
      const uint32_t high = (c >> 2) & (c >> 1) & 0x11111111u;  // codes with bits 2 and 1 set
      c = (c & ~(high * 7u)) | high * 5u;
    }
    code[i] = c;
  }
  return uint32_t(e + 127);
}

template <int D>
__device__ __forceinline__ int64_t page_elem(const DevCache& c, int phys, int h) {
  return (int64_t(phys) * c.H + h) * c.page * D;
}

// Tokens [from, n) of a page's K side, a piece at most, as rows in LDS, the first at `rows` (from
// a multiple of 32, n <= page; whole tiles are read), LOADS 16-byte loads at a time in bf16.
template <int D, bool FP4, int LOADS>
__device__ __forceinline__ void stage_k(const DevCache& c, int phys, int h, int from, int n, __bf16* rows) {
  constexpr int R = lds_row<D>();
  const int tiles = (n + 15) >> 4, tile0 = from >> 4;
  rows -= from * R;
  const int64_t base = page_elem<D>(c, phys, h);
  if constexpr (!FP4) {
    const cu32x4* src = (const cu32x4*)((const __bf16*)c.k + base);
    for (int i0 = tile0 * 2 * D + threadIdx.x; i0 < tiles * 2 * D; i0 += LOADS * kThreads) {
      cu32x4 x[LOADS];
#pragma unroll
      for (int t = 0; t < LOADS; ++t)
        if (i0 + t * kThreads < tiles * 2 * D) x[t] = src[i0 + t * kThreads];
#pragma unroll
      for (int t = 0; t < LOADS; ++t) {
        const int i = i0 + t * kThreads, m = i & 15, sg = (i >> 4) % (D / 8), r = i / (2 * D) * 16 + m;
        if (r < n) *(cu32x4*)(rows + r * R + sg * 8) = x[t];
      }
    }
  } else {  // a thread: the D / 4 channels of lane group g of a token
    static_assert(kPiece / 16 * 64 == kThreads, "a thread a token and lane group");
    constexpr int W = D / 32;
    typedef uint32_t words __attribute__((ext_vector_type(W)));
    const int tile = tile0 + int(threadIdx.x >> 6), g = (threadIdx.x >> 4) & 3, m = threadIdx.x & 15;
    const int r = tile * 16 + m, ch = g * (D / 4);
    if (r < n) {
      const words x = ((const words*)((const uint8_t*)c.k + base / 2))[tile * 64 + (threadIdx.x & 63)];
      const float s = scale_of(c.ks[base / 32 + tile * (D / 2) + (ch >> 5) * 16 + m]);
#pragma unroll
      for (int w = 0; w < W; ++w) *(cbf16x8*)(rows + r * R + ch + w * 8) = fp4_eight(x[w], s);
    }
  }
}

// The same for the V side: a thread turns two neighbouring channels of eight tokens at a time.
template <int D, bool FP4>
__device__ __forceinline__ void stage_v(const DevCache& c, int phys, int h, int from, int n, __bf16* rows) {
  constexpr int R = lds_row<D>(), N = kPiece / 32 * 2 * D / kThreads;
  const int blocks = (n + 31) >> 5, block0 = from >> 5;
  rows -= from * R;
  const int64_t base = page_elem<D>(c, phys, h);
  cbf16x8 x[N][2];
  uint32_t w[N][2];
  cu32x2 sc[N];
  int kb[N], ch[N], g[N];
#pragma unroll
  for (int t = 0; t < N; ++t) {
    const int p = t * kThreads + int(threadIdx.x), y = p % (2 * D);
    kb[t] = block0 + p / (2 * D);
    if constexpr (!FP4) {  // units (ct, g, m) of a block
      g[t] = (y >> 3) & 3;
      ch[t] = (y >> 5) * 16 + (y & 7) * 2;
      const cbf16x8* src = (const cbf16x8*)((const __bf16*)c.v + base) + kb[t] * 4 * D + 2 * y;
      if (kb[t] < blocks) x[t][0] = src[0], x[t][1] = src[1];
    } else {  // (half, g, m, ct)
      const int ct = y & 3, m = ((y >> 2) & 7) * 2, half = y >> 7;
      g[t] = (y >> 5) & 3;
      ch[t] = (half * 4 + ct) * 16 + m;
      const uint32_t* src =
          (const uint32_t*)((const uint8_t*)c.v + base / 2) + kb[t] * 4 * D + half * 256 + g[t] * 64 + m * 4 + ct;
      if (kb[t] < blocks) {
        w[t][0] = src[0], w[t][1] = src[4];
        sc[t] = *(const cu32x2*)(c.vs + base / 32 + kb[t] * D + (g[t] * (D / 32) + (ch[t] >> 5)) * 8);
      }
    }
  }
#pragma unroll
  for (int t = 0; t < N; ++t) {
    if (kb[t] >= blocks) continue;
    if constexpr (FP4) {
#pragma unroll
      for (int z = 0; z < 2; ++z) {
        const cbf16x8 y = fp4_eight(w[t][z], 1.0f);
        // a power of two times an e2m1 value: exact in bf16
#pragma unroll
        for (int j = 0; j < 8; ++j)
          x[t][z][j] = (__bf16)(float(y[j]) * scale_of((sc[t][j >> 2] >> (8 * (j & 3))) & 255u));
      }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int r = kb[t] * 32 + (j >> 2) * 16 + g[t] * 4 + (j & 3);
      const __bf16 a = x[t][0][j], b = x[t][1][j];
      const uint32_t two = uint32_t(__builtin_bit_cast(uint16_t, a)) | uint32_t(__builtin_bit_cast(uint16_t, b)) << 16;
      if (r < n) *(uint32_t*)(rows + r * R + ch[t]) = two;
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
  int64_t page_wgs;  // the first workgroups: for each (page item, head) K, then V in pieces
  uint32_t first;    // of the launch
};

template <int D, bool FP4>
__global__ void __launch_bounds__(kThreads) cache_append_kernel(AppendArgs a) {
  constexpr int R = lds_row<D>();
  constexpr int U = D / 16;
  // one buffer for a piece's rows, the mean's partial sums, and a query workgroup's offsets
  __shared__ __attribute__((aligned(16))) char lds[kPiece * R * 2];
  static_assert(sizeof(lds) >= (kCuLds + 1) * sizeof(int) && sizeof(lds) >= 2 * kThreads * sizeof(double), "");
  __bf16* piece = (__bf16*)lds;
  const int wg = int(a.first + blockIdx.x);
  const int tid = threadIdx.x;

  if (wg >= a.page_wgs) {  // queries: a thread turns one unit of kHeads neighbouring heads
    int* cu_lds = (int*)lds;
    const bool staged = a.b.B <= kCuLds;
    if (staged)
      for (int i = tid; i <= a.b.B; i += kThreads) cu_lds[i] = a.b.cu[i];
    const int groups = (a.Hq + kHeads - 1) / kHeads;
    const int64_t first = (wg - a.page_wgs) * kThreads;
    const int64_t t_first = first / (groups * U);
    const int i = int(first - t_first * (groups * U)) + tid;
    const int64_t t = t_first + i / (groups * U);
    const int u = i % U, h0 = i / U % groups * kHeads;
    __syncthreads();
    if (t >= a.b.n_tokens) return;
    int lo = 0, hi = a.b.B;  // the last b with cu[b] <= t
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if ((staged ? cu_lds[mid] : a.b.cu[mid]) <= t) lo = mid; else hi = mid;
    }
    const int c0 = staged ? cu_lds[lo] : a.b.cu[lo], c1 = staged ? cu_lds[lo + 1] : a.b.cu[lo + 1];
    if (!(c0 <= t && t < c1)) return;  // of no sequence: left as it was
    const int64_t place = int64_t(a.b.lens[lo]) - c1 + t;
    const UnitPlace p = unit_place(a.r, u);
    const __bf16* src = a.q + t * a.q_stride + int64_t(h0) * D;
    __bf16* dst = a.q_out + (t * a.Hq + h0) * D;
    const int n = min(kHeads, a.Hq - h0);
    Chunk2 x[kHeads];
#pragma unroll
    for (int h = 0; h < kHeads; ++h)
      if (h < n) x[h] = Chunk2{*(const cu32x4*)(src + h * D + p.a), *(const cu32x4*)(src + h * D + p.b)};
    const int pos = p.turn ? rope_row(a.r, int(t), place) : -1;
    if (pos >= 0) {
      Turn f;
      load_turn(a.r, u, pos, f);
#pragma unroll
      for (int h = 0; h < kHeads; ++h)
        if (h < n) x[h] = rotate_unit(a.r, x[h], f);
    }
#pragma unroll
    for (int h = 0; h < kHeads; ++h)
      if (h < n) {
        *(cu32x4*)(dst + h * D + p.a) = x[h].a;
        *(cu32x4*)(dst + h * D + p.b) = x[h].b;
      }
    return;
  }

  const int P = a.c.page, sides = 1 + (P + kPiece - 1) / kPiece;  // K, and V in pieces
  const int ih = wg / sides, side = wg - ih * sides;
  const bool vside = side > 0;
  const int h = ih % a.c.H;
  const SeqItem it = find_item(a.b, ih / a.c.H, P, 2);
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

  // the mean's sums: a thread adds two channels of every SEGS-th row
  constexpr int PAIRS = D / 2, SEGS = kThreads / PAIRS;
  const int cp = tid % PAIRS, seg = tid / PAIRS;
  double s0 = 0.0, s1 = 0.0;
  const int p_first = vside ? (side - 1) * kPiece : 0, p_end = vside ? p_first + kPiece : hi;
  for (int p0 = p_first; p0 < p_end; p0 += kPiece) {
    const int r0 = max(lo, p0), r1 = min(hi, p0 + kPiece);  // the piece's new tokens
    if (vside && r0 >= r1) return;
    __bf16* rows = piece - p0 * R;
    if (!vside) {
      stage_k<D, FP4, 1>(a.c, phys, h, p0, min(lo, p0 + kPiece), piece);
      for (int i = tid; i < (r1 - r0) * U; i += kThreads) {
        const int r = r0 + i / U, u = i % U;
        const int64_t t = tok0 + r;
        const UnitPlace p = unit_place(a.r, u);
        const __bf16* src = a.k + t * a.k_stride + int64_t(h) * D;
        Chunk2 x{*(const cu32x4*)(src + p.a), *(const cu32x4*)(src + p.b)};
        if (p.turn) {
          const int pos = rope_row(a.r, int(t), j * P + r);
          if (pos >= 0) {
            Turn f;
            load_turn(a.r, u, pos, f);
            x = rotate_unit(a.r, x, f);
          }
        }
        *(cu32x4*)(rows + r * R + p.a) = x.a;
        *(cu32x4*)(rows + r * R + p.b) = x.b;
      }
    } else {
      for (int i = tid; i < (r1 - r0) * (D / 8); i += kThreads) {
        const int r = r0 + i / (D / 8), x = i % (D / 8);
        const __bf16* src = a.v + (tok0 + r) * a.v_stride + int64_t(h) * D;
        *(cu32x4*)(rows + r * R + x * 8) = *(const cu32x4*)(src + x * 8);
      }
    }
    __syncthreads();

    if constexpr (FP4) {  // codes out (K) or kept in the row's place (V)
      for (int i = tid; i < (r1 - r0) * (D / 32); i += kThreads) {
        const int r = r0 + i / (D / 32), gr = i % (D / 32);
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
        cu32x4* dst = (cu32x4*)((__bf16*)a.c.k + base);
        for (int i = (r0 >> 4) * 2 * D + tid; i < ((r1 + 15) >> 4) * 2 * D; i += kThreads) {
          const int m = i & 15, sg = (i >> 4) % (D / 8), r = i / (2 * D) * 16 + m;
          if (r >= r0 && r < r1) dst[i] = *(cu32x4*)(rows + r * R + sg * 8);
        }
      }
      for (int r = p0 + seg; r < min(hi, p0 + kPiece); r += SEGS) {
        const uint32_t x = *(const uint32_t*)(rows + r * R + cp * 2);
        s0 += double(lo_f(x));
        s1 += double(hi_f(x));
      }
      __syncthreads();  // the next piece overwrites the rows
      continue;
    }
    const uint16_t* codes = (const uint16_t*)rows;
    for (int i = (r0 >> 5) * 4 * D + tid; i < ((r1 + 31) >> 5) * 4 * D; i += kThreads) {
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
        const bool is_new = r >= r0 && r < r1;
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
  if (vside) return;
  // mean key of the page's tokens [0, hi)
  double(*part)[D] = (double(*)[D])lds;  // [SEGS][D]: the rows are no longer read
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
}

struct ReadArgs {
  uint32_t first;  // workgroup of the launch
  int pages;       // of a sequence, at most
  DevCache c;
  DevBatch b;
  __bf16* k;
  __bf16* v;
  int64_t N;
};

// A workgroup copies 64 tokens of a page of one head and side: fragments to LDS rows to raster
// rows. 27673 tokens x 8 heads of 128 in 4 bits, 143 MB: 27 us (5.3 TB/s); with V turned a channel
// at a time, each load waiting for its write, 46, and with 128 tokens a workgroup, fewer of which
// fit a CU, 61. The same tokens in bf16, 227 MB: 48.7 us (4.7 TB/s).
template <int D, bool FP4>
__global__ void __launch_bounds__(kThreads) cache_read_kernel(ReadArgs a) {
  constexpr int R = lds_row<D>();
  __shared__ __attribute__((aligned(16))) __bf16 rows[kPiece * R];
  const int wg = int(a.first + blockIdx.x);
  const bool vside = wg & 1;
  const int P = a.c.page, pieces = (P + kPiece - 1) / kPiece;
  const int from = (wg >> 1) % pieces * kPiece;
  const int bjh = (wg >> 1) / pieces, bj = bjh / a.c.H, h = bjh - bj * a.c.H;
  const int b = bj / a.pages, j = bj - b * a.pages;
  const int64_t to = min(int64_t(a.b.lens[b]), a.N);
  const int n = int(min(to - int64_t(j) * P, int64_t(min(P, from + kPiece))));
  if (n <= from) return;
  const int phys = a.b.table[int64_t(b) * a.b.max_pages + j];
  if (phys < 0 || phys >= a.c.n_pages) return;
  if (vside) stage_v<D, FP4>(a.c, phys, h, from, n, rows);
  else stage_k<D, FP4, 4>(a.c, phys, h, from, n, rows);
  __syncthreads();
  __bf16* dst = (vside ? a.v : a.k) + ((int64_t(b) * a.c.H + h) * a.N + int64_t(j) * P + from) * D;
  for (int i = threadIdx.x; i < (n - from) * (D / 8); i += kThreads) {
    const int r = i / (D / 8), x = i % (D / 8);
    *(cu32x4*)(dst + int64_t(i) * 8) = *(cu32x4*)(rows + r * R + x * 8);
  }
}

int64_t page_workgroups(const DevCache& c, const DevBatch& b) {
  return int64_t(item_base(b.n_tokens, b.B, c.page, 2)) * c.H * (1 + (c.page + kPiece - 1) / kPiece);
}
int64_t query_workgroups(const DevBatch& b, int d, int Hq) {
  return (int64_t(b.n_tokens) * ((Hq + kHeads - 1) / kHeads) * (d / 16) + kThreads - 1) / kThreads;
}

}  // namespace

bool cache_append_fits(const DevCache& c, const DevBatch& b, int d, int Hq) {
  return page_workgroups(c, b) + query_workgroups(b, d, Hq) <= 0x7fffffff;
}

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
  a.page_wgs = page_workgroups(c, b);
  const int64_t wgs = a.page_wgs + query_workgroups(b, d, Hq);
  const auto kernel = d == 128 ? (c.fp4 ? cache_append_kernel<128, true> : cache_append_kernel<128, false>)
                               : (c.fp4 ? cache_append_kernel<64, true> : cache_append_kernel<64, false>);
  return launch_parts(kernel, a, wgs, 1, kThreads, 0, s);
}

hipError_t launch_cache_read(const DevCache& c, const DevBatch& b, int d, int64_t N, void* k,
                             void* v, hipStream_t s) {
  ReadArgs a;
  a.c = c;
  a.b = b;
  a.k = (__bf16*)k;
  a.v = (__bf16*)v;
  a.N = N;
  a.pages = cache_read_pages(c, b, N);
  const int64_t wgs = int64_t(b.B) * a.pages * c.H * 2 * ((c.page + kPiece - 1) / kPiece);
  const auto kernel = d == 128 ? (c.fp4 ? cache_read_kernel<128, true> : cache_read_kernel<128, false>)
                               : (c.fp4 ? cache_read_kernel<64, true> : cache_read_kernel<64, false>);
  return launch_parts(kernel, a, wgs, 1, kThreads, 0, s);
}

}  // namespace spade
