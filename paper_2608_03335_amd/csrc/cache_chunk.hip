// Attention of many new queries over the paged cache (gfx950): chunks of a prompt, new
// frames of a video.
//
// A workgroup takes one K/V head and a run of neighbouring tokens of one sequence: four
// waves of 32 rows each (floor(32 / G) tokens times their G query heads). It walks the
// union of its tokens' page lists in units of 32 keys; a unit's K and V are staged once in
// LDS for the four waves, in the pages' fragment order, which is free of bank conflicts
// and needs no transpose. A wave skips the pages none of its own tokens keeps. The scores
// of a page that only some of its rows keep cost nothing to mask: a row's bias is its
// reference, or infinity where the row does not keep the page.
//
// bf16 units go from memory to LDS directly, into a ring that runs three units ahead of the
// computation: what other workgroups have not yet brought to L2 takes longer than
// two units' computation. 4-bit units run eight ahead as they lie in the page, and are widened to
// bf16 one unit ahead, once for four waves (V's powers of two are applied there: exact).
//
// S^T (32 keys x 32 rows) = K Q^T and O^T += V^T P^T with mfma 32x32x16. The lane's scores
// are then in the order in which a V fragment holds its keys. Softmax as in cache_attn.hip.
//
// Where heads are few, calls that read all tokens share a tile's pages between workgroups and
// join the parts (cache_attn.hip, which chooses).
//
// Bound by the series of a unit's steps (scores, softmax, P V, with a barrier in front) at two
// workgroups a CU; under lists also by waves that wait for the one that keeps a page, and by
// rows that do not keep it. 4680 queries of 12 heads of 128, 40 of 512 pages each: 74 GFLOP in
// 800 us; waves of 32 rows multiply 5.8 times that, of a page that 13 of the tile's 128 rows
// keep, and 355 us pass with the loads alone. 4087 queries of 32 x 4 heads, 64 wide, 32
// pages of 32 each in 4 bits: 34 GFLOP in 169 us, 1.4 times the work, but 182 vector and 122 scalar
// instructions for the eight products of a wave's unit. All tokens, 12 heads of 128, 1200
// queries of 16384 tokens: 116 GFLOP in 170 us (685 TFLOP/s).
//
// What a row must not see: see cache_attn.hip.
#include "cache_attn.h"

namespace spade {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) char lds_char;

constexpr int kWaves = kChunkWaves;
constexpr int kThreads = 64 * kWaves;
constexpr int kTileRows = kChunkRows * kWaves;
constexpr int kSeg = 512;          // pages walked before the masks are built anew
constexpr float kLazy = 8.0f;      // see cache_attn.hip

// LDS of the walk. bf16: a ring of units that are on their way or in use. 4 bits: a ring of
// units as they lie in the page, and two widened ones.
template <int D, bool FP4>
struct Stage {
  static constexpr int SIDE = 32 * D * 2;                // K or V of a unit, bf16
  static constexpr int WIDE = 2 * SIDE;
  static constexpr int PAGE = 34 * D;                    // a 4-bit unit with its scales
  static constexpr int RING = FP4 ? 8 : 4;
  static constexpr int LOADS = FP4 ? 2 : WIDE / 1024 / kWaves;  // a wave's loads of a unit
  static constexpr int BYTES = FP4 ? 2 * WIDE + RING * PAGE : RING * WIDE;
};

struct Seg {
  uint32_t mask[kWaves][kSeg];  // tokens of the wave that keep page i, then entry i of the walk
  int phys[kSeg];               // kept pages in ascending order
  int page[kSeg];               // their place in the sequence
  int wave_n[2][kWaves];
};

// Barrier behind which every wave has at most N loads to LDS in flight and has read what it
// asked of LDS before (the buffers are overwritten next).
template <int N>
__device__ __forceinline__ void unit_barrier() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// 16 (4) bytes a lane from base + off to LDS address dst + 16 (4) lane.
__device__ __forceinline__ void to_lds(const void* base, uint32_t off, uint32_t dst) {
  asm volatile("global_load_lds_dwordx4 %0, %1" ::"v"(off), "s"(base), "{m0}"(dst) : "memory");
}
__device__ __forceinline__ void to_lds4(const void* base, uint32_t off, uint32_t dst) {
  asm volatile("global_load_lds_dword %0, %1" ::"v"(off), "s"(base), "{m0}"(dst) : "memory");
}

template <typename T>
__device__ __forceinline__ const T* uniform(const T* p) {
  const uint64_t x = reinterpret_cast<uint64_t>(p);
  const uint32_t lo = __builtin_amdgcn_readfirstlane(uint32_t(x));
  const uint32_t hi = __builtin_amdgcn_readfirstlane(uint32_t(x >> 32));
  return reinterpret_cast<const T*>(uint64_t(hi) << 32 | lo);
}

__device__ __forceinline__ cbf16x8 scaled_eight(uint32_t x, cu32x2 scales) {
  float f[8];
  const cf32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(x, 1.0f, 0),
               b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(x, 1.0f, 1),
               c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(x, 1.0f, 2),
               d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(x, 1.0f, 3);
  f[0] = a[0], f[1] = a[1], f[2] = b[0], f[3] = b[1], f[4] = c[0], f[5] = c[1], f[6] = d[0], f[7] = d[1];
  cbf16x8 y;
#pragma unroll
  for (int i = 0; i < 8; ++i)
    y[i] = (__bf16)(f[i] * scale_of((scales[i >> 2] >> (8 * (i & 3))) & 255u));
  return y;
}

// Widens a 4-bit unit: each thread 2 D / 256 dwords of either side, 8 values a dword.
template <int D>
__device__ __forceinline__ void widen(const char* raw, char* buf, int tid) {
  constexpr int W = D / 64;  // dwords a thread and side
  typedef uint32_t words __attribute__((ext_vector_type(W == 2 ? 2 : 1)));
  const words k = ((const words*)raw)[tid], v = ((const words*)(raw + 16 * D))[tid];
  const uint8_t* ks = (const uint8_t*)raw + 32 * D;
  const uint8_t* vs = ks + D;
  const int tile = tid >> 7, g = (tid >> 5) & 3, m = (tid >> 1) & 15;
  const float s = scale_of(ks[tile * (D / 2) + (D == 128 ? g : g >> 1) * 16 + m]);
#pragma unroll
  for (int i = 0; i < W; ++i) {
    const int ch = g * (D / 4) + ((tid & 1) * W + i) * 8;  // first of 8 channels
    *(cbf16x8*)(buf + ((tile * (D / 32) + (ch >> 5)) * 64 + ((ch & 31) >> 3) * 16 + m) * 16) =
        fp4_eight(k[i], s);
  }
  char* vb = buf + Stage<D, true>::SIDE;
  // D = 128: column tiles 4 half + 2 (tid & 1) + {0, 1} of lane group g; D = 64: tile tid & 3
  const int ct = D == 128 ? tile * 4 + (tid & 1) * 2 : tid & 3;
  const int vg = D == 128 ? g : tid >> 6, vm = D == 128 ? m : (tid >> 2) & 15;
  const cu32x2 two = ((const cu32x2*)vs)[vg * (D / 32) + (ct >> 1)];
#pragma unroll
  for (int i = 0; i < W; ++i)
    *(cbf16x8*)(vb + (((ct + i) * 4 + vg) * 16 + vm) * 16) = scaled_eight(v[i], two);
}

__device__ __forceinline__ float row_max(float v) {  // over the two lanes of a row
  const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1]));
}

template <int D>
struct Rows {
  cbf16x8 q[D / 16];
  f32x16 o[D / 32];
  float m, l;  // reference and this lane's share of the sum
};

// One staged unit, keys at..at+31. row_in: the lane's row keeps the page. edge (the same for all
// lanes): a row sees the keys below row_seen, and V is cleared from key v_seen on. One path for
// both, with the masks as side steps: two would hold two sets of accumulators.
template <int D>
__device__ __forceinline__ void step(const char* kf, const char* vf, Rows<D>& w, int lane, float scale2,
                                     int at, bool edge, int row_seen, bool row_in, int v_seen) {
  const int key0 = at + 4 * (lane >> 5);  // the lane's keys: key0 + {0..3, 8..11, 16..19, 24..27}
  cbf16x8 k[D / 16];
  cu32x4 v[D / 32][2];
#pragma unroll
  for (int i = 0; i < D / 16; ++i) k[i] = *(const cbf16x8*)(kf + (i >> 1) * 1024 + (i & 1) * 512);
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int c = 0; c < D / 32; ++c) v[c][t] = *(const cu32x4*)(vf + c * 2048 + t * 512);
  __builtin_amdgcn_sched_barrier(0);  // all reads first: else each waits just before its use
  f32x16 s = {};
#pragma unroll
  for (int i = 0; i < D / 16; ++i) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k[i], w.q[i], s, 0, 0, 0);
  if (edge) {
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = key0 + 8 * (i >> 2) + (i & 3) < row_seen ? s[i] : kNegInf;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int key = key0 + 8 * t + (i >> 1) * 16 + (i & 1) * 2;
        const uint32_t keep = (key < v_seen ? 0xffffu : 0u) | (key + 1 < v_seen ? 0xffff0000u : 0u);
#pragma unroll
        for (int c = 0; c < D / 32; ++c) v[c][t][i] &= keep;
      }
  }
  float top = fmaxf(s[0], s[1]);
#pragma unroll
  for (int i = 2; i < 16; i += 2) top = fmaxf(fmaxf(top, s[i]), s[i + 1]);
  top = row_max(top) * scale2;
  top = row_in ? top : kNegInf;
  float m = w.m;
  if (__any(top > m)) {
    m = top > m ? top + kLazy : m;
    const float alpha = w.m == kNegInf ? 0.0f : __builtin_amdgcn_exp2f(w.m - m);
#pragma unroll
    for (int c = 0; c < D / 32; ++c) w.o[c] *= alpha;
    w.l *= alpha;
    w.m = m;
  }
  const float bias = row_in && m != kNegInf ? -m : kNegInf;
  float sum = 0.0f;
  cbf16x8 p[2];
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], scale2, bias));
    sum += e;
    // key 8 (i / 4) + 4 half + i % 4: V fragment 2 t + half holds i / 4 = t and t + 2
    p[(i >> 2) & 1][(i >> 3) * 4 + (i & 3)] = (__bf16)e;
  }
  w.l += sum;
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int c = 0; c < D / 32; ++c)
      w.o[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(cbf16x8, v[c][t]), p[t], w.o[c], 0, 0, 0);
}

template <int D, bool FP4>
__global__ void __launch_bounds__(kThreads, 2) cache_chunk_kernel(AttnArgs a) {
  using ST = Stage<D, FP4>;
  extern __shared__ __attribute__((aligned(16))) char lds[];
  __shared__ Seg sg;
  // each XCD takes a run of neighbouring items of a head and split: they want the same pages
  const int64_t items = a.items, total = items * a.c.H * a.splits, per = (total + 7) >> 3;
  const int64_t wg = a.first + blockIdx.x, slot = wg >> 3, L = (wg & 7) * per + slot;
  if (slot >= per || L >= total) return;
  const int hs = int(L / items), item = int(L - hs * items), h = hs / a.splits, split = hs - h * a.splits;
  JoinHead* head = a.join + int64_t(item) * a.c.H + h;
  const SeqItem it = find_item(a.b, item, a.QT, 1);
  const int skip = it.first * a.QT;
  if (it.b < 0 || skip >= it.n) {
    if (a.splits > 1 && split == 0 && threadIdx.x == 0) *head = JoinHead{0, 0, 0, 0, 0};
    return;
  }
  const int t0 = it.t0 + skip, nq = min(a.QT, it.n - skip);
  Seen seen = seen_of(a, it);
  seen.first += skip * seen.step;
  const int P = a.c.page, upp = P >> 5;
  const int visible = (seen.of(nq - 1) + P - 1) / P;
  // splits share the pages of a long tile evenly
  int splits = 1;
  if (a.splits > 1) {
    splits = min(max((visible * upp + kChunkUnits - 1) / kChunkUnits, 1), a.splits);
    if (split == 0 && threadIdx.x == 0) *head = JoinHead{splits, t0, nq, h * a.G, a.G};
    if (split >= splits) return;
  }
  const int page0 = int(int64_t(visible) * split / splits), pages = int(int64_t(visible) * (split + 1) / splits);
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);

  // the wave's tokens q0..q0+qn-1 of the tile, the lane's row
  const int QW = a.QT / kWaves, q0 = wave * QW, qn = min(max(nq - q0, 0), QW);
  const int r = lane & 31, half = lane >> 5;
  const int qi = r / a.G, gh = r - qi * a.G;
  const bool live = qi < qn;
  const int row_seen = live ? seen.of(q0 + qi) : 0;
  const uint32_t all = qn ? 0xffffffffu >> (32 - qn) : 0;
  const int64_t orow = int64_t(t0 + q0 + qi) * a.Hq + h * a.G + gh;

  Rows<D> w;
#pragma unroll
  for (int k = 0; k < D / 16; ++k)
    w.q[k] = live ? *(const cbf16x8*)(a.q + orow * D + (k >> 1) * 32 + ((k & 1) * 2 + half) * 8)
                  : cbf16x8{};
  const int* table = a.b.table + int64_t(it.b) * a.b.max_pages;
  const int kf_lane = ((lane >> 4) & 1) * (D * 32) + half * 256 + (lane & 15) * 16;
  const int vf_lane = ((lane >> 4) & 1) * 1024 + half * 256 + (lane & 15) * 16;
  const uint32_t lds0 = uint32_t(uintptr_t((lds_char*)lds));

  // only < 0: all tokens at once; else every wave's tokens one by one (see cache_attn.hip)
  for (int only = -1; only < QW; ++only) {
    const int least = qn ? seen.of(q0 + max(only, 0)) : 0;
    const int most = only < 0 ? (qn ? seen.of(q0 + qn - 1) : 0) : only < qn ? least : 0;
    const uint32_t ours = only < 0 ? all : 1u << only;
    w.m = kNegInf;
    w.l = 0.0f;
#pragma unroll
    for (int c = 0; c < D / 32; ++c) w.o[c] = f32x16{};
    for (int seg0 = page0; seg0 < pages; seg0 += kSeg) {
      const int span = min(kSeg, pages - seg0);
      __syncthreads();  // the last segment's masks are no longer read
      if (a.topk) {
        for (int i = tid; i < kSeg; i += kThreads)
#pragma unroll
          for (int v = 0; v < kWaves; ++v) sg.mask[v][i] = 0;
        __syncthreads();
        const int64_t row0 = int64_t(t0) * a.c.H + h;
        for (int i = tid; i < nq * a.topk; i += kThreads) {
          const int q = i / a.topk, k = i - q * a.topk;
          const int64_t row = row0 + int64_t(q) * a.c.H;
          if (k >= a.counts[row]) continue;
          const int j = a.indices[row * a.topk + k];
          if (j >= seg0 && j < seg0 + span && j * P < seen.of(q))
            atomicOr(&sg.mask[q / QW][j - seg0], 1u << (q % QW));
        }
        __syncthreads();
      }
      // the pages that count, in order (an entry's place is not behind its page's: in place)
      int n = 0;
#pragma unroll
      for (int round = 0; round < kSeg / kThreads; ++round) {
        const int i = round * kThreads + tid;
        uint32_t keep[kWaves];
        uint32_t any = a.topk ? 0 : 1;
        if (a.topk)
#pragma unroll
          for (int v = 0; v < kWaves; ++v) any |= keep[v] = sg.mask[v][i];
        const int phys = i < span && any ? table[seg0 + i] : -1;
        const bool ok = phys >= 0 && phys < a.c.n_pages;
        const uint64_t bits = __ballot(ok);
        if (lane == 0) sg.wave_n[round][wave] = __popcll(bits);
        __syncthreads();
        int at = n + __popcll(bits & ((uint64_t(1) << lane) - 1));
#pragma unroll
        for (int v = 0; v < kWaves; ++v) {
          const int x = __builtin_amdgcn_readfirstlane(sg.wave_n[round][v]);
          at += v < wave ? x : 0;
          n += x;
        }
        if (ok) {
          sg.phys[at] = phys;
          sg.page[at] = seg0 + i;
          if (a.topk)
#pragma unroll
            for (int v = 0; v < kWaves; ++v) sg.mask[v][at] = keep[v];
        }
      }
      __syncthreads();
      const int units = n * upp;

      // The cursors of the loads and of the computation know the next entry before they need
      // it: a read of LDS takes as long as four matrix instructions.
      int le = 0, lkb = 0, lbuf = 0, phys = sg.phys[0], next_phys = sg.phys[min(1, kSeg - 1)];
      auto fetch = [&] {
        const int64_t base = (int64_t(__builtin_amdgcn_readfirstlane(phys)) * a.c.H + h) * P * D + lkb * (32 * D);
        if constexpr (FP4) {  // a quarter of the unit a wave: K, K, V, V, and so with the scales
          const bool k = wave < 2;
          const uint32_t dst = lds0 + 2 * ST::WIDE + lbuf * ST::PAGE, part = wave & 1;
          const uint8_t* data = uniform((const uint8_t*)(k ? a.c.k : a.c.v) + (base >> 1) + part * (8 * D));
          const uint8_t* scale = uniform((k ? a.c.ks : a.c.vs) + (base >> 5) + part * (D / 2));
          if (D == 128 || lane < 32) to_lds(data, lane * 16, dst + wave * (8 * D));
          if (lane < D / 8) to_lds4(scale, lane * 4, dst + 32 * D + wave * (D / 2));
        } else {
          const char* kp = (const char*)uniform((const __bf16*)a.c.k + base);
          const char* vp = (const char*)uniform((const __bf16*)a.c.v + base);
          const uint32_t dst = lds0 + lbuf * ST::WIDE;
#pragma unroll
          for (int i = 0; i < ST::LOADS / 2; ++i) {
            const uint32_t off = (wave * (ST::LOADS / 2) + i) * 1024;
            to_lds(kp, off + lane * 16, dst + off);
            to_lds(vp, off + lane * 16, dst + ST::SIDE + off);
          }
        }
        lbuf = lbuf + 1 == ST::RING ? 0 : lbuf + 1;
        if (++lkb == upp) {
          lkb = 0;
          ++le;
          phys = next_phys;
          next_phys = sg.phys[min(le + 1, kSeg - 1)];
        }
      };
      // bf16: unit u + RING - 1 is asked for when unit u begins; 4 bits: unit u + RING, while
      // unit u + 1 is widened
      constexpr int AHEAD = FP4 ? ST::RING : ST::RING - 1;
      for (int u = 0; u < min(units, AHEAD); ++u) fetch();
      if constexpr (FP4) {
        if (units >= AHEAD) unit_barrier<(AHEAD - 1) * ST::LOADS>();
        else unit_barrier<0>();
        if (units > 0) widen<D>(lds + 2 * ST::WIDE, lds, tid);
      }
      int e = 0, kb = 0, buf = 0, raw = 0;
      int page = sg.page[0], next_page = sg.page[1];
      uint32_t mask = sg.mask[wave][0], next_mask = sg.mask[wave][1];
      for (int u = 0; u < units; ++u) {
        // what is needed now has landed: later units may be on their way
        constexpr int FLIGHT = (AHEAD - (FP4 ? 2 : 1)) * ST::LOADS;
        if (u + AHEAD <= units) unit_barrier<FLIGHT>();
        else unit_barrier<0>();
        if (u + AHEAD < units) fetch();
        if constexpr (FP4) {
          raw = raw + 1 == ST::RING ? 0 : raw + 1;
          if (u + 1 < units)
            widen<D>(lds + 2 * ST::WIDE + raw * ST::PAGE, lds + (buf ^ 1) * ST::WIDE, tid);
        }
        const uint32_t who = (a.topk ? __builtin_amdgcn_readfirstlane(mask) : all) & ours;
        const int at = __builtin_amdgcn_readfirstlane(page) * P + kb * 32;
        if (who && at < most) {
          const char* kf = lds + buf * ST::WIDE + kf_lane;
          const char* vf = lds + buf * ST::WIDE + ST::SIDE + vf_lane;
          const bool row_in = live && (who >> qi & 1);
          step<D>(kf, vf, w, lane, a.scale2, at, at + 32 > least, row_seen, row_in, most);
        }
        if (++kb == upp) {
          kb = 0;
          ++e;
          page = next_page;
          mask = next_mask;
          next_page = sg.page[min(e + 1, kSeg - 1)];
          next_mask = sg.mask[wave][min(e + 1, kSeg - 1)];
        }
        buf = buf + 1 == (FP4 ? 2 : ST::RING) ? 0 : buf + 1;
      }
    }
    if (only < 0 && QW > 1) {
      bool bad = false;
#pragma unroll
      for (int c = 0; c < D / 32; ++c)
#pragma unroll
        for (int i = 0; i < 16; ++i) bad |= !(w.o[c][i] == w.o[c][i]);
      if (__syncthreads_or(bad)) continue;
    }
    const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(w.l), __float_as_uint(w.l), false, false);
    const float l = __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
    if (live && (only < 0 || qi == only) && splits > 1) {
      const int row = wave * kChunkRows + r;
      float* po = a.part + ((int64_t(item) * a.c.H + h) * a.splits + split) * (kTileRows * (D + 2));
#pragma unroll
      for (int c = 0; c < D / 32; ++c)
#pragma unroll
        for (int i = 0; i < 16; i += 4)
          *(cf32x4*)(po + row * D + c * 32 + 2 * i + 4 * half) =
              cf32x4{w.o[c][i], w.o[c][i + 1], w.o[c][i + 2], w.o[c][i + 3]};
      if (half == 0) *(cf32x2*)(po + kTileRows * D + row * 2) = cf32x2{w.m, l};
    } else if (live && (only < 0 || qi == only)) {
      const float inv = w.m == kNegInf ? 0.0f : 1.0f / l;
#pragma unroll
      for (int c = 0; c < D / 32; ++c)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
          const cf32x2 x = {w.o[c][i] * inv, w.o[c][i + 1] * inv}, y = {w.o[c][i + 2] * inv, w.o[c][i + 3] * inv};
          *(cu32x2*)(a.o + orow * D + c * 32 + 2 * i + 4 * half) =
              cu32x2{__builtin_bit_cast(uint32_t, __builtin_convertvector(x, cbf16x2)),
                     __builtin_bit_cast(uint32_t, __builtin_convertvector(y, cbf16x2))};
        }
      if (a.lse && half == 0) a.lse[orow] = (w.m + log2f(l)) * kLn2f;
    }
    if (only < 0) break;
  }
}

template <int D, bool FP4>
hipError_t run(const AttnArgs& a, hipStream_t s) {
  const int bytes = Stage<D, FP4>::BYTES;
  if (bytes > 32 * 1024) {
    const hipError_t e = ensure_dynamic_lds((const void*)cache_chunk_kernel<D, FP4>, bytes);
    if (e != hipSuccess) return e;
  }
  const int64_t wgs = (a.items * a.c.H * a.splits + 7) / 8 * 8;
  return launch_parts(cache_chunk_kernel<D, FP4>, a, wgs, 1, kThreads, bytes, s);
}

}  // namespace

hipError_t launch_chunk_attn(const AttnArgs& a, int d, hipStream_t s) {
  if (d == 128) return a.c.fp4 ? run<128, true>(a, s) : run<128, false>(a, s);
  return a.c.fp4 ? run<64, true>(a, s) : run<64, false>(a, s);
}

}  // namespace spade
