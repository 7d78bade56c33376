// fe_tree_attn.hip -- attention of draft-tree nodes over a paged cache (gfx950).
//
// The T * G rows of one (sequence, KV head) -- its nodes times the G query heads
// that share the KV head -- read the same keys, so they are the columns of one
// pair of matrix products over the cache: S^T = K Q^T, O^T = V^T P^T.  A
// workgroup takes a tile of TR of these rows and walks the keys once, with the
// running maximum and sum of a softmax per row.
//
//  * In the accumulators a lane holds keys of one row, which is what the second
//    product wants as its right operand once V's keys are taken in the same order
//    (the transposing LDS read delivers them so): probabilities never move between
//    lanes, and a row's maximum and sum need an exchange with lane ^ 32 (and ^ 16
//    in tiles of 16) only.
//  * Keys go through registers into LDS: a tile is loaded (16 bytes a lane) while
//    the one before is worked on, and 8-bit codes become bf16 (or fp32) there, once
//    per workgroup.  With a power of two as the scale that is exact.
//  * RW waves share a tile, side by side on rows; KW groups of them take the tiles
//    in turn and add up at the end.  RW = 1: every wave streams keys of its own, one
//    LDS buffer and no barrier.  RW = 4, 8: a key is staged once per 128 or 256 rows,
//    in two buffers, one barrier a tile.
//  * The tiles of all (sequence, row tile, KV head) segments are numbered and cut
//    into equal ranges, one per workgroup, whatever the lengths: a segment that
//    ranges share leaves partial sums, joined in order by a second launch.  A
//    range leaves at most two partials (the segment it starts in and the one it
//    ends in), so their number does not depend on the lengths either.
//  * Only keys past what every row of the tile sees are masked.  A masked score is
//    replaced, so what it was does not matter; in a value row an infinity or NaN
//    would still come through as 0 * inf, so from a masked tile on that holds one,
//    keys are added one by one at the end, each row over those it sees.
//
// Scores, probabilities' sum and accumulators are fp32; in bf16 the probabilities
// are rounded as the matrix instruction takes them, and summed as rounded.
//
// What bounds it (the two launches under a kernel trace): few rows, the cache's
// bytes -- 32 sequences, one token, 280 MB of 8-bit rows: 55 + 5 us, 4.7 TB/s, where
// a copy reaches 5.2.  Many rows, the pipes that a tile goes through one after the
// other: 1024 nodes of 32 heads behind 8192 keys, 146 GFLOP, 179 + 12 us, 765
// TFLOP/s where a large library product reaches 1300; of 5900 cycles a tile (64
// keys, 256 rows) the matrix pipe is busy for 2050, LDS reads and the softmax for
// about as many each.  Reading the next keys' pieces under the softmax did not help
// (173 -> 184 us: registers).  A few short sequences, latency: a workgroup's setup is
// about 20000 cycles with its first keys' way from memory, and the partials' way
// through memory costs 5 to 8 us more.
#include <algorithm>
#include <atomic>
#include <type_traits>

#include "fe_attn_unit.h"
#include "fe_paged.h"

namespace fe {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr float kLog2e = 1.4426950408889634f;

// Keys per tile: 32, or as many as give every lane of RW waves a 16-byte load of an
// 8-bit row.
constexpr int tile_keys(int RW, int D) { return RW * 1024 / D > 32 ? RW * 1024 / D : 32; }

// Shape of one variant: RW waves side by side on MF rows each (the side of the
// matrix instructions' tile), KW groups of them taking tiles of TK keys in turn.
template <typename T, int D, int MF_, int RW_, int KW_> struct Shape {
  static constexpr int MF = MF_, RW = RW_, KW = KW_;
  static constexpr int TK = tile_keys(RW, D);
  static constexpr int IK = TK * KW;             // keys per work item
  static constexpr int TR = MF * RW;        // rows per tile
  static constexpr int NT = 64 * RW * KW;        // threads
  static constexpr int NBUF = RW == 1 ? 1 : 2;   // LDS buffers per group
  static constexpr int RB = D * (int)sizeof(T);  // bytes per row in LDS
  static constexpr int BUF = 2 * TK * RB;        // K rows, then V rows
  static constexpr int LDS = KW * NBUF * BUF;
};

// A value that is the same in every lane, where the compiler can see it (in scalar
// registers, and branches on it taken by the wave as a whole).
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ long uniform(long x) {
  return (long)((uint64_t)(uint32_t)uniform((int)(x >> 32)) << 32 | (uint32_t)uniform((int)x));
}

// A value the compiler cannot compute ahead of a seldom taken branch, so that the
// branch's addresses hold no registers outside it.
template <typename V> __device__ __forceinline__ V opaque(V x) {
  asm volatile("" : "+v"(x));
  return x;
}

__device__ __forceinline__ uint32_t lds_address(const void *p) {
  return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void *)p;
}
template <typename V> __device__ __forceinline__ V lds_read(uint32_t at) {
  return *(__attribute__((address_space(3))) const V *)(uintptr_t)at;
}
__device__ __forceinline__ void lds_write(uint32_t at, const u32x4 &w) {
  *(__attribute__((address_space(3))) u32x4 *)(uintptr_t)at = w;
}
__device__ __forceinline__ u32x2 lds_read_tr(uint32_t at) {
  return __builtin_bit_cast(
      u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4 *)(uintptr_t)at));
}

// ---- the split ------------------------------------------------------------------

// One sequence's rows and keys as a row tile sees them.
struct Span {
  int P, n, live;  // prefix, nodes, rows that get written
  bool bad;
};
__device__ __forceinline__ Span span_of(const TreeArgs &a, int b) {
  Span s;
  s.P = a.lens[b];
  s.n = a.counts ? a.counts[b] : a.T;
  const bool nbad = s.n < 0 || s.n > a.T;
  if (nbad) s.n = a.T;
  s.bad = nbad || s.P < 0 || (long)s.P + s.n > a.c.max_len;
  s.live = s.n * (a.Hq / a.c.Hkv);
  return s;
}
// Keys that row tile rt (TR rows) of a sequence reads: [0, end); every row of it
// sees [0, all).
__device__ __forceinline__ int keys_end(const TreeArgs &a, const Span &s, int rt, int TR) {
  if (s.bad) return 0;
  if (a.mask) return s.P + s.n;
  return s.P + (min((rt + 1) * TR, s.live) - 1) / (a.Hq / a.c.Hkv) + 1;
}
// Starting and ending a segment costs about as much as kSegItems of its work items
// (its lengths, pages, queries and first keys are fetched one after the other, and
// its sums written), so where every workgroup gets several items a segment counts
// that many more.  With 0, 1, 2, 3, 5: one token each of 32 ragged histories 127, 111,
// 100, 93, 95 us, 32 ragged trees 292, 269, 251, 240, 240 (as the kernels then were).
constexpr int kSegItems = 3;

// Work items of a segment: steps over its keys (none where the tile has no row).
__device__ __forceinline__ int items_of(const TreeArgs &a, const Span &s, int rt, int TR, int IK) {
  return rt * TR >= s.live ? 0 : max(1, (keys_end(a, s, rt, TR) + IK - 1) / IK);
}

// Sums of a wave's values up to each lane (below 2^32: an item count is at most 2^25).
__device__ __forceinline__ uint32_t wave_incl_scan(uint32_t x) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t y = __shfl_up(x, o, 64);
    if (lane >= o) x += y;
  }
  return x;
}

// Equal ranges of `total` items over W workgroups; none is empty (W is at most
// total), so every range between a segment's first and last holds a part of it.
struct Ranges {
  long total, W;
  __device__ __forceinline__ Ranges(long items, int wgs) : total(items), W(items < wgs ? items : wgs) {}
  // products below 2^32 are the rule, and a 64-bit division costs 4 times theirs
  __device__ __forceinline__ static long div(long x, long y) {
    return (x | y) >> 32 ? x / y : (long)((uint32_t)x / (uint32_t)y);
  }
  __device__ __forceinline__ long begin(long w) const { return div(total * w, W); }
  // the range that holds item x
  __device__ __forceinline__ long owner(long x) const {
    const long w = div((x + 1) * W + total - 1, total) - 1;
    return w < W - 1 ? w : W - 1;
  }
};

// Workspace: per range two partials (slot 2w: the segment the range starts inside
// of, 2w + 1: the one it ends inside of): the accumulators of RW waves as the lanes
// hold them, [wave][D / MF][registers / 4][lane][4], so that writing and reading them
// is one run of memory, and a row's (max, sum), [TR]; then the items before every
// (sequence, row tile), E + 1 of them.
template <int D> struct Work {
  float *p;
  long slots;
  int TR;
  __device__ f32x4 *o(long slot) const { return (f32x4 *)(p + slot * TR * D); }
  __device__ float2 *ml(long slot) const { return (float2 *)(p + slots * TR * D) + slot * TR; }
  __host__ __device__ long *before() const { return (long *)(p + slots * TR * (D + 2)); }
};

// Two of a word's e4m3 codes, times a power of two, as bf16 (exact).
template <bool HI> __device__ __forceinline__ uint32_t f8_bf16(uint32_t w, float sc) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, sc, HI));
}

// ---- one tile of keys: global memory -> registers -> LDS ---------------------------

// 16-byte piece p of row R (rows of VPR pieces) in LDS: pieces are permuted within
// a row so that sixteen rows' reads of one piece meet sixteen different banks, and
// so do four rows' reads of four neighbouring pieces (the transposing read).
template <int VPR> __device__ __forceinline__ int piece_at(int R, int p) {
  if constexpr (VPR == 8)
    return R * 8 + (p ^ ((((R >> 1) & 1) << 2) | ((R >> 2) & 3)));
  else
    return R * VPR + (p ^ (((R & 3) << 2) | ((R >> 2) & 3)));
}

// A wave's rows in one load are at most 16 neighbours (and a page holds whole runs
// of 16), so their address is wave-uniform: the rows that the runs of the next 1024
// keys start at sit in one register, a lane per run, and each load picks its own
// with a readlane.
template <typename T, typename S, int D, int RW, int TK, int IK> struct Tile {
  static constexpr int PS = D * (int)sizeof(S) / 16;  // 16-byte pieces of a stored row
  static constexpr int VPR = D * (int)sizeof(T) / 16;
  static constexpr int SPAN = 64 / PS;                // rows of one load of a wave
  static constexpr int STEP = RW * SPAN;              // rows between a thread's loads
  static constexpr int NL = TK / STEP;                // loads per thread, K (as many V)
  static_assert(SPAN >= 1 && SPAN <= 16 && NL >= 1 && TK % STEP == 0, "whole loads inside runs of 16 rows");
  static constexpr int WIN = 1024 / IK;               // tiles per register of runs
  static constexpr bool F8 = sizeof(S) == 1;
  u32x4 k[NL], v[NL];
  uint32_t sk[NL], sv[NL];  // scale bytes
  int window;               // which 1024 keys of the run of tiles `run` is for
  int run, run_next;        // lane l: first row of keys 16 l .. + 15 of this window, of the next; -1: a bad page
  uint32_t badp;            // bit i: load i's page lies outside the pool
  int rw, lrow, lpc;        // this wave; this lane's row and piece in its load
  uint32_t loff, rowb;

  __device__ __forceinline__ void init(const PagedView &c, int rw_, int lane) {
    rw = rw_;
    lrow = lane / PS;
    lpc = lane % PS;
    rowb = c.Hkv * D * (int)sizeof(S);
    loff = lrow * rowb + 16 * lpc;
  }
  __device__ __forceinline__ int row(int i) const { return i * STEP + rw * SPAN + lrow; }
  __device__ __forceinline__ static int runs(const PagedView &c, const int32_t *table, int w0, int end) {
    return runs1(c, table, min(w0 + 16 * (int)(threadIdx.x & 63), (end - 1) & ~15));
  }
  // The row of position pos; -1 on a bad page.
  __device__ __forceinline__ static int runs1(const PagedView &c, const int32_t *table, int pos) {
    const int pg = table[pos >> c.shift];
    return (unsigned)pg < (unsigned)c.n_pages ? (pg << c.shift) + (pos & ((1 << c.shift) - 1)) : -1;
  }
  // The first two windows of a run of tiles that starts at key k0.
  __device__ __forceinline__ void pages(const PagedView &c, const int32_t *table, int k0, int end) {
    window = 0;
    run = runs(c, table, k0, end);
    run_next = runs(c, table, min(k0 + 1024, end), end);
  }
  // Loads tile j of the run (keys k0 ..); rows past end are some row of a page that
  // belongs to the sequence.
  __device__ __forceinline__ void load(const PagedView &c, const int32_t *table, int hk, int j, int k0, int end) {
    if (j / WIN != window) {
      window = j / WIN;
      run = run_next;
      run_next = runs(c, table, min(k0 - j % WIN * IK + 1024, end), end);
    }
    badp = 0;
    const char *kb = (const char *)c.k + hk * (D * (int)sizeof(S)), *vb = (const char *)c.v + hk * (D * (int)sizeof(S));
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int R0 = i * STEP + rw * SPAN;  // uniform
      const int first = __builtin_amdgcn_readlane(run, (j % WIN * IK + R0) / 16);
      if (first < 0) badp |= 1u << i;
      const uint32_t r = (uint32_t)max(first, 0) + R0 % 16;
      const uint64_t at = (uint64_t)r * rowb;
      k[i] = *reinterpret_cast<const u32x4 *>(kb + at + loff);
      v[i] = *reinterpret_cast<const u32x4 *>(vb + at + loff);
      if constexpr (F8) {
        sk[i] = (c.ks + hk * c.rows() + r)[(uint32_t)lrow];
        sv[i] = (c.vs + hk * c.rows() + r)[(uint32_t)lrow];
      }
    }
  }
  // Load i's piece to LDS, `at` being where load 0's goes: the rows between them
  // only add bits to the row's number, so the permutation is ^ a constant.
  __device__ __forceinline__ static void put(uint32_t at, int i, const u32x4 &w, uint32_t s) {
    const uint32_t to = (at ^ (16 * (piece_at<VPR>(i * STEP, 0) - i * STEP * VPR))) + i * STEP * VPR * 16;
    if constexpr (!F8) {
      lds_write(to, w);
    } else {
      const float sc = scale_of(s);
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const uint32_t a = w[2 * q], b = w[2 * q + 1];
        if constexpr (sizeof(T) == 2) {
          lds_write(to ^ (16 * q), u32x4{f8_bf16<false>(a, sc), f8_bf16<true>(a, sc), f8_bf16<false>(b, sc), f8_bf16<true>(b, sc)});
        } else {
          lds_write(to ^ (32 * q), __builtin_bit_cast(u32x4, f8x4_to_f(a) * sc));
          lds_write(to ^ (32 * q + 16), __builtin_bit_cast(u32x4, f8x4_to_f(b) * sc));
        }
      }
    }
  }
  // Writes the tile.  masked: rows from `left` on become zeros, a row on a bad page
  // NaN keys (and zero values); returns whether a value this thread wrote is not
  // finite.
  template <bool masked> __device__ __forceinline__ bool store(uint32_t lds, int left) {
    const uint32_t at = opaque(lds + 16 * piece_at<VPR>(row(0), lpc * (int)(sizeof(T) / sizeof(S))));
    bool odd = false;
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int R = row(i);
      u32x4 kw = k[i], vw = v[i];
      if constexpr (masked) {
        if (badp >> i & 1) {
          kw = u32x4(0xffffffffu);
          vw = u32x4(0u);
        }
        if (R >= left) kw = vw = u32x4(0u);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const uint32_t x = vw[w];
          if constexpr (F8) {
            const uint32_t y = (x & 0x7f7f7f7fu) + 0x01010101u;  // a NaN code is 127: bit 7 comes up
            odd |= (y & 0x80808080u) != 0;
          } else if constexpr (sizeof(S) == 2) {
            odd |= (x & 0x7f80u) == 0x7f80u || (x & 0x7f800000u) == 0x7f800000u;
          } else {
            odd |= (x & 0x7f800000u) == 0x7f800000u;
          }
        }
      }
      put(at, i, kw, F8 ? sk[i] : 0);
      put(at + TK * D * (int)sizeof(T), i, vw, F8 ? sv[i] : 0);
    }
    return odd;
  }
};

// ---- the kernel -------------------------------------------------------------------

// The matrix instructions with tiles of MF x MF.  A step multiplies one 16-byte
// piece of every lane's left row (lane % MF) with one of its right column; lane
// group lane / MF of NG takes its own piece.  Register 4 q + e of a result holds
// row 4 (NG q + lane / MF) + e of column lane % MF.
template <int MF> struct Acc { typedef f32x16 type; };
template <> struct Acc<16> { typedef f32x4 type; };
template <int MF>
__device__ __forceinline__ typename Acc<MF>::type one_mm(float a, float b, typename Acc<MF>::type c) {
  if constexpr (MF == 32)
    return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
}
template <typename T, int MF>
__device__ __forceinline__ typename Acc<MF>::type step_mm(const u32x4 &a, const u32x4 &b, typename Acc<MF>::type c) {
  if constexpr (sizeof(T) == 2) {
    if constexpr (MF == 32)
      return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    else
      return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  } else {
    const f32x4 x = __builtin_bit_cast(f32x4, a), y = __builtin_bit_cast(f32x4, b);
#pragma unroll
    for (int w = 0; w < 4; ++w) c = one_mm<MF>(x[w], y[w], c);
    return c;
  }
}

// Bytes c .. c + 3 of a mask row of T: one (unaligned) load where T >= 4, moved
// inside the row and shifted back; bytes outside the row are 0.
__device__ __forceinline__ uint32_t mask_word(const uint8_t *mp, int c, int T) {
  uint32_t w = 0;
  int at = 0;
  if (T >= 4) {
    at = min(max(c, 0), T - 4);
    __builtin_memcpy(&w, mp + at, 4);
  } else {
    for (int i = 0; i < T; ++i) w |= (uint32_t)mp[i] << 8 * i;
  }
  const int d = c - at;
  return d >= 4 || d <= -4 ? 0u : d >= 0 ? w >> 8 * d : w << -8 * d;
}

template <typename T, typename S, int D, int MF, int RW, int KW>
__global__ __launch_bounds__(64 * RW * KW, sizeof(T) == 2 ? 2 : 1) void k_tree_attn(TreeArgs a, int nrt, int W_) {
  using Sh = Shape<T, D, MF, RW, KW>;
  using V = typename Acc<MF>::type;
  constexpr int TK = Sh::TK, IK = Sh::IK, TR = Sh::TR, NT = Sh::NT, NS = TK / 32, NDT = D / MF;
  constexpr int NG = 64 / MF, NSUB = 32 / MF;          // lane groups; tiles of 32 keys
  constexpr int NQ = MF * MF / 256;                    // runs of 4 registers of a result
  constexpr int VPR = D * (int)sizeof(T) / 16;
  constexpr int NC = VPR / NG;                         // steps along a key
  constexpr int NR = 32 / NG, NPW = NR * sizeof(T) / 4;  // scores of a lane's 32 keys, registers of their weights
  __shared__ __attribute__((aligned(16))) unsigned char s_mem[Sh::LDS];
  __shared__ float s_ml[KW > 1 ? KW * RW * 64 : 1][2];
  __shared__ long s_scan[NT / 64];
  __shared__ int s_segs[NT / 64];
  __shared__ long s_first[2];
  __shared__ uint32_t s_odd[Sh::NBUF][RW * KW];
  const PagedView &c = a.c;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int grp = wave / RW, rw = wave % RW;
  const int n = lane % MF, h = lane / MF;
  const int G = a.Hq / c.Hkv, E = a.B * nrt;
  // the items of every segment, this range of them, and the segment it starts in
  Work<D> work{a.ws, 2L * W_, TR};
  long total = 0, before = 0;  // items of all, and of those before this thread's
  int segs = 0, segs_before = 0;
  uint32_t mine = 0;
  // The counts of NT entries, added to the running sums.
  auto count = [&](int e0, long &sum, int &nseg) __attribute__((always_inline)) {
    const int e = e0 + tid;
    mine = e < E ? items_of(a, span_of(a, e / nrt), e % nrt, TR, IK) : 0;
    const uint32_t inc = wave_incl_scan(mine);
    const uint64_t some = __builtin_amdgcn_ballot_w64(mine > 0);
    if (lane == 63) {
      s_scan[wave] = inc;
      s_segs[wave] = __popcll(some);
    }
    __syncthreads();
    before = sum + inc - mine;
    segs_before = nseg + __popcll(some & ((1ull << lane) - 1));
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) {
      if (w < wave) {
        before += s_scan[w];
        segs_before += s_segs[w];
      }
      sum += s_scan[w];
      nseg += s_segs[w];
    }
  };
  for (int e0 = 0; e0 < E; e0 += NT) {
    if (e0 > 0) __syncthreads();
    count(e0, total, segs);
  }
  total = uniform(total);
  segs = uniform(segs);
  // (with one item a segment is never cut, and no second launch joins it)
  const int extra = c.max_len > IK && total * c.Hkv > 2L * W_ ? kSegItems : 0;
  const Ranges rg((total + (long)extra * segs) * c.Hkv, W_);
  if (rg.total == 0) {
    if (blockIdx.x == 0)
      for (int e0 = tid; e0 <= E; e0 += NT) work.before()[e0] = 0;
    return;
  }
  if (blockIdx.x >= rg.W) return;
  // neighbouring ranges on one XCD: workgroups go round the 8 of them
  const int xcd = blockIdx.x % 8, wg = (int)(xcd * (rg.W / 8) + min((long)xcd, rg.W % 8)) + blockIdx.x / 8;
  const long x0 = rg.begin(wg), x1 = rg.begin(wg + 1);
  auto find = [&](int e0) __attribute__((always_inline)) {
    before += (long)extra * segs_before;
    if (blockIdx.x == 0 && e0 + tid < E) work.before()[e0 + tid] = before;
    const long lo = before * c.Hkv;
    if (mine > 0 && lo <= x0 && x0 < lo + (long)(mine + extra) * c.Hkv) {
      s_first[0] = e0 + tid;
      s_first[1] = lo;
    }
  };
  if (E <= NT) {
    find(0);
  } else {  // a second walk: the first kept only its last stretch
    long sum = 0;
    int nseg = 0;
    for (int e0 = 0; e0 < E; e0 += NT) {
      __syncthreads();
      count(e0, sum, nseg);
      find(e0);
      if (blockIdx.x > 0 && (uniform(sum) + (long)extra * uniform(nseg)) * c.Hkv > x0) break;
    }
  }
  if (blockIdx.x == 0 && tid == 0) work.before()[E] = rg.total / c.Hkv;
  __syncthreads();
  typedef Tile<T, S, D, RW, TK, IK> Loads;
  Loads tile;  // the next keys, on their way to LDS
  tile.init(c, rw, lane);
  int e = (int)uniform(s_first[0]);
  long at = uniform(s_first[1]);  // first item of entry e
  unsigned char *bufs = s_mem + grp * Sh::NBUF * Sh::BUF;
  const uint32_t bufs_at = lds_address(bufs);

  for (long x = x0; x < x1;) {
    const int b = e / nrt, rt = e % nrt;
    const Span sp = span_of(a, b);
    const int steps = items_of(a, sp, rt, TR, IK), it = steps > 0 ? steps + extra : 0;
    if (it == 0 || x >= at + (long)it * c.Hkv) {
      at += (long)it * c.Hkv;
      ++e;
      continue;
    }
    const int hk = (int)(x - at) / it, i0 = (int)(x - at) % it;  // below 2^31: keys * heads are at most 2^36
    const int ni = (int)min((long)(it - i0), x1 - x);
    x += ni;
    const int end = keys_end(a, sp, rt, TR);
    const int vis_all = sp.bad ? 0 : sp.P + (a.mask ? 0 : rt * TR / G + 1);  // keys every row sees
    const int32_t *table = c.pages + (size_t)b * c.max_pages;
    const int kbeg = i0 * IK + grp * TK;
    // the group's tiles: keys kbeg + j * IK, j < nj (as many rounds for every group)
    const int nj = i0 < steps && end > 0 ? min(ni, steps - i0) : 0;
    const int own = kbeg < end ? min(nj, (end - kbeg + IK - 1) / IK) : 0;
    auto has = [&](int j) __attribute__((always_inline)) { return j < own; };
    // this lane's row: node, head, and q, a 16-byte piece per step: the right operand
    const int row = rt * TR + MF * rw + n, rowc = min(row, sp.live - 1);
    const int node = rowc / G, head = hk * G + rowc % G;
    u32x4 qf[NC];
    {
      const T *qp = (const T *)a.q + ((long)b * a.T + node) * a.qs + (long)head * D;
#pragma unroll
      for (int cc = 0; cc < NC; ++cc) qf[cc] = *reinterpret_cast<const u32x4 *>((const char *)qp + 16 * (NG * cc + h));
    }
    if (has(0)) {
      tile.pages(c, table, kbeg, end);
      tile.load(c, table, hk, 0, kbeg, end);
    }
    const bool wlive = rt * TR + MF * rw < sp.live;  // some row of this wave is there
    const float scl = a.scale * kLog2e;
    float m = -INFINITY, l = 0.f;  // running maximum (log2 units) and sum
    V o[NDT];
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt) o[dt] = V(0.f);
    uint32_t pw[NPW];           // probabilities as the second product takes them
    u32x2 vf[NR / 8 * NDT][2];  // bf16: values of 32 keys
    // A masked tile that holds an infinity or NaN among its values, and those after
    // it, are left for the end: 0 * inf would come through the product to rows that
    // do not see the key.
    int j_odd = own;
    // S^T = K Q^T, then probabilities and their sum.
    auto scores = [&](int j, int u) __attribute__((always_inline)) {
      const int k0 = kbeg + j * IK + 32 * u;
      // piece NG cc + h of row n: ^ 16 NG cc
      const uint32_t ka = opaque(bufs_at + (j % Sh::NBUF) * Sh::BUF + 32 * u * Sh::RB + 16 * piece_at<VPR>(n, h));
      V sv[NSUB];
#pragma unroll
      for (int t = 0; t < NSUB; ++t) sv[t] = V(0.f);
      // reads first, eight at a time: left to itself the compiler reads into one set
      // of registers and waits out the LDS before every product
      constexpr int KB = NC * NSUB < 8 ? NC * NSUB : 8;
#pragma unroll
      for (int c0 = 0; c0 < NC * NSUB; c0 += KB) {
        u32x4 kf[KB];
#pragma unroll
        for (int i = 0; i < KB; ++i) {
          const int cc = (c0 + i) / NSUB, t = (c0 + i) % NSUB;
          kf[i] = lds_read<u32x4>((ka ^ (16 * NG * cc)) + t * MF * Sh::RB);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < KB; ++i) {
          const int cc = (c0 + i) / NSUB, t = (c0 + i) % NSUB;
          sv[t] = step_mm<T, MF>(kf[i], qf[cc], sv[t]);
        }
      }
      if constexpr (sizeof(T) == 2) {
        // the values' reads go out before the scores are worked on.
        // Keys 4 (NG i + h) + 0 .. 3 and those of i + 1, dim MF dt + n: the transposing
        // read (lane 4 e + d of 16 names key e, dims 4 d .. + 3, and gets dim lane % 16
        // of the four keys); the dims of step dt lie ^ 2 MF dt
        const uint32_t vb = bufs_at + (j % Sh::NBUF) * Sh::BUF + (TK + 32 * u) * Sh::RB;
        const int R = 4 * h + (lane >> 2 & 3), pc = (MF == 32 ? 2 * (lane >> 4 & 1) : 0) + (lane >> 1 & 1);
        const uint32_t va0 = opaque(vb + 16 * piece_at<VPR>(R, pc) + 8 * (lane & 1));
        const uint32_t va1 = opaque(vb + 16 * piece_at<VPR>(R + 4 * NG, pc) + 8 * (lane & 1));
#pragma unroll
        for (int i = 0; i < NR / 4; i += 2)
#pragma unroll
          for (int dt = 0; dt < NDT; ++dt) {
            vf[i / 2 * NDT + dt][0] = lds_read_tr((va0 ^ (2 * MF * dt)) + 4 * NG * i * Sh::RB);
            vf[i / 2 * NDT + dt][1] = lds_read_tr((va1 ^ (2 * MF * dt)) + 4 * NG * i * Sh::RB);
          }
        __builtin_amdgcn_sched_barrier(0);
      }
      // log2 units from the maximum on; score 4 q + e: key k0 + 4 (NG q + h) + e
      const float mr = m == -INFINITY ? 0.f : m;
      float s[NR];
#pragma unroll
      for (int r = 0; r < NR; ++r) s[r] = sv[r / (4 * NQ)][r % (4 * NQ)] * scl - mr;
      if (k0 + 32 > vis_all) {
        const uint8_t *mp = opaque(a.mask ? a.mask + ((size_t)b * a.T + node) * a.T : nullptr);
        const int c0 = opaque(k0 - sp.P + 4 * h);
        uint32_t sn = 0;
#pragma unroll
        for (int i = 0; i < NR / 4; ++i) {  // four neighbouring keys
          const int cn = c0 + 4 * NG * i;
          const uint32_t own = mp ? mask_word(mp, cn, a.T) : 0u;
#pragma unroll
          for (int v = 0; v < 4; ++v) {
            const uint32_t in_mask = mp ? (own >> 8 * v & 255) != 0 : cn + v <= node;
            const uint32_t inside = cn + v < sp.n;
            sn |= ((uint32_t)(cn + v < 0) | (inside & in_mask)) << (4 * i + v);
          }
        }
#pragma unroll
        for (int r = 0; r < NR; ++r) s[r] = (sn >> r & 1) ? s[r] : -INFINITY;
      }
      float mx = -INFINITY;
#pragma unroll
      for (int r = 0; r < NR; r += 2) mx = fmaxf(fmaxf(mx, s[r]), s[r + 1]);
      if constexpr (MF == 16) mx = xor16_max(mx);
      mx = xor32_max(mx);
      // the maximum is raised only when a score passes it by 2^8: probabilities
      // stay below that, and the accumulators are seldom rescaled
      const bool up = mx > (m == -INFINITY ? -INFINITY : kLazyMax);
      if (__builtin_amdgcn_ballot_w64(up)) {
        const float by = up ? mx : 0.f, alpha = __builtin_amdgcn_exp2f(-by);
        if (up) m = mr + by;
        l *= alpha;
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt) o[dt] *= alpha;
#pragma unroll
        for (int r = 0; r < NR; ++r) s[r] -= by;
      }
#pragma unroll
      for (int r = 0; r < NR; r += 2) {
        const float p0 = __builtin_amdgcn_exp2f(s[r]), p1 = __builtin_amdgcn_exp2f(s[r + 1]);
        if constexpr (sizeof(T) == 2) {
          // the sum takes the rounded values, so the result is a weighted mean
          pw[r / 2] = f2bf2(p0, p1);
          l = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, pw[r / 2]),
                                              __builtin_bit_cast(bf16x2_t, 0x3f803f80u), l, false);
        } else {
          pw[r] = __float_as_uint(p0);
          pw[r + 1] = __float_as_uint(p1);
          l += p0 + p1;
        }
      }
    };
    // O^T += V^T P^T.
    auto values = [&](int j, int u) __attribute__((always_inline)) {
      if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int i = 0; i < NR / 4; i += 2) {
          const u32x4 pf = {pw[2 * i], pw[2 * i + 1], pw[2 * i + 2], pw[2 * i + 3]};
#pragma unroll
          for (int dt = 0; dt < NDT; ++dt) {
            const u32x2 v0 = vf[i / 2 * NDT + dt][0], v1 = vf[i / 2 * NDT + dt][1];
            o[dt] = step_mm<T, MF>(u32x4{v0.x, v0.y, v1.x, v1.y}, pf, o[dt]);
          }
        }
      } else {
        const uint32_t vb = bufs_at + (j % Sh::NBUF) * Sh::BUF + (TK + 32 * u) * Sh::RB;
#pragma unroll
        for (int r = 0; r < NR; ++r) {
          const int key = 4 * (NG * (r / 4) + h) + r % 4;
#pragma unroll
          for (int dt = 0; dt < NDT; ++dt) {
            const int by = 4 * (MF * dt + n);
            const float vf = lds_read<float>(vb + 16 * piece_at<VPR>(key, by / 16) + by % 16);
            o[dt] = one_mm<MF>(vf, __uint_as_float(pw[r]), o[dt]);
          }
        }
      }
    };
    // One copy of everything in one loop: a workgroup runs through its code once or a
    // few times, and fetching it is a part of what a short call takes.
#pragma unroll 1
    for (int j = 0; j < nj; ++j) {
      const int at_buf = j % Sh::NBUF;
      const bool masked = kbeg + j * IK + TK > vis_all;
      bool odd = false;
      if (has(j)) {
        // Into the buffer of tile j - NBUF: with two, its readers are past barrier j - 1
        // (a wave that shares its tiles with no other needs one).
        const uint32_t to = bufs_at + at_buf * Sh::BUF;
        if (masked || tile.badp != 0)
          odd = __builtin_amdgcn_ballot_w64(tile.template store<true>(to, end - kbeg - j * IK)) != 0;
        else
          tile.template store<false>(to, 0);
        // past the end the last tile again: a condition here would have the compiler
        // move registers that are still being loaded, and wait for them
        const int jl = min(j + 1, own - 1);
        tile.load(c, table, hk, jl, kbeg + jl * IK, end);
      }
      if constexpr (RW > 1) {
        if (masked && lane == 0) s_odd[at_buf][wave] = odd;
        __syncthreads();
        if (masked) {
#pragma unroll
          for (int w = 0; w < RW; ++w) odd |= s_odd[at_buf][grp * RW + w] != 0;
        }
      }
      if (odd && masked) j_odd = min(j_odd, j);
      if (!wlive || j >= j_odd) continue;
#pragma unroll 1
      for (int u = 0; u < NS; ++u) {
        scores(j, u);
        values(j, u);
      }
    }
    // The tiles that were left: a key at a time, from memory, every row over the keys
    // it sees.
    if (j_odd < own && wlive) {
#pragma unroll 1
      for (int i = 0; i < (own - j_odd) * TK; ++i) {
        const int pos = kbeg + (j_odd + i / TK) * IK + i % TK, cn = pos - sp.P;
        if (pos >= end) continue;
        const int first = uniform(Loads::runs1(c, table, pos));
        const long r = max(first, 0);
        const S *kr = (const S *)c.k + (r * c.Hkv + hk) * D, *vr = (const S *)c.v + (r * c.Hkv + hk) * D;
        const float ks = sizeof(S) == 1 ? scale_of(c.ks[hk * c.rows() + r]) : 1.f;
        const float vs = sizeof(S) == 1 ? scale_of(c.vs[hk * c.rows() + r]) : 1.f;
        float dot = 0.f;
#pragma unroll
        for (int cc = 0; cc < NC; ++cc) {
          constexpr int EP = 16 / sizeof(T);  // q's values in a piece
#pragma unroll
          for (int w = 0; w < EP; w += 4) {
            const f32x4 kv = load4<S>(kr + EP * (NG * cc + h) + w);
            f32x4 qv;
            if constexpr (sizeof(T) == 4) {
              qv = __builtin_bit_cast(f32x4, qf[cc]);
            } else {
              const uint32_t q0 = qf[cc][w / 2], q1 = qf[cc][w / 2 + 1];
              qv = f32x4{__uint_as_float(q0 << 16), __uint_as_float(q0 & 0xffff0000u), __uint_as_float(q1 << 16),
                         __uint_as_float(q1 & 0xffff0000u)};
            }
            dot += qv.x * kv.x + qv.y * kv.y + qv.z * kv.z + qv.w * kv.w;
          }
        }
        if constexpr (MF == 16) dot = xor16_sum(dot);
        dot = xor32_sum(dot) * ks * scl;
        if (first < 0) dot = __int_as_float(0x7fc00000);
        const bool vis =
            cn < 0 || (a.mask ? a.mask[((size_t)b * a.T + node) * a.T + cn] != 0 : cn <= node);
        const float mn = vis ? fmaxf(m, dot) : m, mr = mn == -INFINITY ? 0.f : mn;
        const float alpha = sexp2(m, mr), p = vis ? __builtin_amdgcn_exp2f(dot - mr) : 0.f;
        m = mn;
        l = l * alpha + (h == 0 ? p : 0.f);  // the groups' sums are added up below
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
          for (int q4 = 0; q4 < NQ; ++q4) {
            const f32x4 vv = load4<S>(vr + MF * dt + 4 * (NG * q4 + h));
#pragma unroll
            for (int w4 = 0; w4 < 4; ++w4) {
              const float old = o[dt][4 * q4 + w4] * alpha;
              o[dt][4 * q4 + w4] = vis ? old + p * (vv[w4] * vs) : old;
            }
            __builtin_amdgcn_sched_barrier(0);  // few registers: this is seldom run
          }
      }
    }
    if constexpr (MF == 16) l = xor16_sum(l);
    l = xor32_sum(l);

    // groups add up: group g > 0 leaves its sums in LDS, group 0 takes them in order
    if constexpr (KW > 1) {
      f32x4 *so = reinterpret_cast<f32x4 *>(s_mem);  // [(KW - 1) RW][NDT NQ][64]
      static_assert((KW - 1) * RW * NDT * NQ * 64 * 16 <= Sh::LDS, "sums fit the tiles' buffers");
      __syncthreads();
      if (grp > 0) {
        const int at_w = (grp - 1) * RW + rw;
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
          for (int g8 = 0; g8 < NQ; ++g8)
            so[(at_w * NDT * NQ + NQ * dt + g8) * 64 + lane] =
                f32x4{o[dt][4 * g8], o[dt][4 * g8 + 1], o[dt][4 * g8 + 2], o[dt][4 * g8 + 3]};
        s_ml[at_w * 64 + lane][0] = m;
        s_ml[at_w * 64 + lane][1] = l;
      }
      __syncthreads();
      if (grp == 0) {
        float mm = m;
#pragma unroll
        for (int g = 1; g < KW; ++g) mm = fmaxf(mm, s_ml[((g - 1) * RW + rw) * 64 + lane][0]);
        const float sc0 = sexp2(m, mm);
        l *= sc0;
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt) o[dt] *= sc0;
#pragma unroll 1
        for (int g = 1; g < KW; ++g) {
          const int at_w = (g - 1) * RW + rw;
          const float scg = sexp2(s_ml[at_w * 64 + lane][0], mm);
          l += s_ml[at_w * 64 + lane][1] * scg;
#pragma unroll
          for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
            for (int g8 = 0; g8 < NQ; ++g8) {
              const f32x4 w = so[(at_w * NDT * NQ + NQ * dt + g8) * 64 + lane];
#pragma unroll
              for (int w4 = 0; w4 < 4; ++w4) o[dt][4 * g8 + w4] += w[w4] * scg;
            }
        }
        m = mm;
      }
    }
    if (grp == 0 && row < sp.live) {
      if (ni == it) {  // the whole segment
        const float inv = sp.bad ? __int_as_float(0x7fc00000) : l == 0.f ? 0.f : 1.f / l;
        T *op = (T *)a.out + (((long)b * a.T + node) * a.Hq + head) * D + 4 * h;
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
          for (int g8 = 0; g8 < NQ; ++g8) {
            const f32x4 w = f32x4{o[dt][4 * g8], o[dt][4 * g8 + 1], o[dt][4 * g8 + 2], o[dt][4 * g8 + 3]} * inv;
            if constexpr (sizeof(T) == 2)
              *reinterpret_cast<u32x2 *>(op + MF * dt + 4 * NG * g8) = u32x2{f2bf2(w.x, w.y), f2bf2(w.z, w.w)};
            else
              *reinterpret_cast<f32x4 *>(op + MF * dt + 4 * NG * g8) = w;
          }
      } else {
        const long slot = 2L * wg + (i0 > 0 ? 0 : 1);
        f32x4 *po = work.o(slot) + rw * NDT * NQ * 64 + lane;
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
          for (int g8 = 0; g8 < NQ; ++g8)
            po[(NQ * dt + g8) * 64] = f32x4{o[dt][4 * g8], o[dt][4 * g8 + 1], o[dt][4 * g8 + 2], o[dt][4 * g8 + 3]};
        if (h == 0) work.ml(slot)[MF * rw + n] = float2{m, l};
      }
    }
    __syncthreads();  // LDS is free for the next segment
  }
}

// Joins the partials of one segment in the order of their ranges: a wave per MF rows
// and MF dims, a lane as it was in the kernel above, and as many waves of segment
// (sequence, row tile, KV head) blockIdx.x as hold it.  Bound by the partials' bytes:
// 17 us for up to 67 MB of them (256 ranges of 256 rows), 4 to 8 us where latency
// counts.
template <typename T, int D, int MF>
__global__ __launch_bounds__(256) void k_tree_join(TreeArgs a, int nrt, int W_, int TR) {
  constexpr int NDT = D / MF, NG = 64 / MF, NQ = MF * MF / 256, AT = 8 / NQ;
  const PagedView &c = a.c;
  const Work<D> work{a.ws, 2L * W_, TR};
  const int E = a.B * nrt, e = blockIdx.x / c.Hkv, hk = blockIdx.x % c.Hkv;
  const long all = work.before()[E], before = work.before()[e], it = work.before()[e + 1] - before;
  const Span sp = span_of(a, e / nrt);
  if (it == 0) return;
  const Ranges rg(all * c.Hkv, W_);
  const long S = before * c.Hkv + hk * it;
  const long w0 = rg.owner(S), w1 = rg.owner(S + it - 1);
  if (w0 == w1) return;  // one range held it all and wrote the rows
  const int lane = threadIdx.x & 63, n = lane % MF, h = lane / MF;
  const int unit = uniform((int)(blockIdx.y * 4 + (threadIdx.x >> 6))), rw = unit / NDT, dt = unit % NDT;
  const int row = (e % nrt) * TR + MF * rw + n;
  if (row >= sp.live || MF * rw >= TR) return;
  // o += the parts' sums, l += theirs, over the running maximum m; AT parts at a time
  float m = -INFINITY, l = 0.f;
  f32x4 o[NQ];
#pragma unroll
  for (int q = 0; q < NQ; ++q) o[q] = f32x4(0.f);
  auto add = [&](long w, auto kParts) __attribute__((always_inline)) {
    constexpr int N = decltype(kParts)::value;
    float2 ml[N];
    f32x4 part[N][NQ];
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const long slot = w + u == w0 ? 2 * w0 + 1 : 2 * (w + u);
      ml[u] = work.ml(slot)[MF * rw + n];
#pragma unroll
      for (int q = 0; q < NQ; ++q) part[u][q] = work.o(slot)[(NQ * unit + q) * 64 + lane];
    }
    float mn = m;
#pragma unroll
    for (int u = 0; u < N; ++u) mn = fmaxf(mn, ml[u].x);
    const float sc = sexp2(m, mn);
    m = mn;
    l *= sc;
#pragma unroll
    for (int q = 0; q < NQ; ++q) o[q] *= sc;
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const float su = sexp2(ml[u].x, m);
      l += ml[u].y * su;
      // a part of no weight may hold anything
#pragma unroll
      for (int q = 0; q < NQ; ++q) o[q] += su > 0.f ? part[u][q] * su : f32x4(0.f);
    }
  };
  long w = w0;
  for (; w + AT <= w1 + 1; w += AT) add(w, std::integral_constant<int, AT>());
  if (AT > 4 && w + 4 <= w1 + 1) {
    add(w, std::integral_constant<int, 4>());
    w += 4;
  }
  if (AT > 2 && w + 2 <= w1 + 1) {
    add(w, std::integral_constant<int, 2>());
    w += 2;
  }
  if (w <= w1) add(w, std::integral_constant<int, 1>());
  const float inv = sp.bad ? __int_as_float(0x7fc00000) : l == 0.f ? 0.f : 1.f / l;
  const int G = a.Hq / c.Hkv;
  T *op = (T *)a.out + (((long)(e / nrt) * a.T + row / G) * a.Hq + hk * G + row % G) * D + MF * dt + 4 * h;
#pragma unroll
  for (int q = 0; q < NQ; ++q) {
    const f32x4 y = o[q] * inv;
    if constexpr (sizeof(T) == 2)
      *reinterpret_cast<u32x2 *>(op + 4 * NG * q) = u32x2{f2bf2(y.x, y.y), f2bf2(y.z, y.w)};
    else
      *reinterpret_cast<f32x4 *>(op + 4 * NG * q) = y;
  }
}

// ---- host ---------------------------------------------------------------------------

// Compute units of the current device (asked once per device).
int compute_units() {
  static std::atomic<int> known[64];
  int d = 0;
  if (hipGetDevice(&d) != hipSuccess || d < 0 || d >= 64) return 256;
  int n = known[d].load(std::memory_order_relaxed);
  if (n == 0) {
    if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, d) != hipSuccess || n <= 0) n = 256;
    known[d].store(n, std::memory_order_relaxed);
  }
  return n;
}

// The launch of a call: the variant, row tiles per sequence, ranges, and whether a
// segment may be cut at all.
struct Plan {
  int variant, nrt, W;
  bool join;
};
constexpr int kMaxCus = 512;

// The variants: MF, RW, KW, workgroups per compute unit.  The last is fp32's, whose
// operands take twice the registers.
constexpr int kShapes[4][4] = {{16, 1, 4, 2}, {32, 4, 2, 1}, {32, 8, 1, 1}, {32, 4, 1, 1}};

// The variant for `rows` per (sequence, KV head) and `keys` over all of these.  Few
// rows in all, counted in tiles of 16: a workgroup of 16 rows starts soonest and
// leaves the smallest partial sums; more row tiles then read a key more often, from
// L2.  Many: a key is staged once for 128 rows, or for 256, whose partial sums are
// twice as large: up to 2^16 keys only where one tile holds all rows (204 rows over
// 1024 keys: 26 us in tiles of 128, 22 in one of 256).  Measured with 8 KV heads of 128 dims and 2048 keys a
// sequence (us; 16 / 128 / 256 rows at a time; * taken):
//   rows   bf16, 1 seq.      bf16, 32            8 bits, 1         8 bits, 32
//    16   *14 /  19 /  19    59 / *47 /   57    *12 / 19 /  18   *33 /  47 /   54
//    32   *16 /  20 /  19    63 / *48 /   58    *14 / 20 /  19    39 / *47 /   55
//   128    28 / *23 /  22   162 / *61 /   68    *17 / 23 /  22   133 / *54 /   62
//   256    30 /  30 / *33   289 / 108 /  *93    *21 / 30 /  32   261 /  98 /  *83
//   512    33 / *24 /  34   578 / 209 / *177     28 / *28 / 34   522 / 191 / *163
// fp32, 32 sequences, 16 / 128 rows at a time: 16 rows 131 / 400, 32 rows 225 / 400,
// 64 rows 424 / 405.
int variant_of(int rows, int dt, bool f8, long keys) {
  if (dt == kF32) return rows <= 32 ? 0 : 3;
  const long tiles = (rows + 15) / 16;
  if (f8 ? rows <= 16 || keys * tiles <= 1L << 18 : rows <= 32 && keys * tiles <= 1L << 17) return 0;
  return rows <= 128 || (rows > 256 && keys <= 1L << 16) ? 1 : 2;
}

Plan plan_of(const PagedView &c, int B, int T, int Hq, int dt, int cus) {
  const int rows = T * (Hq / c.Hkv);
  Plan p;
  p.variant = variant_of(rows, dt, c.dtype == kF8, (long)B * c.Hkv * c.max_len);
  const int *sh = kShapes[p.variant];
  const int TR = sh[0] * sh[1], IK = sh[2] * tile_keys(sh[1], c.D);
  p.nrt = (rows + TR - 1) / TR;
  const long most = ((long)c.max_len + IK - 1) / IK;
  const long items = (long)B * p.nrt * c.Hkv * most;
  p.W = (int)std::min<long>(items, (long)cus * (dt == kF32 ? 1 : sh[3]));
  p.join = most > 1 && p.W > 0;
  return p;
}

template <typename T, typename S, int D, int V> hipError_t launch(const TreeArgs &a, const Plan &p, hipStream_t s) {
  using Sh = Shape<T, D, kShapes[V][0], kShapes[V][1], kShapes[V][2]>;
  k_tree_attn<T, S, D, Sh::MF, Sh::RW, Sh::KW><<<p.W, Sh::NT, 0, s>>>(a, p.nrt, p.W);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !p.join) return e;
  const int waves = std::min<long>(Sh::RW, ((long)a.T * (a.Hq / a.c.Hkv) + Sh::MF - 1) / Sh::MF) * (D / Sh::MF);
  k_tree_join<T, D, Sh::MF><<<dim3(a.B * p.nrt * a.c.Hkv, (waves + 3) / 4), 256, 0, s>>>(a, p.nrt, p.W, Sh::TR);
  return hipGetLastError();
}

template <typename T, typename S, int D> hipError_t by_rows(const TreeArgs &a, const Plan &p, hipStream_t s) {
  if (p.variant == 0) return launch<T, S, D, 0>(a, p, s);
  if constexpr (sizeof(T) == 4)
    return launch<T, S, D, 3>(a, p, s);
  else
    return p.variant == 1 ? launch<T, S, D, 1>(a, p, s) : launch<T, S, D, 2>(a, p, s);
}

template <typename T, typename S> hipError_t by_dim(const TreeArgs &a, const Plan &p, hipStream_t s) {
  return a.c.D == 64 ? by_rows<T, S, 64>(a, p, s) : by_rows<T, S, 128>(a, p, s);
}

}  // namespace

size_t tree_attention_ws(const PagedView &c, int B, int T, int Hq, int dt) {
  const Plan p = plan_of(c, B, T, Hq, dt, kMaxCus);
  const size_t rows = 2 * (size_t)p.W * kShapes[p.variant][0] * kShapes[p.variant][1];
  return (rows * (c.D + 2) * 4 + ((size_t)B * p.nrt + 1) * 8 + 255) & ~(size_t)255;
}

hipError_t tree_attention(const TreeArgs &a, int dt, hipStream_t s) {
  const Plan p = plan_of(a.c, a.B, a.T, a.Hq, dt, std::min(compute_units(), kMaxCus));
  if (dt == kF32) return a.c.dtype == kF8 ? by_dim<float, uint8_t>(a, p, s) : by_dim<float, float>(a, p, s);
  return a.c.dtype == kF8 ? by_dim<uint16_t, uint8_t>(a, p, s) : by_dim<uint16_t, uint16_t>(a, p, s);
}

}  // namespace fe
