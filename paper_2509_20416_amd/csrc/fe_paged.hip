// fe_paged.hip -- the paged cache around tree-attention verification: rows
// appended (rotated, kept as they are or coded in 8 bits), read back, and moved
// behind the prefix after acceptance (gfx950).  All three are bound by bytes (or,
// for a few rows, by the latency of one launch).
#include <algorithm>

#include "fe_paged.h"

namespace fe {
namespace {

// ---- append -----------------------------------------------------------------------
// One workgroup per new row (b, i): the row's angles once (double precision, 8
// bytes of product and the sine and cosine of the reduced angle, so positions past
// 2^24 turn by the right amount), shared by all its heads.  A lane takes 8
// neighbouring dims of a head, so 16-byte loads and stores throughout; the other
// half of its pairs (half layout) is a second load from the same lines.  Bound by
// bytes: 8192 rows with 64 query and 8 KV heads of 128 dims, rotated, the cache in 8
// bits, 319 MB in 63 us, 5.0 TB/s.
//
// Up to kFewRows rows their heads are spread over as many workgroups as take them in
// one step, which computes the angles more often and waits for one load instead of
// several (8 KV heads and 32 query heads of 128 dims, us, spread / not): 32 rows 4.0 /
// 6.0, 256 rows 4.8 / 6.5, 512 rows 6.4 / 7.1, 1024 rows 9.4 / 8.5.
constexpr int kFewRows = 512;

template <typename T, bool F8, int D, bool ROPE>
__global__ __launch_bounds__(256) void k_cache_append(PagedView c, int T_, const int32_t *__restrict__ starts,
                                                      const int32_t *__restrict__ counts,
                                                      const int32_t *__restrict__ positions, RopeArgs rope,
                                                      const T *__restrict__ k, long ks,
                                                      const T *__restrict__ v, long vs,
                                                      const T *__restrict__ q, long qs, int Hq,
                                                      T *__restrict__ q_out) {
  constexpr int LPH = D / 8;  // lanes per head
  __shared__ double s_cs[2][D / 2];
  const int r = blockIdx.x, b = r / T_, i = r % T_;
  if (counts && i >= counts[b]) return;
  const int start = starts[b];
  const long slot = (long)start + i;
  const long row = start >= 0 && slot < c.max_len ? c.row(b, (int)slot) : -1;
  if constexpr (ROPE) {
    const int m = threadIdx.x;
    if (m < rope.rot / 2) {
      const double pos = positions ? (double)positions[r] : (double)slot;
      double sn, cs;
      sincos(pos * rope.freqs[m], &sn, &cs);
      s_cs[0][m] = cs * (double)rope.magnitude;
      s_cs[1][m] = sn * (double)rope.magnitude;
    }
    __syncthreads();
  }
  const int d0 = 8 * (threadIdx.x % LPH), half = rope.rot / 2;
  const int nq = q ? Hq : 0, units = nq + 2 * c.Hkv;
  for (int u = blockIdx.y * (256 / LPH) + threadIdx.x / LPH; u < units; u += gridDim.y * (256 / LPH)) {
    const int kind = u < nq ? 0 : u < nq + c.Hkv ? 1 : 2;  // query, key, value
    const int h = kind == 0 ? u : kind == 1 ? u - nq : u - nq - c.Hkv;
    const T *src = (kind == 0 ? q + r * qs : kind == 1 ? k + r * ks : v + r * vs) + (long)h * D;
    f32x8 y = load8<T>(src + d0);
    if (ROPE && kind != 2 && d0 < rope.rot) {
      if (rope.interleaved) {
        const f32x8 x = y;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const double cs = s_cs[0][d0 / 2 + e], sn = s_cs[1][d0 / 2 + e];
          if (sizeof(T) == 4 || (F8 && kind == 1)) {
            y[2 * e] = (float)(x[2 * e] * cs - x[2 * e + 1] * sn);
            y[2 * e + 1] = (float)(x[2 * e + 1] * cs + x[2 * e] * sn);
          } else {
            y[2 * e] = x[2 * e] * (float)cs - x[2 * e + 1] * (float)sn;
            y[2 * e + 1] = x[2 * e + 1] * (float)cs + x[2 * e] * (float)sn;
          }
        }
      } else {
        const bool low = d0 < half;
        const int m0 = low ? d0 : d0 - half;
        const f32x8 p = load8<T>(src + (low ? d0 + half : d0 - half));
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const double cs = s_cs[0][m0 + e], sn = low ? -s_cs[1][m0 + e] : s_cs[1][m0 + e];
          if (sizeof(T) == 4 || (F8 && kind == 1))
            y[e] = (float)(y[e] * cs + p[e] * sn);
          else
            y[e] = y[e] * (float)cs + p[e] * (float)sn;
        }
      }
    }
    if (kind == 0) {
      store8<T>(q_out + ((long)r * Hq + h) * D + d0, y);
      continue;
    }
    if (row < 0) continue;
    const long at = (row * c.Hkv + h) * D + d0;
    if constexpr (F8) {
      float mx = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const bool fin = fabsf(y[e]) < INFINITY;
        mx = fin ? fmaxf(mx, fabsf(y[e])) : mx;
        y[e] = fin ? y[e] : __int_as_float(0x7fc00000);
      }
      mx = group_max<LPH>(mx);
      // 448 = 1.75 * 2^8: s = exponent - 8, one more where the mantissa is past .75
      const uint32_t w = __float_as_uint(mx);
      const int s = max((int)(w >> 23) - 8 + ((w & 0x7fffffu) > 0x600000u ? 1 : 0), 1);
      y *= scale_of(254 - s);
      u32x2 o;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        int x = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * e], y[4 * e + 1], 0, false);
        o[e] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[4 * e + 2], y[4 * e + 3], x, true);
      }
      *reinterpret_cast<u32x2 *>((uint8_t *)(kind == 1 ? c.k : c.v) + at) = o;
      if (threadIdx.x % LPH == 0) (kind == 1 ? c.ks : c.vs)[h * c.rows() + row] = (uint8_t)s;
    } else {
      store8<T>((T *)(kind == 1 ? c.k : c.v) + at, y);
    }
  }
}

// ---- gather -----------------------------------------------------------------------
// The sequence of packed row r: the number of ends cu[1 .. B] at or below it,
// counted 64 at a time by the wave (r is wave-uniform).
__device__ __forceinline__ int seq_of(const int32_t *__restrict__ cu, int B, int r) {
  int n = 0;
  for (int j0 = 0; j0 < B; j0 += 64) {
    const int j = j0 + (threadIdx.x & 63);
    const uint64_t m = __builtin_amdgcn_ballot_w64(j < B && cu[j + 1] <= r);
    n += __popcll(m);
    if (~m) break;
  }
  return n;
}

// One wave per packed row, so that its sequence and page are wave-uniform; a lane
// takes the same 16 bytes of stored keys and values (8 values of fp32) at a time.
// Bound by bytes: 833 MB of 32 histories, 8 bits to bf16, in 176 us, 4.7 TB/s.
template <typename T, typename S, int D>
__global__ __launch_bounds__(256) void k_cache_gather(PagedView c, int B, const int32_t *__restrict__ starts,
                                                      const int32_t *__restrict__ cu, int n_rows,
                                                      T *__restrict__ ko, T *__restrict__ vo) {
  constexpr int NV = sizeof(S) == 1 ? 2 : 1;        // runs of 8 values
  const int per = c.Hkv * (D / (8 * NV)), lane = threadIdx.x & 63;
  for (long rl = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6)); rl < n_rows; rl += gridDim.x * 4) {
    const int r = (int)rl, b = seq_of(cu, B, r);
    if (b >= B || r < cu[0]) continue;
    const long pos = (starts ? (long)starts[b] : 0) + r - cu[b];
    const long row = pos >= 0 && pos < c.max_len ? c.row(b, (int)pos) : -1;
    const long from = max(row, 0L) * c.Hkv * D, to = (long)r * c.Hkv * D;
    for (int p = lane; p < per; p += 64) {
      const int h = p / (D / (8 * NV));
      f32x8 y[2][NV];
#pragma unroll
      for (int w = 0; w < 2; ++w)
        if (w ? vo : ko) {
#pragma unroll
          for (int i = 0; i < NV; ++i) y[w][i] = load8<S>((const S *)(w ? c.v : c.k) + from + 8 * (NV * p + i));
          if constexpr (sizeof(S) == 1) {
            const float sc = scale_of((w ? c.vs : c.ks)[h * c.rows() + max(row, 0L)]);
#pragma unroll
            for (int i = 0; i < NV; ++i) y[w][i] *= sc;
          }
        }
#pragma unroll
      for (int w = 0; w < 2; ++w)
        if (T *dst = w ? vo : ko) {
#pragma unroll
          for (int i = 0; i < NV; ++i)
            store8<T>(dst + to + 8 * (NV * p + i), row < 0 ? f32x8(__int_as_float(0x7fc00000)) : y[w][i]);
        }
    }
  }
}

// ---- commit -----------------------------------------------------------------------
struct CommitArgs {
  CommitPool pool[kCommitLayers];
};

// One workgroup per (layer, sequence).  A thread owns 16-byte columns of the
// rows: it loads its column of every source row before it stores any, so rows
// that are both source and destination need no order between threads.  Bound by
// latency, lengths to table to rows: 4.8 us for one sequence in 5 layers, 9.2 us for
// 32 in 32 layers (14.8 MB).
__global__ __launch_bounds__(256) void k_cache_commit(PagedView c, CommitArgs a, int first, int T, int n_paths,
                                                      int depth, const int32_t *__restrict__ lens,
                                                      const int32_t *__restrict__ retrieve,
                                                      const int32_t *__restrict__ path,
                                                      const int32_t *__restrict__ len,
                                                      int32_t *__restrict__ new_lens) {
  const int b = blockIdx.y, layer = blockIdx.x;
  __shared__ long s_src[kCommitDepth], s_dst[kCommitDepth];
  __shared__ int s_bad;
  const int P = lens[b], n = len[b], pt = path[b];
  if (threadIdx.x == 0) s_bad = n < 0 || n > depth || pt < 0 || pt >= n_paths || P < 0;
  __syncthreads();
  const bool ok = !s_bad;
  __syncthreads();
  if (ok && (int)threadIdx.x <= n) {  // t = 0: the root's own place has to exist too
    const int t = threadIdx.x;
    const int node = t ? retrieve[((size_t)b * n_paths + pt) * (depth + 1) + t] : 0;
    long src = -1, dst = -1;
    if (node >= 0 && node < T && (long)P + node < c.max_len && (long)P + t < c.max_len) {
      src = c.row(b, P + node);
      dst = c.row(b, P + t);
    }
    if (src < 0 || dst < 0) s_bad = 1;
    if (t) {
      s_src[t - 1] = src;
      s_dst[t - 1] = dst;
    }
  }
  __syncthreads();
  if (first && layer == 0 && threadIdx.x == 0) new_lens[b] = s_bad ? -1 : P + 1 + n;
  if (s_bad || n == 0) return;
  const CommitPool pool = a.pool[layer];
  const int es = c.dtype == kF32 ? 4 : c.dtype == kBf16 ? 2 : 1;
  const int rb = c.Hkv * c.D * es, per = rb / 16;
  for (int p = threadIdx.x; p < 2 * per; p += 256) {
    char *base = p < per ? pool.k + 16 * p : pool.v + 16 * (p - per);
    u32x4 w[kCommitDepth];
#pragma unroll
    for (int t = 0; t < kCommitDepth; ++t)
      if (t < n) w[t] = *reinterpret_cast<const u32x4 *>(base + s_src[t] * rb);
#pragma unroll
    for (int t = 0; t < kCommitDepth; ++t)
      if (t < n) *reinterpret_cast<u32x4 *>(base + s_dst[t] * rb) = w[t];
  }
  if (c.dtype == kF8)
    for (int p = threadIdx.x; p < 2 * c.Hkv; p += 256) {
      uint8_t *base = p < c.Hkv ? pool.ks + p * c.rows() : pool.vs + (p - c.Hkv) * c.rows();
      uint8_t w[kCommitDepth];
#pragma unroll
      for (int t = 0; t < kCommitDepth; ++t)
        if (t < n) w[t] = base[s_src[t]];
#pragma unroll
      for (int t = 0; t < kCommitDepth; ++t)
        if (t < n) base[s_dst[t]] = w[t];
    }
}

template <typename T, bool F8, int D>
hipError_t append_d(const PagedView &c, int B, int T_, const int32_t *starts, const int32_t *counts,
                    const int32_t *positions, const RopeArgs &rope, const void *k, long ks, const void *v,
                    long vs, const void *q, long qs, int Hq, void *q_out, hipStream_t s) {
  const int heads = (q ? Hq : 0) + 2 * c.Hkv, split = B * T_ <= kFewRows ? (heads * (D / 8) + 255) / 256 : 1;
  auto go = [&](auto kern) {
    kern<<<dim3(B * T_, split), 256, 0, s>>>(c, T_, starts, counts, positions, rope, (const T *)k, ks, (const T *)v, vs,
                                (const T *)q, qs, Hq, (T *)q_out);
    return hipGetLastError();
  };
  return rope.freqs ? go(k_cache_append<T, F8, D, true>) : go(k_cache_append<T, F8, D, false>);
}

template <typename T, typename S>
hipError_t gather_t(const PagedView &c, int B, const int32_t *starts, const int32_t *cu, int n_rows, void *ko,
                    void *vo, hipStream_t s) {
  const int grid = (int)std::min<long>(((long)n_rows + 3) / 4, 65536);
  if (c.D == 64)
    k_cache_gather<T, S, 64><<<grid, 256, 0, s>>>(c, B, starts, cu, n_rows, (T *)ko, (T *)vo);
  else
    k_cache_gather<T, S, 128><<<grid, 256, 0, s>>>(c, B, starts, cu, n_rows, (T *)ko, (T *)vo);
  return hipGetLastError();
}

}  // namespace

hipError_t cache_append(const PagedView &c, int B, int T, const int32_t *starts, const int32_t *counts,
                        const int32_t *positions, const RopeArgs &rope, int dt, const void *k, long ks,
                        const void *v, long vs, const void *q, long qs, int Hq, void *q_out,
                        hipStream_t s) {
  auto go = [&](auto f) { return f(c, B, T, starts, counts, positions, rope, k, ks, v, vs, q, qs, Hq, q_out, s); };
  const bool f8 = c.dtype == kF8, d64 = c.D == 64;
  if (dt == kF32)
    return f8 ? (d64 ? go(append_d<float, true, 64>) : go(append_d<float, true, 128>))
              : (d64 ? go(append_d<float, false, 64>) : go(append_d<float, false, 128>));
  return f8 ? (d64 ? go(append_d<uint16_t, true, 64>) : go(append_d<uint16_t, true, 128>))
            : (d64 ? go(append_d<uint16_t, false, 64>) : go(append_d<uint16_t, false, 128>));
}

hipError_t cache_gather(const PagedView &c, int B, const int32_t *starts, const int32_t *cu, int n_rows, int dt,
                        void *k_out, void *v_out, hipStream_t s) {
  auto go = [&](auto f) { return f(c, B, starts, cu, n_rows, k_out, v_out, s); };
  if (dt == kF32)
    return c.dtype == kF32    ? go(gather_t<float, float>)
           : c.dtype == kBf16 ? go(gather_t<float, uint16_t>)
                              : go(gather_t<float, uint8_t>);
  return c.dtype == kF32    ? go(gather_t<uint16_t, float>)
         : c.dtype == kBf16 ? go(gather_t<uint16_t, uint16_t>)
                            : go(gather_t<uint16_t, uint8_t>);
}

hipError_t cache_commit(const PagedView &c, const CommitPool *pools, int n_layers, int B, int T, int n_paths,
                        int depth, const int32_t *lens, const int32_t *retrieve, const int32_t *path,
                        const int32_t *len, int32_t *new_lens, hipStream_t s) {
  for (int l0 = 0; l0 < n_layers; l0 += kCommitLayers) {
    CommitArgs a;
    const int n = n_layers - l0 < kCommitLayers ? n_layers - l0 : kCommitLayers;
    for (int l = 0; l < n; ++l) a.pool[l] = pools[l0 + l];
    k_cache_commit<<<dim3(n, B), 256, 0, s>>>(c, a, l0 == 0, T, n_paths, depth, lens, retrieve, path, len,
                                              new_lens);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace fe
