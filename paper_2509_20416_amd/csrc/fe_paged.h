// fe_paged.h -- the paged cache as its kernels see it (gfx950).  Not part of the
// public ABI.
#pragma once

#include "fe_internal.h"

namespace fe {

// Cache types (include/fe.h fe_dtype).
constexpr int kF32 = 0, kBf16 = 1, kF8 = 2;

// A batch's view of one layer's cache.
struct PagedView {
  void *k, *v;              // [n_pages << shift, Hkv, D]
  uint8_t *ks, *vs;         // 8-bit caches: [Hkv, n_pages << shift] scale bytes
  const int32_t *pages;     // [B, max_pages]
  int n_pages, shift, max_pages, max_len, Hkv, D, dtype;
  __host__ __device__ long rows() const { return (long)n_pages << shift; }
  // Row of position pos, 0 <= pos < max_len, of sequence b; -1 on a page outside
  // the pool.
  __device__ __forceinline__ long row(int b, int pos) const {
    const int pg = pages[(size_t)b * max_pages + (pos >> shift)];
    if ((unsigned)pg >= (unsigned)n_pages) return -1;
    return ((long)pg << shift) + (pos & ((1 << shift) - 1));
  }
};

typedef float f32x8 __attribute__((ext_vector_type(8)));

// 2^(s - 127) of a scale byte s (1 .. 254).
__device__ __forceinline__ float scale_of(uint32_t s) { return __uint_as_float(s << 23); }

// Four e4m3 codes -> fp32, exact (NaN codes give NaN).
__device__ __forceinline__ f32x4 f8x4_to_f(uint32_t w) {
  const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false);
  const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  return f32x4{lo[0], lo[1], hi[0], hi[1]};
}

// Eight stored values -> fp32; p: the piece's first element.
template <typename T> __device__ __forceinline__ f32x8 load8(const T *p);
template <> __device__ __forceinline__ f32x8 load8<float>(const float *p) {
  const f32x4 a = *reinterpret_cast<const f32x4 *>(p), b = *reinterpret_cast<const f32x4 *>(p + 4);
  return f32x8{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
}
template <> __device__ __forceinline__ f32x8 load8<uint16_t>(const uint16_t *p) {
  const u32x4 w = *reinterpret_cast<const u32x4 *>(p);
  f32x8 f;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    f[2 * e] = __uint_as_float(w[e] << 16);
    f[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
  }
  return f;
}
template <> __device__ __forceinline__ f32x8 load8<uint8_t>(const uint8_t *p) {
  const u32x2 w = *reinterpret_cast<const u32x2 *>(p);
  const f32x4 a = f8x4_to_f(w.x), b = f8x4_to_f(w.y);
  return f32x8{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
}
template <typename T> __device__ __forceinline__ f32x4 load4(const T *p);
template <> __device__ __forceinline__ f32x4 load4<float>(const float *p) { return *reinterpret_cast<const f32x4 *>(p); }
template <> __device__ __forceinline__ f32x4 load4<uint16_t>(const uint16_t *p) {
  const u32x2 w = *reinterpret_cast<const u32x2 *>(p);
  return f32x4{__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xffff0000u), __uint_as_float(w.y << 16),
               __uint_as_float(w.y & 0xffff0000u)};
}
template <> __device__ __forceinline__ f32x4 load4<uint8_t>(const uint8_t *p) {
  return f8x4_to_f(*reinterpret_cast<const uint32_t *>(p));
}
template <typename T> __device__ __forceinline__ void store8(T *p, const f32x8 &f);
template <> __device__ __forceinline__ void store8<float>(float *p, const f32x8 &f) {
  *reinterpret_cast<f32x4 *>(p) = f32x4{f[0], f[1], f[2], f[3]};
  *reinterpret_cast<f32x4 *>(p + 4) = f32x4{f[4], f[5], f[6], f[7]};
}
template <> __device__ __forceinline__ void store8<uint16_t>(uint16_t *p, const f32x8 &f) {
  *reinterpret_cast<u32x4 *>(p) =
      u32x4{f2bf2(f[0], f[1]), f2bf2(f[2], f[3]), f2bf2(f[4], f[5]), f2bf2(f[6], f[7])};
}

// Launchers; the entry points in fe_paged_api.hip have checked the arguments.
struct RopeArgs {
  const double *freqs;  // null: no rotation
  int rot, interleaved;
  float magnitude;
};
hipError_t cache_append(const PagedView &c, int B, int T, const int32_t *starts, const int32_t *counts,
                        const int32_t *positions, const RopeArgs &rope, int dt, const void *k, long ks,
                        const void *v, long vs, const void *q, long qs, int Hq, void *q_out,
                        hipStream_t s);
hipError_t cache_gather(const PagedView &c, int B, const int32_t *starts, const int32_t *cu, int n_rows,
                        int dt, void *k_out, void *v_out, hipStream_t s);
// One layer's pool in a commit launch.
struct CommitPool {
  char *k, *v;
  uint8_t *ks, *vs;
};
constexpr int kCommitLayers = 64;  // layers per launch: their pools are kernel arguments
constexpr int kCommitDepth = 16;
hipError_t cache_commit(const PagedView &c, const CommitPool *pools, int n_layers, int B, int T,
                        int n_paths, int depth, const int32_t *lens, const int32_t *retrieve,
                        const int32_t *path, const int32_t *len, int32_t *new_lens, hipStream_t s);
struct TreeArgs {
  PagedView c;
  int B, T, Hq;
  const int32_t *lens, *counts;
  const uint8_t *mask;
  const void *q;
  long qs;
  float scale;
  void *out;
  float *ws;
};
hipError_t tree_attention(const TreeArgs &a, int dt, hipStream_t s);
size_t tree_attention_ws(const PagedView &c, int B, int T, int Hq, int dt);

}  // namespace fe
