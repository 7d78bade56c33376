// fe_tree_attn.hip -- attention of draft-tree nodes over a paged cache (gfx950).
#include "fe_paged.h"

namespace fe {
namespace {

// One wave per (sequence, node, query head): a key at a time, its score summed
// over the wave, running maximum and sum.
template <typename T, typename S, int D>
__global__ __launch_bounds__(256) void k_tree_attn_rows(TreeArgs a) {
  constexpr int E = D / 64;
  const PagedView &c = a.c;
  const long w = (long)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  if (w >= (long)a.B * a.T * a.Hq) return;
  const int h = w % a.Hq, t = w / a.Hq % a.T, b = w / a.Hq / a.T, hk = h / (a.Hq / c.Hkv);
  const int P = a.lens[b], n = a.counts ? a.counts[b] : a.T;
  const bool bad = P < 0 || n < 0 || n > a.T || (long)P + n > c.max_len;
  if (n >= 0 && n <= a.T && t >= n) return;
  T *out = (T *)a.out + (((long)b * a.T + t) * a.Hq + h) * D + E * lane;
  const T *qp = (const T *)a.q + ((long)b * a.T + t) * a.qs + (long)h * D + E * lane;
  float q[E], o[E];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    q[e] = Elt<T>::to_f(qp[e]) * (a.scale * 1.4426950408889634f);
    o[e] = 0.f;
  }
  float m = -INFINITY, l = 0.f;
  const int end = bad ? 0 : P + n;
  for (int j = 0; j < end; ++j) {
    const int node = j - P;
    if (node >= 0 && !(a.mask ? a.mask[((long)b * a.T + t) * a.T + node] != 0 : node <= t)) continue;
    const long row = c.row(b, j);
    float k[E], v[E];
    if (row < 0) {
#pragma unroll
      for (int e = 0; e < E; ++e) k[e] = v[e] = __int_as_float(0x7fc00000);
    } else {
      const long at = (row * c.Hkv + hk) * D + E * lane;
      if constexpr (sizeof(S) == 1) {
        const float sk = scale_of(c.ks[hk * c.rows() + row]), sv = scale_of(c.vs[hk * c.rows() + row]);
#pragma unroll
        for (int e = 0; e < E; ++e) {
          k[e] = f8x4_to_f(((const uint8_t *)c.k)[at + e]).x * sk;
          v[e] = f8x4_to_f(((const uint8_t *)c.v)[at + e]).x * sv;
        }
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e) {
          k[e] = Elt<S>::to_f(((const S *)c.k)[at + e]);
          v[e] = Elt<S>::to_f(((const S *)c.v)[at + e]);
        }
      }
    }
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) s += q[e] * k[e];
    s = group_sum<64>(s);
    const float mn = fmaxf(m, s), al = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mn);
    const float p = __builtin_amdgcn_exp2f(s - (mn == -INFINITY ? 0.f : mn));
    m = mn;
    l = l * al + p;
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = o[e] * al + p * v[e];
  }
  const float inv = bad ? __int_as_float(0x7fc00000) : l == 0.f ? 0.f : 1.f / l;
#pragma unroll
  for (int e = 0; e < E; ++e) out[e] = Elt<T>::from_f(o[e] * inv);
}

template <typename T, typename S>
hipError_t rows_t(const TreeArgs &a, hipStream_t s) {
  const long waves = (long)a.B * a.T * a.Hq;
  if (a.c.D == 64)
    k_tree_attn_rows<T, S, 64><<<(waves + 3) / 4, 256, 0, s>>>(a);
  else
    k_tree_attn_rows<T, S, 128><<<(waves + 3) / 4, 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

size_t tree_attention_ws(const PagedView &, int, int, int, int) { return 256; }

hipError_t tree_attention(const TreeArgs &a, int dt, hipStream_t s) {
  if (dt == kF32) return a.c.dtype == kF8 ? rows_t<float, uint8_t>(a, s) : rows_t<float, float>(a, s);
  return a.c.dtype == kF8 ? rows_t<uint16_t, uint8_t>(a, s) : rows_t<uint16_t, uint16_t>(a, s);
}

}  // namespace fe
