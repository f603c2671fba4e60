// Attention with a window and sinks, one row by one wave: the definition, walked 64 keys (or queries) at a time, a lane each, in float32.  Only what a row sees is read, so that
// nothing else reaches its results.
#pragma once
#include "mixers.h"

// sum over d of a[x] b[x], d a multiple of 8
template <typename T>
__device__ __forceinline__ float window_dot(const T* __restrict__ a, const T* __restrict__ b, int d) {
  float s = 0.f;
  for (int x = 0; x < d; x += 8) {
    Vec8<T> u, v;
    u.load(a + x);
    v.load(b + x);
#pragma unroll
    for (int e = 0; e < 8; e++) s = fmaf(u.v[e], v.v[e], s);
  }
  return s;
}
// The keys of row i are first the sinks before its window, `ns` of them, then the window from lo on.
struct WindowKeys {
  int ns, lo, n;
  __device__ __forceinline__ WindowKeys(const WindowGeom& g, int i) {
    lo = max(0, i - g.window + 1);
    ns = min(g.sinks, lo);
    n = ns + i + 1 - lo;
  }
  __device__ __forceinline__ int key(int c) const { return c < ns ? c : lo + c - ns; }
};
// The queries that see key j are rows j .. end - 1.
__device__ __forceinline__ int window_queries_end(const WindowGeom& g, int j) { return j < g.sinks ? g.seq : (int)min((long long)g.seq, (long long)j + g.window); }

#define WR_COLS 2  // columns of a row that a lane holds: d <= 128
// o and lse of row i of sequence b, head h.  qkv: of the sequence's first row.
template <typename T>
__device__ __forceinline__ void window_row_fwd(const WindowGeom& g, const T* __restrict__ qkv, int h, int i, T* __restrict__ orow, float* __restrict__ lrow) {
  const int lane = threadIdx.x & 63, d = g.d, hk = h / (g.nq / g.nkv);
  const size_t ld = (size_t)(g.nq + 2 * g.nkv) * d;
  const T *q = qkv + i * ld + (size_t)h * d, *k = qkv + (size_t)(g.nq + hk) * d, *v = k + (size_t)g.nkv * d;
  const WindowKeys keys(g, i);
  float m = -INFINITY, l = 0.f, acc[WR_COLS] = {};
  for (int c0 = 0; c0 < keys.n; c0 += 64) {
    const int c = c0 + lane;
    const bool on = c < keys.n;
    const float s = on ? window_dot(q, k + keys.key(c) * ld, d) * g.scale : -INFINITY;
    const float mn = fmaxf(m, wave_max(s)), ref = mn == -INFINITY ? 0.f : mn;
    const float alpha = m == -INFINITY ? 0.f : expf(m - ref), p = on ? expf(s - ref) : 0.f;
    l = (m == -INFINITY ? 0.f : l * alpha) + wave_sum(p);
#pragma unroll
    for (int x = 0; x < WR_COLS; x++) acc[x] = m == -INFINITY ? 0.f : acc[x] * alpha;
    m = mn;
    const int many = min(64, keys.n - c0);
    for (int e = 0; e < many; e++) {
      const float pe = __shfl(p, e, 64);
      const T* row = v + keys.key(c0 + e) * ld;
#pragma unroll
      for (int x = 0; x < WR_COLS; x++)
        if (lane + 64 * x < d) acc[x] = fmaf(pe, to_f32(row[lane + 64 * x]), acc[x]);
    }
  }
#pragma unroll
  for (int x = 0; x < WR_COLS; x++)
    if (lane + 64 * x < d) orow[lane + 64 * x] = from_f32<T>(m == -INFINITY ? NAN : acc[x] / l);
  if (lane == 0) *lrow = m + logf(l);
}
// dq of row i; delta: of the row.
template <typename T>
__device__ __forceinline__ void window_row_dq(const WindowGeom& g, const T* __restrict__ qkv, const T* __restrict__ dorow, float lse, float delta, int h, int i, T* __restrict__ dq) {
  const int lane = threadIdx.x & 63, d = g.d, hk = h / (g.nq / g.nkv);
  const size_t ld = (size_t)(g.nq + 2 * g.nkv) * d;
  const T *q = qkv + i * ld + (size_t)h * d, *k = qkv + (size_t)(g.nq + hk) * d, *v = k + (size_t)g.nkv * d;
  const WindowKeys keys(g, i);
  float acc[WR_COLS] = {};
  for (int c0 = 0; c0 < keys.n; c0 += 64) {
    const int c = c0 + lane;
    float ds = 0.f;
    if (c < keys.n) {
      const size_t at = keys.key(c) * ld;
      ds = expf(window_dot(q, k + at, d) * g.scale - lse) * (window_dot(dorow, v + at, d) - delta);
    }
    const int many = min(64, keys.n - c0);
    for (int e = 0; e < many; e++) {
      const float w = __shfl(ds, e, 64);
      const T* row = k + keys.key(c0 + e) * ld;
#pragma unroll
      for (int x = 0; x < WR_COLS; x++)
        if (lane + 64 * x < d) acc[x] = fmaf(w, to_f32(row[lane + 64 * x]), acc[x]);
    }
  }
#pragma unroll
  for (int x = 0; x < WR_COLS; x++)
    if (lane + 64 * x < d) dq[lane + 64 * x] = from_f32<T>(acc[x] * g.scale);
}
// dk and dv of key j, key/value head hk.  dout, lse, delta: of the sequence's first row (lse, delta: of head 0, `tokens` a head).
template <typename T>
__device__ __forceinline__ void window_row_dkv(const WindowGeom& g, const T* __restrict__ qkv, const T* __restrict__ dout, const float* __restrict__ lse, const float* __restrict__ delta,
                                               size_t tokens, int hk, int j, T* __restrict__ dk, T* __restrict__ dv) {
  const int lane = threadIdx.x & 63, d = g.d, grp = g.nq / g.nkv, end = window_queries_end(g, j);
  const size_t ld = (size_t)(g.nq + 2 * g.nkv) * d, ldo = (size_t)g.nq * d;
  const T *k = qkv + j * ld + (size_t)(g.nq + hk) * d, *v = k + (size_t)g.nkv * d;
  float ak[WR_COLS] = {}, av[WR_COLS] = {};
  for (int h = hk * grp; h < (hk + 1) * grp; h++) {
    const T *q = qkv + (size_t)h * d, *dor = dout + (size_t)h * d;
    for (int i0 = j; i0 < end; i0 += 64) {
      const int i = i0 + lane;
      float p = 0.f, ds = 0.f;
      if (i < end) {
        p = expf(window_dot(k, q + i * ld, d) * g.scale - lse[h * tokens + i]);
        ds = p * (window_dot(v, dor + i * ldo, d) - delta[h * tokens + i]);
      }
      const int many = min(64, end - i0);
      for (int e = 0; e < many; e++) {
        const float pe = __shfl(p, e, 64), we = __shfl(ds, e, 64);
        const T *qr = q + (i0 + e) * ld, *dr = dor + (i0 + e) * ldo;
#pragma unroll
        for (int x = 0; x < WR_COLS; x++)
          if (lane + 64 * x < d) {
            ak[x] = fmaf(we, to_f32(qr[lane + 64 * x]), ak[x]);
            av[x] = fmaf(pe, to_f32(dr[lane + 64 * x]), av[x]);
          }
      }
    }
  }
#pragma unroll
  for (int x = 0; x < WR_COLS; x++)
    if (lane + 64 * x < d) {
      dk[lane + 64 * x] = from_f32<T>(ak[x] * g.scale);
      dv[lane + 64 * x] = from_f32<T>(av[x]);
    }
}
