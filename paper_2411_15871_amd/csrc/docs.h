// Packed documents: what dh_docs_plan leaves in a micro-batch's table, and attention one row at a time.
#pragma once
#include "common.h"

// The table: a head of DOCS_HEAD ints, then three ints a row (arrays lo, hi, pre of T): the row's document is rows lo .. hi-1 and its prefix ends before row
// `pre`.  Rows of no document have lo = hi = pre = their own index.  So row r sees keys lo[r] .. max(r + 1, pre[r]) - 1, and key j is seen by
// rows (j < pre[j] ? lo[j] : j) .. hi[j] - 1.  All four borders ascend with the row.
#define DOCS_HEAD 16
enum { DOCS_LIVE0 = 0, DOCS_LIVE1 = 1 };  // head: the rows of documents are [live0, live1)
struct DocsView {
  int T;
  const int32_t *head, *lo, *hi, *pre;
};
static inline DocsView docs_view(const dh_docs* docs) {
  const int32_t* t = (const int32_t*)docs->table;
  return {docs->T, t, t + DOCS_HEAD, t + DOCS_HEAD + (size_t)docs->T, t + DOCS_HEAD + 2 * (size_t)docs->T};
}

// A scaled score under the cap, and the cap's slope there.
__device__ __forceinline__ float docs_capped(float x, float cap, float& slope) {
  if (cap <= 0.f) { slope = 1.f; return x; }
  const float t = tanhf(x / cap);
  slope = 1.f - t * t;
  return cap * t;
}
// Dot product of d elements (a multiple of 8); a is read at wave-uniform addresses.
template <typename T>
__device__ __forceinline__ float docs_dot(const T* a, const T* b, int d) {
  float s = 0.f;
  for (int c = 0; c < d; c += 8) {
    Vec8<T> x, y;
    x.load(a + c);
    y.load(b + c);
#pragma unroll
    for (int i = 0; i < 8; i++) s = fmaf(x.v[i], y.v[i], s);
  }
  return s;
}
// acc[c] += sum over the wave's lanes i of w(lane i) * row(i)[lane + 64 c], over the lanes whose bit in `which` is set: what is not asked for is not touched, so
// that an infinity or a NaN there stays there.
template <typename T>
__device__ __forceinline__ void docs_add_rows(float (&acc)[4], float w, unsigned long long which, const T* rows, size_t ld, int d) {
  const int lane = threadIdx.x & 63;
  while (which) {
    const int i = __builtin_ctzll(which);
    which &= which - 1;
    const float wi = __shfl(w, i, 64);
    const T* r = rows + i * ld;
#pragma unroll
    for (int c = 0; c < 4; c++)
      if (lane + 64 * c < d) acc[c] = fmaf(wi, to_f32(r[lane + 64 * c]), acc[c]);
  }
}

// Attention of one row by one wave, a lane per key of 64: plain sums over exactly the keys the row sees.  Forward over keys [j0, j1): unnormalised output
// (lane's columns lane + 64 c), running maximum and sum (natural units).
template <typename T>
__device__ __forceinline__ void docs_row_fwd(const T* q, const T* k, const T* v, size_t ld, int j0, int j1, int d, float scale, float cap, float (&acc)[4], float& m, float& l) {
  const int lane = threadIdx.x & 63;
  for (int j = j0; j < j1; j += 64) {
    const bool on = j + lane < j1;
    float slope, y = on ? docs_capped(docs_dot(q, k + (size_t)(j + lane) * ld, d) * scale, cap, slope) : -INFINITY;
    const float mn = fmaxf(m, wave_max(y));
    const float a = mn == -INFINITY ? 1.f : expf(m - mn), p = on ? (mn == -INFINITY ? y - mn : expf(y - mn)) : 0.f;  // all scores minus infinity: no softmax
    l = l * a + wave_sum(p);
#pragma unroll
    for (int c = 0; c < 4; c++) acc[c] *= a;
    docs_add_rows(acc, p, __ballot(on), v + (size_t)j * ld, ld, d);
    m = mn;
  }
}
// dQ of one row over keys [j0, j1), unscaled; dout: its gradient, lse and delta its statistics.
template <typename T>
__device__ __forceinline__ void docs_row_dq(const T* q, const T* dout, const T* k, const T* v, size_t ld, int j0, int j1, int d, float scale, float cap, float lse, float delta,
                                            float (&acc)[4]) {
  const int lane = threadIdx.x & 63;
  for (int j = j0; j < j1; j += 64) {
    const bool on = j + lane < j1;
    float ds = 0.f;
    if (on) {
      float slope;
      const float y = docs_capped(docs_dot(q, k + (size_t)(j + lane) * ld, d) * scale, cap, slope);
      ds = expf(y - lse) * (docs_dot(dout, v + (size_t)(j + lane) * ld, d) - delta) * slope;
    }
    docs_add_rows(acc, ds, __ballot(on), k + (size_t)j * ld, ld, d);
  }
}
// dK (unscaled) and dV of one key over rows [i0, i1) of one head; q, dout, lse, delta: of row 0.
template <typename T>
__device__ __forceinline__ void docs_row_dkv(const T* k, const T* v, const T* q, size_t ld, const T* dout, size_t ldo, const float* lse, const float* delta, int i0, int i1, int d,
                                             float scale, float cap, float (&dk)[4], float (&dv)[4]) {
  const int lane = threadIdx.x & 63;
  for (int i = i0; i < i1; i += 64) {
    const bool on = i + lane < i1;
    float p = 0.f, ds = 0.f;
    if (on) {
      float slope;
      const float y = docs_capped(docs_dot(k, q + (size_t)(i + lane) * ld, d) * scale, cap, slope);
      p = expf(y - lse[i + lane]);
      ds = p * (docs_dot(v, dout + (size_t)(i + lane) * ldo, d) - delta[i + lane]) * slope;
    }
    docs_add_rows(dv, p, __ballot(on), dout + (size_t)i * ldo, ldo, d);
    docs_add_rows(dk, ds, __ballot(on), q + (size_t)i * ld, ld, d);
  }
}
