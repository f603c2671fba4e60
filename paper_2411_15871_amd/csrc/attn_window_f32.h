// float32 attention with a sliding window and sinks (part of attn_f32.hip, whose fragments and layouts it uses): a block owns 16 rows (queries, or keys for dK/dV) of one head, its waves take the
// 16-row tiles of the sinks and of the window in turn and meet in LDS at the end, in wave order.  Tiles that some row of the block does not see whole are summed over what counts alone
// (accumulate_seen).  Bound by latency, as the other float32 kernels: 2 x 64 tokens of 4 heads of 64, window 16, a training step, 33 us with a wave a row.
#pragma once
#include "window.h"

// The tiles that queries i0 .. i0 + 15 meet: [0, ns) of the sinks, then from w0 to w1.
struct Window32 {
  int ns, w0, w1;
  __device__ __forceinline__ Window32(const WindowGeom& g, int i0) {
    w0 = max(0, i0 - g.window + 1) / 16;
    w1 = (min(i0 + 16, g.seq) + 15) / 16;
    ns = min((g.sinks + 15) / 16, w0);
  }
  __device__ __forceinline__ int count() const { return ns + w1 - w0; }
  __device__ __forceinline__ int first(int x) const { return (x < ns ? x : w0 + x - ns) * 16; }  // key of the x-th tile
};
__device__ __forceinline__ bool window32_partial(const WindowGeom& g, int i0, int j0) { return j0 + 15 > i0 || (j0 < i0 + 16 - g.window && j0 + 16 > g.sinks); }
__device__ __forceinline__ bool window32_counts(const WindowGeom& g, int i, int j) { return (uint32_t)(j - (i - g.window + 1)) < (uint32_t)g.window || j < min(g.sinks, i + 1); }

// grid (16-row tiles, nq, batch)
template <int DT>
__global__ __launch_bounds__(64 * a32_waves<DT>()) void attn_window_fwd_f32_kernel(const WindowGeom w, const float* __restrict__ qkv, float* __restrict__ o, float* __restrict__ lse) {
  constexpr int A32_WAVES = a32_waves<DT>(), LD = DT * 16 + 4;
  __shared__ float ms[A32_WAVES][16], ls[A32_WAVES][16];
  extern __shared__ float os[];  // [16 queries][LD]
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane & 15, g = lane >> 4, d = w.d, nq = w.nq, nkv = w.nkv, seq = w.seq;
  const int h = blockIdx.y, hk = h / (nq / nkv), i0 = (gridDim.x - 1 - blockIdx.x) * 16, iq = i0 + l16, ld = (nq + 2 * nkv) * d;
  const size_t t0 = (size_t)blockIdx.z * seq;
  const float* rows = qkv + t0 * ld;
  RowFrag<DT> q;
  q.load(rows + (size_t)min(iq, seq - 1) * ld + (size_t)h * d, iq < seq, g, d);
#pragma unroll
  for (int c = 0; c < DT; c++)
#pragma unroll
    for (int e = 0; e < 4; e++) q.v[c][e] *= w.scale;
  const Window32 tiles(w, i0);
  const float* kbase = rows + (size_t)(nq + hk) * d;
  const float* vbase = kbase + (size_t)nkv * d;
  float m = -INFINITY, l = 0.f;
  f32x4 acc[DT];
#pragma unroll
  for (int c = 0; c < DT; c++) acc[c] = f32x4{0.f, 0.f, 0.f, 0.f};
  auto tile = [&](auto partial, int j0) {
    RowFrag<DT> k;
    k.load(kbase + (size_t)min(j0 + l16, seq - 1) * ld, true, g, d);
    ColFrag<DT> vc;
    vc.start(vbase, ld, j0, seq - 1, l16, g, d);
    f32x4 s = dot_tile<DT>(k, q);  // rows = keys, column = query
    int seen = 0;
    if (partial) {
#pragma unroll
      for (int e = 0; e < 4; e++) {
        if (window32_counts(w, iq, j0 + 4 * g + e)) seen |= 1 << e;
        else s[e] = -INFINITY;
      }
    }
    const float mn = fmaxf(m, group_max(fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]))));
    if (__any(mn > m)) {
      const float alpha = mn == -INFINITY ? 1.f : expf(m - mn);  // a row may see no key of the tile
      l *= alpha;
#pragma unroll
      for (int c = 0; c < DT; c++) acc[c] *= alpha;
      m = mn;
    }
    f32x4 p;
#pragma unroll
    for (int e = 0; e < 4; e++) p[e] = s[e] == -INFINITY ? 0.f : expf(s[e] - m);
    l += group_sum(p[0] + p[1] + p[2] + p[3]);
    vc.accumulate_seen(acc, p, partial, seen);
  };
  for (int t = wave; t < tiles.count(); t += A32_WAVES) with_partial<DT>(window32_partial(w, i0, tiles.first(t)), [&](auto partial) { tile(partial, tiles.first(t)); });
  if (g == 0) { ms[wave][l16] = m; ls[wave][l16] = l; }
  __syncthreads();
  float M = ms[0][l16], L = 0.f;
#pragma unroll
  for (int x = 1; x < A32_WAVES; x++) M = fmaxf(M, ms[x][l16]);
#pragma unroll
  for (int x = 0; x < A32_WAVES; x++) L += ls[x][l16] == 0.f ? 0.f : ls[x][l16] * expf(ms[x][l16] - M);
  // every score the row sees is minus infinity (or a NaN, whose L is one): no softmax, o is a NaN; lse is minus infinity, the logarithm of no weight at all
  const float f = M == -INFINITY ? NAN : l == 0.f ? 0.f : expf(m - M) / L;
  for (int x = 0; x < A32_WAVES; x++) {  // the waves' shares, added in wave order
    if (wave == x) {
#pragma unroll
      for (int c = 0; c < DT; c++) {
        f32x4* dst = reinterpret_cast<f32x4*>(os + l16 * LD + 16 * c + 4 * g);
        const f32x4 y = acc[c] * f;
        *dst = x == 0 ? y : *dst + y;
      }
    }
    __syncthreads();
  }
  for (int x = threadIdx.x; x < 16 * (d / 4); x += blockDim.x) {
    const int r = x / (d / 4), c4 = (x % (d / 4)) * 4;
    if (i0 + r < seq) *reinterpret_cast<f32x4*>(o + (t0 + i0 + r) * nq * d + (size_t)h * d + c4) = *reinterpret_cast<const f32x4*>(os + r * LD + c4);
  }
  if (wave == 0 && g == 0 && iq < seq) lse[(size_t)h * w.batch * seq + t0 + iq] = M + logf(L);
}

struct Window32Bwd {
  WindowGeom w;
  const float *qkv, *o, *dout, *lse;
  float *dqkv, *delta;
};
// dQ of rows i0 .. i0 + 15 of head h, sequence b; also stores their delta.
template <int DT>
__device__ __forceinline__ void window32_dq(const Window32Bwd& a, int i0, int h, int b, float* os) {
  constexpr int A32_WAVES = a32_waves<DT>(), LD = DT * 16 + 4;
  const WindowGeom& w = a.w;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane & 15, g = lane >> 4, d = w.d, nq = w.nq, nkv = w.nkv, seq = w.seq;
  const int hk = h / (nq / nkv), iq = i0 + l16, row = min(iq, seq - 1), ld = (nq + 2 * nkv) * d;
  const size_t t0 = (size_t)b * seq, head = (size_t)h * w.batch * seq + t0, at = ((t0 + row) * nq + h) * d;
  const float* rows = a.qkv + t0 * ld;
  RowFrag<DT> q, dof;
  dof.load(a.dout + at, iq < seq, g, d);
  const float dl = row_delta<DT>(dof, a.o + at, iq < seq, g, d);
  if (wave == 0 && g == 0 && iq < seq) a.delta[head + iq] = dl;
  q.load(rows + (size_t)row * ld + (size_t)h * d, iq < seq, g, d);
#pragma unroll
  for (int c = 0; c < DT; c++)
#pragma unroll
    for (int e = 0; e < 4; e++) q.v[c][e] *= w.scale;
  const float Lq = a.lse[head + row];
  const Window32 tiles(w, i0);
  const float* kbase = rows + (size_t)(nq + hk) * d;
  const float* vbase = kbase + (size_t)nkv * d;
  f32x4 acc[DT];
#pragma unroll
  for (int c = 0; c < DT; c++) acc[c] = f32x4{0.f, 0.f, 0.f, 0.f};
  auto tile = [&](auto partial, int j0) {
    const size_t krow = (size_t)min(j0 + l16, seq - 1) * ld;
    RowFrag<DT> k, vv;
    k.load(kbase + krow, true, g, d);
    vv.load(vbase + krow, true, g, d);
    ColFrag<DT> kc;
    kc.start(kbase, ld, j0, seq - 1, l16, g, d);
    const f32x4 s = dot_tile<DT>(k, q);
    const f32x4 dp = dot_tile<DT>(vv, dof);
    f32x4 ds;
    int seen = 0;
#pragma unroll
    for (int e = 0; e < 4; e++) {
      const bool counts = !partial || window32_counts(w, iq, j0 + 4 * g + e);
      ds[e] = counts ? expf(s[e] - Lq) * (dp[e] - dl) : 0.f;
      seen |= counts ? 1 << e : 0;
    }
    kc.accumulate_seen(acc, ds, partial, seen);
  };
  for (int t = wave; t < tiles.count(); t += A32_WAVES) with_partial<DT>(window32_partial(w, i0, tiles.first(t)), [&](auto partial) { tile(partial, tiles.first(t)); });
  for (int x = 0; x < A32_WAVES; x++) {
    if (wave == x) {
#pragma unroll
      for (int c = 0; c < DT; c++) {
        f32x4* dst = reinterpret_cast<f32x4*>(os + l16 * LD + 16 * c + 4 * g);
        *dst = x == 0 ? acc[c] : *dst + acc[c];
      }
    }
    __syncthreads();
  }
  for (int x = threadIdx.x; x < 16 * (d / 4); x += blockDim.x) {
    const int r = x / (d / 4), c4 = (x % (d / 4)) * 4;
    if (i0 + r < seq) *reinterpret_cast<f32x4*>(a.dqkv + (t0 + i0 + r) * ld + (size_t)h * d + c4) = *reinterpret_cast<const f32x4*>(os + r * LD + c4) * w.scale;
  }
}
// dK, dV of keys j0 .. j0 + 15 of key/value head hk: every (query head of the group, query tile) pair.  OWN_DELTA: delta is formed here, since the dQ tiles may not have stored it yet.
template <int DT, bool OWN_DELTA>
__device__ __forceinline__ void window32_dkv(const Window32Bwd& a, int j0, int hk, int b, float* os) {  // os: [16 keys][dK | dV], row pitch 2*DT*16 + 4
  constexpr int A32_WAVES = a32_waves<DT>(), LD = 2 * DT * 16 + 4;
  const WindowGeom& w = a.w;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane & 15, g = lane >> 4, d = w.d, nq = w.nq, nkv = w.nkv, seq = w.seq;
  const int grp = nq / nkv, jk = j0 + l16, ld = (nq + 2 * nkv) * d;
  const size_t t0 = (size_t)b * seq, T = (size_t)w.batch * seq;
  const float* rows = a.qkv + t0 * ld;
  const float* krow = rows + (size_t)min(jk, seq - 1) * ld + (size_t)(nq + hk) * d;
  RowFrag<DT> k, vv;
  k.load(krow, jk < seq, g, d);
  vv.load(krow + (size_t)nkv * d, jk < seq, g, d);
#pragma unroll
  for (int c = 0; c < DT; c++)
#pragma unroll
    for (int e = 0; e < 4; e++) k.v[c][e] *= w.scale;
  const int n = max(0, window_queries_end(w, jk) - jk), plain = max(j0, w.sinks);  // plain: the first key that is no sink, whose window ends first
  const int all1 = plain < j0 + 16 ? window_queries_end(w, plain) : seq, tile0 = j0 / 16, tiles = (window_queries_end(w, j0 < w.sinks ? j0 : j0 + 15) + 15) / 16 - tile0;
  f32x4 dk[DT], dv[DT];
#pragma unroll
  for (int c = 0; c < DT; c++) dk[c] = dv[c] = f32x4{0.f, 0.f, 0.f, 0.f};
  auto tile = [&](auto partial, int h, int i0) {  // partial: some queries of the tile do not see some of the keys
    const size_t row = t0 + min(i0 + l16, seq - 1);
    const float* qb = rows + (size_t)h * d;
    const float* ob = a.dout + t0 * nq * d + (size_t)h * d;
    RowFrag<DT> q, dof;
    q.load(a.qkv + row * ld + (size_t)h * d, true, g, d);
    dof.load(a.dout + (row * nq + h) * d, true, g, d);
    ColFrag<DT> qc, oc;
    oc.start(ob, (size_t)nq * d, i0, seq - 1, l16, g, d);
    qc.start(qb, ld, i0, seq - 1, l16, g, d);
    float own = 0.f;
    if constexpr (OWN_DELTA) own = row_delta<DT>(dof, a.o + (row * nq + h) * d, true, g, d);
    const f32x4 s = dot_tile<DT>(q, k);  // rows = queries, column = key
    const f32x4 dp = dot_tile<DT>(dof, vv);
    f32x4 p, ds;
    int seen = 0;
#pragma unroll
    for (int e = 0; e < 4; e++) {
      const int i = i0 + 4 * g + e;
      const size_t st = (size_t)h * T + t0 + min(i, seq - 1);
      const bool counts = !partial || (uint32_t)(i - jk) < (uint32_t)n;
      p[e] = counts ? expf(s[e] - a.lse[st]) : 0.f;
      const float dl = OWN_DELTA ? __shfl(own, 4 * g + e, 64) : a.delta[st];  // lane l16 holds row i0 + l16's
      ds[e] = counts ? p[e] * (dp[e] - dl) : 0.f;
      seen |= counts ? 1 << e : 0;
    }
    oc.accumulate_seen(dv, p, partial, seen);
    qc.accumulate_seen(dk, ds, partial, seen);
  };
  for (int x = wave; x < grp * tiles; x += A32_WAVES) {
    const int h = hk * grp + x / tiles, i0 = (tile0 + x % tiles) * 16;
    with_partial<DT>(i0 < j0 + 15 || i0 + 16 > all1, [&](auto partial) { tile(partial, h, i0); });
  }
  for (int x = 0; x < A32_WAVES; x++) {
    if (wave == x) {
#pragma unroll
      for (int c = 0; c < DT; c++) {
        f32x4* dst = reinterpret_cast<f32x4*>(os + l16 * LD + 16 * c + 4 * g);
        f32x4* dst2 = reinterpret_cast<f32x4*>(os + l16 * LD + DT * 16 + 16 * c + 4 * g);
        *dst = x == 0 ? dk[c] : *dst + dk[c];
        *dst2 = x == 0 ? dv[c] : *dst2 + dv[c];
      }
    }
    __syncthreads();
  }
  for (int x = threadIdx.x; x < 16 * (d / 4); x += blockDim.x) {
    const int r = x / (d / 4), c4 = (x % (d / 4)) * 4;
    if (j0 + r >= seq) continue;
    float* dst = a.dqkv + (t0 + j0 + r) * ld + (size_t)(nq + hk) * d + c4;
    *reinterpret_cast<f32x4*>(dst) = *reinterpret_cast<const f32x4*>(os + r * LD + c4) * w.scale;  // (k took the scale for its scores)
    *reinterpret_cast<f32x4*>(dst + (size_t)nkv * d) = *reinterpret_cast<const f32x4*>(os + r * LD + DT * 16 + c4);
  }
}
// The two as launches of their own, grids (tiles, nq, batch) and (tiles, nkv, batch), and as one, grid (tiles, nkv + nq, batch); see bwd_f32.
template <int DT>
__global__ __launch_bounds__(64 * a32_waves<DT>()) void attn_window_dq_f32_kernel(const Window32Bwd a) {
  extern __shared__ float os[];
  window32_dq<DT>(a, (gridDim.x - 1 - blockIdx.x) * 16, blockIdx.y, blockIdx.z, os);
}
template <int DT>
__global__ __launch_bounds__(64 * a32_waves<DT>()) void attn_window_dkv_f32_kernel(const Window32Bwd a) {
  extern __shared__ float os[];
  window32_dkv<DT, false>(a, blockIdx.x * 16, blockIdx.y, blockIdx.z, os);
}
template <int DT>
__global__ __launch_bounds__(64 * a32_waves<DT>()) void attn_window_bwd_f32_kernel(const Window32Bwd a) {
  extern __shared__ float os[];
  if ((int)blockIdx.y < a.w.nkv) window32_dkv<DT, true>(a, blockIdx.x * 16, blockIdx.y, blockIdx.z, os);
  else window32_dq<DT>(a, (gridDim.x - 1 - blockIdx.x) * 16, blockIdx.y - a.w.nkv, blockIdx.z, os);
}

// ------------------------------------------------------------------------------------ host side
static WindowGeom window32_geom(WindowGeom g) {
  g.window = std::min(g.window, g.seq);
  g.sinks = std::min(g.sinks, g.seq);
  return g;
}
template <int DT>
static int window_fwd_f32(const WindowGeom& g, const float* qkv, float* o, float* lse, hipStream_t stream) {
  attn_window_fwd_f32_kernel<DT><<<dim3((g.seq + 15) / 16, g.nq, g.batch), 64 * a32_waves<DT>(), 16 * (DT * 16 + 4) * sizeof(float), stream>>>(g, qkv, o, lse);
  DH_LAUNCH_CHECK();
  return DH_OK;
}
int dh_launch_window_fwd_f32(const WindowGeom& g0, const float* qkv, float* o, float* lse, hipStream_t stream) {
  const WindowGeom g = window32_geom(g0);
  if (g.d <= 32) return window_fwd_f32<2>(g, qkv, o, lse, stream);
  if (g.d <= 64) return window_fwd_f32<4>(g, qkv, o, lse, stream);
  return window_fwd_f32<8>(g, qkv, o, lse, stream);
}
template <int DT>
static int window_bwd_f32(const Window32Bwd& a, hipStream_t stream) {
  const int tiles = (a.w.seq + 15) / 16, nq = a.w.nq, nkv = a.w.nkv, batch = a.w.batch;
  const size_t lds_q = 16 * (DT * 16 + 4) * sizeof(float), lds_k = 16 * (2 * DT * 16 + 4) * sizeof(float);
  if ((long long)tiles * (nq + nkv) * batch <= A32_ONE_LAUNCH) {
    attn_window_bwd_f32_kernel<DT><<<dim3(tiles, nkv + nq, batch), 64 * a32_waves<DT>(), lds_k, stream>>>(a);
    DH_LAUNCH_CHECK();
    return DH_OK;
  }
  attn_window_dq_f32_kernel<DT><<<dim3(tiles, nq, batch), 64 * a32_waves<DT>(), lds_q, stream>>>(a);
  DH_LAUNCH_CHECK();
  attn_window_dkv_f32_kernel<DT><<<dim3(tiles, nkv, batch), 64 * a32_waves<DT>(), lds_k, stream>>>(a);
  DH_LAUNCH_CHECK();
  return DH_OK;
}
int dh_launch_window_bwd_f32(const WindowGeom& g, const float* qkv, const float* o, const float* dout, const float* lse, float* dqkv, float* delta, hipStream_t stream) {
  const Window32Bwd a = {window32_geom(g), qkv, o, dout, lse, dqkv, delta};
  if (g.d <= 32) return window_bwd_f32<2>(a, stream);
  if (g.d <= 64) return window_bwd_f32<4>(a, stream);
  return window_bwd_f32<8>(a, stream);
}
