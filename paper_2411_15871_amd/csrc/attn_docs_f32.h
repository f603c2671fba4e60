// float32 attention over packed documents (part of attn_f32.hip, whose fragments and layouts it uses): a block owns 16 rows (queries, or keys for dK/dV) of one head,
// its waves take the 16-row tiles that any of them meets in turn and meet in LDS at the end, in wave order.  What a row sees is an interval (docs.h); tiles that some row of
// the block does not see whole are summed over what counts alone (accumulate_seen).  Bound by latency, as the kernels for equal sequences: 128 rows of 4 heads of 64, a
// training step, 110 us with a wave a row.
#pragma once
#include "docs.h"

// The interval [at, at + n) of a lane's row (empty: of no document), and the block's: tiles [t0, t1) of 16 rows, every row of a document sees [all0, all1).
struct Docs32 { int at, n, t0, t1, all0, all1; };
__device__ __forceinline__ Docs32 docs32(bool live, int from, int end) {
  const uint32_t rows = (uint32_t)__ballot(live) & 0xffffu;  // the four lane groups hold the same 16 rows
  Docs32 s = {from, live ? end - from : 0, 0, 0, 0, 0};
  if (rows != 0) {
    const int first = __builtin_ctz(rows), last = 31 - __builtin_clz(rows);
    s.t0 = __builtin_amdgcn_readlane(from, first) / 16;
    s.t1 = (__builtin_amdgcn_readlane(end, last) + 15) / 16;
    s.all0 = __builtin_amdgcn_readlane(from, last);
    s.all1 = __builtin_amdgcn_readlane(end, first);
  }
  return s;
}
// ColFrag over rows clamped to [first, last] of the buffer behind base.
template <int DT>
__device__ __forceinline__ void docs32_cols(ColFrag<DT>& c, const float* base, size_t ld, int row0, int first, int last, int l16, int g, int d) {
  const int shift = max(first - row0, 0);  // rows before `first` repeat it: only the first document's first tile has any
  if (shift == 0) {
    c.start(base, ld, row0, last, l16, g, d);
    return;
  }
  c.base = base; c.ld = ld; c.row0 = row0; c.row_last = last; c.l16 = l16; c.g = g; c.d = d;
  if constexpr (ColFrag<DT>::EARLY) {
#pragma unroll
    for (int e = 0; e < 4; e++)
#pragma unroll
      for (int x = 0; x < DT; x++) c.x[x][e] = 16 * x + l16 < d ? base[(size_t)max(first, min(row0 + 4 * g + e, last)) * ld + 16 * x + l16] : 0.f;
  }
}

// Tiles of a launch, 16 rows each: a launch's threads along x are counted in 32 bits (2^23 tiles of 512 threads no longer fit).  A longer micro-batch takes several
// launches, of tiles from tile0 on.
#define A32_TILES (1 << 22)

// grid (16-row tiles, nq)
template <int DT>
__global__ __launch_bounds__(64 * a32_waves<DT>()) void attn_docs_fwd_f32_kernel(const DocsAttn a, int tile0, const float* __restrict__ qkv, float* __restrict__ o, float* __restrict__ lse) {
  constexpr int A32_WAVES = a32_waves<DT>(), LD = DT * 16 + 4;
  __shared__ float ms[A32_WAVES][16], ls[A32_WAVES][16];
  extern __shared__ float os[];  // [16 queries][LD]
  const DocsView& v = a.v;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane & 15, g = lane >> 4, d = a.d, nq = a.nq, nkv = a.nkv, T = v.T;
  const int h = blockIdx.y, hk = h / (nq / nkv), i0 = (tile0 + (int)(gridDim.x - 1 - blockIdx.x)) * 16, iq = i0 + l16, row = min(iq, T - 1), ld = (nq + 2 * nkv) * d;
  if (!docs_fits(v, nq, nkv)) return;
  const int live0 = v.head[DOCS_LIVE0], key_last = v.head[DOCS_LIVE1] - 1;
  const int lo = v.lo[row], hi = v.hi[row], end = max(iq + 1, v.pre[row]);
  RowFrag<DT> q;
  q.load(qkv + (size_t)row * ld + (size_t)h * d, iq < T, g, d);
#pragma unroll
  for (int c = 0; c < DT; c++)
#pragma unroll
    for (int e = 0; e < 4; e++) q.v[c][e] *= a.scale;
  const bool live = iq < T && hi > lo;
  const Docs32 see = docs32(live, lo, end);
  const float* kbase = qkv + (size_t)(nq + hk) * d;
  const float* vbase = kbase + (size_t)nkv * d;
  float m = -INFINITY, l = 0.f;
  f32x4 acc[DT];
#pragma unroll
  for (int c = 0; c < DT; c++) acc[c] = f32x4{0.f, 0.f, 0.f, 0.f};
  auto tile = [&](auto partial, int j0) {  // partial: some keys of the tile are not seen by some of the queries
    RowFrag<DT> k;
    k.load(kbase + (size_t)max(live0, min(j0 + l16, key_last)) * ld, true, g, d);
    ColFrag<DT> vc;
    docs32_cols<DT>(vc, vbase, ld, j0, live0, key_last, l16, g, d);
    f32x4 s = dot_tile<DT>(k, q);  // rows = keys, column = query
    int seen = 0;
#pragma unroll
    for (int e = 0; e < 4; e++) {
      float slope;
      s[e] = docs_capped(s[e], a.cap, slope);
      if (partial) {
        if ((uint32_t)(j0 + 4 * g + e - see.at) < (uint32_t)see.n) seen |= 1 << e;
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
  for (int t = see.t0 + wave; t < see.t1; t += A32_WAVES) {
    with_partial<DT>(t * 16 < see.all0 || t * 16 + 16 > see.all1, [&](auto partial) { tile(partial, t * 16); });
  }
  if (g == 0) { ms[wave][l16] = m; ls[wave][l16] = l; }
  __syncthreads();
  float M = ms[0][l16], L = 0.f;
#pragma unroll
  for (int w = 1; w < A32_WAVES; w++) M = fmaxf(M, ms[w][l16]);
#pragma unroll
  for (int w = 0; w < A32_WAVES; w++) L += ls[w][l16] == 0.f ? 0.f : ls[w][l16] * expf(ms[w][l16] - M);
  // every score the row sees is minus infinity (or a NaN, whose L is one): no softmax, o is a NaN; lse is minus infinity, the logarithm of no weight at all
  const float f = M == -INFINITY ? NAN : l == 0.f ? 0.f : expf(m - M) / L;
  for (int w = 0; w < A32_WAVES; w++) {  // the waves' shares, added in wave order
    if (wave == w) {
#pragma unroll
      for (int c = 0; c < DT; c++) {
        f32x4* dst = reinterpret_cast<f32x4*>(os + l16 * LD + 16 * c + 4 * g);
        const f32x4 x = acc[c] * f;
        *dst = w == 0 ? x : *dst + x;
      }
    }
    __syncthreads();
  }
  const uint32_t rows = (uint32_t)__ballot(live) & 0xffffu;
  for (int x = threadIdx.x; x < 16 * (d / 4); x += blockDim.x) {
    const int r = x / (d / 4), c4 = (x % (d / 4)) * 4;
    if ((rows >> r) & 1) *reinterpret_cast<f32x4*>(o + (size_t)(i0 + r) * nq * d + (size_t)h * d + c4) = *reinterpret_cast<const f32x4*>(os + r * LD + c4);
  }
  if (wave == 0 && g == 0 && live) lse[(size_t)h * T + row] = M + logf(L);
}

struct Docs32Bwd {
  DocsAttn a;
  const float *qkv, *o, *dout, *lse;
  float *dqkv, *delta;
};
// dQ of rows 16 tile .. of head h; also stores their delta.
template <int DT>
__device__ __forceinline__ void docs32_dq(const Docs32Bwd& b, int tile_q, int h, float* os) {
  constexpr int A32_WAVES = a32_waves<DT>(), LD = DT * 16 + 4;
  const DocsAttn& a = b.a;
  const DocsView& v = a.v;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane & 15, g = lane >> 4, d = a.d, nq = a.nq, nkv = a.nkv, T = v.T;
  const int hk = h / (nq / nkv), i0 = tile_q * 16, iq = i0 + l16, row = min(iq, T - 1), ld = (nq + 2 * nkv) * d;
  const int live0 = v.head[DOCS_LIVE0], key_last = v.head[DOCS_LIVE1] - 1;
  const int lo = v.lo[row], hi = v.hi[row], end = max(iq + 1, v.pre[row]);
  const bool live = iq < T && hi > lo;
  const size_t at = ((size_t)row * nq + h) * d;
  RowFrag<DT> q, dof;
  dof.load(b.dout + at, iq < T, g, d);
  const float dl = row_delta<DT>(dof, b.o + at, iq < T, g, d);
  if (wave == 0 && g == 0 && live) b.delta[(size_t)h * T + row] = dl;
  q.load(b.qkv + (size_t)row * ld + (size_t)h * d, iq < T, g, d);
#pragma unroll
  for (int c = 0; c < DT; c++)
#pragma unroll
    for (int e = 0; e < 4; e++) q.v[c][e] *= a.scale;
  const float Lq = b.lse[(size_t)h * T + row];
  const Docs32 see = docs32(live, lo, end);
  const float* kbase = b.qkv + (size_t)(nq + hk) * d;
  const float* vbase = kbase + (size_t)nkv * d;
  f32x4 acc[DT];
#pragma unroll
  for (int c = 0; c < DT; c++) acc[c] = f32x4{0.f, 0.f, 0.f, 0.f};
  auto tile = [&](auto partial, int j0) {
    const size_t krow = (size_t)max(live0, min(j0 + l16, key_last)) * ld;
    RowFrag<DT> k, vv;
    k.load(kbase + krow, true, g, d);
    vv.load(vbase + krow, true, g, d);
    ColFrag<DT> kc;
    docs32_cols<DT>(kc, kbase, ld, j0, live0, key_last, l16, g, d);
    const f32x4 s = dot_tile<DT>(k, q);
    const f32x4 dp = dot_tile<DT>(vv, dof);
    f32x4 ds;
    int seen = 0;
#pragma unroll
    for (int e = 0; e < 4; e++) {
      const bool counts = !partial || (uint32_t)(j0 + 4 * g + e - see.at) < (uint32_t)see.n;
      float slope;
      const float y = docs_capped(s[e], a.cap, slope);
      ds[e] = counts ? expf(y - Lq) * (dp[e] - dl) * slope : 0.f;
      seen |= counts ? 1 << e : 0;
    }
    kc.accumulate_seen(acc, ds, partial, seen);
  };
  for (int t = see.t0 + wave; t < see.t1; t += A32_WAVES) {
    with_partial<DT>(t * 16 < see.all0 || t * 16 + 16 > see.all1, [&](auto partial) { tile(partial, t * 16); });
  }
  for (int w = 0; w < A32_WAVES; w++) {
    if (wave == w) {
#pragma unroll
      for (int c = 0; c < DT; c++) {
        f32x4* dst = reinterpret_cast<f32x4*>(os + l16 * LD + 16 * c + 4 * g);
        *dst = w == 0 ? acc[c] : *dst + acc[c];
      }
    }
    __syncthreads();
  }
  const uint32_t rows = (uint32_t)__ballot(live) & 0xffffu;
  for (int x = threadIdx.x; x < 16 * (d / 4); x += blockDim.x) {
    const int r = x / (d / 4), c4 = (x % (d / 4)) * 4;
    if ((rows >> r) & 1) *reinterpret_cast<f32x4*>(b.dqkv + (size_t)(i0 + r) * ld + (size_t)h * d + c4) = *reinterpret_cast<const f32x4*>(os + r * LD + c4) * a.scale;
  }
}
// dK, dV of keys 16 tile .. of key/value head hk: every (query head of the group, query tile) pair.  OWN_DELTA: delta is formed here, since the dQ tiles may not have stored it yet.
template <int DT, bool OWN_DELTA>
__device__ __forceinline__ void docs32_dkv(const Docs32Bwd& b, int tile_k, int hk, float* os) {  // os: [16 keys][dK | dV], row pitch 2*DT*16 + 4
  constexpr int A32_WAVES = a32_waves<DT>(), LD = 2 * DT * 16 + 4;
  const DocsAttn& a = b.a;
  const DocsView& v = a.v;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane & 15, g = lane >> 4, d = a.d, nq = a.nq, nkv = a.nkv, T = v.T;
  const int grp = nq / nkv, j0 = tile_k * 16, jk = j0 + l16, row_k = min(jk, T - 1), ld = (nq + 2 * nkv) * d;
  const int live0 = v.head[DOCS_LIVE0], q_last = v.head[DOCS_LIVE1] - 1;
  const int lo = v.lo[row_k], end = v.hi[row_k], from = jk < v.pre[row_k] ? lo : jk;
  const bool live = jk < T && end > lo;
  const float* krow = b.qkv + (size_t)row_k * ld + (size_t)(nq + hk) * d;
  RowFrag<DT> k, vv;
  k.load(krow, jk < T, g, d);
  vv.load(krow + (size_t)nkv * d, jk < T, g, d);
#pragma unroll
  for (int c = 0; c < DT; c++)
#pragma unroll
    for (int e = 0; e < 4; e++) k.v[c][e] *= a.scale;
  const Docs32 see = docs32(live, from, end);
  f32x4 dk[DT], dv[DT];
#pragma unroll
  for (int c = 0; c < DT; c++) dk[c] = dv[c] = f32x4{0.f, 0.f, 0.f, 0.f};
  auto tile = [&](auto partial, int h, int i0) {  // partial: some queries of the tile do not see some of the keys
    const size_t row = (size_t)max(live0, min(i0 + l16, q_last));
    const float* qb = b.qkv + (size_t)h * d;
    const float* ob = b.dout + (size_t)h * d;
    RowFrag<DT> q, dof;
    q.load(qb + row * ld, true, g, d);
    dof.load(ob + row * nq * d, true, g, d);
    ColFrag<DT> qc, oc;
    docs32_cols<DT>(oc, ob, (size_t)nq * d, i0, live0, q_last, l16, g, d);
    docs32_cols<DT>(qc, qb, ld, i0, live0, q_last, l16, g, d);
    float own = 0.f;
    if constexpr (OWN_DELTA) own = row_delta<DT>(dof, b.o + row * nq * d + (size_t)h * d, true, g, d);
    const f32x4 s = dot_tile<DT>(q, k);  // rows = queries, column = key
    const f32x4 dp = dot_tile<DT>(dof, vv);
    f32x4 p, ds;
    int seen = 0;
#pragma unroll
    for (int e = 0; e < 4; e++) {
      const int i = i0 + 4 * g + e;
      const size_t st = (size_t)h * T + max(live0, min(i, q_last));
      const bool counts = !partial || (uint32_t)(i - see.at) < (uint32_t)see.n;
      float slope;
      const float y = docs_capped(s[e], a.cap, slope);
      p[e] = counts ? expf(y - b.lse[st]) : 0.f;
      const float dl = OWN_DELTA ? __shfl(own, 4 * g + e, 64) : b.delta[st];  // lane l16 holds row i0 + l16's
      ds[e] = counts ? p[e] * (dp[e] - dl) * slope : 0.f;
      seen |= counts ? 1 << e : 0;
    }
    oc.accumulate_seen(dv, p, partial, seen);
    qc.accumulate_seen(dk, ds, partial, seen);
  };
  const int tiles = see.t1 - see.t0;
  for (int x = wave; x < grp * tiles; x += A32_WAVES) {
    const int h = hk * grp + x / tiles, i0 = (see.t0 + x % tiles) * 16;
    with_partial<DT>(i0 < see.all0 || i0 + 16 > see.all1, [&](auto partial) { tile(partial, h, i0); });
  }
  for (int w = 0; w < A32_WAVES; w++) {
    if (wave == w) {
#pragma unroll
      for (int c = 0; c < DT; c++) {
        f32x4* dst = reinterpret_cast<f32x4*>(os + l16 * LD + 16 * c + 4 * g);
        f32x4* dst2 = reinterpret_cast<f32x4*>(os + l16 * LD + DT * 16 + 16 * c + 4 * g);
        *dst = w == 0 ? dk[c] : *dst + dk[c];
        *dst2 = w == 0 ? dv[c] : *dst2 + dv[c];
      }
    }
    __syncthreads();
  }
  const uint32_t rows = (uint32_t)__ballot(live) & 0xffffu;
  for (int x = threadIdx.x; x < 16 * (d / 4); x += blockDim.x) {
    const int r = x / (d / 4), c4 = (x % (d / 4)) * 4;
    if (!((rows >> r) & 1)) continue;
    float* dst = b.dqkv + (size_t)(j0 + r) * ld + (size_t)(nq + hk) * d + c4;
    *reinterpret_cast<f32x4*>(dst) = *reinterpret_cast<const f32x4*>(os + r * LD + c4) * a.scale;
    *reinterpret_cast<f32x4*>(dst + (size_t)nkv * d) = *reinterpret_cast<const f32x4*>(os + r * LD + DT * 16 + c4);
  }
}
// The two as launches of their own, grids (tiles, nq) and (tiles, nkv), and as one, grid (tiles, nkv + nq); see bwd_f32.
template <int DT>
__global__ __launch_bounds__(64 * a32_waves<DT>()) void attn_docs_dq_f32_kernel(const Docs32Bwd b, int tile0) {
  extern __shared__ float os[];
  if (docs_fits(b.a.v, b.a.nq, b.a.nkv)) docs32_dq<DT>(b, tile0 + (int)gridDim.x - 1 - blockIdx.x, blockIdx.y, os);
}
template <int DT>
__global__ __launch_bounds__(64 * a32_waves<DT>()) void attn_docs_dkv_f32_kernel(const Docs32Bwd b, int tile0) {
  extern __shared__ float os[];
  if (docs_fits(b.a.v, b.a.nq, b.a.nkv)) docs32_dkv<DT, false>(b, tile0 + blockIdx.x, blockIdx.y, os);
}
template <int DT>
__global__ __launch_bounds__(64 * a32_waves<DT>()) void attn_docs_bwd_f32_kernel(const Docs32Bwd b) {
  extern __shared__ float os[];
  if (!docs_fits(b.a.v, b.a.nq, b.a.nkv)) return;
  if ((int)blockIdx.y < b.a.nkv) docs32_dkv<DT, true>(b, blockIdx.x, blockIdx.y, os);
  else docs32_dq<DT>(b, gridDim.x - 1 - blockIdx.x, blockIdx.y - b.a.nkv, os);
}

// ------------------------------------------------------------------------------------ host side
template <int DT>
static int docs_fwd_f32(const DocsAttn& a, const float* qkv, float* o, float* lse, hipStream_t stream) {
  const int tiles = (a.v.T + 15) / 16;
  for (int t = 0; t < tiles; t += A32_TILES) {
    attn_docs_fwd_f32_kernel<DT><<<dim3(std::min(tiles - t, A32_TILES), a.nq), 64 * a32_waves<DT>(), 16 * (DT * 16 + 4) * sizeof(float), stream>>>(a, t, qkv, o, lse);
    DH_LAUNCH_CHECK();
  }
  return DH_OK;
}
int dh_launch_attn_docs_fwd_f32(const DocsAttn& a, const float* qkv, float* o, float* lse, hipStream_t stream) {
  if (a.d <= 32) return docs_fwd_f32<2>(a, qkv, o, lse, stream);
  if (a.d <= 64) return docs_fwd_f32<4>(a, qkv, o, lse, stream);
  if (a.d <= 128) return docs_fwd_f32<8>(a, qkv, o, lse, stream);
  return docs_fwd_f32<16>(a, qkv, o, lse, stream);
}
template <int DT>
static int docs_bwd_f32(const Docs32Bwd& b, hipStream_t stream) {
  const int tiles = (b.a.v.T + 15) / 16, nq = b.a.nq, nkv = b.a.nkv;
  const size_t lds_q = 16 * (DT * 16 + 4) * sizeof(float), lds_k = 16 * (2 * DT * 16 + 4) * sizeof(float);
  if constexpr (DT <= 8) {
    if ((long long)tiles * (nq + nkv) <= A32_ONE_LAUNCH) {
      attn_docs_bwd_f32_kernel<DT><<<dim3(tiles, nkv + nq), 64 * a32_waves<DT>(), lds_k, stream>>>(b);
      DH_LAUNCH_CHECK();
      return DH_OK;
    }
  }
  for (int t = 0; t < tiles; t += A32_TILES) {
    attn_docs_dq_f32_kernel<DT><<<dim3(std::min(tiles - t, A32_TILES), nq), 64 * a32_waves<DT>(), lds_q, stream>>>(b, t);
    DH_LAUNCH_CHECK();
  }
  for (int t = 0; t < tiles; t += A32_TILES) {  // behind all of dQ, which leaves the rows' delta
    attn_docs_dkv_f32_kernel<DT><<<dim3(std::min(tiles - t, A32_TILES), nkv), 64 * a32_waves<DT>(), lds_k, stream>>>(b, t);
    DH_LAUNCH_CHECK();
  }
  return DH_OK;
}
int dh_launch_attn_docs_bwd_f32(const DocsAttn& a, const float* qkv, const float* o, const float* dout, const float* lse, float* dqkv, float* delta, hipStream_t stream) {
  const Docs32Bwd b = {a, qkv, o, dout, lse, dqkv, delta};
  if (a.d <= 32) return docs_bwd_f32<2>(b, stream);
  if (a.d <= 64) return docs_bwd_f32<4>(b, stream);
  if (a.d <= 128) return docs_bwd_f32<8>(b, stream);
  return docs_bwd_f32<16>(b, stream);
}
