// bf16 attention with a sliding window and sinks on the matrix cores, forward and backward (part of attn_bf16.hip, whose tiles, fragments and layouts it uses).
//
// A block of 128 queries walks the 64-key tiles of the sinks that lie before its window, then those of its window up to the diagonal: about (window + 128 + sinks) / 64 tiles whatever the
// row's length.  Which keys of a tile a row sees is two comparisons an element (one behind the sinks), made only where some row of the wave does not see the whole tile.  A block of 128 keys
// walks, head after head of its group, the query tiles from its own position to the window's end; blocks that hold sinks walk on to the row's end.  Where blocks are few, or rounds of them would leave
// the chip idle, their walks are cut into units whose partial results a launch behind adds in order (4096 rows of 4:1 heads, window 1024, backward pass 121 -> 75 us).
//
// Probabilities and their gradients round to bf16 before the products that take them, as the causal kernels' do: matrix instructions of the full rate take nothing else.
//
// Masked probabilities are zeros, and a zero times an infinity or a NaN of a row that is not seen is a NaN: a wave whose result is not finite looks, as the kernels of packed documents do, whether
// its masked tiles hold such values that a row does not see, and only then walks its tiles again (window_again_*).  8192 rows of 32:8 heads, window
// 1024, us: forward 170 -> 260 with one token of NaNs, 150 with nothing else; backward 600 -> 1930 (one token), 1860 (a gradient's row), 1940 (nothing else).
//
// Bound by matrix products (4 D flops a visible pair forward, 10 of the backward pass, which do 14 here: dQ and dK/dV each form S and dP for themselves) from windows of some hundred on, below that
// by what a block begins and ends with.
#pragma once
#include "window.h"

#define WB_BLOCK 128
#define WB_Y 32768  // blocks of a row along the launch's y, further ones along z
struct WindowTiled {
  WindowGeom g;   // window and sinks at most seq
  int blocks;     // of 128 rows, a sequence
  int parts;      // forward: units that share a block's tiles
  // dK/dV: a key block's walk is cut into units of `chunk` tiles, blocks that hold sinks (they walk on to the row's end) into others.  One unit: the block writes its results itself.
  int plain_units, plain_chunk, sink_blocks, sink_units, sink_chunk;
  float exp_scale;  // score -> exponent of 2
};
__host__ __device__ static inline int window_units(const WindowTiled& p) { return (p.blocks - p.sink_blocks) * p.plain_units + p.sink_blocks * p.sink_units; }  // of dK/dV, a head
// Partial results of a head's dK/dV: [units of the blocks without sinks, if these are cut][units of the others, if these are].
__host__ __device__ static inline int window_parts(const WindowTiled& p) {
  return (p.plain_units > 1 ? (p.blocks - p.sink_blocks) * p.plain_units : 0) + (p.sink_units > 1 ? p.sink_blocks * p.sink_units : 0);
}
struct WindowKeys128 { int jb, chunk, f0, f1, q0, nt, part; };  // a unit: key block, its run of tiles [f0, f1), counted through the heads of the group, nt of each head from row q0 on; partial result or -1
__host__ __device__ static inline int window_key_tiles(const WindowTiled& p, int jb) {  // of one head
  const int j0 = jb * WB_BLOCK, q0 = j0 / AB_KT * AB_KT;
  const long long end = jb < p.sink_blocks ? p.g.seq : (long long)j0 + WB_BLOCK - 1 + p.g.window;
  return (int)(((end < p.g.seq ? end : p.g.seq) - q0 + AB_KT - 1) / AB_KT);
}
__device__ __forceinline__ WindowKeys128 window_keys128(const WindowTiled& p, int unit, int grp) {
  const int plain = (p.blocks - p.sink_blocks) * p.plain_units;
  const bool sink = unit >= plain;
  const int id = sink ? unit - plain : unit, units = sink ? p.sink_units : p.plain_units, ch = sink ? p.sink_chunk : p.plain_chunk;
  WindowKeys128 k;
  k.jb = id / units + (sink ? 0 : p.sink_blocks);
  k.chunk = id % units;
  k.q0 = k.jb * WB_BLOCK / AB_KT * AB_KT;
  k.nt = window_key_tiles(p, k.jb);
  k.f0 = min(k.chunk * ch, grp * k.nt);
  k.f1 = min(k.f0 + ch, grp * k.nt);
  k.part = units == 1 ? -1 : id + (sink && p.plain_units > 1 ? plain : 0);
  return k;
}
// Heads of a group next to one another on the same XCD (workgroups go to the eight in turn), whose L2 then holds their keys and values once.
__device__ __forceinline__ int window_head(int x, int n) { return n % 8 == 0 ? (x & 7) * (n >> 3) + (x >> 3) : x; }
struct WindowUnit { int id, b; };
__device__ __forceinline__ WindowUnit window_unit(int batch) { return {(int)(blockIdx.z / batch) * WB_Y + (int)blockIdx.y, (int)(blockIdx.z % batch)}; }
static dim3 window_grid(int heads, int units, int batch) { return dim3(heads, std::min(units, WB_Y), (unsigned)(((long long)units + WB_Y - 1) / WB_Y) * batch); }

// Key tiles of query block ib: [0, ns) of the sinks, then from w0 to w1.
struct WindowTiles {
  int ns, w0, w1;
  __host__ __device__ WindowTiles(const WindowGeom& g, int ib) {
    const int lo = ib * WB_BLOCK - g.window + 1;
    w0 = lo > 0 ? lo / AB_KT : 0;
    const int end = g.seq - ib * WB_BLOCK < WB_BLOCK ? g.seq : (ib + 1) * WB_BLOCK, s = (g.sinks + AB_KT - 1) / AB_KT;
    w1 = (end + AB_KT - 1) / AB_KT;
    ns = s < w0 ? s : w0;
  }
  __host__ __device__ int count() const { return ns + w1 - w0; }
  __device__ int tile(int f) const { return f < ns ? f : w0 + f - ns; }
};
// What the 32 rows from iw on see of the tile of keys from kb on.
struct WindowSeen {
  int iw, iq, window, sinks;
  __device__ __forceinline__ bool none(int kb) const { return kb > iw + 31 || (kb + AB_KT <= iw - window + 1 && kb >= sinks); }
  __device__ __forceinline__ bool part(int kb) const { return kb + AB_KT - 1 > iw || (kb < iw + 31 - window + 1 && kb + AB_KT > sinks); }
  // f(mt, r, seen) for every element of the lane's column
  template <class F>
  __device__ __forceinline__ void each(int kb, int kg, F f) const {
    const int at = kb + 4 * kg - (iq - window + 1), ahead = min(sinks, iq + 1) - kb - 4 * kg;  // (a copy of its own for tiles behind the sinks costs dQ the 25 registers it has not)
#pragma unroll
    for (int mt = 0; mt < 2; mt++)
#pragma unroll
      for (int r = 0; r < 16; r++) {
        const int e = mt * 32 + 8 * (r >> 2) + (r & 3);
        f(mt, r, (uint32_t)(at + e) < (uint32_t)window || e < ahead);
        if ((r & 3) == 3) __builtin_amdgcn_sched_barrier(0);  // (32 comparisons ahead of their use take more scalar registers than there are)
      }
  }
};

// ---- Results that are not finite: attn_docs_bf16.h's steps, where what a row sees is two intervals, the sinks before its window and the window.
// The lane's interval and the wave's, as docs_seen; rows behind the sequence's end are copies of its last one.
__device__ __forceinline__ DocsSeen window_interval(const WindowGeom& g, int iw, bool window) {
  const int last = min(iw + 31, g.seq - 1), i = min(iw + (docs_lane() & 31), last);
  auto lo = [&](int row) { return max(0, row - g.window + 1); };
  if (window) return {lo(i), i + 1 - lo(i), lo(iw), last + 1, lo(last), iw + 1};
  return {0, min(g.sinks, lo(i)), 0, min(g.sinks, lo(last)), 0, min(g.sinks, lo(iw))};
}
// f(first row, interval) for tiles [f0, f1) of a query block, for each of the two intervals that some row of the wave has there.
template <class F>
__device__ __forceinline__ void window_again_tiles(const WindowGeom& g, const WindowTiles& tiles, int iw, int f0, int f1, F f) {
#pragma unroll 1
  for (int x = 2 * f0; x < 2 * f1; x++) {
    const int kb = tiles.tile(x >> 1) * AB_KT;
    const DocsSeen see = window_interval(g, iw, x & 1);
    if (kb < see.any1 && kb + AB_KT > see.any0) f(kb, see);
  }
}
// f(first row, the lane's seen rows) for those of them that some row of the wave does not see whole.
template <class F>
__device__ __forceinline__ void window_masked_tiles(const WindowGeom& g, const WindowTiles& tiles, int iw, int f0, int f1, F f) {
  const WindowSeen see = {iw, 0, g.window, g.sinks};
#pragma unroll 1
  for (int x = f0; x < f1; x++) {
    const int kb = tiles.tile(x) * AB_KT;
    if (!see.none(kb) && see.part(kb)) f(kb, docs_bits(window_interval(g, iw, false), kb) | docs_bits(window_interval(g, iw, true), kb));
  }
}

// ================================================================================ forward
// The rows `bad` of a wave again, as docs_again_fwd.  q, o, lse: of the wave's first row; part_o, part_ml: likewise, of a part, or nullptr.
template <int D>
__device__ __forceinline__ void window_again_fwd(const WindowTiled& p, const WindowTiles& tiles, int iw, int f0, int f1, bool bad, const DocsRows& k, const DocsRows& v, const bf16_t* q, bf16_t* o,
                                                 float* lse, float* part_o, float* part_ml, char* tile) {
  const WindowGeom& g = p.g;
  bool arrives = false, none = false;
  window_masked_tiles(g, tiles, iw, f0, f1, [&](int kb, uint64_t seen) {
    const DocsOdd odd = docs_odd<D>(v, kb, DOCS_ODD);
    arrives |= (odd.some & ~seen) != 0;
    none |= (odd.all & seen) != 0;
  });
  const uint64_t rows = __ballot(bad && arrives && !none);
  if (rows == 0) return;
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the first results of these rows, which other lanes have stored, are in place
  const int lane = docs_lane(), r = lane & 31;
  DocsTiled softmax = {};
  softmax.exp_scale = p.exp_scale;
  float m = -3.0e38f, l = 0.f;
  f32x16 ot[D / 32];
#pragma unroll
  for (int dt = 0; dt < D / 32; dt++) acc_zero<false>(ot[dt]);
  window_again_tiles(g, tiles, iw, f0, f1, [&](int kb, const DocsSeen& see) {
    f32x16 st[2];
    docs_again_scores<D>(st, tile, k, kb, q + (size_t)min(r, g.seq - 1 - iw) * k.ld, true);
    docs_softmax<D, false, true>(softmax, see, kb, lane >> 5, st, ot, m, l);
    docs_again_add<D>(ot, st, tile, v, kb, see);
  });
  const bool on = ((rows | rows >> 32) >> r) & 1;
  if (part_o) {
    docs_again_out<D>(ot, 1.f, part_o + (size_t)r * D, on);
    if (on) { part_ml[r * 2] = m; part_ml[r * 2 + 1] = l; }
  } else {
    docs_again_out<D>(ot, 1.f / l, o + (size_t)r * g.nq * D, on);
    if (on) lse[r] = (m + log2f(l)) * 0.6931471805599453f;
  }
}
// grid: window_grid(nq, blocks * parts, batch)
template <int D>
__global__ __launch_bounds__(AB_THREADS, 2) void attn_window_fwd_bf16_kernel(const WindowTiled p, const bf16_t* __restrict__ qkv, bf16_t* __restrict__ o, float* __restrict__ lse,
                                                                         float* __restrict__ part_o, float* __restrict__ part_ml) {
  using TL = ATile<D>;
  extern __shared__ __attribute__((aligned(1024))) char smem[];  // K ring, then V ring
  const lds_char* sm = (const lds_char*)smem;
  const WindowGeom& g = p.g;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l32 = lane & 31, kg = lane >> 5;
  const int nq = g.nq, nkv = g.nkv, h = window_head(blockIdx.x, nq), hk = h / (nq / nkv), ld = (nq + 2 * nkv) * D, seq = g.seq;
  const WindowUnit u = window_unit(g.batch);
  if (u.id >= p.blocks * p.parts) return;
  const int ib = p.blocks - 1 - u.id / p.parts, part = u.id % p.parts;  // the longest first
  const WindowTiles tiles(g, ib);
  const int f0 = (int)((long long)part * tiles.count() / p.parts), f1 = (int)((long long)(part + 1) * tiles.count() / p.parts);
  const size_t t0 = (size_t)u.b * seq;
  const int iw = ib * WB_BLOCK + wave * 32, iq = iw + l32, row = min(iq, seq - 1);
  const bf16_t* rows = qkv + t0 * ld;
  const char* kbase = reinterpret_cast<const char*>(rows + (size_t)(nq + hk) * D);
  const char* vbase = kbase + (size_t)nkv * D * sizeof(bf16_t);
  const size_t tstride = (size_t)AB_KT * ld * sizeof(bf16_t);
  uint32_t voff[TL::IPW];
  tile_voff<D>(voff, ld, wave, lane, AB_KT);
  const uint32_t ldsK = lds_address(smem), ldsV = ldsK + AF_RING * TL::BYTES;
  auto issue = [&](int t, int slot) {
    const int valid = seq - t * AB_KT;
    if (valid >= AB_KT) {
      tile_dma<D>(kbase + t * tstride, voff, ldsK + slot * TL::BYTES, wave);
      tile_dma<D>(vbase + t * tstride, voff, ldsV + slot * TL::BYTES, wave);
    } else {
      uint32_t vc[TL::IPW];
      tile_voff<D>(vc, ld, wave, lane, valid);
      tile_dma<D>(kbase + t * tstride, vc, ldsK + slot * TL::BYTES, wave);
      tile_dma<D>(vbase + t * tstride, vc, ldsV + slot * TL::BYTES, wave);
    }
  };
  if (f0 < f1) issue(tiles.tile(f0), 0);
  bf16x8 qf[D / 16];
  load_row_frags<D>(qf, rows + (size_t)row * ld + (size_t)h * D, iq < seq, kg);
  FragAddr<D> fa;
  fa.init(lane);
  f32x16 ot[D / 32];
  float m = -3.0e38f, l = 0.f;  // finite: a tile that a row does not see leaves it alone
#pragma unroll
  for (int dt = 0; dt < D / 32; dt++)
#pragma unroll
    for (int r = 0; r < 16; r++) ot[dt][r] = 0.f;
  pin_frags(qf);
  const WindowSeen see = {iw, iq, g.window, g.sinks};
  int slot = 0;
  for (int f = f0; f < f1; f++, slot ^= 1) {
    dma_wait<0>();
    __syncthreads();  // tile f is visible; every wave is done with tile f-1, whose slot tile f+1 reuses
    if (f + 1 < f1) issue(tiles.tile(f + 1), slot ^ 1);
    const int kb = tiles.tile(f) * AB_KT;
    if (see.none(kb)) continue;
    TilePtrs<D> Kp, Vp;
    Kp.set(sm + slot * TL::BYTES, fa);
    Vp.set(sm + (AF_RING + slot) * TL::BYTES, fa);
    f32x16 st[2];
    score_tiles<D>(st, Kp, qf);
    if (see.part(kb)) see.each(kb, kg, [&](int mt, int r, bool on) { st[mt][r] = on ? st[mt][r] : -INFINITY; });
    float mx = max_of(st[0][0], st[1][0]);
#pragma unroll
    for (int r = 1; r < 16; r++) mx = max_of(mx, max_of(st[0][r], st[1][r]));
    mx = across_halves(mx, [](float a, float b) { return max_of(a, b); });
    const float mnew = mx * p.exp_scale;
    if (__any(mnew > m + AF_TAU)) {  // the reference maximum moves where a row's probabilities would grow beyond 2^AF_TAU
      const float mn = max_of(m, mnew), alpha = fast_exp2(m - mn);
      l *= alpha;
      m = mn;
#pragma unroll
      for (int dt = 0; dt < D / 32; dt++)
#pragma unroll
        for (int r = 0; r < 16; r++) ot[dt][r] *= alpha;
    }
    float rs = 0.f;
#pragma unroll
    for (int mt = 0; mt < 2; mt++)
#pragma unroll
      for (int r = 0; r < 16; r++) {
        const float x = fast_exp2(fmaf(st[mt][r], p.exp_scale, -m));
        st[mt][r] = x;
        rs += x;
      }
    l += across_halves(rs, [](float a, float b) { return a + b; });
#pragma unroll
    for (int mt = 0; mt < 2; mt++)
#pragma unroll
      for (int c = 0; c < 2; c++) {
        const bf16x8 pf = pack_rows(st[mt], c);
        const int ro = (mt * 32 + 16 * c) * TL::LD * 2;
#pragma unroll
        for (int dt = 0; dt < D / 32; dt++) ot[dt] = MFMA(lds_frag_tr(Vp.t0[dt], Vp.t1[dt], ro), pf, ot[dt]);
      }
  }
  __syncthreads();  // every wave is done with the K/V rings: their LDS serves the output turn
  const int live = seq - iw;  // rows of the wave that there are
  const size_t head = (size_t)h * g.batch * seq + t0;
  const bool bad = l32 < live && docs_not_finite<D / 32>(ot) && l == l;
  bf16_t* orow = o + ((t0 + iw) * nq + h) * D;
  float *prow = nullptr, *pml = nullptr;
  if (p.parts > 1) {
    const size_t unit = (((size_t)u.b * nq + h) * p.blocks + ib) * p.parts + part;
    prow = part_o + (unit * WB_BLOCK + wave * 32) * D;
    pml = part_ml + (unit * WB_BLOCK + wave * 32) * 2;
    wave_rows_out_f32<D>(
        wave_region<float, D>(smem, wave), lane,
        [&](int dt, int q4) { return f32x4{ot[dt][4 * q4], ot[dt][4 * q4 + 1], ot[dt][4 * q4 + 2], ot[dt][4 * q4 + 3]}; },
        [&](int r) { return r < live ? prow + (size_t)r * D : nullptr; });
    if (lane < 32 && lane < live) {
      pml[l32 * 2] = m;
      pml[l32 * 2 + 1] = l;
    }
  } else {
    const float inv = 1.0f / l;
    wave_rows_out_bf16<D>(
        wave_region<bf16_t, D>(smem, wave), lane,
        [&](int dt, int q4) { return f32x4{ot[dt][4 * q4] * inv, ot[dt][4 * q4 + 1] * inv, ot[dt][4 * q4 + 2] * inv, ot[dt][4 * q4 + 3] * inv}; },
        [&](int r) { return r < live ? orow + (size_t)r * nq * D : nullptr; });
    if (lane < 32 && lane < live) lse[head + iq] = (m + log2f(l)) * 0.6931471805599453f;
  }
  if (!__any(bad)) return;
  const DocsRows k = {rows + (size_t)(nq + hk) * D, (size_t)ld, 0, docs_scalar(seq) - 1}, v = {k.base + (size_t)nkv * D, (size_t)ld, 0, k.last};
  window_again_fwd<D>(p, tiles, docs_scalar(iw), docs_scalar(f0), docs_scalar(f1), bad, k, v, rows + (size_t)iw * ld + (size_t)h * D, orow, lse + head + iw, prow, pml,
                      wave_region<char, D>(smem, wave));
}

// Merges the parts of every block.  grid (nq, ceil(seq / 16), batch): 16 rows a block, 16 lanes a row
template <int D>
__global__ __launch_bounds__(256) void attn_window_combine_kernel(const WindowTiled p, const float* __restrict__ part_o, const float* __restrict__ part_ml, bf16_t* __restrict__ o,
                                                                  float* __restrict__ lse) {
  const WindowGeom& g = p.g;
  const int h = blockIdx.x, b = blockIdx.z, nq = g.nq, i = blockIdx.y * 16 + (threadIdx.x >> 4), row = min(i, g.seq - 1);
  constexpr int CPT = D / 16;
  const int c0 = (threadIdx.x & 15) * CPT, ib = row / WB_BLOCK;
  const size_t t0 = (size_t)b * g.seq, unit = (((size_t)b * nq + h) * p.blocks + ib) * p.parts, at = unit * WB_BLOCK + row % WB_BLOCK;
  float M = -3.0e38f;
#pragma unroll 4
  for (int c = 0; c < p.parts; c++) M = max_of(M, part_ml[(at + (size_t)c * WB_BLOCK) * 2]);
  float L = 0.f, acc[CPT];
#pragma unroll
  for (int e = 0; e < CPT; e++) acc[e] = 0.f;
#pragma unroll 4
  for (int c = 0; c < p.parts; c++) {
    const size_t x = at + (size_t)c * WB_BLOCK;
    const float lc = part_ml[x * 2 + 1], w = lc == 0.f ? 0.f : fast_exp2(part_ml[x * 2] - M);  // no weight: this part holds no key of the row
    L += w * lc;
#pragma unroll
    for (int e = 0; e < CPT; e += 4) {
      const f32x4 v = *reinterpret_cast<const f32x4*>(part_o + x * D + c0 + e);
      acc[e] += w * v[0]; acc[e + 1] += w * v[1]; acc[e + 2] += w * v[2]; acc[e + 3] += w * v[3];
    }
  }
  if (i >= g.seq) return;
  const float inv = 1.0f / L;
  bf16_t* orow = o + ((t0 + row) * nq + h) * D;
#pragma unroll
  for (int e = 0; e < CPT; e += 4) {
    const bf16x4 x = {(bf16_t)(acc[e] * inv), (bf16_t)(acc[e + 1] * inv), (bf16_t)(acc[e + 2] * inv), (bf16_t)(acc[e + 3] * inv)};
    *reinterpret_cast<bf16x4*>(orow + c0 + e) = x;
  }
  if (c0 == 0) lse[(size_t)h * g.batch * g.seq + t0 + row] = (M + log2f(L)) * 0.6931471805599453f;
}

// ================================================================================ backward: dQ
// The rows `bad` of a wave again, as docs_again_dq.  q, dout, dq: of the wave's first row.
template <int D>
__device__ __forceinline__ void window_again_dq(const WindowTiled& p, const WindowTiles& tiles, int iw, bool bad, float l2, float dl, const DocsRows& k, const DocsRows& v, const bf16_t* q,
                                                const bf16_t* dout, bf16_t* dq, char* tile) {
  const WindowGeom& g = p.g;
  const int lane = docs_lane(), r = lane & 31, at = min(r, g.seq - 1 - iw), n = tiles.count();
  const size_t ldo = (size_t)g.nq * D;
  bool arrives = (docs_odd<D>({dout + at * ldo, 0, 0, 0}, 0, DOCS_LARGE).some >> lane) & 1;
  window_masked_tiles(g, tiles, iw, 0, n, [&](int kb, uint64_t seen) {
    arrives |= ((docs_odd<D>(k, kb, DOCS_ODD).some | docs_odd<D>(v, kb, DOCS_LARGE).some) & ~seen) != 0;
  });
  const uint64_t rows = __ballot(bad && arrives);
  if (rows == 0) return;
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the first results of these rows, which other lanes have stored, are in place
  f32x16 acc[D / 32];
#pragma unroll
  for (int dt = 0; dt < D / 32; dt++) acc_zero<false>(acc[dt]);
  window_again_tiles(g, tiles, iw, 0, n, [&](int kb, const DocsSeen& see) {
    f32x16 st[2], dp[2];
    docs_again_scores<D>(st, tile, k, kb, q + at * k.ld, true);
    docs_again_scores<D>(dp, tile, v, kb, dout + at * ldo, true);
    const uint64_t seen = docs_bits(see, kb);
#pragma unroll
    for (int mt = 0; mt < 2; mt++)
#pragma unroll
      for (int i = 0; i < 16; i++)
        st[mt][i] = docs_where((uint32_t)(seen >> (32 * mt)) >> (4 * (lane >> 5)), 8 * (i >> 2) + (i & 3), fast_exp2(fmaf(st[mt][i], p.exp_scale, -l2)) * (dp[mt][i] - dl));
    docs_again_add<D>(acc, st, tile, k, kb, see);
  });
  docs_again_out<D>(acc, g.scale, dq + r * k.ld, ((rows | rows >> 32) >> r) & 1);
}
// As docs_dq_block: block ib of head h, sequence b.  STORE: leaves the rows' delta and lse2 for the dK/dV launch behind it; otherwise attn_window_prep_kernel has.
template <int D, bool STORE>
__device__ __forceinline__ void window_dq_block(const WindowTiled& p, int ib, int h, int b, const bf16_t* __restrict__ qkv, const bf16_t* __restrict__ o, const bf16_t* __restrict__ dout,
                                                const float* __restrict__ lse, float* __restrict__ lse2, float* __restrict__ delta, bf16_t* __restrict__ dqkv) {
  using TL = ATile<D>;
  constexpr int RING = 2;
  extern __shared__ __attribute__((aligned(1024))) char smem[];  // K ring, then V ring
  const lds_char* sm = (const lds_char*)smem;
  const WindowGeom& g = p.g;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l32 = lane & 31, kg = lane >> 5;
  const int nq = g.nq, nkv = g.nkv, hk = h / (nq / nkv), ld = (nq + 2 * nkv) * D, seq = g.seq;
  const WindowTiles tiles(g, ib);
  const int f1 = tiles.count();
  const size_t t0 = (size_t)b * seq, head = (size_t)h * g.batch * seq + t0;
  const int iw = ib * WB_BLOCK + wave * 32, iq = iw + l32, row = min(iq, seq - 1);
  const bf16_t* rows = qkv + t0 * ld;
  const char* kbase = reinterpret_cast<const char*>(rows + (size_t)(nq + hk) * D);
  const char* vbase = kbase + (size_t)nkv * D * sizeof(bf16_t);
  const size_t tstride = (size_t)AB_KT * ld * sizeof(bf16_t);
  uint32_t voff[TL::IPW];
  tile_voff<D>(voff, ld, wave, lane, AB_KT);
  const uint32_t ldsK = lds_address(smem), ldsV = ldsK + RING * TL::BYTES;
  auto issue = [&](int t, int slot) {
    const int valid = seq - t * AB_KT;
    if (valid >= AB_KT) {
      tile_dma<D>(kbase + t * tstride, voff, ldsK + slot * TL::BYTES, wave);
      tile_dma<D>(vbase + t * tstride, voff, ldsV + slot * TL::BYTES, wave);
    } else {
      uint32_t vc[TL::IPW];
      tile_voff<D>(vc, ld, wave, lane, valid);
      tile_dma<D>(kbase + t * tstride, vc, ldsK + slot * TL::BYTES, wave);
      tile_dma<D>(vbase + t * tstride, vc, ldsV + slot * TL::BYTES, wave);
    }
  };
  issue(tiles.tile(0), 0);
  const size_t at = ((t0 + row) * nq + h) * D;
  bf16x8 qf[D / 16], dof[D / 16];
  load_row_frags<D>(qf, rows + (size_t)row * ld + (size_t)h * D, iq < seq, kg);
  load_row_frags<D>(dof, dout + at, iq < seq, kg);
  float l2 = lse[head + row] * LOG2E, dl = 0.f;
  {
    bf16x8 of[D / 16];
    load_row_frags<D>(of, o + at, iq < seq, kg);
#pragma unroll
    for (int ks = 0; ks < D / 16; ks++)
#pragma unroll
      for (int e = 0; e < 8; e++) dl = fmaf((float)dof[ks][e], (float)of[ks][e], dl);
    dl += __shfl_xor(dl, 32, 64);
  }
  if (STORE && kg == 0 && iq < seq) {
    delta[head + iq] = dl;
    lse2[head + iq] = l2;
  }
  const WindowSeen see = {iw, iq, g.window, g.sinks};
  f32x16 dqt[D / 32];
#pragma unroll
  for (int dt = 0; dt < D / 32; dt++) acc_zero<false>(dqt[dt]);
  FragAddr<D> fa;
  fa.init(lane);
  pin_frags(qf);
  pin_frags(dof);
  pin_scalar(l2);
  pin_scalar(dl);
  TilePtrs<D> Kp;
  Kp.set(sm, fa);
  int slot = 0;
  for (int f = 0; f < f1; f++, docs_shift<D>(Kp, slot ? -(int)TL::BYTES : (int)TL::BYTES), slot ^= 1) {
    dma_wait<0>();
    __syncthreads();
    if (f + 1 < f1) issue(tiles.tile(f + 1), slot ^ 1);
    const int kb = tiles.tile(f) * AB_KT;
    if (see.none(kb)) continue;
    f32x16 st[2], dp[2];
    score_tiles2<D, RING * TL::BYTES, 1>(st, Kp, qf, dp, dof, [&](int j) {  // P^T from S^T beside the dP^T products
      constexpr int N = 32 / (D / 16);
#pragma unroll
      for (int i = 0; i < N; i++) {
        const int x = j * N + i;
        st[x >> 4][x & 15] = fast_exp2(fmaf(st[x >> 4][x & 15], p.exp_scale, -l2));
      }
    });
    TrFrags<D> fr;
    tr_fetch<D>(fr, Kp, 0);
    if (see.part(kb)) see.each(kb, kg, [&](int mt, int r, bool on) { st[mt][r] = on ? st[mt][r] : 0.f; });
    auto ds_quarter = [&](int q) {  // dS^T = P^T (dP^T - delta), one quarter ahead of the products that take it
#pragma unroll
      for (int r = 8 * (q & 1); r < 8 * (q & 1) + 8; r++) st[q >> 1][r] *= dp[q >> 1][r] - dl;
    };
    ds_quarter(0);
    acc_tile_tr<D, false, false>(dqt, fr, Kp, st, Kp, [&](int q) { if (q + 1 < 4) ds_quarter(q + 1); });
  }
  __syncthreads();
  const int live = seq - iw;
  bf16_t* out = dqkv + (t0 + iw) * ld + (size_t)h * D;
  const bool bad = l32 < live && docs_not_finite<D / 32>(dqt) && l2 == l2 && __builtin_isfinite(dl);
  const float scale = g.scale;
  wave_rows_out_bf16<D>(
      wave_region<bf16_t, D>(smem, wave), lane,
      [&](int dt, int q4) { return f32x4{dqt[dt][4 * q4] * scale, dqt[dt][4 * q4 + 1] * scale, dqt[dt][4 * q4 + 2] * scale, dqt[dt][4 * q4 + 3] * scale}; },
      [&](int r) { return r < live ? out + (size_t)r * ld : nullptr; });
  if (!__any(bad)) return;
  const DocsRows k = {rows + (size_t)(nq + hk) * D, (size_t)ld, 0, docs_scalar(seq) - 1}, v = {k.base + (size_t)nkv * D, (size_t)ld, 0, k.last};
  window_again_dq<D>(p, tiles, docs_scalar(iw), bad, l2, dl, k, v, rows + (size_t)iw * ld + (size_t)h * D, dout + ((t0 + iw) * nq + h) * D, out, wave_region<char, D>(smem, wave));
}

// ================================================================================ backward: dK, dV
// The walk of dkv_pinned: query tiles from position q0 on.
struct WindowWalk {
  int jw, jk, n, any1, all1, whole;  // a lane's key sees n rows from jk on; some key of the wave rows up to any1, all keys up to all1; tiles below `whole` are whole
  __device__ __forceinline__ bool idle(int qb) const { return qb >= any1 || qb + AB_KT <= jw; }
  __device__ __forceinline__ bool partial(int qb) const { return qb < jw + 31 || qb + AB_KT > all1; }
  __device__ __forceinline__ uint32_t rows() const { return (uint32_t)n; }
  __device__ __forceinline__ bool ragged(int ti) const { return ti >= whole; }
};
// Unit `unit` of key/value head hk, sequence b: the blocks without sinks, which are of one length, then the short units of the others, which fill up the last round.
template <int D>
__device__ __forceinline__ void window_dkv_block(const WindowTiled& p, int unit, int hk, int b, const bf16_t* __restrict__ qkv, const bf16_t* __restrict__ dout,
                                                 const float* __restrict__ lse2, const float* __restrict__ delta, bf16_t* __restrict__ dqkv, float* __restrict__ part) {
  using TL = ATile<D>;
  constexpr bool PINNED = D == 128;
  extern __shared__ __attribute__((aligned(1024))) char smem[];  // Q ring, dO ring, lse2 ring, delta ring
  const lds_char* sm = (const lds_char*)smem;
  const WindowGeom& g = p.g;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l32 = lane & 31, kg = lane >> 5;
  const int nq = g.nq, nkv = g.nkv, grp = nq / nkv, hq = hk * grp, ld = (nq + 2 * nkv) * D, ldo = nq * D, seq = g.seq;
  if (unit >= window_units(p)) return;
  const WindowKeys128 k = window_keys128(p, unit, grp);
  const int q0 = k.q0, nt = k.nt, f0 = k.f0, f1 = k.f1;
  if (f0 >= f1) return;  // a shorter block has fewer tiles than units; the merge knows
  const size_t t0 = (size_t)b * seq, T = (size_t)g.batch * seq;
  const int jw = k.jb * WB_BLOCK + wave * 32, jk = jw + l32, row = min(jk, seq - 1), live = seq - jw;
  float* prow = part + ((((size_t)b * nkv + hk) * window_parts(p) + k.part) * WB_BLOCK + wave * 32) * (2 * D);
  const bf16_t* rows = qkv + t0 * ld;
  const bf16_t* kcol = rows + (size_t)(nq + hk) * D;
  const char* qbase = reinterpret_cast<const char*>(rows + (size_t)q0 * ld + (size_t)hq * D);
  const char* obase = reinterpret_cast<const char*>(dout + (t0 + q0) * ldo + (size_t)hq * D);
  float* lse_s = reinterpret_cast<float*>(smem + 2 * AB_RING * TL::BYTES);
  float* del_s = lse_s + AB_RING * AB_KT;
  uint32_t vq[TL::IPW], vo[TL::IPW];
  tile_voff<D>(vq, ld, wave, lane, AB_KT);
  tile_voff<D>(vo, ldo, wave, lane, AB_KT);
#pragma unroll
  for (int j = 0; j < TL::IPW; j++) { vq[j] -= j * 1024; vo[j] -= j * 1024; }  // for tile_dma_at: transfer j moves rows from 512 j / D on, of at least 2 D bytes
  const uint32_t ldsQ = lds_address(smem), ldsO = ldsQ + AB_RING * TL::BYTES;
  const size_t qstride = (size_t)AB_KT * ld * sizeof(bf16_t), ostride = (size_t)AB_KT * ldo * sizeof(bf16_t);
  int gi = f0 / nt, ti = f0 - gi * nt;  // head of the group and tile to transfer next
  int tc = ti;                          // tile to work off next
  const uint32_t ldsS = ldsQ + 2 * AB_RING * TL::BYTES + (wave & 1) * AB_RING * AB_KT * sizeof(float);  // even waves transfer lse2, odd ones delta
  const float* srow = ((wave & 1) ? delta : lse2) + (size_t)hq * T + t0 + q0;
  auto issue = [&](int slot) {
    const int end = min(AB_KT - 1, seq - 1 - q0 - ti * AB_KT);
    const char* qp = qbase + ti * qstride + gi * (D * sizeof(bf16_t));
    const char* op = obase + ti * ostride + gi * (D * sizeof(bf16_t));
    if (end == AB_KT - 1) {
      tile_dma_at<D>(qp, vq, ldsQ + slot * TL::BYTES, wave);
      tile_dma_at<D>(op, vo, ldsO + slot * TL::BYTES, wave);
    } else {
      uint32_t vc[TL::IPW];
      docs_voff<D>(vc, ld, wave, lane, 0, end);
      tile_dma<D>(qp, vc, ldsQ + slot * TL::BYTES, wave);
      docs_voff<D>(vc, ldo, wave, lane, 0, end);
      tile_dma<D>(op, vc, ldsO + slot * TL::BYTES, wave);
    }
    dma4_base(srow + (size_t)gi * T + (size_t)ti * AB_KT, (uint32_t)(min(lane, end) * sizeof(float)), ldsS + slot * AB_KT * sizeof(float));
    if (++ti == nt) { ti = 0; gi++; }
  };
  if constexpr (!PINNED) issue(0);
  bf16x8 kf[D / 16], vf[D / 16];
  load_row_frags<D>(kf, kcol + (size_t)row * ld, jk < seq, kg);
  load_row_frags<D>(vf, kcol + (size_t)row * ld + (size_t)nkv * D, jk < seq, kg);
  f32x16 dkt[D / 32], dvt[D / 32];
  constexpr bool AGPR = D == 128;
#pragma unroll
  for (int dt = 0; dt < D / 32; dt++) { acc_zero<AGPR>(dkt[dt]); acc_zero<AGPR>(dvt[dt]); }
  FragAddr<D> fa;
  fa.init(lane);
  pin_frags(kf);
  pin_frags(vf);
  const int end = window_queries_end(g, jk), first_plain = max(jw, g.sinks);  // the wave's first key that is no sink: the one whose window ends first
  const WindowWalk walk = {jw, jk, max(0, end - jk), window_queries_end(g, jw < g.sinks ? jw : jw + 31), first_plain < jw + 32 ? window_queries_end(g, first_plain) : seq, (seq - q0) / AB_KT};
  if constexpr (PINNED) {
    dkv_pinned(walk, issue, sm, fa, kf, vf, dkt, dvt, qbase, obase, srow, T, qstride, ostride, vq, vo, ldsQ, ldsS, wave, lane, kg, q0, nt, f0, f1, gi, ti, tc, p.exp_scale);
  } else {
    if (f0 + 1 < f1) issue(1);
    int slot = 0;
    for (int f = f0; f < f1; f++, slot = slot == AB_RING - 1 ? 0 : slot + 1) {
      if (f + 1 < f1) dma_wait<2 * TL::IPW + 1>(); else dma_wait<0>();
      __syncthreads();
      if (f + 2 < f1) issue(slot == 0 ? AB_RING - 1 : slot - 1);
      const int qb = q0 + tc * AB_KT;
      if (++tc == nt) tc = 0;
      if (walk.idle(qb)) continue;
      TilePtrs<D> Qp, Op;
      Qp.set(sm + slot * TL::BYTES, fa);
      Op.set(sm + (AB_RING + slot) * TL::BYTES, fa);
      const float* ls = lse_s + slot * AB_KT;
      const float* ds = del_s + slot * AB_KT;
      f32x4 lv[8];  // rows 32*mt + 8*q4 + 4*kg + e of the tile at [4*mt + q4]
#pragma unroll
      for (int x = 0; x < 8; x++) lv[x] = *reinterpret_cast<const f32x4*>(ls + 8 * x + 4 * kg);
      f32x16 st[2], dp[2];
      score_tiles2<D, AB_RING * TL::BYTES, 3>(st, Qp, kf, dp, vf, [&](int j) {  // P from S beside the dP products
        constexpr int N = 8 / (D / 16) > 0 ? 8 / (D / 16) : 1;
#pragma unroll
        for (int i = 0; i < N; i++) {
          const int x = j * N + i, mt = x >> 2, q4 = x & 3;
#pragma unroll
          for (int e = 0; e < 4; e++) st[mt][4 * q4 + e] = fast_exp2(fmaf(st[mt][4 * q4 + e], p.exp_scale, -lv[x][e]));
        }
      });
      TrFrags<D> fr;
      tr_fetch<D>(fr, Op, 0);
#pragma unroll
      for (int x = 0; x < 8; x++) lv[x] = *reinterpret_cast<const f32x4*>(ds + 8 * x + 4 * kg);
      if (walk.partial(qb)) {
        const int first = qb + 4 * kg - jk;
#pragma unroll
        for (int mt = 0; mt < 2; mt++)
#pragma unroll
          for (int r = 0; r < 16; r++) {
            st[mt][r] = (uint32_t)(first + mt * 32 + 8 * (r >> 2) + (r & 3)) < walk.rows() ? st[mt][r] : 0.f;
            if ((r & 3) == 3) __builtin_amdgcn_sched_barrier(0);
          }
      }
      acc_tile_tr<D, true, AGPR>(dvt, fr, Op, st, Qp, [&](int q) {
#pragma unroll
        for (int r = 8 * (q & 1); r < 8 * (q & 1) + 8; r++) st[q >> 1][r] *= dp[q >> 1][r] - lv[4 * (q >> 1) + (r >> 2)][r & 3];
      });
      acc_tile_tr<D, false, AGPR>(dkt, fr, Qp, st, Qp, [](int) {});
    }
  }
  acc_settle<AGPR>(dkt);
  acc_settle<AGPR>(dvt);
  __syncthreads();  // every wave is done with the Q/dO rings: their LDS serves the output turn (dK, then dV)
  const float scale = g.scale;
  auto dk_quad = [&](int dt, int q4) { return f32x4{dkt[dt][4 * q4] * scale, dkt[dt][4 * q4 + 1] * scale, dkt[dt][4 * q4 + 2] * scale, dkt[dt][4 * q4 + 3] * scale}; };
  auto dv_quad = [&](int dt, int q4) { return f32x4{dvt[dt][4 * q4], dvt[dt][4 * q4 + 1], dvt[dt][4 * q4 + 2], dvt[dt][4 * q4 + 3]}; };
  const bool bad = l32 < live && (docs_not_finite<D / 32>(dkt) || docs_not_finite<D / 32>(dvt));
  bf16_t* out = dqkv + (t0 + jw) * ld + (size_t)(nq + hk) * D;
  if (k.part >= 0) {
    float* reg = wave_region<float, D>(smem, wave);
    wave_rows_out_f32<D>(reg, lane, dk_quad, [&](int r) { return r < live ? prow + (size_t)r * (2 * D) : nullptr; });
    __builtin_amdgcn_wave_barrier();
    wave_rows_out_f32<D>(reg, lane, dv_quad, [&](int r) { return r < live ? prow + (size_t)r * (2 * D) + D : nullptr; });
  } else {
    bf16_t* reg = wave_region<bf16_t, D>(smem, wave);
    wave_rows_out_bf16<D>(reg, lane, dk_quad, [&](int r) { return r < live ? out + (size_t)r * ld : nullptr; });
    __builtin_amdgcn_wave_barrier();
    wave_rows_out_bf16<D>(reg, lane, dv_quad, [&](int r) { return r < live ? out + (size_t)r * ld + (size_t)nkv * D : nullptr; });
  }
  if (!__any(bad)) return;
  const int keys = docs_scalar(jw), last = docs_scalar(seq) - 1, h0 = docs_scalar(hq), mine = min(keys + (docs_lane() & 31), last), from = docs_scalar(q0);
  const DocsSeen see = {mine, window_queries_end(g, mine) - mine, keys, docs_scalar(walk.any1), min(keys + 31, last), docs_scalar(walk.all1)};
  const DocsUnit run = {0, docs_scalar(f0), docs_scalar(f1), k.part};
  const DocsSpan span = {from / AB_KT, docs_scalar(nt), 0, 0};
  const DocsRows q = {rows + (size_t)h0 * D, (size_t)ld, 0, last}, e = {dout + t0 * ldo + (size_t)h0 * D, (size_t)ldo, 0, last};
  DocsTiled docs = {};
  docs.a.v.T = (int)T;
  docs.exp_scale = p.exp_scale;
  docs_again_dkv<D, false>(docs, see, bad, run, span, q, e, lse2 + (size_t)h0 * T + t0, delta + (size_t)h0 * T + t0, kcol + (size_t)keys * ld, ld, (size_t)nkv * D, out, prow, scale,
                           wave_region<char, D>(smem, wave));
}
// Delta and lse2 of every row, as attn_bwd_prep_kernel: the numbers the dQ blocks use.  Two lanes a row of a head.
template <int D>
__global__ __launch_bounds__(64) void attn_window_prep_kernel(const WindowGeom g, const bf16_t* __restrict__ o, const bf16_t* __restrict__ dout, const float* __restrict__ lse, float* __restrict__ lse2,
                                                              float* __restrict__ delta) {
  const size_t T = (size_t)g.batch * g.seq, i = (size_t)blockIdx.x * 32 + (threadIdx.x >> 1);
  if (i >= T * g.nq) return;
  const int kg = threadIdx.x & 1, h = (int)(i % g.nq);
  const size_t t = i / g.nq, at = (size_t)h * T + t;
  const bf16_t *orow = o + i * D + kg * 8, *drow = dout + i * D + kg * 8;
  bf16x8 a[D / 16], b[D / 16];
#pragma unroll
  for (int ks = 0; ks < D / 16; ks++) {
    a[ks] = *reinterpret_cast<const bf16x8*>(drow + ks * 16);
    b[ks] = *reinterpret_cast<const bf16x8*>(orow + ks * 16);
  }
  float half = 0.f;
#pragma unroll
  for (int ks = 0; ks < D / 16; ks++)
#pragma unroll
    for (int e = 0; e < 8; e++) half = fmaf((float)a[ks][e], (float)b[ks][e], half);
  const float other = __shfl_xor(half, 1, 64);
  if (kg == 0) {
    delta[at] = half + other;
    lse2[at] = lse[at] * LOG2E;
  }
}
// The two as launches of their own (dQ first: it stores what the dK/dV blocks read), grids window_grid(nq, blocks, batch) and window_grid(nkv, units, batch) ...
template <int D>
__global__ __launch_bounds__(AB_THREADS, 2) void attn_window_dq_bf16_kernel(const WindowTiled p, const bf16_t* __restrict__ qkv, const bf16_t* __restrict__ o, const bf16_t* __restrict__ dout,
                                                                        const float* __restrict__ lse, float* __restrict__ lse2, float* __restrict__ delta, bf16_t* __restrict__ dqkv) {
  const WindowUnit u = window_unit(p.g.batch);
  if (u.id < p.blocks) window_dq_block<D, true>(p, p.blocks - 1 - u.id, window_head(blockIdx.x, p.g.nq), u.b, qkv, o, dout, lse, lse2, delta, dqkv);
}
template <int D>
__global__ __launch_bounds__(AB_THREADS) void attn_window_dkv_bf16_kernel(const WindowTiled p, const bf16_t* __restrict__ qkv, const bf16_t* __restrict__ dout,
                                                                          const float* __restrict__ lse2, const float* __restrict__ delta, bf16_t* __restrict__ dqkv, float* __restrict__ part) {
  const WindowUnit u = window_unit(p.g.batch);
  window_dkv_block<D>(p, u.id, window_head(blockIdx.x, p.g.nkv), u.b, qkv, dout, lse2, delta, dqkv, part);
}
// ... and as one, behind attn_window_prep_kernel, for grids that leave units of the chip idle: dK/dV units (the longer ones) first.  grid (units * nkv + blocks * nq, batch)
template <int D>
__global__ __launch_bounds__(AB_THREADS) void attn_window_bwd_bf16_kernel(const WindowTiled p, const bf16_t* __restrict__ qkv, const bf16_t* __restrict__ o, const bf16_t* __restrict__ dout,
                                                                          const float* __restrict__ lse, float* __restrict__ lse2, float* __restrict__ delta, bf16_t* __restrict__ dqkv,
                                                                          float* __restrict__ part) {
  const int nq = p.g.nq, nkv = p.g.nkv, n_k = window_units(p) * nkv, id = blockIdx.x;
  if (id < n_k) {
    const int unit = __builtin_amdgcn_readfirstlane(id / nkv);
    window_dkv_block<D>(p, unit, id - unit * nkv, blockIdx.y, qkv, dout, lse2, delta, dqkv, part);
  } else {
    const int x = id - n_k, block = __builtin_amdgcn_readfirstlane(x / nq);
    window_dq_block<D, false>(p, p.blocks - 1 - block, x - block * nq, blockIdx.y, qkv, o, dout, lse, lse2, delta, dqkv);
  }
}
// Adds the units of key blocks [first, first + y / 32) in order.  grid (nkv, blocks * 32, batch): 4 keys a block, a wave each
template <int D>
__global__ __launch_bounds__(256) void attn_window_merge_kernel(const WindowTiled p, int first, const float* __restrict__ part, bf16_t* __restrict__ dqkv) {
  const WindowGeom& g = p.g;
  const int hk = blockIdx.x, b = blockIdx.z, j = first * WB_BLOCK + blockIdx.y * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, nkv = g.nkv, jb = j / WB_BLOCK;
  if (j >= g.seq) return;
  constexpr int CPL = 2 * D / 64;
  const int ld = (g.nq + 2 * nkv) * D, tiles = (g.nq / nkv) * window_key_tiles(p, jb);
  const bool sink = jb < p.sink_blocks;
  const int ch = sink ? p.sink_chunk : p.plain_chunk, units = (tiles + ch - 1) / ch, plain = (p.blocks - p.sink_blocks) * p.plain_units;
  const int at = sink ? jb * p.sink_units + (p.plain_units > 1 ? plain : 0) : (jb - p.sink_blocks) * p.plain_units;
  const float* from = part + ((((size_t)b * nkv + hk) * window_parts(p) + at) * WB_BLOCK + j % WB_BLOCK) * (2 * D) + lane * CPL;
  float s[CPL] = {};
#pragma unroll 8
  for (int c = 0; c < units; c++)
#pragma unroll
    for (int e = 0; e < CPL; e++) s[e] += from[(size_t)c * WB_BLOCK * 2 * D + e];
  bf16_t* dk = dqkv + ((size_t)b * g.seq + j) * ld + (size_t)(g.nq + hk) * D;
  const int c0 = lane * CPL;
#pragma unroll
  for (int e = 0; e < CPL; e++) (c0 < D ? dk + c0 : dk + (size_t)nkv * D + c0 - D)[e] = (bf16_t)s[e];
}

// ------------------------------------------------------------------------------------ host side
// Whether both halves of the backward pass go out as one launch: up to so many 128-row blocks of all heads.  us, two launches and one, by blocks: D = 128: 128 (1000 rows of 8 heads, window 300) 41.8 and
// 26.9, 160 (4096 rows of 4:1, window 1024) 83.9 and 74.7, 512 (2 x 2048 of 8, window 512) 69.1 and 69.5, 640 (4096 of 16:4, window 1024) 161 and 175; D = 64: 128 23.6 and 16.0, 512 38.7 and
// 37.7, 1280 (4 x 2048 of 16:4, window 256) 94.7 and 91.7, 2560 (8192 of 32:8, window 512) 191 and 205.
#define WB_ONE_128 512
#define WB_ONE_64 1280
// Tiles that a part of a forward block holds at least.  us, 4 and 8: 2 x 2048 rows of 8 heads, window 512, 32.4 and 21.8; 2 x 2001 of 8 heads of 64, window 300, 17.7 and 13.6; 1000 of 8,
// window 300, 15.5 and 17.2.
#define WB_PART 8
static WindowTiled window_tiled(const WindowGeom& g0) {
  WindowTiled p = {};
  p.g = g0;
  p.g.window = std::min(g0.window, g0.seq);
  p.g.sinks = std::min(g0.sinks, g0.seq);
  p.blocks = (g0.seq + WB_BLOCK - 1) / WB_BLOCK;
  p.exp_scale = (float)(1.4426950408889634 / sqrt((double)g0.d));
  // forward: parts until the chip's units have two blocks each
  const long long have = (long long)g0.batch * g0.nq * p.blocks;
  const WindowTiles longest(p.g, p.blocks - 1);
  p.parts = (int)std::max(1ll, std::min(2ll * attn_num_cus() / std::max(1ll, have), (long long)longest.count() / WB_PART));
  // dK/dV: the number of units a block without sinks is cut into whose launch is expected to be through first, in tiles of one unit: rounds of resident units (two a unit of the chip at D = 64), each
  // with three tiles for its beginning and end, and for a cut the merge's launch and its way through memory.
  const int grp = g0.nq / g0.nkv, slots = attn_num_cus() * (g0.d == 64 ? 2 : 1);
  p.sink_blocks = (p.g.sinks + WB_BLOCK - 1) / WB_BLOCK;
  const long long pairs = (long long)g0.batch * g0.nkv, plain_blocks = pairs * (p.blocks - p.sink_blocks);
  p.plain_units = 1;
  p.plain_chunk = p.blocks > p.sink_blocks ? grp * window_key_tiles(p, p.sink_blocks) : 1;  // the first is as long as any
  if (plain_blocks > 0 && plain_blocks < 2 * slots) {
    const int tiles = p.plain_chunk;
    double best = 1e30;
    for (int u = 1; u <= 16 && (u == 1 || tiles / u >= 4); u++) {
      const long long n = plain_blocks * u;
      const double cost = (double)((n + slots - 1) / slots) * ((tiles + u - 1) / u + 3) + (u > 1 ? 2.5 + n * (g0.d / 128.0) * 0.03 : 0.0);
      if (cost < best) {
        best = cost;
        p.plain_units = u;
        p.plain_chunk = (tiles + u - 1) / u;
      }
    }
  }
  // Blocks that hold sinks walk on to the row's end.  Where they are few they are cut into units, about as many as the chip has units, of four tiles at least; more than eight fill the chip uncut.
  const int whole = grp * ((g0.seq + AB_KT - 1) / AB_KT);
  const long long sink_tiles = pairs * p.sink_blocks * whole;
  p.sink_chunk = (int)std::max({4ll, (sink_tiles + attn_num_cus() - 1) / attn_num_cus(), (whole + 63ll) / 64});
  p.sink_units = p.sink_blocks > 0 && p.sink_blocks <= 8 ? (whole + p.sink_chunk - 1) / p.sink_chunk : 1;
  if (p.sink_units == 1) p.sink_chunk = whole;
  return p;
}
size_t dh_window_fwd_bf16_ws_bytes(const WindowGeom& g) {
  const WindowTiled p = window_tiled(g);
  return p.parts == 1 ? 0 : (size_t)g.batch * g.nq * p.blocks * p.parts * WB_BLOCK * (g.d + 2) * sizeof(float);
}
template <int D>
static int window_fwd(const WindowTiled& p, const bf16_t* qkv, bf16_t* o, float* lse, float* ws, hipStream_t s) {
  static bool ready[DH_MAX_DEVICES] = {};
  const WindowGeom& g = p.g;
  const size_t lds = 2 * AF_RING * (size_t)ATile<D>::BYTES;
  bool& set = ready[dh_device_index()];
  if (!set) {
    if (int rc = set_lds(attn_window_fwd_bf16_kernel<D>, lds)) return rc;
    set = true;
  }
  float* part_ml = ws + (size_t)g.batch * g.nq * p.blocks * p.parts * WB_BLOCK * D;
  attn_window_fwd_bf16_kernel<D><<<window_grid(g.nq, p.blocks * p.parts, g.batch), AB_THREADS, lds, s>>>(p, qkv, o, lse, ws, part_ml);
  DH_LAUNCH_CHECK();
  if (p.parts > 1) {  // few blocks: ceil(seq / 16) fits the launch's y
    attn_window_combine_kernel<D><<<dim3(g.nq, (g.seq + 15) / 16, g.batch), 256, 0, s>>>(p, ws, part_ml, o, lse);
    DH_LAUNCH_CHECK();
  }
  return DH_OK;
}
int dh_launch_window_fwd_bf16(const WindowGeom& g, const bf16_t* qkv, bf16_t* o, float* lse, void* ws, hipStream_t s) {
  const WindowTiled p = window_tiled(g);
  return g.d == 128 ? window_fwd<128>(p, qkv, o, lse, (float*)ws, s) : window_fwd<64>(p, qkv, o, lse, (float*)ws, s);
}
size_t dh_window_bwd_bf16_ws_bytes(const WindowGeom& g) {
  const WindowTiled p = window_tiled(g);
  return dh_align_up((size_t)g.nq * g.batch * g.seq * sizeof(float), 256) +
         (size_t)g.batch * g.nkv * window_parts(p) * WB_BLOCK * 2 * g.d * sizeof(float);
}
template <int D>
static int window_bwd(const WindowTiled& p, const bf16_t* qkv, const bf16_t* o, const bf16_t* dout, const float* lse, bf16_t* dqkv, float* delta, char* ws, hipStream_t s) {
  static bool ready[DH_MAX_DEVICES] = {};
  const WindowGeom& g = p.g;
  const size_t lds_dq = 4 * (size_t)ATile<D>::BYTES, lds_dkv = 2 * AB_RING * ((size_t)ATile<D>::BYTES + AB_KT * sizeof(float));
  bool& set = ready[dh_device_index()];
  if (!set) {
    if (int rc = set_lds(attn_window_dq_bf16_kernel<D>, lds_dq)) return rc;
    if (int rc = set_lds(attn_window_dkv_bf16_kernel<D>, lds_dkv)) return rc;
    if (int rc = set_lds(attn_window_bwd_bf16_kernel<D>, lds_dkv)) return rc;
    set = true;
  }
  float *lse2 = (float*)ws, *part = (float*)(ws + dh_align_up((size_t)g.nq * g.batch * g.seq * sizeof(float), 256));
  if ((long long)p.blocks * (g.nq + g.nkv) * g.batch <= (D == 128 ? WB_ONE_128 : WB_ONE_64)) {
    attn_window_prep_kernel<D><<<(unsigned)(((size_t)g.batch * g.seq * g.nq + 31) / 32), 64, 0, s>>>(g, o, dout, lse, lse2, delta);
    DH_LAUNCH_CHECK();
    attn_window_bwd_bf16_kernel<D><<<dim3(window_units(p) * g.nkv + p.blocks * g.nq, g.batch), AB_THREADS, lds_dkv, s>>>(p, qkv, o, dout, lse, lse2, delta, dqkv, part);
    DH_LAUNCH_CHECK();
  } else {
    attn_window_dq_bf16_kernel<D><<<window_grid(g.nq, p.blocks, g.batch), AB_THREADS, lds_dq, s>>>(p, qkv, o, dout, lse, lse2, delta, dqkv);
    DH_LAUNCH_CHECK();
    attn_window_dkv_bf16_kernel<D><<<window_grid(g.nkv, window_units(p), g.batch), AB_THREADS, lds_dkv, s>>>(p, qkv, dout, lse2, delta, dqkv, part);
    DH_LAUNCH_CHECK();
  }
  const int first = p.sink_units > 1 ? 0 : p.sink_blocks, cut = (p.plain_units > 1 ? p.blocks : p.sink_blocks) - first;  // blocks that were cut: few enough for the launch's y
  if (cut > 0 && (p.plain_units > 1 || p.sink_units > 1)) {
    attn_window_merge_kernel<D><<<dim3(g.nkv, cut * (WB_BLOCK / 4), g.batch), 256, 0, s>>>(p, first, part, dqkv);
    DH_LAUNCH_CHECK();
  }
  return DH_OK;
}
int dh_launch_window_bwd_bf16(const WindowGeom& g, const bf16_t* qkv, const bf16_t* o, const bf16_t* dout, const float* lse, bf16_t* dqkv, float* delta, void* ws, hipStream_t s) {
  const WindowTiled p = window_tiled(g);
  return g.d == 128 ? window_bwd<128>(p, qkv, o, dout, lse, dqkv, delta, (char*)ws, s) : window_bwd<64>(p, qkv, o, dout, lse, dqkv, delta, (char*)ws, s);
}
