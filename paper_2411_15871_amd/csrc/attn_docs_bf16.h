// bf16 attention over packed documents on the matrix cores, forward and backward (part of attn_bf16.hip, whose tiles, fragments and layouts it uses).
//
// A block of 128 rows lies anywhere in the packed row of documents and walks the one run of 64-row tiles that any of its rows meets (borders ascend with the row): the
// documents need no padding, and a block of short documents walks few tiles.  What a lane's row sees inside a tile is an interval, one comparison an element, and only
// tiles that some row of the wave does not see whole are masked.  The runs come from the lists that dh_docs_plan has made (docs.h): longest first, long ones cut, partial
// results merged in order by a launch behind.
//
// Probabilities and their gradients round to bf16 before the products that take them, as the causal kernels' do: matrix instructions of the full rate take nothing else.  Errors against 64 bits,
// relative norms, with float32 in their place and so: o 1.65e-3 and 1.95e-3, gradients 2.2e-3 and 2.9e-3 (rounding the results alone makes 1.65e-3).
//
// Masked probabilities are zeros, and a zero times an infinity or a NaN of a row that is not seen is a NaN.  A wave whose result is not finite looks whether its masked tiles hold any
// such row; only then it walks its tiles again (docs_again_*), with the infinities and NaNs of masked tiles added to the rows that see them alone.  Rows outside all documents enter
// no tile, transfers take the nearest row of a document instead, and what a lane makes of such a row of its own goes nowhere.
//
// CAP: x = cap tanh(x / cap) as cap - 2 cap r with r = 1 / (1 + e^(2x/cap)), one exponential and one reciprocal more an element, whose limits (r = 0, 1) are right where the
// exponential is infinite or zero; its slope is 4 (r - r r), off by at most 2^-22, of which the factor 4 waits for the end.  The exponent of 2 of a probability is
// one multiply-add of r.
#pragma once
#include "docs.h"

struct DocsTiled {
  DocsAttn a;
  float exp_scale;  // score -> exponent of 2 without a cap; with one: score -> log2 of e^(2x/cap)
  float cap_log2;   // cap * log2(e)
};
// Visible interval of a lane's row, [at, at + n): empty for rows of no document; and the wave's: some row sees [any0, any1), every row of a document [all0, all1).
struct DocsSeen { int at, n, any0, any1, all0, all1; };
__device__ __forceinline__ DocsSeen docs_seen(bool live, int from, int end) {
  const uint32_t rows = (uint32_t)__ballot(live);  // both halves of a wave hold the same 32 rows
  DocsSeen s = {from, live ? end - from : 0, INT32_MAX, INT32_MIN, INT32_MAX, INT32_MIN};
  if (rows != 0) {
    const int first = __builtin_ctz(rows), last = 31 - __builtin_clz(rows);
    s.any0 = __builtin_amdgcn_readlane(from, first);
    s.any1 = __builtin_amdgcn_readlane(end, last);
    s.all0 = __builtin_amdgcn_readlane(from, last);
    s.all1 = __builtin_amdgcn_readlane(end, first);
  }
  return s;
}
// Per-lane byte offsets as tile_voff, rows clamped to [first, last].
template <int D>
__device__ __forceinline__ void docs_voff(uint32_t (&v)[ATile<D>::IPW], int ld, int wave, int lane, int first, int last) {
  using TL = ATile<D>;
#pragma unroll
  for (int j = 0; j < TL::IPW; j++) {
    const int p = (wave * TL::IPW + j) * 64 + lane;
    const int row = p / TL::CPR, c = (p % TL::CPR) ^ TL::swz(row);
    v[j] = (uint32_t)(((size_t)max(first, min(row, last)) * ld + c * 8) * sizeof(bf16_t));
  }
}
// Moves a tile's lane pointers by a number of bytes, in the same registers: pointers that are formed anew for each tile need their offsets' registers as well, and where these do not
// suffice the offsets come from scratch, in whose counter of loads the next tile's transfer stands ahead of them.
template <int D>
__device__ __forceinline__ void docs_shift(TilePtrs<D>& p, int bytes) {
  auto by = [&](const lds_char*& q) {
    q += bytes;
    asm volatile("" : "+v"(q));
  };
#pragma unroll
  for (int ks = 0; ks < D / 16; ks++) by(p.dir[ks]);
#pragma unroll
  for (int dt = 0; dt < D / 32; dt++) { by(p.t0[dt]); by(p.t1[dt]); }
}
// Whether any of N accumulator tiles holds an infinity or a NaN.  (__builtin_bit_cast of an element of a vector takes the vector's first one: elements are read as numbers.)
template <int N>
__device__ __forceinline__ bool docs_not_finite(const f32x16 (&t)[N]) {
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < N; i++)
#pragma unroll
    for (int r = 0; r < 16; r++) m = max_of(m, __builtin_fabsf(t[i][r]));
  return !(m < INFINITY);
}

// ---- Results that are not finite.  What follows is a wave's own and stands behind its stores: it finds out which of its 32 rows may hold what they do not see, and makes these again.  One
// tile at a time, in the LDS where the rows have left through.  Nothing of it may lengthen the tile loops: lane numbers are taken anew (docs_lane), accumulators are its own.
#define DOCS_ODD 0x7f80u    // bits without the sign from which on a bf16 number is an infinity or a NaN
#define DOCS_LARGE 0x5d80u  // 2^60: products of two smaller ones, summed over a head, are finite
__device__ __forceinline__ int docs_lane() {
  int lane = threadIdx.x & 63;
  asm volatile("" : "+v"(lane));
  return lane;
}
// A scalar taken anew: with more vector arithmetic hanging off the tile loop's own, the compiler keeps those in vector registers, which transfers do not take.
__device__ __forceinline__ int docs_scalar(int x) { return __builtin_amdgcn_readfirstlane(x); }
// 64 rows of D columns from row0 on, clamped to [first, last]; base: their columns of row 0.
struct DocsRows {
  const bf16_t* base;
  size_t ld;
  int first, last;
  __device__ __forceinline__ const bf16_t* row(int i) const { return base + (size_t)max(first, min(i, last)) * ld; }
};
// Bit r: row r of the 64 holds a number of bits `large` or more; holds nothing but infinities and NaNs.
struct DocsOdd { uint64_t some, all; };
template <int D>
__device__ __forceinline__ DocsOdd docs_odd(const DocsRows& rows, int row0, uint32_t large) {
  const uint4* x = reinterpret_cast<const uint4*>(rows.row(row0 + docs_lane()));
  uint32_t top = 0, low = 0x7fffu;
#pragma unroll 2
  for (int c = 0; c < D / 8; c++) {
    const uint4 v = x[c];
    auto word = [&](uint32_t w) {
      const uint32_t a = w & 0x7fffu, b = (w >> 16) & 0x7fffu;
      top = max(top, max(a, b));
      low = min(low, min(a, b));
    };
    word(v.x); word(v.y); word(v.z); word(v.w);
  }
  return {__ballot(top >= large), __ballot(low >= DOCS_ODD)};
}
// Of the 64 rows from row0 on: those in the lane's interval.
__device__ __forceinline__ uint64_t docs_bits(const DocsSeen& see, int row0) {
  const int a = max(see.at - row0, 0), b = min(see.at + see.n - row0, 64);
  return a < b ? (~0ull >> (64 - (b - a))) << a : 0;
}
__device__ __forceinline__ bool docs_masked(const DocsSeen& see, int row0) { return row0 < see.all0 || row0 + AB_KT > see.all1; }
// x where bit `bit` of `seen` is set, else zero, without a comparison (32 of these ahead of their use take more scalar registers than there are).
__device__ __forceinline__ float docs_where(uint32_t seen, int bit, float x) {
  return __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, x) & (uint32_t)__builtin_amdgcn_sbfe((int)seen, bit, 1));
}
// Between accesses to the wave's LDS in different layouts: they stay in order.
__device__ __forceinline__ void docs_wave_order() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_wave_barrier();
}
// f(first row) for the tiles [f0, f1) that some row of the wave sees.
template <class F>
__device__ __forceinline__ void docs_again_tiles(const DocsSeen& see, int f0, int f1, F f) {
#pragma unroll 1
  for (int t = max(f0, see.any0 / AB_KT); t < f1 && t * AB_KT < see.any1; t++) f(t * AB_KT);
}
// 64 rows from row0 on to a tile as a transfer lays it out; clean: zeros in the place of infinities and NaNs.
template <int D>
__device__ __forceinline__ void docs_again_load(char* tile, const DocsRows& rows, int row0, bool clean) {
  using TL = ATile<D>;
  const uint32_t least = clean ? DOCS_ODD : 0x8000u;
  docs_wave_order();
#pragma unroll 2
  for (int i = docs_lane(); i < AB_KT * TL::CPR; i += 64) {
    const int r = i / TL::CPR, c = (i % TL::CPR) * 8;
    uint4 v = *reinterpret_cast<const uint4*>(rows.row(row0 + r) + c);
    auto word = [&](uint32_t w) { return ((w & 0x7fffu) >= least ? 0u : w & 0xffffu) | (((w >> 16) & 0x7fffu) >= least ? 0u : w & 0xffff0000u); };
    v = make_uint4(word(v.x), word(v.y), word(v.z), word(v.w));
    *reinterpret_cast<uint4*>(tile + TL::off(r, c) * 2) = v;
  }
  docs_wave_order();
}
// Score tiles of the 64 rows from row0 on against the lane's own row.
template <int D>
__device__ __forceinline__ void docs_again_scores(f32x16 (&st)[2], char* tile, const DocsRows& rows, int row0, const bf16_t* own, bool valid) {
  docs_again_load<D>(tile, rows, row0, false);
  const int lane = docs_lane(), l32 = lane & 31, kg = lane >> 5;
  bf16x8 b[D / 16];
  load_row_frags<D>(b, own, valid, kg);
#pragma unroll
  for (int mt = 0; mt < 2; mt++)
#pragma unroll
    for (int r = 0; r < 16; r++) st[mt][r] = 0.f;
#pragma unroll
  for (int ks = 0; ks < D / 16; ks++) {
    const lds_char* at = (const lds_char*)tile + ATile<D>::off(l32, ks * 16 + kg * 8) * 2;
    st[0] = MFMA(lds_frag(at, 0), b[ks], st[0]);
    st[1] = MFMA(lds_frag(at, 32 * ATile<D>::LD * 2), b[ks], st[1]);
    __builtin_amdgcn_sched_barrier(0);
  }
}
// acc += rows^T w over 64 rows: w[mt][r] is the lane's weight of row 32 mt + 8 (r / 4) + 4 kg + r % 4.  In a masked tile the infinities and NaNs stay out of the products; those of its
// rows are added to the lanes that see them, one row at a time.
template <int D>
__device__ __forceinline__ void docs_again_add(f32x16 (&acc)[D / 32], const f32x16 (&w)[2], char* tile, const DocsRows& rows, int row0, const DocsSeen& see) {
  uint64_t odd = docs_masked(see, row0) ? docs_odd<D>(rows, row0, DOCS_ODD).some : 0;
  docs_again_load<D>(tile, rows, row0, odd != 0);
  const int lane = docs_lane(), kg = lane >> 5;
  FragAddr<D> fa;
  fa.init(lane);
  const lds_char* sm = (const lds_char*)tile;
#pragma unroll
  for (int g = 0; g < 4; g++) {
    const bf16x8 pf = pack_rows(w[g >> 1], g & 1);
#pragma unroll
    for (int dt = 0; dt < D / 32; dt++) acc[dt] = MFMA(lds_frag_tr(sm + fa.tr0[dt], sm + fa.tr1[dt], g * 16 * ATile<D>::LD * 2), pf, acc[dt]);
    __builtin_amdgcn_sched_barrier(0);
  }
  if (odd == 0) return;
  docs_wave_order();
  float* weights = reinterpret_cast<float*>(tile) + (lane & 31);  // [64 rows][32 lanes], in the place of the tile
#pragma unroll
  for (int mt = 0; mt < 2; mt++)
#pragma unroll
    for (int r = 0; r < 16; r++) weights[(32 * mt + 8 * (r >> 2) + 4 * kg + (r & 3)) * 32] = w[mt][r];
  docs_wave_order();
  const uint64_t seen = docs_bits(see, row0);
#pragma unroll 1
  for (; odd != 0; odd &= odd - 1) {
    const int j = __builtin_ctzll(odd);
    const float x = weights[j * 32];
    const bool on = (seen >> j) & 1;
    const bf16_t* row = rows.row(row0 + j) + 4 * kg;
#pragma unroll
    for (int dt = 0; dt < D / 32; dt++) {
#pragma unroll
      for (int q4 = 0; q4 < 4; q4++) {
        const bf16x4 v = *reinterpret_cast<const bf16x4*>(row + dt * 32 + 8 * q4);
#pragma unroll
        for (int e = 0; e < 4; e++)
          if (on && !__builtin_isfinite((float)v[e])) acc[dt][4 * q4 + e] = fmaf(x, (float)v[e], acc[dt][4 * q4 + e]);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  }
}
// The lane's row (its half of the columns) times f to `to`, float32 or bf16.
template <int D, typename T>
__device__ __forceinline__ void docs_again_out(const f32x16 (&acc)[D / 32], float f, T* to, bool on) {
  to += 4 * (docs_lane() >> 5);
#pragma unroll
  for (int dt = 0; dt < D / 32; dt++)
#pragma unroll
    for (int r = 0; r < 16; r++)
      if (on) to[dt * 32 + 8 * (r >> 2) + (r & 3)] = from_f32<T>(acc[dt][r] * f);
}
// r of a score under the cap, k = exp_scale.
__device__ __forceinline__ float docs_cap_r(float s, float k) { return __builtin_amdgcn_rcpf(1.f + fast_exp2(s * k)); }
// ================================================================================ forward
// The tile's scores become probabilities; running maximum m, sum l and accumulators follow.
template <int D, bool CAP, bool AGAIN>
__device__ __forceinline__ void docs_softmax(const DocsTiled& p, const DocsSeen& see, int kb, int kg, f32x16 (&st)[2], f32x16 (&ot)[D / 32], float& m, float& l) {
  if constexpr (CAP) {
#pragma unroll
    for (int mt = 0; mt < 2; mt++)
#pragma unroll
      for (int r = 0; r < 16; r++) st[mt][r] = docs_cap_r(st[mt][r], p.exp_scale);
  }
  if (docs_masked(see, kb)) {
#pragma unroll
    for (int mt = 0; mt < 2; mt++)
#pragma unroll
      for (int r = 0; r < 16; r++) {
        st[mt][r] = (uint32_t)(kb + mt * 32 + 8 * (r >> 2) + 4 * kg + (r & 3) - see.at) < (uint32_t)see.n ? st[mt][r] : CAP ? INFINITY : -INFINITY;
        if constexpr (AGAIN || (CAP && D == 64)) { if ((r & 3) == 3) __builtin_amdgcn_sched_barrier(0); }  // (32 comparisons ahead of their use take more scalar registers than there are)
      }
  }
  auto larger = [](float a, float b) { return CAP ? min_of(a, b) : max_of(a, b); };  // of the scores: the smaller r
  float mx = larger(st[0][0], st[1][0]);
#pragma unroll
  for (int r = 1; r < 16; r++) mx = larger(mx, larger(st[0][r], st[1][r]));
  mx = larger(mx, __shfl_xor(mx, 32, 64));
  const float scale = CAP ? -2.f * p.cap_log2 : p.exp_scale, mnew = CAP ? fmaf(scale, mx, p.cap_log2) : mx * scale;
  float rs = 0.f;
  if (__any(mnew > m + AF_TAU)) {  // the reference maximum moves where a row's probabilities would grow beyond 2^AF_TAU
    const float mn = max_of(m, mnew);
    const float alpha = fast_exp2(m - mn);
    l *= alpha;
    m = mn;
#pragma unroll
    for (int dt = 0; dt < D / 32; dt++)
#pragma unroll
      for (int r = 0; r < 16; r++) ot[dt][r] *= alpha;
  }
  const float off = CAP ? p.cap_log2 - m : -m;
#pragma unroll
  for (int mt = 0; mt < 2; mt++)
#pragma unroll
    for (int r = 0; r < 16; r++) {
      const float x = fast_exp2(fmaf(st[mt][r], scale, off));
      st[mt][r] = x;
      rs += x;
    }
  rs += __shfl_xor(rs, 32, 64);
  l += rs;
}
// The rows `bad` of a wave again where they may hold what they do not see.  A row whose sum is a NaN has seen one among its scores (each of its results is one) and is not asked for; the
// others are right as they are unless a masked tile holds an infinity or a NaN that they do not see, or a row sees there a key that makes each of its results one or the other.
// q, o, lse: of the wave's first row, part_o, part_ml: likewise, of a unit with a slot.
template <int D, bool CAP>
__device__ __forceinline__ void docs_again_fwd(const DocsTiled& p, const DocsSeen& see, bool bad, const DocsUnit& u, const DocsRows& k, const DocsRows& v, const bf16_t* q, size_t ld, bf16_t* o,
                                               size_t ldo, float* lse, float* part_o, float* part_ml, char* tile) {
  bool arrives = false, none = false;
  docs_again_tiles(see, u.f0, u.f1, [&](int kb) {
    if (!docs_masked(see, kb)) return;
    const DocsOdd odd = docs_odd<D>(v, kb, DOCS_ODD);
    const uint64_t seen = docs_bits(see, kb);
    arrives |= (odd.some & ~seen) != 0;
    none |= (odd.all & seen) != 0;
  });
  const uint64_t rows = __ballot(bad && arrives && !none);
  if (rows == 0) return;
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the first results of these rows, which other lanes have stored, are in place
  const int lane = docs_lane(), r = lane & 31;
  float m = -3.0e38f, l = 0.f;
  f32x16 ot[D / 32];
#pragma unroll
  for (int dt = 0; dt < D / 32; dt++) acc_zero<false>(ot[dt]);
  docs_again_tiles(see, u.f0, u.f1, [&](int kb) {
    f32x16 st[2];
    docs_again_scores<D>(st, tile, k, kb, q + (see.n > 0 ? r : 0) * ld, see.n > 0);
    docs_softmax<D, CAP, true>(p, see, kb, lane >> 5, st, ot, m, l);
    docs_again_add<D>(ot, st, tile, v, kb, see);
  });
  const bool on = ((rows | rows >> 32) >> r) & 1;
  if (u.slot >= 0) {
    docs_again_out<D>(ot, 1.f, part_o + (size_t)r * D, on);
    if (on) { part_ml[r * 2] = m; part_ml[r * 2 + 1] = l; }
  } else {
    docs_again_out<D>(ot, 1.f / l, o + r * ldo, on);
    if (on) lse[r] = (m + log2f(l)) * 0.6931471805599453f;
  }
}
// grid (units * nq)
template <int D, bool CAP>
__global__ __launch_bounds__(AB_THREADS, 2) void attn_docs_fwd_bf16_kernel(const DocsTiled p, const bf16_t* __restrict__ qkv, bf16_t* __restrict__ o, float* __restrict__ lse,
                                                                       float* __restrict__ part_o, float* __restrict__ part_ml) {
  using TL = ATile<D>;
  extern __shared__ __attribute__((aligned(1024))) char smem[];  // K ring, then V ring
  const lds_char* sm = (const lds_char*)smem;
  const DocsView& v = p.a.v;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l32 = lane & 31, kg = lane >> 5;
  const int nq = p.a.nq, nkv = p.a.nkv, h = blockIdx.x % nq, id = blockIdx.x / nq, hk = h / (nq / nkv), ld = (nq + 2 * nkv) * D, T = v.T;
  const DocsUnit u = v.q.units[id];  // fetched beside the head
  if (!docs_fits(v, nq, nkv) || id >= v.head[v.q.counts]) return;
  const int live0 = v.head[DOCS_LIVE0], live1 = v.head[DOCS_LIVE1];
  const int iw = (u.block2 >> 1) * DOCS_BLOCK + wave * 32, iq = iw + l32, row = min(iq, T - 1);
  const bf16_t* kcol = qkv + (size_t)(nq + hk) * D;
  const char* kbase = reinterpret_cast<const char*>(kcol);
  const char* vbase = reinterpret_cast<const char*>(kcol + (size_t)nkv * D);
  const size_t tstride = (size_t)AB_KT * ld * sizeof(bf16_t);
  uint32_t voff[TL::IPW];
  tile_voff<D>(voff, ld, wave, lane, AB_KT);
  const uint32_t ldsK = lds_address(smem), ldsV = ldsK + AF_RING * TL::BYTES;
  auto issue = [&](int t, int slot) {
    const int first = live0 - t * AB_KT, last = live1 - 1 - t * AB_KT;
    if (first <= 0 && last >= AB_KT - 1) {
      tile_dma<D>(kbase + t * tstride, voff, ldsK + slot * TL::BYTES, wave);
      tile_dma<D>(vbase + t * tstride, voff, ldsV + slot * TL::BYTES, wave);
    } else {
      uint32_t vc[TL::IPW];
      docs_voff<D>(vc, ld, wave, lane, max(first, 0), min(last, AB_KT - 1));
      tile_dma<D>(kbase + t * tstride, vc, ldsK + slot * TL::BYTES, wave);
      tile_dma<D>(vbase + t * tstride, vc, ldsV + slot * TL::BYTES, wave);
    }
  };
  issue(u.f0, 0);  // the first tile, the row's table entries and its fragments are on their way together
  const int lo = v.lo[row], hi = v.hi[row], end = max(iq + 1, v.pre[row]);
  bf16x8 qf[D / 16];
  load_row_frags<D>(qf, qkv + (size_t)row * ld + (size_t)h * D, iq < T, kg);
  FragAddr<D> fa;
  fa.init(lane);
  f32x16 ot[D / 32];
  float m = -3.0e38f, l = 0.f;  // finite: a tile that a row does not see leaves it alone
#pragma unroll
  for (int dt = 0; dt < D / 32; dt++)
#pragma unroll
    for (int r = 0; r < 16; r++) ot[dt][r] = 0.f;
  pin_frags(qf);
  const bool live = iq < T && hi > lo;
  const DocsSeen see = docs_seen(live, lo, end);
  int slot = 0;
  for (int t = u.f0; t < u.f1; t++, slot ^= 1) {
    dma_wait<0>();
    __syncthreads();  // tile t is visible; every wave is done with tile t-1, whose slot tile t+1 reuses
    if (t + 1 < u.f1) issue(t + 1, slot ^ 1);
    const int kb = t * AB_KT;
    if (kb >= see.any1 || kb + AB_KT <= see.any0) continue;  // no key of the tile is visible to any row of this wave
    TilePtrs<D> Kp, Vp;
    Kp.set(sm + slot * TL::BYTES, fa);
    Vp.set(sm + (AF_RING + slot) * TL::BYTES, fa);
    f32x16 st[2];
    score_tiles<D>(st, Kp, qf);
    docs_softmax<D, CAP, false>(p, see, kb, kg, st, ot, m, l);
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
  const bool bad = live && docs_not_finite<D / 32>(ot) && l < INFINITY;
  const uint32_t store = (uint32_t)__ballot(live);
  float* prow = part_o + ((size_t)u.slot * nq + h) * DOCS_BLOCK * D + (size_t)wave * 32 * D;
  float* pml = part_ml + (((size_t)u.slot * nq + h) * DOCS_BLOCK + wave * 32) * 2;
  bf16_t* orow = o + (size_t)iw * nq * D + (size_t)h * D;
  float* lrow = lse + (size_t)h * T + iw;
  if (u.slot >= 0) {  // partial result of this unit
    wave_rows_out_f32<D>(
        wave_region<float, D>(smem, wave), lane,
        [&](int dt, int q4) { return f32x4{ot[dt][4 * q4], ot[dt][4 * q4 + 1], ot[dt][4 * q4 + 2], ot[dt][4 * q4 + 3]}; },
        [&](int r) { return (store >> r) & 1 ? prow + (size_t)r * D : nullptr; });
    if (lane < 32 && (store >> lane) & 1) {
      pml[l32 * 2] = m;
      pml[l32 * 2 + 1] = l;
    }
  } else {
    const float inv = 1.0f / l;
    wave_rows_out_bf16<D>(
        wave_region<bf16_t, D>(smem, wave), lane,
        [&](int dt, int q4) { return f32x4{ot[dt][4 * q4] * inv, ot[dt][4 * q4 + 1] * inv, ot[dt][4 * q4 + 2] * inv, ot[dt][4 * q4 + 3] * inv}; },
        [&](int r) { return (store >> r) & 1 ? orow + (size_t)r * nq * D : nullptr; });
    if (lane < 32 && (store >> lane) & 1) lrow[l32] = (m + log2f(l)) * 0.6931471805599453f;
  }
  if (__any(bad)) {
    const int first = docs_scalar(live0), last = docs_scalar(live1) - 1;
    const DocsUnit unit = {0, docs_scalar(u.f0), docs_scalar(u.f1), docs_scalar(u.slot)};
    const DocsRows k = {kcol, (size_t)ld, first, last}, v = {kcol + (size_t)nkv * D, (size_t)ld, first, last};
    docs_again_fwd<D, CAP>(p, see, bad, unit, k, v, qkv + (size_t)iw * ld + (size_t)h * D, ld, orow, (size_t)nq * D, lrow, prow, pml, wave_region<char, D>(smem, wave));
  }
}

// Merges the units of the query blocks that were cut, as attn_fwd_combine_kernel.  grid (8 * blocks that may be cut, nq): 16 rows a block, D/16 columns of a row a thread.
template <int D>
__global__ __launch_bounds__(256) void attn_docs_combine_kernel(const DocsTiled p, const float* __restrict__ part_o, const float* __restrict__ part_ml, bf16_t* __restrict__ o,
                                                                float* __restrict__ lse) {
  const DocsView& v = p.a.v;
  const int nq = p.a.nq, k = blockIdx.x >> 3, h = blockIdx.y;
  const DocsSplit s = v.q.splits[k];
  if (!docs_fits(v, nq, p.a.nkv) || k >= v.head[v.q.counts + 1]) return;
  const int r = (blockIdx.x & 7) * 16 + (threadIdx.x >> 4), i = s.block * DOCS_BLOCK + r;
  if (i >= v.T || v.hi[i] <= v.lo[i]) return;
  constexpr int CPT = D / 16;
  const int c0 = (threadIdx.x & 15) * CPT;
  const size_t unit = ((size_t)s.slot * nq + h) * DOCS_BLOCK + r, step = (size_t)nq * DOCS_BLOCK;  // rows of the first unit's partial result, and to the next unit's
  float M = -3.0e38f;
#pragma unroll 8
  for (int c = 0; c < s.n; c++) M = max_of(M, part_ml[(unit + c * step) * 2]);
  float L = 0.f, acc[CPT];
#pragma unroll
  for (int e = 0; e < CPT; e++) acc[e] = 0.f;
  for (int c = 0; c < s.n; c++) {
    const float lc = part_ml[(unit + c * step) * 2 + 1];
    if (lc == 0.f) continue;  // this unit's tiles hold no key of the row
    const float w = exp2f(part_ml[(unit + c * step) * 2] - M);
    L += w * lc;
    const float* po = part_o + (unit + c * step) * D + c0;
#pragma unroll
    for (int e = 0; e < CPT; e += 4) {
      const f32x4 x = *reinterpret_cast<const f32x4*>(po + e);
      acc[e] += w * x[0]; acc[e + 1] += w * x[1]; acc[e + 2] += w * x[2]; acc[e + 3] += w * x[3];
    }
  }
  const float inv = 1.0f / L;
  bf16_t* orow = o + ((size_t)i * nq + h) * D + c0;
#pragma unroll
  for (int e = 0; e < CPT; e += 4) {
    bf16x4 x = {(bf16_t)(acc[e] * inv), (bf16_t)(acc[e + 1] * inv), (bf16_t)(acc[e + 2] * inv), (bf16_t)(acc[e + 3] * inv)};
    *reinterpret_cast<bf16x4*>(orow + e) = x;
  }
  if (c0 == 0) lse[(size_t)h * v.T + i] = (M + log2f(L)) * 0.6931471805599453f;
}

// ================================================================================ backward: dQ
// The rows `bad` of a wave again, as docs_again_fwd.  A row whose lse is a NaN, or whose delta is not finite, has no finite result at all and is not asked for.  What is masked here is the gradient of a score, so that
// no product over an unseen row counts; products that may pass float32's range are taken for infinities.  q, dout, dq: of the wave's first row, part: likewise, of a unit with a slot.
template <int D, bool CAP>
__device__ __forceinline__ void docs_again_dq(const DocsTiled& p, const DocsSeen& see, bool bad, float l2, float dl, const DocsUnit& u, const DocsRows& k, const DocsRows& v, const bf16_t* q,
                                              size_t ld, const bf16_t* dout, size_t ldo, bf16_t* dq, float* part, float scale, char* tile) {
  const int lane = docs_lane(), r = lane & 31, at = see.n > 0 ? r : 0;
  bool arrives = (docs_odd<D>({dout + at * ldo, 0, 0, 0}, 0, DOCS_LARGE).some >> lane) & 1;
  docs_again_tiles(see, u.f0, u.f1, [&](int kb) {
    if (docs_masked(see, kb)) arrives |= ((docs_odd<D>(k, kb, DOCS_ODD).some | docs_odd<D>(v, kb, DOCS_LARGE).some) & ~docs_bits(see, kb)) != 0;
  });
  const uint64_t rows = __ballot(bad && arrives);
  if (rows == 0) return;
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the first results of these rows, which other lanes have stored, are in place
  f32x16 acc[D / 32];
#pragma unroll
  for (int dt = 0; dt < D / 32; dt++) acc_zero<false>(acc[dt]);
  docs_again_tiles(see, u.f0, u.f1, [&](int kb) {
    f32x16 st[2], dp[2];
    docs_again_scores<D>(st, tile, k, kb, q + at * ld, see.n > 0);
    docs_again_scores<D>(dp, tile, v, kb, dout + at * ldo, see.n > 0);
    const uint64_t seen = docs_bits(see, kb);
#pragma unroll
    for (int mt = 0; mt < 2; mt++)
#pragma unroll
      for (int i = 0; i < 16; i++) {
        float x;
        if constexpr (CAP) {
          const float c = docs_cap_r(st[mt][i], p.exp_scale);
          x = fast_exp2(fmaf(-2.f * p.cap_log2, c, l2)) * fmaf(-c, c, c);
        } else {
          x = fast_exp2(fmaf(st[mt][i], p.exp_scale, -l2));
        }
        st[mt][i] = docs_where((uint32_t)(seen >> (32 * mt)) >> (4 * (lane >> 5)), 8 * (i >> 2) + (i & 3), x * (dp[mt][i] - dl));
      }
    docs_again_add<D>(acc, st, tile, k, kb, see);
  });
  const bool on = ((rows | rows >> 32) >> r) & 1;
  if (u.slot >= 0) docs_again_out<D>(acc, 1.f, part + (size_t)r * D, on);
  else docs_again_out<D>(acc, scale, dq + r * ld, on);
}
// As attn_bwd_dq_block, unit id of head h.  STORE: the first unit of a block also stores its rows' delta and lse2 for the dK/dV launch behind it; otherwise
// attn_docs_prep_kernel has.
#define DOCS_DQ_RING 2
template <int D, bool CAP, bool STORE>
__device__ __forceinline__ void docs_dq_block(const DocsTiled& p, int id, int h, const bf16_t* __restrict__ qkv, const bf16_t* __restrict__ o, const bf16_t* __restrict__ dout,
                                              const float* __restrict__ lse, float* __restrict__ lse2, float* __restrict__ delta, bf16_t* __restrict__ dqkv, float* __restrict__ part) {
  using TL = ATile<D>;
  extern __shared__ __attribute__((aligned(1024))) char smem[];  // K ring, then V ring
  const lds_char* sm = (const lds_char*)smem;
  const DocsView& v = p.a.v;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l32 = lane & 31, kg = lane >> 5;
  const int nq = p.a.nq, nkv = p.a.nkv, hk = h / (nq / nkv), ld = (nq + 2 * nkv) * D, T = v.T;
  const DocsUnit u = v.q.units[id];  // fetched beside the head
  if (!docs_fits(v, nq, nkv) || id >= v.head[v.q.counts]) return;
  const int live0 = v.head[DOCS_LIVE0], live1 = v.head[DOCS_LIVE1];
  const int iw = (u.block2 >> 1) * DOCS_BLOCK + wave * 32, iq = iw + l32, row = min(iq, T - 1);
  const bf16_t* kcol = qkv + (size_t)(nq + hk) * D;
  const char* kbase = reinterpret_cast<const char*>(kcol);
  const char* vbase = reinterpret_cast<const char*>(kcol + (size_t)nkv * D);
  const size_t tstride = (size_t)AB_KT * ld * sizeof(bf16_t);
  uint32_t voff[TL::IPW];
  tile_voff<D>(voff, ld, wave, lane, AB_KT);
  const uint32_t ldsK = lds_address(smem), ldsV = ldsK + DOCS_DQ_RING * TL::BYTES;
  auto issue = [&](int t, int slot) {
    const int first = live0 - t * AB_KT, last = live1 - 1 - t * AB_KT;
    if (first <= 0 && last >= AB_KT - 1) {
      tile_dma<D>(kbase + t * tstride, voff, ldsK + slot * TL::BYTES, wave);
      tile_dma<D>(vbase + t * tstride, voff, ldsV + slot * TL::BYTES, wave);
    } else {
      uint32_t vc[TL::IPW];
      docs_voff<D>(vc, ld, wave, lane, max(first, 0), min(last, AB_KT - 1));
      tile_dma<D>(kbase + t * tstride, vc, ldsK + slot * TL::BYTES, wave);
      tile_dma<D>(vbase + t * tstride, vc, ldsV + slot * TL::BYTES, wave);
    }
  };
  issue(u.f0, 0);  // the first tile, the row's table entries and its fragments are on their way together
  const int lo = v.lo[row], hi = v.hi[row], end = max(iq + 1, v.pre[row]);
  bf16x8 qf[D / 16], dof[D / 16];
  load_row_frags<D>(qf, qkv + (size_t)row * ld + (size_t)h * D, iq < T, kg);
  load_row_frags<D>(dof, dout + ((size_t)row * nq + h) * D, iq < T, kg);
  float l2 = lse[(size_t)h * T + row];
  float dl = 0.f;
  {
    bf16x8 of[D / 16];
    load_row_frags<D>(of, o + ((size_t)row * nq + h) * D, iq < T, kg);
#pragma unroll
    for (int ks = 0; ks < D / 16; ks++)
#pragma unroll
      for (int e = 0; e < 8; e++) dl = fmaf((float)dof[ks][e], (float)of[ks][e], dl);
    dl += __shfl_xor(dl, 32, 64);
  }
  const bool live = iq < T && hi > lo;
  l2 = CAP ? p.cap_log2 - l2 * LOG2E : l2 * LOG2E;  // with a cap: what the exponent adds to the multiple of r
  if (STORE && (u.block2 & 1) && kg == 0 && live) {
    delta[(size_t)h * T + row] = dl;
    lse2[(size_t)h * T + row] = l2;
  }
  const DocsSeen see = docs_seen(live, lo, end);
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
  for (int t = u.f0; t < u.f1; t++, docs_shift<D>(Kp, slot ? -(int)TL::BYTES : (int)TL::BYTES), slot ^= 1) {
    dma_wait<0>();
    __syncthreads();
    if (t + 1 < u.f1) issue(t + 1, slot ^ 1);
    const int kb = t * AB_KT;
    if (kb >= see.any1 || kb + AB_KT <= see.any0) continue;
    f32x16 st[2], dp[2];
    // P^T from S^T beside the dP^T products
    score_tiles2<D, DOCS_DQ_RING * TL::BYTES, 1>(st, Kp, qf, dp, dof, [&](int j) {
      constexpr int N = 32 / (D / 16);
#pragma unroll
      for (int i = 0; i < N; i++) {
        const int x = j * N + i;
        const float s = st[x >> 4][x & 15];
        if constexpr (CAP) {
          const float r = docs_cap_r(s, p.exp_scale);
          st[x >> 4][x & 15] = fast_exp2(fmaf(-2.f * p.cap_log2, r, l2)) * fmaf(-r, r, r);  // times the slope at once: dQ needs no probability by itself
        } else {
          st[x >> 4][x & 15] = fast_exp2(fmaf(s, p.exp_scale, -l2));
        }
      }
    });
    TrFrags<D> fr;
    tr_fetch<D>(fr, Kp, 0);
    if (kb < see.all0 || kb + AB_KT > see.all1) {
#pragma unroll
      for (int mt = 0; mt < 2; mt++)
#pragma unroll
        for (int r = 0; r < 16; r++)
          st[mt][r] = (uint32_t)(kb + mt * 32 + 8 * (r >> 2) + 4 * kg + (r & 3) - see.at) < (uint32_t)see.n ? st[mt][r] : 0.f;
    }
    // dS^T = P^T (dP^T - delta) (P^T with its slope), one quarter (8 registers of a tile) ahead of the products that consume it
    auto ds_quarter = [&](int g) {
#pragma unroll
      for (int r = 8 * (g & 1); r < 8 * (g & 1) + 8; r++) st[g >> 1][r] *= dp[g >> 1][r] - dl;
    };
    ds_quarter(0);
    acc_tile_tr<D, false, false>(dqt, fr, Kp, st, Kp, [&](int g) { if (g + 1 < 4) ds_quarter(g + 1); });
  }
  __syncthreads();
  const bool bad = live && docs_not_finite<D / 32>(dqt) && l2 == l2 && __builtin_isfinite(dl);
  const uint32_t store = (uint32_t)__ballot(live);
  float* prow = part + (((size_t)u.slot * nq + h) * DOCS_BLOCK + wave * 32) * D;
  bf16_t* out = dqkv + (size_t)iw * ld + (size_t)h * D;
  const float scale = CAP ? 4.f * p.a.scale : p.a.scale;
  if (u.slot >= 0) {
    wave_rows_out_f32<D>(
        wave_region<float, D>(smem, wave), lane,
        [&](int dt, int q4) { return f32x4{dqt[dt][4 * q4], dqt[dt][4 * q4 + 1], dqt[dt][4 * q4 + 2], dqt[dt][4 * q4 + 3]}; },
        [&](int r) { return (store >> r) & 1 ? prow + (size_t)r * D : nullptr; });
  } else {
    wave_rows_out_bf16<D>(
        wave_region<bf16_t, D>(smem, wave), lane,
        [&](int dt, int q4) { return f32x4{dqt[dt][4 * q4] * scale, dqt[dt][4 * q4 + 1] * scale, dqt[dt][4 * q4 + 2] * scale, dqt[dt][4 * q4 + 3] * scale}; },
        [&](int r) { return (store >> r) & 1 ? out + (size_t)r * ld : nullptr; });
  }
  if (__any(bad)) {
    const int first = docs_scalar(live0), last = docs_scalar(live1) - 1;
    const DocsUnit unit = {0, docs_scalar(u.f0), docs_scalar(u.f1), docs_scalar(u.slot)};
    const DocsRows k = {kcol, (size_t)ld, first, last}, v = {kcol + (size_t)nkv * D, (size_t)ld, first, last};
    docs_again_dq<D, CAP>(p, see, bad, l2, dl, unit, k, v, qkv + (size_t)iw * ld + (size_t)h * D, ld, dout + ((size_t)iw * nq + h) * D, (size_t)nq * D, out, prow, scale,
                          wave_region<char, D>(smem, wave));
  }
}

// ================================================================================ backward: dK, dV
// The walk of dkv_pinned.
struct DocsWalk {
  DocsSeen see;
  int jk, live0, live1;  // whole tiles begin at live0 .. live1, from the first tile's row on
  __device__ __forceinline__ bool idle(int qb) const { return qb >= see.any1 || qb + AB_KT <= see.any0; }
  __device__ __forceinline__ bool partial(int qb) const { return qb < see.all0 || qb + AB_KT > see.all1; }
  __device__ __forceinline__ uint32_t rows() const { return (uint32_t)see.n; }
  __device__ __forceinline__ bool ragged(int ti) const { return ti * AB_KT < live0 || ti * AB_KT > live1; }
};
// The keys `bad` of a wave again, as docs_again_fwd.  Keys that see a row whose lse is a NaN, or one whose gradient holds nothing but infinities and NaNs, have no finite result at all.
// q, dout, lse2, delta: of the group's first head; k: of the wave's first key, v: so many columns behind; dk: likewise, part: likewise, of a unit with a slot.
template <int D, bool CAP>
__device__ __forceinline__ void docs_again_dkv(const DocsTiled& p, const DocsSeen& see, bool bad, const DocsUnit& u, const DocsSpan& span, const DocsRows& q0, const DocsRows& g0,
                                               const float* lse2, const float* delta, const bf16_t* k, size_t ld, size_t v_off, bf16_t* dk, float* part, float scale, char* tile) {
  const int lane = docs_lane(), r = lane & 31, T = p.a.v.T;
  k += (see.n > 0 ? r : 0) * ld;
  // f(rows of Q, rows of dO, statistics of the head, first row) for every tile of the unit that the wave sees, head after head
  auto tiles = [&](auto f) {
#pragma unroll 1
    for (int h = 0; h * span.n < u.f1; h++) {
      const DocsRows q = {q0.base + h * D, q0.ld, q0.first, q0.last}, g = {g0.base + h * D, g0.ld, g0.first, g0.last};
      docs_again_tiles(see, span.first + max(u.f0 - h * span.n, 0), span.first + min(u.f1 - h * span.n, span.n), [&](int qb) { f(q, g, (size_t)h * T, qb); });
    }
  };
  bool arrives = ((docs_odd<D>({k, 0, 0, 0}, 0, DOCS_LARGE).some | docs_odd<D>({k + v_off, 0, 0, 0}, 0, DOCS_LARGE).some) >> lane) & 1, none = false;
  tiles([&](const DocsRows& q, const DocsRows& g, size_t head, int qb) {
    if (!docs_masked(see, qb)) return;
    const size_t at = head + max(q.first, min(qb + lane, q.last));
    const DocsOdd odd = docs_odd<D>(g, qb, DOCS_LARGE);
    const float sum = lse2[at];
    const uint64_t no_delta = __ballot(!__builtin_isfinite(delta[at])), seen = docs_bits(see, qb);
    arrives |= ((odd.some | docs_odd<D>(q, qb, DOCS_LARGE).some | __ballot(!__builtin_isfinite(sum)) | no_delta) & ~seen) != 0;
    none |= ((odd.all | __ballot(sum != sum)) & seen) != 0;
  });
  const uint64_t rows = __ballot(bad && arrives && !none);
  if (rows == 0) return;
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the first results of these rows, which other lanes have stored, are in place
  const bool on = ((rows | rows >> 32) >> r) & 1;
#pragma unroll 1
  for (int pass = 0; pass < 2; pass++) {  // dV, then dK: both at once take more registers than the tile loop
    f32x16 acc[D / 32];
#pragma unroll
    for (int dt = 0; dt < D / 32; dt++) acc_zero<false>(acc[dt]);
    tiles([&](const DocsRows& q, const DocsRows& g, size_t head, int qb) {
      f32x16 st[2], dp[2];
      docs_again_scores<D>(st, tile, q, qb, k, see.n > 0);
      docs_again_scores<D>(dp, tile, g, qb, k + v_off, see.n > 0);
      docs_wave_order();
      float* stats = reinterpret_cast<float*>(tile);  // in the place of the tile: lse2 of the 64 rows, then delta
      const size_t at = head + max(q.first, min(qb + lane, q.last));
      stats[lane] = lse2[at];
      stats[64 + lane] = delta[at];
      docs_wave_order();
      const uint64_t seen = docs_bits(see, qb);
#pragma unroll
      for (int mt = 0; mt < 2; mt++)
#pragma unroll
        for (int q4 = 0; q4 < 4; q4++) {
          const uint32_t word = (uint32_t)(seen >> (32 * mt)) >> (4 * (lane >> 5));
          const float* of = stats + 32 * mt + 8 * q4 + 4 * (lane >> 5);
          const f32x4 sums = *reinterpret_cast<const f32x4*>(of), deltas = *reinterpret_cast<const f32x4*>(of + 64);
#pragma unroll
          for (int e = 0; e < 4; e++) {
            float x, slope = 1.f;
            if constexpr (CAP) {
              const float c = docs_cap_r(st[mt][4 * q4 + e], p.exp_scale);
              x = fast_exp2(fmaf(-2.f * p.cap_log2, c, sums[e]));
              slope = fmaf(-c, c, c);
            } else {
              x = fast_exp2(fmaf(st[mt][4 * q4 + e], p.exp_scale, -sums[e]));
            }
            st[mt][4 * q4 + e] = docs_where(word, 8 * q4 + e, pass == 0 ? x : x * (dp[mt][4 * q4 + e] - deltas[e]) * slope);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      docs_again_add<D>(acc, st, tile, pass == 0 ? g : q, qb, see);
    });
    const int column = pass == 0 ? D : 0;
    if (u.slot >= 0) docs_again_out<D>(acc, pass == 0 ? 1.f : scale, part + (size_t)r * (2 * D) + column, on);
    else docs_again_out<D>(acc, pass == 0 ? 1.f : scale, dk + r * ld + (pass == 0 ? v_off : 0), on);
  }
}
// As attn_bwd_dkv_block, at D = 128 without a cap with its pinned loop, otherwise in phases: a block owns 128 keys of a key/value head and walks the query tiles of the group's heads, one head after the other.  Unit id of key/value head hk.
template <int D, bool CAP>
__device__ __forceinline__ void docs_dkv_block(const DocsTiled& p, int id, int hk, const bf16_t* __restrict__ qkv, const bf16_t* __restrict__ dout,
                                               const float* __restrict__ lse2, const float* __restrict__ delta, bf16_t* __restrict__ dqkv, float* __restrict__ part) {
  using TL = ATile<D>;
  constexpr bool AGPR = D == 128, PINNED = D == 128 && !CAP;
  extern __shared__ __attribute__((aligned(1024))) char smem[];  // Q ring, dO ring, lse2 ring, delta ring
  const lds_char* sm = (const lds_char*)smem;
  const DocsView& v = p.a.v;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l32 = lane & 31, kg = lane >> 5;
  const int nq = p.a.nq, nkv = p.a.nkv, grp = nq / nkv, hq = hk * grp, ld = (nq + 2 * nkv) * D, ldo = nq * D, T = v.T;
  const DocsUnit u = v.k.units[id];  // fetched beside the head
  const DocsSpan span = v.k.spans[id];
  if (!docs_fits(v, nq, nkv) || id >= v.head[v.k.counts]) return;
  const int live0 = v.head[DOCS_LIVE0], live1 = v.head[DOCS_LIVE1];
  const int jw = (u.block2 >> 1) * DOCS_BLOCK + wave * 32, jk = jw + l32, row = min(jk, T - 1);
  const bf16_t* kcol = qkv + (size_t)(nq + hk) * D;
  const int q0 = span.first * AB_KT;  // tiles are counted from here
  const char* qbase = reinterpret_cast<const char*>(qkv + (size_t)q0 * ld + (size_t)hq * D);
  const char* obase = reinterpret_cast<const char*>(dout + (size_t)q0 * ldo + (size_t)hq * D);
  float* lse_s = reinterpret_cast<float*>(smem + 2 * AB_RING * TL::BYTES);
  float* del_s = lse_s + AB_RING * AB_KT;
  uint32_t vq[TL::IPW], vo[TL::IPW];
  tile_voff<D>(vq, ld, wave, lane, AB_KT);
  tile_voff<D>(vo, ldo, wave, lane, AB_KT);
#pragma unroll
  for (int j = 0; j < TL::IPW; j++) { vq[j] -= j * 1024; vo[j] -= j * 1024; }  // for tile_dma_at: transfer j moves rows from 512 j / D on, of at least 2 D bytes
  const uint32_t ldsQ = lds_address(smem), ldsO = ldsQ + AB_RING * TL::BYTES;
  const int nt = span.n, f0 = u.f0, f1 = u.f1;
  const size_t qstride = (size_t)AB_KT * ld * sizeof(bf16_t), ostride = (size_t)AB_KT * ldo * sizeof(bf16_t);
  int gi = f0 / nt, ti = f0 - gi * nt;  // head of the group and tile to transfer next
  int tc = ti;                          // tile to work off next
  const uint32_t ldsS = ldsQ + 2 * AB_RING * TL::BYTES + (wave & 1) * AB_RING * AB_KT * sizeof(float);  // even waves transfer lse2, odd ones delta
  const float* srow = ((wave & 1) ? delta : lse2) + (size_t)hq * T + q0;
  auto issue = [&](int slot) {
    const int first = max(0, live0 - q0 - ti * AB_KT), last = min(AB_KT - 1, live1 - 1 - q0 - ti * AB_KT);
    const char* qp = qbase + ti * qstride + gi * (D * sizeof(bf16_t));
    const char* op = obase + ti * ostride + gi * (D * sizeof(bf16_t));
    if (first == 0 && last == AB_KT - 1) {
      tile_dma_at<D>(qp, vq, ldsQ + slot * TL::BYTES, wave);
      tile_dma_at<D>(op, vo, ldsO + slot * TL::BYTES, wave);
    } else {
      uint32_t vc[TL::IPW];
      docs_voff<D>(vc, ld, wave, lane, first, last);
      tile_dma<D>(qp, vc, ldsQ + slot * TL::BYTES, wave);
      docs_voff<D>(vc, ldo, wave, lane, first, last);
      tile_dma<D>(op, vc, ldsO + slot * TL::BYTES, wave);
    }
    dma4_base(srow + (size_t)gi * T + (size_t)ti * AB_KT, (uint32_t)(max(first, min(lane, last)) * sizeof(float)), ldsS + slot * AB_KT * sizeof(float));
    if (++ti == nt) { ti = 0; gi++; }
  };
  if constexpr (!PINNED) issue(0);  // the first tile, the key's table entries and its fragments are on their way together
  const int lo = v.lo[row], end = v.hi[row], pre = v.pre[row];
  bf16x8 kf[D / 16], vf[D / 16];
  load_row_frags<D>(kf, kcol + (size_t)row * ld, jk < T, kg);
  load_row_frags<D>(vf, kcol + (size_t)row * ld + (size_t)nkv * D, jk < T, kg);
  f32x16 dkt[D / 32], dvt[D / 32];
#pragma unroll
  for (int dt = 0; dt < D / 32; dt++) { acc_zero<AGPR>(dkt[dt]); acc_zero<AGPR>(dvt[dt]); }
  FragAddr<D> fa;
  fa.init(lane);
  pin_frags(kf);
  pin_frags(vf);
  const bool live = jk < T && end > lo;
  const int from = jk < pre ? lo : jk;
  const DocsSeen see = docs_seen(live, from, end);
  if constexpr (PINNED) {
    const DocsWalk walk = {see, see.at, live0 - q0, live1 - q0 - AB_KT};
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
      if (qb >= see.any1 || qb + AB_KT <= see.any0) continue;  // no query of the tile sees any key of this wave
      TilePtrs<D> Qp, Op;
      Qp.set(sm + slot * TL::BYTES, fa);
      Op.set(sm + (AB_RING + slot) * TL::BYTES, fa);
      const float* ls = lse_s + slot * AB_KT;
      const float* ds = del_s + slot * AB_KT;
      // With slopes besides, statistics are read where they are used: 248 registers let two blocks share a unit, 277 did not (5000 rows on 16:4 heads 360 us, 272 this way).
      constexpr bool LATE = CAP && D == 64;
      f32x4 lv[LATE ? 1 : 8];  // rows 32*mt + 8*q4 + 4*kg + e of the tile at [4*mt + q4]
      if constexpr (!LATE) {
#pragma unroll
        for (int x = 0; x < 8; x++) lv[x] = *reinterpret_cast<const f32x4*>(ls + 8 * x + 4 * kg);
      }
      f32x16 st[2], dp[2], slope[CAP ? 2 : 1];
      // P from S beside the dP products
      score_tiles2<D, AB_RING * TL::BYTES, 3>(st, Qp, kf, dp, vf, [&](int j) {
        constexpr int N = 8 / (D / 16) > 0 ? 8 / (D / 16) : 1;
#pragma unroll
        for (int i = 0; i < N; i++) {
          const int x = j * N + i, mt = x >> 2, q4 = x & 3;
          if constexpr (LATE) lv[0] = *reinterpret_cast<const f32x4*>(ls + 8 * x + 4 * kg);
#pragma unroll
          for (int e = 0; e < 4; e++) {
            const float s = st[mt][4 * q4 + e];
            if constexpr (CAP) {
              const float r = docs_cap_r(s, p.exp_scale);
              st[mt][4 * q4 + e] = fast_exp2(fmaf(-2.f * p.cap_log2, r, lv[LATE ? 0 : x][e]));
              slope[mt][4 * q4 + e] = fmaf(-r, r, r);
            } else {
              st[mt][4 * q4 + e] = fast_exp2(fmaf(s, p.exp_scale, -lv[x][e]));
            }
          }
        }
      });
      TrFrags<D> fr;
      tr_fetch<D>(fr, Op, 0);
      if constexpr (!LATE) {
#pragma unroll
        for (int x = 0; x < 8; x++) lv[x] = *reinterpret_cast<const f32x4*>(ds + 8 * x + 4 * kg);
      }
      if (qb < see.all0 || qb + AB_KT > see.all1) {
        const int first = qb + 4 * kg - see.at;
#pragma unroll
        for (int mt = 0; mt < 2; mt++)
#pragma unroll
          for (int r = 0; r < 16; r++) {
            st[mt][r] = (uint32_t)(first + mt * 32 + 8 * (r >> 2) + (r & 3)) < (uint32_t)see.n ? st[mt][r] : 0.f;
            if ((r & 3) == 3) __builtin_amdgcn_sched_barrier(0);
          }
      }
      acc_tile_tr<D, true, AGPR>(dvt, fr, Op, st, Qp, [&](int g) {
#pragma unroll
        for (int r = 8 * (g & 1); r < 8 * (g & 1) + 8; r++) {
          if constexpr (LATE) { if ((r & 3) == 0) lv[0] = *reinterpret_cast<const f32x4*>(ds + 8 * (4 * (g >> 1) + (r >> 2)) + 4 * kg); }
          st[g >> 1][r] *= dp[g >> 1][r] - lv[LATE ? 0 : 4 * (g >> 1) + (r >> 2)][r & 3];
          if constexpr (CAP) st[g >> 1][r] *= slope[g >> 1][r];
        }
      });
      acc_tile_tr<D, false, AGPR>(dkt, fr, Qp, st, Qp, [](int) {});
    }
  }
  acc_settle<AGPR>(dkt);
  acc_settle<AGPR>(dvt);
  __syncthreads();  // every wave is done with the Q/dO rings: their LDS serves the output turn (dK, then dV)
  const bool bad = live && (docs_not_finite<D / 32>(dkt) || docs_not_finite<D / 32>(dvt));
  const uint32_t store = (uint32_t)__ballot(live);
  const float scale = CAP ? 4.f * p.a.scale : p.a.scale;
  auto dk_quad = [&](int dt, int q4) {
    return f32x4{dkt[dt][4 * q4] * scale, dkt[dt][4 * q4 + 1] * scale, dkt[dt][4 * q4 + 2] * scale, dkt[dt][4 * q4 + 3] * scale};
  };
  auto dv_quad = [&](int dt, int q4) { return f32x4{dvt[dt][4 * q4], dvt[dt][4 * q4 + 1], dvt[dt][4 * q4 + 2], dvt[dt][4 * q4 + 3]}; };
  float* prow = part + (((size_t)u.slot * nkv + hk) * DOCS_BLOCK + wave * 32) * (2 * D);
  bf16_t* out = dqkv + (size_t)jw * ld + (size_t)(nq + hk) * D;
  if (u.slot >= 0) {
    float* reg = wave_region<float, D>(smem, wave);
    wave_rows_out_f32<D>(reg, lane, dk_quad, [&](int r) { return (store >> r) & 1 ? prow + (size_t)r * (2 * D) : nullptr; });
    __builtin_amdgcn_wave_barrier();
    wave_rows_out_f32<D>(reg, lane, dv_quad, [&](int r) { return (store >> r) & 1 ? prow + (size_t)r * (2 * D) + D : nullptr; });
  } else {
    bf16_t* reg = wave_region<bf16_t, D>(smem, wave);
    wave_rows_out_bf16<D>(reg, lane, dk_quad, [&](int r) { return (store >> r) & 1 ? out + (size_t)r * ld : nullptr; });
    __builtin_amdgcn_wave_barrier();
    wave_rows_out_bf16<D>(reg, lane, dv_quad, [&](int r) { return (store >> r) & 1 ? out + (size_t)r * ld + (size_t)nkv * D : nullptr; });
  }
  if (__any(bad)) {
    const int first = docs_scalar(live0), last = docs_scalar(live1) - 1, h0 = docs_scalar(hq), key = docs_scalar(jw);
    const DocsUnit unit = {0, docs_scalar(u.f0), docs_scalar(u.f1), docs_scalar(u.slot)};
    const DocsSpan run = {docs_scalar(span.first), docs_scalar(span.n), 0, 0};
    const DocsRows q = {qkv + (size_t)h0 * D, (size_t)ld, first, last}, g = {dout + (size_t)h0 * D, (size_t)ldo, first, last};
    docs_again_dkv<D, CAP>(p, see, bad, unit, run, q, g, lse2 + (size_t)h0 * T, delta + (size_t)h0 * T, qkv + (size_t)key * ld + (size_t)(nq + docs_scalar(hk)) * D, ld, (size_t)nkv * D, out, prow,
                           scale, wave_region<char, D>(smem, wave));
  }
}

// Delta and lse2 (with a cap: cap_log2 - lse2) of every row of a document, as attn_bwd_prep_kernel: the numbers the dQ blocks use.  Like these it stores nothing if the table
// was made for other sizes; the table's entries are fetched beside the rows.
template <int D, bool CAP>
__global__ __launch_bounds__(64) void attn_docs_prep_kernel(const DocsTiled p, const bf16_t* __restrict__ o, const bf16_t* __restrict__ dout, const float* __restrict__ lse, float* __restrict__ lse2,
                                                            float* __restrict__ delta) {
  const DocsView& v = p.a.v;
  const int T = v.T, nq = p.a.nq;
  const size_t i = (size_t)blockIdx.x * 32 + (threadIdx.x >> 1);
  if (i >= (size_t)T * nq) return;
  const int kg = threadIdx.x & 1, h = (int)(i % nq);
  const size_t t = i / nq, at = (size_t)h * T + t;
  const bf16_t* orow = o + (t * nq + h) * D + kg * 8;
  const bf16_t* drow = dout + (t * nq + h) * D + kg * 8;
  const float l = lse[at] * LOG2E;
  const bool ours = docs_fits(v, nq, p.a.nkv) & (v.hi[t] > v.lo[t]);
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
  if (kg == 0 && ours) {
    delta[at] = half + other;
    lse2[at] = CAP ? p.cap_log2 - l : l;
  }
}
// The two as launches of their own (dQ first: it stores the rows' statistics that the dK/dV blocks read), grids (units * nq) and (units * nkv) ...
template <int D, bool CAP>
__global__ __launch_bounds__(AB_THREADS, 2) void attn_docs_dq_bf16_kernel(const DocsTiled p, const bf16_t* __restrict__ qkv, const bf16_t* __restrict__ o, const bf16_t* __restrict__ dout,
                                                                      const float* __restrict__ lse, float* __restrict__ lse2, float* __restrict__ delta, bf16_t* __restrict__ dqkv,
                                                                      float* __restrict__ part) {
  docs_dq_block<D, CAP, true>(p, blockIdx.x / p.a.nq, blockIdx.x % p.a.nq, qkv, o, dout, lse, lse2, delta, dqkv, part);
}
template <int D, bool CAP>
__global__ __launch_bounds__(AB_THREADS) void attn_docs_dkv_bf16_kernel(const DocsTiled p, const bf16_t* __restrict__ qkv, const bf16_t* __restrict__ dout,
                                                                        const float* __restrict__ lse2, const float* __restrict__ delta, bf16_t* __restrict__ dqkv,
                                                                        float* __restrict__ part) {
  docs_dkv_block<D, CAP>(p, blockIdx.x / p.a.nkv, blockIdx.x % p.a.nkv, qkv, dout, lse2, delta, dqkv, part);
}
// ... and as one, behind attn_docs_prep_kernel, for grids that leave units of the chip idle: dK/dV units (the longer ones) first.  grid (units_k * nkv + units_q * nq)
template <int D, bool CAP>
__global__ __launch_bounds__(AB_THREADS) void attn_docs_bwd_bf16_kernel(const DocsTiled p, const bf16_t* __restrict__ qkv, const bf16_t* __restrict__ o, const bf16_t* __restrict__ dout,
                                                                        const float* __restrict__ lse, float* __restrict__ lse2, float* __restrict__ delta, bf16_t* __restrict__ dqkv,
                                                                        float* __restrict__ part_q, float* __restrict__ part_kv) {
  const DocsView& v = p.a.v;
  const int nq = p.a.nq, nkv = p.a.nkv;
  // the units there are, not the room for them: blocks without work between the two kinds would hold up the second (17 documents in 4096 rows on 4:1 heads 40.6 -> 38.9 us, 1000 rows of 8 heads 29.3 -> 28.2)
  const unsigned n_k = (unsigned)min(max(v.head[v.k.counts], 0), v.k.cap.units) * nkv;
  if (blockIdx.x < n_k) {
    docs_dkv_block<D, CAP>(p, blockIdx.x / nkv, blockIdx.x % nkv, qkv, dout, lse2, delta, dqkv, part_kv);
  } else {
    const int id = (blockIdx.x - n_k) / nq;
    if (id < v.q.cap.units) docs_dq_block<D, CAP, false>(p, id, (blockIdx.x - n_k) % nq, qkv, o, dout, lse, lse2, delta, dqkv, part_q);
  }
}

// Adds the units of the blocks that were cut, in order: rows of dQ (scaled here) and of [dK | dV].  The first nb_q blocks are (16 * blocks that may be cut, nq) of dQ, 8 rows
// each; the rest (32 * blocks, nkv) of dK/dV, 4 rows each.
template <int D>
__global__ __launch_bounds__(256) void attn_docs_reduce_kernel(const DocsTiled p, const float* __restrict__ part_q, const float* __restrict__ part_kv, bf16_t* __restrict__ dqkv, unsigned nb_q,
                                                               unsigned gqx, unsigned gkx) {
  const DocsView& v = p.a.v;
  const int nq = p.a.nq, nkv = p.a.nkv, ld = (nq + 2 * nkv) * D;
  unsigned id = blockIdx.x;
  const bool q = id < nb_q;
  if (!q) id -= nb_q;
  const unsigned gx = q ? gqx : gkx, x = id % gx;
  const int h = id / gx, k = q ? x >> 4 : x >> 5, r0 = q ? (x & 15) * 8 : (x & 31) * 4, width = q ? D : 2 * D, heads = q ? nq : nkv;
  const DocsList& list = q ? v.q : v.k;
  const DocsSplit s = list.splits[k];
  if (!docs_fits(v, nq, nkv) || k >= v.head[list.counts + 1]) return;
  const float* part = q ? part_q : part_kv;
  const size_t unit = ((size_t)s.slot * heads + h) * DOCS_BLOCK, step = (size_t)heads * DOCS_BLOCK * width;
  const int e = threadIdx.x, row = r0 + e / (width / 4), c4 = (e % (width / 4)) * 4, i = s.block * DOCS_BLOCK + row;
  if (row >= r0 + (q ? 8 : 4) || i >= v.T || v.hi[i] <= v.lo[i]) return;
  f32x4 t = {0.f, 0.f, 0.f, 0.f};
  const float* from = part + (unit + row) * width + c4;
#pragma unroll 8
  for (int c = 0; c < s.n; c++) t += __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(from + c * step));
  const float f = !q ? 1.f : p.a.cap > 0.f ? 4.f * p.a.scale : p.a.scale;
  bf16x4 out = {(bf16_t)(t[0] * f), (bf16_t)(t[1] * f), (bf16_t)(t[2] * f), (bf16_t)(t[3] * f)};
  bf16_t* dst = dqkv + (size_t)i * ld + (q ? (size_t)h * D + c4 : c4 < D ? (size_t)(nq + h) * D + c4 : (size_t)(nq + nkv + h) * D + (c4 - D));
  *reinterpret_cast<bf16x4*>(dst) = out;
}

// ------------------------------------------------------------------------------------ host side
static DocsTiled docs_tiled(const DocsAttn& a) {
  const double log2e = 1.4426950408889634;
  return {a, (float)(a.cap > 0.f ? 2.0 * log2e / sqrt((double)a.d) / a.cap : log2e / sqrt((double)a.d)), (float)(a.cap * log2e)};
}

size_t dh_attn_docs_fwd_bf16_ws_bytes(int T, int nq, int nkv, int d) {
  return (size_t)docs_view(nullptr, T, nq, nkv, d, false).q.cap.slots * nq * DOCS_BLOCK * ((size_t)d + 2) * sizeof(float);
}

template <int D, bool CAP>
static int docs_fwd(const DocsTiled& p, const bf16_t* qkv, bf16_t* o, float* lse, float* ws, hipStream_t stream) {
  static bool ready[DH_MAX_DEVICES] = {};
  const size_t lds = 2 * AF_RING * (size_t)ATile<D>::BYTES;
  bool& set = ready[dh_device_index()];
  if (!set) {
    if (int rc = set_lds(attn_docs_fwd_bf16_kernel<D, CAP>, lds)) return rc;
    set = true;
  }
  const DocsCaps& q = p.a.v.q.cap;
  float* part_ml = ws + (size_t)q.slots * p.a.nq * DOCS_BLOCK * D;
  attn_docs_fwd_bf16_kernel<D, CAP><<<(unsigned)q.units * p.a.nq, AB_THREADS, lds, stream>>>(p, qkv, o, lse, ws, part_ml);
  DH_LAUNCH_CHECK();
  if (q.splits > 0) {
    attn_docs_combine_kernel<D><<<dim3(8 * q.splits, p.a.nq), 256, 0, stream>>>(p, ws, part_ml, o, lse);
    DH_LAUNCH_CHECK();
  }
  return DH_OK;
}
int dh_launch_attn_docs_fwd_bf16(const DocsAttn& a, const bf16_t* qkv, bf16_t* o, float* lse, void* ws, size_t, hipStream_t stream) {
  const DocsTiled p = docs_tiled(a);
  if (a.d == 128) return a.cap > 0.f ? docs_fwd<128, true>(p, qkv, o, lse, (float*)ws, stream) : docs_fwd<128, false>(p, qkv, o, lse, (float*)ws, stream);
  return a.cap > 0.f ? docs_fwd<64, true>(p, qkv, o, lse, (float*)ws, stream) : docs_fwd<64, false>(p, qkv, o, lse, (float*)ws, stream);
}

struct DocsBwdLayout { size_t lse2, dkv, dq, total; };
static DocsBwdLayout docs_bwd_layout(const DocsView& v, int nq, int nkv, int d) {
  DocsBwdLayout l;
  size_t at = 0;
  l.lse2 = at; at += dh_align_up((size_t)nq * v.T * sizeof(float), 256);
  l.dkv = at; at += (size_t)v.k.cap.slots * nkv * DOCS_BLOCK * 2 * d * sizeof(float);
  l.dq = at; at += (size_t)v.q.cap.slots * nq * DOCS_BLOCK * d * sizeof(float);
  l.total = at;
  return l;
}
size_t dh_attn_docs_bwd_bf16_ws_bytes(int T, int nq, int nkv, int d) { return docs_bwd_layout(docs_view(nullptr, T, nq, nkv, d, true), nq, nkv, d).total; }

template <int D, bool CAP>
static int docs_bwd(const DocsTiled& p, const bf16_t* qkv, const bf16_t* o, const bf16_t* dout, const float* lse, bf16_t* dqkv, float* delta, char* ws, hipStream_t stream) {
  static bool ready[DH_MAX_DEVICES] = {};
  const size_t lds_dq = 2 * DOCS_DQ_RING * (size_t)ATile<D>::BYTES, lds_dkv = 2 * AB_RING * ((size_t)ATile<D>::BYTES + AB_KT * sizeof(float));
  bool& set = ready[dh_device_index()];
  if (!set) {
    if (int rc = set_lds(attn_docs_dq_bf16_kernel<D, CAP>, lds_dq)) return rc;
    if (int rc = set_lds(attn_docs_dkv_bf16_kernel<D, CAP>, lds_dkv)) return rc;
    if (int rc = set_lds(attn_docs_bwd_bf16_kernel<D, CAP>, lds_dkv)) return rc;
    set = true;
  }
  const int nq = p.a.nq, nkv = p.a.nkv;
  const DocsCaps &q = p.a.v.q.cap, &k = p.a.v.k.cap;
  const DocsBwdLayout l = docs_bwd_layout(p.a.v, nq, nkv, D);
  float *lse2 = (float*)(ws + l.lse2), *part_kv = (float*)(ws + l.dkv), *part_q = (float*)(ws + l.dq);
  // One launch: the two halves' blocks fill each other's units.  Its blocks have the registers and LDS of dK/dV, so that large grids of dQ blocks, two a unit by themselves, lose
  // more than they gain at D = 128.  us, two launches and one, by blocks: D = 128: 128 (1000 rows of 8 heads) 41 and 28, 512 (4096 rows of 8) 68 and 57, 768 (8:4 x 8192) 157 and 147,
  // 960 (16:4 x 6144) 262 and 261, 1024 (8 x 8192) 149 and 151, capped 174 and 184, 1536 (8:4 x 16384) 1763 and 1820, 2560 (32:8 x 8192) 691 and 777.  D = 64, where two fit either
  // way: 512 59.2 and 48.4, 1280 240 and 219, 4096 978 and 983; capped 1280 302 and 273, 2500 318 and 296, 4000 433 and 434.
  if (docs_one_launch(p.a.v.T, nq, nkv, D == 128 ? DOCS_ONE_128 : 4 * DOCS_ONE_64)) {
    attn_docs_prep_kernel<D, CAP><<<(unsigned)(((size_t)p.a.v.T * nq + 31) / 32), 64, 0, stream>>>(p, o, dout, lse, lse2, delta);
    DH_LAUNCH_CHECK();
    attn_docs_bwd_bf16_kernel<D, CAP><<<(unsigned)k.units * nkv + (unsigned)q.units * nq, AB_THREADS, lds_dkv, stream>>>(p, qkv, o, dout, lse, lse2, delta, dqkv, part_q, part_kv);
    DH_LAUNCH_CHECK();
  } else {
    attn_docs_dq_bf16_kernel<D, CAP><<<(unsigned)q.units * nq, AB_THREADS, lds_dq, stream>>>(p, qkv, o, dout, lse, lse2, delta, dqkv, part_q);
    DH_LAUNCH_CHECK();
    attn_docs_dkv_bf16_kernel<D, CAP><<<(unsigned)k.units * nkv, AB_THREADS, lds_dkv, stream>>>(p, qkv, dout, lse2, delta, dqkv, part_kv);
    DH_LAUNCH_CHECK();
  }
  const unsigned gqx = 16 * q.splits, gkx = 32 * k.splits, nb_q = gqx * nq, nb_k = gkx * nkv;
  if (nb_q + nb_k > 0) {
    attn_docs_reduce_kernel<D><<<nb_q + nb_k, 256, 0, stream>>>(p, part_q, part_kv, dqkv, nb_q, gqx, gkx);
    DH_LAUNCH_CHECK();
  }
  return DH_OK;
}
int dh_launch_attn_docs_bwd_bf16(const DocsAttn& a, const bf16_t* qkv, const bf16_t* o, const bf16_t* dout, const float* lse, bf16_t* dqkv, float* delta, void* ws, size_t,
                                 hipStream_t stream) {
  const DocsTiled p = docs_tiled(a);
  if (a.d == 128)
    return a.cap > 0.f ? docs_bwd<128, true>(p, qkv, o, dout, lse, dqkv, delta, (char*)ws, stream) : docs_bwd<128, false>(p, qkv, o, dout, lse, dqkv, delta, (char*)ws, stream);
  return a.cap > 0.f ? docs_bwd<64, true>(p, qkv, o, dout, lse, dqkv, delta, (char*)ws, stream) : docs_bwd<64, false>(p, qkv, o, dout, lse, dqkv, delta, (char*)ws, stream);
}
