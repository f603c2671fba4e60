// bf16 linear attention with a decay for each head on the matrix cores, forward and backward.
//
// A row is walked in chunks of 32 tokens.  With S the state before a chunk, r = 0 .. n-1 the tokens of it,
//   o_r = scale sum_{j <= r} lambda^(r-j) (q_r k_j) v_j + scale lambda^(r+1) S^T q_r,      S' = lambda^n S + sum_j lambda^(n-1-j) k_j v_j^T.
// All three gradients are this form again with other rows in the three places: dq from (dout, v, k) and the states S^T; dk from (v, dout, q) and dv from (k, q, dout), walked from the
// end, each summed over the query heads of the group, with the state R = sum of scale q dout^T (whose gradient of the state arrives undecayed: powers r and n-r in the place of r+1 and n-1-r).
//
// A wave owns 32 columns of the state, all D rows of it, in float32 accumulators (so the block of D / 32 waves has the whole state in registers), and the same 32 columns of the results.  All
// products of a chunk then need no exchange between waves: scores are formed by each wave for itself (8 of 26 matrix instructions a chunk at D = 128), transposed, so that they feed the next
// product from the registers they were formed in, and so does the state, rounded to bf16.  The state's row index is permuted (LinFrag) so that its accumulators meet q's fragments as these lie in LDS.
//
// Long rows are cut into pieces that run side by side: a first launch sums each piece's own contribution to the state, a second one carries the states along the pieces, a third makes
// the results.  States that leave the call come from products whose weighted rows are split into three bf16 terms (24 bits: float32's own): EXACT.  Within a piece the state only feeds
// bf16 products, and its weighted rows are rounded once.
//
// Bound by memory: q, k, v, o once, k and v again for the pieces' states.
#include <algorithm>
#include <type_traits>
#include "attn_tiles.h"
#include "dma.h"
#include "linattn.h"

#ifndef LIN_OCC
#define LIN_OCC 2
#endif
#define LC 32  // tokens of a chunk

// One pass in the form above.
struct LinPass {
  const bf16_t *q, *k, *v;  // of the first head
  bf16_t* out;
  int ldq, ldk, ldv, ldo;
  const float* state;       // OUT: before each piece [batch][nkv][pieces][D][D]; otherwise not read
  float* sum;               // !OUT: where the pieces' contributions go, likewise; OUT && EXACT: the state at the end [batch][nkv][D][D] (or nullptr)
  int transposed;           // state is read with its indexes exchanged
};
struct LinArgs {
  LinGeom g;
  int pieces, per;  // per: chunks of a piece
  LinPass pass[3];
};

// Fragments of 32-token tiles.  tr: as FragAddr's transposed reads; tp: the same with bits 2 and 3 of the column exchanged, so that accumulator row 8a + 4b + e (of 16) of a product with it holds
// column 8b + 4a + e, and pack_rows of the accumulators has eight neighbouring columns in a lane, like a direct read.
template <int D>
struct LinFrag {
  int dir[D / 16], tr[2], tp[D / 32][2];
  __device__ __forceinline__ void init(int lane, int wave) {
    using TL = ATile<D>;
    const int l32 = lane & 31, kg = lane >> 5, s = lane & 15, h16 = (lane >> 4) & 1, c = (s & 3) << 2, p = ((s & 1) << 3) | ((s & 2) << 1);
#pragma unroll
    for (int ks = 0; ks < D / 16; ks++) dir[ks] = TL::off(l32, ks * 16 + kg * 8) * 2;
#pragma unroll
    for (int i = 0; i < 2; i++) {
      tr[i] = TL::off(8 * i + 4 * kg + (s >> 2), wave * 32 + h16 * 16 + c) * 2;
#pragma unroll
      for (int dt = 0; dt < D / 32; dt++) tp[dt][i] = TL::off(8 * i + 4 * kg + (s >> 2), dt * 32 + h16 * 16 + p) * 2;
    }
  }
};
__device__ __forceinline__ int lin_row(int dt, int r, int kg) { return 32 * dt + 16 * (r >> 3) + 8 * kg + (r & 7); }  // state row of accumulator register r
__device__ __forceinline__ int lin_token(int c, int e, int kg) { return 16 * c + 8 * (e >> 2) + 4 * kg + (e & 3); }    // token of element e of fragment c

// lambda^m; log2 of lambda may be minus infinity
__device__ __forceinline__ float lin_pow(float l2, int m) { return m == 0 ? 1.f : fast_exp2(l2 * (float)m); }

// GROUPED: the query role is shared by the group's heads and the other two come from each of them (dk, dv and the states R), otherwise the other way
// round.  REV: from the row's end.
template <int D, bool GROUPED, bool REV, bool EXACT, bool OUT>
__device__ __forceinline__ void lin_walk(const LinArgs& a, const LinPass& p, int piece, int hk, int b, char* smem) {
  using TL = ATile<D>;
  constexpr int W = D / 32, KS = D / 16, TILE = LC * D * 2, IPW = 2;
  const lds_char* sm = (const lds_char*)smem;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l32 = lane & 31, kg = lane >> 5;
  const LinGeom& g = a.g;
  const int grp = g.nq / g.nkv, chunks = (g.seq + LC - 1) / LC, c0 = piece * a.per, c1 = min(chunks, c0 + a.per), heads = GROUPED || OUT ? grp : 1;
  const size_t t0 = (size_t)b * g.seq;
  const float l2 = g.log_decay[hk] * LOG2E;
  // LDS: two slots each of Q, K, V tiles.  (A third, with transfers two steps ahead, brings nothing: 131 -> 133 us for 8192 tokens x 32 heads.)
  const uint32_t lds = lds_address(smem);
  uint32_t off[3][IPW];
  auto offsets = [&](uint32_t (&v)[IPW], int ld, int last) {
#pragma unroll
    for (int j = 0; j < IPW; j++) {
      const int x = (wave * IPW + j) * 64 + lane, row = x / TL::CPR, c = (x % TL::CPR) ^ TL::swz(row);
      v[j] = (uint32_t)((min(row, last) * (size_t)ld + c * 8) * sizeof(bf16_t));
    }
  };
  offsets(off[0], p.ldq, LC - 1);
  offsets(off[1], p.ldk, LC - 1);
  offsets(off[2], p.ldv, LC - 1);
  auto transfer = [&](int which, const bf16_t* base, int ld, int head, int chunk, int slot) {
    const char* at = reinterpret_cast<const char*>(base + (t0 + (size_t)chunk * LC) * ld + (size_t)head * D);
    const int last = min(LC, g.seq - chunk * LC) - 1;
    const uint32_t to = lds + (which * 2 + slot) * TILE + wave * IPW * 1024;
    if (last == LC - 1) {
#pragma unroll
      for (int j = 0; j < IPW; j++) dma16_base(at, off[which][j], to + j * 1024);
    } else {
      uint32_t v[IPW];
      offsets(v, ld, last);
#pragma unroll
      for (int j = 0; j < IPW; j++) dma16_base(at, v[j], to + j * 1024);
    }
  };
  const int nc = c1 - c0, steps = nc * heads;
  auto chunk_of = [&](int n) { return REV ? c1 - 1 - n : c0 + n; };
  int in = 0, ih = 0;  // of the step to transfer next
  auto issue = [&]() {
    const int chunk = chunk_of(in), slot_s = (in * heads + ih) & 1, slot_c = in & 1;
    if (OUT && (!GROUPED || ih == 0)) transfer(0, p.q, p.ldq, GROUPED ? hk : hk * grp + ih, chunk, GROUPED ? slot_c : slot_s);
    if (GROUPED || ih == 0) {
      transfer(1, p.k, p.ldk, GROUPED ? hk * grp + ih : hk, chunk, GROUPED ? slot_s : slot_c);
      transfer(2, p.v, p.ldv, GROUPED ? hk * grp + ih : hk, chunk, GROUPED ? slot_s : slot_c);
    }
    if (++ih == heads) { ih = 0; in++; }
  };
  issue();
  LinFrag<D> fa;
  fa.init(lane, wave);
  f32x16 S[W];
  {
    const float* from = OUT ? p.state + (((size_t)b * g.nkv + hk) * a.pieces + piece) * D * D : nullptr;
#pragma unroll
    for (int dt = 0; dt < W; dt++)
#pragma unroll
      for (int r = 0; r < 16; r++) {
        const int x = lin_row(dt, r, kg), y = wave * 32 + l32;
        S[dt][r] = OUT && p.state ? from[p.transposed ? (size_t)y * D + x : (size_t)x * D + y] : 0.f;
      }
  }
  // powers: of a score, of the state a token reads, of a row on its way into the state (fragment 1; fragment 0 of a whole chunk: 16 tokens further from the end, or nearer)
  const float f_score = g.scale, f_read = GROUPED ? 1.f : g.scale, f_in = GROUPED ? g.scale : 1.f;
  float weight[OUT ? 16 : 1], into[2][8], whole, read;
  uint32_t seen;
  auto powers = [&](int left) {  // of a chunk of so many tokens: rows behind them are copies of the last one, which count for nothing
    seen = 0;
#pragma unroll
    for (int r = 0; r < 16; r++) {
      const int j = lin_token(r >> 3, r & 7, kg);
      seen |= (REV ? j >= l32 && j < left : j <= l32) ? 1u << r : 0u;
    }
#pragma unroll
    for (int c = 0; c < 2; c++)
#pragma unroll
      for (int e = 0; e < 8; e++) {
        const int t = lin_token(c, e, kg);
        into[c][e] = t < left ? f_in * lin_pow(l2, REV ? 1 + t : left - 1 - t) : 0.f;
      }
    whole = lin_pow(l2, left);
    read = f_read * (REV ? l32 < left ? lin_pow(l2, left - 1 - l32) : 0.f : lin_pow(l2, l32 + 1));
  };
  if constexpr (OUT) {
#pragma unroll
    for (int r = 0; r < 16; r++) weight[r] = f_score * lin_pow(l2, max(0, REV ? lin_token(r >> 3, r & 7, kg) - l32 : l32 - lin_token(r >> 3, r & 7, kg)));
  }
  int known = LC;  // tokens of the chunk that the powers are for
  powers(LC);
  f32x16 ot;
  bf16x8 qf[OUT ? KS : 1];
  int n = 0, h = 0;
  for (int s = 0; s < steps; s++) {
    // this step's tiles are here once the transfers before the last step's stores are through
    if constexpr (OUT && !GROUPED) { if (s > 0) dma_wait<2>(); else dma_wait<0>(); }
    else dma_wait<0>();
    __syncthreads();  // and every wave is done with the step before, whose slots the next one takes
    if (s + 1 < steps) issue();
    const int chunk = chunk_of(n), left = min(LC, g.seq - chunk * LC), slot_s = s & 1, slot_c = n & 1, slot_q = GROUPED ? slot_c : slot_s, slot_k = GROUPED ? slot_s : slot_c;
    const lds_char *Qt = sm + slot_q * TILE, *Kt = sm + (2 + slot_k) * TILE, *Vt = sm + (4 + slot_k) * TILE;
    if (left != known) powers(known = left);
    bf16x8 vf[2];
#pragma unroll
    for (int c = 0; c < 2; c++) vf[c] = lds_frag_tr(Vt + fa.tr[0], Vt + fa.tr[1], c * 16 * TL::LD * 2);
    if constexpr (OUT) {
      if (!GROUPED || h == 0) {
#pragma unroll
        for (int ks = 0; ks < KS; ks++) qf[ks] = lds_frag(Qt + fa.dir[ks], 0);
      }
      // Tokens whose value holds an infinity or a NaN in this wave's columns: a zero times it would reach the tokens that do not see it.  They stay out of the product and are added
      // one by one.
      uint32_t odd = 0;
      bf16x8 vs[2] = {vf[0], vf[1]};
      {
        typedef __attribute__((ext_vector_type(8))) unsigned short u16x8;
        const u16x8 m0 = __builtin_bit_cast(u16x8, vf[0]) & (unsigned short)0x7fff, m1 = __builtin_bit_cast(u16x8, vf[1]) & (unsigned short)0x7fff;
        const u16x8 m = __builtin_elementwise_max(m0, m1);
        const auto m4 = __builtin_elementwise_max(__builtin_shufflevector(m, m, 0, 1, 2, 3), __builtin_shufflevector(m, m, 4, 5, 6, 7));
        const auto m2 = __builtin_elementwise_max(__builtin_shufflevector(m4, m4, 0, 1), __builtin_shufflevector(m4, m4, 2, 3));
        if (__any(m2[0] >= 0x7f80 || m2[1] >= 0x7f80)) {
#pragma unroll
          for (int e = 0; e < 8; e++) {
            const uint64_t x = __ballot(m0[e] >= 0x7f80), y = __ballot(m1[e] >= 0x7f80);
            odd |= ((uint32_t)x ? 1u << lin_token(0, e, 0) : 0) | ((uint32_t)(x >> 32) ? 1u << lin_token(0, e, 1) : 0);
            odd |= ((uint32_t)y ? 1u << lin_token(1, e, 0) : 0) | ((uint32_t)(y >> 32) ? 1u << lin_token(1, e, 1) : 0);
          }
#pragma unroll
          for (int e = 0; e < 8; e++) {
            vs[0][e] = (odd >> lin_token(0, e, kg)) & 1 ? (bf16_t)0.f : vf[0][e];
            vs[1][e] = (odd >> lin_token(1, e, kg)) & 1 ? (bf16_t)0.f : vf[1][e];
          }
        }
      }
      f32x16 st;
#pragma unroll
      for (int r = 0; r < 16; r++) st[r] = 0.f;
      if (!GROUPED || h == 0) {
#pragma unroll
        for (int r = 0; r < 16; r++) ot[r] = 0.f;
#pragma unroll
        for (int ks = 0; ks < KS; ks++) ot = MFMA(pack_rows(S[ks >> 1], ks & 1), qf[ks], ot);
#pragma unroll
        for (int r = 0; r < 16; r++) ot[r] *= read;
      }
#pragma unroll
      for (int ks = 0; ks < KS; ks++) st = MFMA(lds_frag(Kt + fa.dir[ks], 0), qf[ks], st);
#pragma unroll
      for (int r = 0; r < 16; r++)  // what is not seen becomes a zero whatever it is
        st[r] = __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, st[r] * weight[r]) & (uint32_t)__builtin_amdgcn_sbfe((int)seen, r, 1));
      const bf16x8 pf[2] = {pack_rows(st, 0), pack_rows(st, 1)};
      ot = MFMA(vs[0], pf[0], ot);
      ot = MFMA(vs[1], pf[1], ot);
      if (odd != 0) {
#pragma unroll 1
        for (; odd != 0; odd &= odd - 1) {
          const int j = __builtin_ctz(odd);
          bf16x8 v0, v1;
#pragma unroll
          for (int e = 0; e < 8; e++) {
            v0[e] = lin_token(0, e, kg) == j ? vf[0][e] : (bf16_t)0.f;
            v1[e] = lin_token(1, e, kg) == j ? vf[1][e] : (bf16_t)0.f;
          }
          f32x16 add;
#pragma unroll
          for (int r = 0; r < 16; r++) add[r] = 0.f;
          add = MFMA(v0, pf[0], add);
          add = MFMA(v1, pf[1], add);
          const bool here = REV ? j >= l32 : j <= l32;
#pragma unroll
          for (int r = 0; r < 16; r++) ot[r] = here ? ot[r] + add[r] : ot[r];
        }
      }
      if (!GROUPED || h == heads - 1) {  // a lane has a token's columns 8 q4 + 4 kg .. of 32; halves are exchanged so that it stores 16 bytes
        bf16_t* row = p.out + (t0 + (size_t)chunk * LC + l32) * p.ldo + (size_t)(GROUPED ? hk : hk * grp + h) * D + wave * 32 + 8 * kg;
#pragma unroll
        for (int c = 0; c < 2; c++) {
          const uint4 u = __builtin_bit_cast(uint4, pack_rows(ot, c));
          const auto x = __builtin_amdgcn_permlane32_swap(u.x, u.z, false, false);
          const auto y = __builtin_amdgcn_permlane32_swap(u.y, u.w, false, false);
          if (l32 < left) *reinterpret_cast<uint4*>(row + 16 * c) = make_uint4((uint32_t)x[0], (uint32_t)y[0], (uint32_t)x[1], (uint32_t)y[1]);
        }
      }
    }
    if (GROUPED || h == heads - 1) {  // into the state
      if (!GROUPED || h == 0) {
#pragma unroll
        for (int dt = 0; dt < W; dt++)
#pragma unroll
          for (int r = 0; r < 16; r++) S[dt][r] *= whole;
      }
#pragma unroll
      for (int c = 0; c < 2; c++) {
        bf16x8 hi, mid, lo;
#pragma unroll
        for (int e = 0; e < 8; e++) {
          const float x = (float)vf[c][e] * into[c][e];
          hi[e] = (bf16_t)x;
          if constexpr (EXACT) {
            const float y = x - (float)hi[e];
            mid[e] = (bf16_t)y;
            lo[e] = (bf16_t)(y - (float)mid[e]);
          }
        }
#pragma unroll
        for (int dt = 0; dt < W; dt++) {
          const bf16x8 kf = lds_frag_tr(Kt + fa.tp[dt][0], Kt + fa.tp[dt][1], c * 16 * TL::LD * 2);
          S[dt] = MFMA(kf, hi, S[dt]);
          if constexpr (EXACT) {
            S[dt] = MFMA(kf, mid, S[dt]);
            S[dt] = MFMA(kf, lo, S[dt]);
          }
        }
      }
    }
    if (++h == heads) { h = 0; n++; }
  }
  if constexpr (EXACT) {
    if (!p.sum) return;
    float* to = p.sum + (OUT ? ((size_t)b * g.nkv + hk) : ((size_t)b * g.nkv + hk) * a.pieces + piece) * D * D;
#pragma unroll
    for (int dt = 0; dt < W; dt++)
#pragma unroll
      for (int r = 0; r < 16; r++) to[(size_t)lin_row(dt, r, kg) * D + wave * 32 + l32] = S[dt][r];
  }
}

// The forward pass: OUT its results, otherwise the pieces' contributions to the states.  grid (pieces, nkv, batch)
template <int D, bool EXACT, bool OUT>
__global__ __launch_bounds__(2 * D, LIN_OCC) void lin_fwd_kernel(const LinArgs a) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  lin_walk<D, false, false, EXACT, OUT>(a, a.pass[0], blockIdx.x, blockIdx.y, blockIdx.z, smem);
}
// The backward pass: dq, dk and dv (OUT), otherwise the pieces' contributions to S and R.  grid (pieces, nkv * (OUT ? 3 : 2), batch)
template <int D, bool EXACT, bool OUT>
__global__ __launch_bounds__(2 * D, LIN_OCC) void lin_bwd_kernel(const LinArgs a) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const int nkv = a.g.nkv, y = blockIdx.y, b = blockIdx.z;
  if (y < nkv) lin_walk<D, false, false, EXACT && !OUT, OUT>(a, a.pass[0], blockIdx.x, y, b, smem);
  else if (y < 2 * nkv) lin_walk<D, true, true, EXACT && !OUT, OUT>(a, a.pass[1], blockIdx.x, y - nkv, b, smem);
  else if constexpr (OUT) lin_walk<D, true, true, EXACT, OUT>(a, a.pass[2], blockIdx.x, y - 2 * nkv, b, smem);
}
// Carries the states along the pieces: each piece's contribution gives place to the state before it.  REV: from the end, after the same of the S of a backward pass.
// grid (D * D / 1024, nkv * passes, batch), four elements a thread
struct LinCarry { float* sums; const float* first; float* last; int rev; };
template <int D>
__global__ __launch_bounds__(256) void lin_carry_kernel(const LinArgs a, const LinCarry c0, const LinCarry c1) {
  const LinGeom& g = a.g;
  const int b = blockIdx.z, hk = blockIdx.y % g.nkv, e = (blockIdx.x * 256 + threadIdx.x) * 4;
  const LinCarry& c = (int)blockIdx.y >= g.nkv ? c1 : c0;
  const size_t head = (size_t)b * g.nkv + hk;
  const float l2 = g.log_decay[hk] * LOG2E;
  const int len = a.per * LC;
  f32x4 run = {0.f, 0.f, 0.f, 0.f};
  if (c.first) run = *reinterpret_cast<const f32x4*>(c.first + head * D * D + e);
  const float f = lin_pow(l2, len), f_last = lin_pow(l2, g.seq - (a.pieces - 1) * len);
  float* at = c.sums + head * a.pieces * D * D + e;
#pragma unroll 4
  for (int i = 0; i < a.pieces; i++) {
    const int s = c.rev ? a.pieces - 1 - i : i;
    f32x4* x = reinterpret_cast<f32x4*>(at + (size_t)s * D * D);
    const f32x4 sum = *x;
    *x = run;
    const float w = s == a.pieces - 1 ? f_last : f;
    run = run * w + sum;
  }
  if (c.last) *reinterpret_cast<f32x4*>(c.last + head * D * D + e) = run;
}

// ------------------------------------------------------------------------------------ host side
// Pieces of a row: enough that the chip's units have two blocks each, none below LIN_LEAST chunks.
#define LIN_LEAST 4
#ifndef LIN_BLOCKS
#define LIN_BLOCKS 512
#endif
struct LinCut { int pieces, per; };
static LinCut lin_cut(const LinGeom& g, bool bwd) {
  const long long chunks = (g.seq + LC - 1) / LC, blocks = (long long)g.batch * g.nkv * (bwd ? 3 : 1);
  const long long want = std::max(1ll, std::min((LIN_BLOCKS + blocks - 1) / blocks, chunks / LIN_LEAST));
  const int per = (int)((chunks + want - 1) / want);
  return {(int)((chunks + per - 1) / per), per};
}
static size_t lin_states(const LinGeom& g, int pieces) { return (size_t)g.batch * g.nkv * pieces * g.d * g.d; }
size_t dh_linattn_bf16_ws_bytes(const LinGeom& g, bool bwd) {
  const LinCut c = lin_cut(g, bwd);
  return c.pieces == 1 ? 0 : (bwd ? 2 : 1) * lin_states(g, c.pieces) * sizeof(float);
}
template <int D>
static int lin_fwd(const LinGeom& g, const bf16_t* qkv, const float* state_in, bf16_t* o, float* state_out, float* ws, hipStream_t s) {
  const int ld = (g.nq + 2 * g.nkv) * D;
  const LinCut c = lin_cut(g, false);
  LinArgs a = {g, c.pieces, c.per, {}};
  a.pass[0] = {qkv, qkv + (size_t)g.nq * D, qkv + (size_t)(g.nq + g.nkv) * D, o, ld, ld, ld, g.nq * D, state_in, state_out, 0};
  const dim3 grid(c.pieces, g.nkv, g.batch);
  const size_t lds = 6 * LC * D * 2;
  if (c.pieces > 1) {
    a.pass[0].state = nullptr;
    a.pass[0].sum = ws;
    lin_fwd_kernel<D, true, false><<<grid, 2 * D, lds, s>>>(a);
    DH_LAUNCH_CHECK();
    lin_carry_kernel<D><<<dim3(D * D / 1024, g.nkv, g.batch), 256, 0, s>>>(a, {ws, state_in, state_out, 0}, {});
    DH_LAUNCH_CHECK();
    a.pass[0].state = ws;
  } else if (state_out) {
    lin_fwd_kernel<D, true, true><<<grid, 2 * D, lds, s>>>(a);
    DH_LAUNCH_CHECK();
    return DH_OK;
  }
  lin_fwd_kernel<D, false, true><<<grid, 2 * D, lds, s>>>(a);
  DH_LAUNCH_CHECK();
  return DH_OK;
}
int dh_launch_linattn_fwd_bf16(const LinGeom& g, const bf16_t* qkv, const float* state_in, bf16_t* o, float* state_out, void* ws, hipStream_t s) {
  return g.d == 128 ? lin_fwd<128>(g, qkv, state_in, o, state_out, (float*)ws, s) : lin_fwd<64>(g, qkv, state_in, o, state_out, (float*)ws, s);
}
template <int D>
static int lin_bwd(const LinGeom& g, const bf16_t* qkv, const float* state_in, const bf16_t* dout, const float* dstate_out, bf16_t* dqkv, float* dstate_in, float* ws, hipStream_t s) {
  const int ld = (g.nq + 2 * g.nkv) * D, ldo = g.nq * D;
  const size_t kc = (size_t)g.nq * D, vc = kc + (size_t)g.nkv * D;
  const bf16_t *q = qkv, *k = qkv + kc, *v = qkv + vc;
  const LinCut c = lin_cut(g, true);
  LinArgs a = {g, c.pieces, c.per, {}};
  a.pass[0] = {dout, v, k, dqkv, ldo, ld, ld, ld, state_in, nullptr, 1};
  a.pass[1] = {v, dout, q, dqkv + kc, ld, ldo, ld, ld, dstate_out, nullptr, 1};
  a.pass[2] = {k, q, dout, dqkv + vc, ld, ld, ldo, ld, dstate_out, dstate_in, 0};
  const size_t lds = 6 * LC * D * 2;
  const dim3 grid(c.pieces, g.nkv * 3, g.batch);
  if (c.pieces > 1) {
    float* R = ws + lin_states(g, c.pieces);
    LinArgs f = a;
    f.pass[0] = {nullptr, k, v, nullptr, 0, ld, ld, 0, nullptr, ws, 0};
    f.pass[1] = {nullptr, q, dout, nullptr, 0, ld, ldo, 0, nullptr, R, 0};
    lin_bwd_kernel<D, true, false><<<dim3(c.pieces, g.nkv * 2, g.batch), 2 * D, lds, s>>>(f);
    DH_LAUNCH_CHECK();
    lin_carry_kernel<D><<<dim3(D * D / 1024, g.nkv * 2, g.batch), 256, 0, s>>>(a, {ws, state_in, nullptr, 0}, {R, dstate_out, dstate_in, 1});
    DH_LAUNCH_CHECK();
    a.pass[0].state = ws;
    a.pass[1].state = a.pass[2].state = R;
    a.pass[2].sum = nullptr;
  } else if (dstate_in) {
    lin_bwd_kernel<D, true, true><<<grid, 2 * D, lds, s>>>(a);
    DH_LAUNCH_CHECK();
    return DH_OK;
  }
  lin_bwd_kernel<D, false, true><<<grid, 2 * D, lds, s>>>(a);
  DH_LAUNCH_CHECK();
  return DH_OK;
}
int dh_launch_linattn_bwd_bf16(const LinGeom& g, const bf16_t* qkv, const float* state_in, const bf16_t* dout, const float* dstate_out, bf16_t* dqkv, float* dstate_in, void* ws,
                               hipStream_t s) {
  return g.d == 128 ? lin_bwd<128>(g, qkv, state_in, dout, dstate_out, dqkv, dstate_in, (float*)ws, s) : lin_bwd<64>(g, qkv, state_in, dout, dstate_out, dqkv, dstate_in, (float*)ws, s);
}
