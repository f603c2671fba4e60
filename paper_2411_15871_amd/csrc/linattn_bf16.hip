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
// products that take it rounded to bf16, as they take the weighted scores, and its weighted rows go in two terms: with one, errors against 64 bits (relative norms, where the result's own
// rounding makes 1.7e-3) were 2.7e-3 and are 2.3e-3, for 103 and 109 us at 8192 tokens x 32 heads.
//
// Bound by memory: q, k, v, o once, k and v again for the pieces' states.
#include <algorithm>
#include "attn_tiles.h"
#include "dma.h"
#include "linattn.h"


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
  LinPass pass[2];
};
// dk and dv together.
struct LinGrads {
  const bf16_t *qkv, *dout;
  bf16_t* dqkv;
  const float* state;  // R behind each piece
  float* sum;          // EXACT: the gradient of the state before the row (or nullptr)
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


// The lane's number taken anew: what only heads of no memory need is made in their branches and takes no registers of the loops around these.
__device__ __forceinline__ int lin_lane() {
  int lane = threadIdx.x & 63;
  asm volatile("" : "+v"(lane));
  return lane;
}
// The register of a score tile that holds the score of the lane's token (its column) with itself, or -1: the other half of the wave has it.
__device__ __forceinline__ int lin_own(int lane) { return ((lane >> 2) & 1) == lane >> 5 ? 4 * ((lane & 31) >> 3) + (lane & 3) : -1; }

// What a chunk's arithmetic multiplies by.  Powers of lambda: of a score, of the state that a token reads, of a row on its way into the state.  REV: the row is walked from its end.
template <bool REV>
struct LinPowers {
  float weight[16], into[2][8], whole, read;
  bool alone;     // each token sees itself alone
  uint32_t seen;  // bit r: the lane's token sees that of score register r
  int left;       // tokens of the chunk
  __device__ __forceinline__ void scores(float l2, float f, int lane) {
    const int l32 = lane & 31, kg = lane >> 5;
#pragma unroll
    for (int r = 0; r < 16; r++) weight[r] = f * lin_pow(l2, max(0, REV ? lin_token(r >> 3, r & 7, kg) - l32 : l32 - lin_token(r >> 3, r & 7, kg)));
  }
  __device__ __forceinline__ void chunk(int n, float l2, float f_read, float f_in, int lane) {  // rows behind the chunk's n are copies of its last one, which count for nothing
    const int l32 = lane & 31, kg = lane >> 5;
    left = n;
    alone = lin_alone(l2);
    seen = 0;
#pragma unroll
    for (int r = 0; r < 16; r++) {
      const int j = lin_token(r >> 3, r & 7, kg);
      seen |= (REV ? j >= l32 && j < n : j <= l32) ? 1u << r : 0u;
    }
    if (alone) {
      const int own = lin_own(lin_lane());
      seen &= own >= 0 ? 1u << own : 0u;
    }
#pragma unroll
    for (int c = 0; c < 2; c++)
#pragma unroll
      for (int e = 0; e < 8; e++) {
        const int t = lin_token(c, e, kg);
        into[c][e] = t < n ? f_in * lin_pow(l2, REV ? 1 + t : n - 1 - t) : 0.f;
      }
    whole = lin_pow(l2, n);
    read = f_read * (REV ? l32 < n ? lin_pow(l2, n - 1 - l32) : 0.f : lin_pow(l2, l32 + 1));
  }
};
// The values of 32 tokens in a wave's columns, as the matrix instruction takes them.
struct LinValues {
  bf16x8 all[2];
  uint32_t odd;  // tokens that hold an infinity or a NaN, which a zero's product would carry to tokens that do not see them
  __device__ __forceinline__ void load(const lds_char* t0, const lds_char* t1, int row_bytes) {
#pragma unroll
    for (int c = 0; c < 2; c++) all[c] = lds_frag_tr(t0, t1, c * 16 * row_bytes);
  }
  __device__ __forceinline__ void look() {
    typedef __attribute__((ext_vector_type(8))) unsigned short u16x8;
    odd = 0;
    const u16x8 m0 = __builtin_bit_cast(u16x8, all[0]) & (unsigned short)0x7fff, m1 = __builtin_bit_cast(u16x8, all[1]) & (unsigned short)0x7fff;
    const u16x8 m = __builtin_elementwise_max(m0, m1);
    const auto m4 = __builtin_elementwise_max(__builtin_shufflevector(m, m, 0, 1, 2, 3), __builtin_shufflevector(m, m, 4, 5, 6, 7));
    const auto m2 = __builtin_elementwise_max(__builtin_shufflevector(m4, m4, 0, 1), __builtin_shufflevector(m4, m4, 2, 3));
    if (!__any(m2[0] >= 0x7f80 || m2[1] >= 0x7f80)) return;
#pragma unroll
    for (int e = 0; e < 8; e++) {
      const uint64_t x = __ballot(m0[e] >= 0x7f80), y = __ballot(m1[e] >= 0x7f80);
      odd |= ((uint32_t)x ? 1u << lin_token(0, e, 0) : 0) | ((uint32_t)(x >> 32) ? 1u << lin_token(0, e, 1) : 0);
      odd |= ((uint32_t)y ? 1u << lin_token(1, e, 0) : 0) | ((uint32_t)(y >> 32) ? 1u << lin_token(1, e, 1) : 0);
    }
  }
};
__device__ __forceinline__ void lin_zero(f32x16& t) {
#pragma unroll
  for (int r = 0; r < 16; r++) t[r] = 0.f;
}
// ot += values * (weighted scores st); what is not seen becomes a zero whatever it is.
template <bool REV>
__device__ __forceinline__ void lin_inside(f32x16& ot, f32x16& st, const LinPowers<REV>& p, const LinValues& v, int lane) {
  const int l32 = lane & 31, kg = lane >> 5;
#pragma unroll
  for (int r = 0; r < 16; r++)
    st[r] = __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, st[r] * p.weight[r]) & (uint32_t)__builtin_amdgcn_sbfe((int)p.seen, r, 1));
  const bf16x8 pf[2] = {pack_rows(st, 0), pack_rows(st, 1)};
  if (v.odd == 0) {
    ot = MFMA(v.all[0], pf[0], ot);
    ot = MFMA(v.all[1], pf[1], ot);
    return;
  }
  bf16x8 kept[2];  // the others
#pragma unroll
  for (int c = 0; c < 2; c++)
#pragma unroll
    for (int e = 0; e < 8; e++) kept[c][e] = (v.odd >> lin_token(c, e, kg)) & 1 ? (bf16_t)0.f : v.all[c][e];
  ot = MFMA(kept[0], pf[0], ot);
  ot = MFMA(kept[1], pf[1], ot);
#pragma unroll 1
  for (uint32_t odd = v.odd; odd != 0; odd &= odd - 1) {  // token by token, to those that see it
    const int j = __builtin_ctz(odd);
    bf16x8 v0, v1;
#pragma unroll
    for (int e = 0; e < 8; e++) {
      v0[e] = lin_token(0, e, kg) == j ? v.all[0][e] : (bf16_t)0.f;
      v1[e] = lin_token(1, e, kg) == j ? v.all[1][e] : (bf16_t)0.f;
    }
    f32x16 add;
    lin_zero(add);
    add = MFMA(v0, pf[0], add);
    add = MFMA(v1, pf[1], add);
    const bool here = p.alone ? j == l32 : REV ? j >= l32 : j <= l32;
#pragma unroll
    for (int r = 0; r < 16; r++) ot[r] = here ? ot[r] + add[r] : ot[r];
  }
}
// Where a wave does little else (sums of states) fragments are asked for ahead, and what is asked for stays in its place: left to the compiler each is read right before the product that takes it,
// which then waits for LDS.  Elsewhere the waves of a SIMD cover such waits, and registers count for more.
#define LIN_PIN() __builtin_amdgcn_sched_barrier(0)
template <int D>
struct LinRows {  // a tile's transposed fragments of 16 tokens
  bf16x8 f[D / 32];
  __device__ __forceinline__ void load(const LinFrag<D>& fa, const lds_char* rows, int c) {
#pragma unroll
    for (int dt = 0; dt < D / 32; dt++) f[dt] = lds_frag_tr(rows + fa.tp[dt][0], rows + fa.tp[dt][1], c * 16 * D * 2);
  }
};
// S += rows^T * (values on their way into the state), these weighted and taken in TERMS bf16 terms.  PIN: the fragments are in `ahead` already.
template <int D, int TERMS, bool PIN>
__device__ __forceinline__ void lin_into(f32x16 (&S)[D / 32], const LinFrag<D>& fa, const lds_char* rows, const LinRows<D> (&ahead)[2], const bf16x8 (&v)[2], const float (&into)[2][8]) {
#pragma unroll
  for (int c = 0; c < 2; c++) {
    bf16x8 hi, mid, lo;
#pragma unroll
    for (int e = 0; e < 8; e++) {
      const float x = (float)v[c][e] * into[c][e];
      hi[e] = (bf16_t)x;
      if constexpr (TERMS > 1) {
        const float y = x - (float)hi[e];
        mid[e] = (bf16_t)y;
        if constexpr (TERMS > 2) lo[e] = (bf16_t)(y - (float)mid[e]);
      }
    }
    LinRows<D> k;
    if constexpr (PIN) k = ahead[c];
    else k.load(fa, rows, c);
#pragma unroll
    for (int dt = 0; dt < D / 32; dt++) S[dt] = MFMA(k.f[dt], hi, S[dt]);
    if constexpr (TERMS > 1) {
#pragma unroll
      for (int dt = 0; dt < D / 32; dt++) S[dt] = MFMA(k.f[dt], mid, S[dt]);
    }
    if constexpr (TERMS > 2) {
#pragma unroll
      for (int dt = 0; dt < D / 32; dt++) S[dt] = MFMA(k.f[dt], lo, S[dt]);
    }
  }
}
// The state behind tokens that see themselves alone: the last one's k v^T.  (Within the row it stays zero.)
template <int D>
__device__ __forceinline__ void lin_state_alone(f32x16 (&S)[D / 32], const lds_char* Kt, const lds_char* Vt, int last, int wave) {
  using TL = ATile<D>;
  const int lane = lin_lane(), l32 = lane & 31, kg = lane >> 5;
  const float v = (float)*reinterpret_cast<const __attribute__((address_space(3))) bf16_t*>(Vt + (TL::off(last, wave * 32 + (l32 & ~3)) + (l32 & 3)) * 2);
#pragma unroll
  for (int dt = 0; dt < D / 32; dt++)
#pragma unroll
    for (int c = 0; c < 2; c++) {
      const bf16x8 k = lds_frag(Kt + TL::off(last, 32 * dt + 16 * c + 8 * kg) * 2, 0);
#pragma unroll
      for (int e = 0; e < 8; e++) S[dt][8 * c + e] = (float)k[e] * v;
    }
}
// The state a wave begins with (its 32 columns; transposed: of the transposed one), and the one it leaves.
template <int D>
__device__ __forceinline__ void lin_state_load(f32x16 (&S)[D / 32], const float* from, bool transposed, int wave, int lane) {
  const int l32 = lane & 31, kg = lane >> 5, y = wave * 32 + l32;
#pragma unroll
  for (int dt = 0; dt < D / 32; dt++)
#pragma unroll
    for (int r = 0; r < 16; r++) {
      const int x = lin_row(dt, r, kg);
      S[dt][r] = from ? from[transposed ? (size_t)y * D + x : (size_t)x * D + y] : 0.f;
    }
}
template <int D>
__device__ __forceinline__ void lin_state_store(const f32x16 (&S)[D / 32], float* to, int wave, int lane) {
#pragma unroll
  for (int dt = 0; dt < D / 32; dt++)
#pragma unroll
    for (int r = 0; r < 16; r++) to[(size_t)lin_row(dt, r, lane >> 5) * D + wave * 32 + (lane & 31)] = S[dt][r];
}
// A lane has a token's columns 8 q4 + 4 kg .. of 32: halves are exchanged so that it stores 16 bytes twice.  row: of the lane's token, from the wave's columns on.
__device__ __forceinline__ void lin_out(const f32x16& ot, bf16_t* row, bool on, int lane) {
#pragma unroll
  for (int c = 0; c < 2; c++) {
    const uint4 u = __builtin_bit_cast(uint4, pack_rows(ot, c));
    const auto x = __builtin_amdgcn_permlane32_swap(u.x, u.z, false, false);
    const auto y = __builtin_amdgcn_permlane32_swap(u.y, u.w, false, false);
    if (on) *reinterpret_cast<uint4*>(row + 8 * (lane >> 5) + 16 * c) = make_uint4((uint32_t)x[0], (uint32_t)y[0], (uint32_t)x[1], (uint32_t)y[1]);
  }
}
// Transfers of 32-token tiles to LDS, D / 16 KiB a tile, two a wave.
template <int D>
struct LinTransfer {
  static constexpr int TILE = LC * D * 2;
  __device__ static __forceinline__ void offsets(uint32_t (&v)[2], int ld, int last, int wave, int lane) {
    using TL = ATile<D>;
#pragma unroll
    for (int j = 0; j < 2; j++) {
      const int x = (wave * 2 + j) * 64 + lane, row = x / TL::CPR, c = (x % TL::CPR) ^ TL::swz(row);
      v[j] = (uint32_t)((min(row, last) * (size_t)ld + c * 8) * sizeof(bf16_t));
    }
  }
  // rows from `base` on; rows behind row `last` are copies of it.  off: offsets of a whole tile.
  __device__ static __forceinline__ void go(const bf16_t* base, int ld, const uint32_t (&off)[2], int last, uint32_t to, int wave, int lane) {
    to += wave * 2048;
    if (last == LC - 1) {
#pragma unroll
      for (int j = 0; j < 2; j++) dma16_base(base, off[j], to + j * 1024);
    } else {
      uint32_t v[2];
      offsets(v, ld, last, wave, lane);
#pragma unroll
      for (int j = 0; j < 2; j++) dma16_base(base, v[j], to + j * 1024);
    }
  }
};

// The pass in its first form, a state for the group and a query row for each of its heads (o, dq), which TEAMS of D / 32 waves share out; or, with !OUT, sums for the states alone: GROUPED and REV: of R, over the group's heads, from
// the row's end.  LDS: two slots each of each team's Q tiles and of K and V tiles.  (More of them, with transfers further ahead, bring
// nothing: results of 8192 tokens x 32 heads 131 -> 133 us, sums with three steps ahead 1 %.)
template <int D, bool GROUPED, bool REV, bool EXACT, bool OUT, int TEAMS = 1>
__device__ __forceinline__ void lin_walk(const LinArgs& a, const LinPass& p, int piece, int hk, int b, char* smem) {
  static_assert(!(GROUPED && OUT) && (OUT || TEAMS == 1), "lin_walk_kv; a team a head");
  using TR = LinTransfer<D>;
  constexpr int W = D / 32, KS = D / 16;
  const lds_char* sm = (const lds_char*)smem;
  const int lane = threadIdx.x & 63, both = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), team = TEAMS > 1 ? both / W : 0, wave = both - team * W, l32 = lane & 31;
  const LinGeom& g = a.g;
  const int grp = g.nq / g.nkv, chunks = (g.seq + LC - 1) / LC, c0 = piece * a.per, c1 = min(chunks, c0 + a.per), heads = GROUPED ? grp : OUT ? (grp + TEAMS - 1) / TEAMS : 1;
  const size_t t0 = (size_t)b * g.seq;
  const float l2 = g.log_decay[hk] * LOG2E, f_in = GROUPED ? g.scale : 1.f;
  const uint32_t lds = lds_address(smem);
  // offsets of q's rows and of k's, or (sums) of k's and v's; with results k and v lie in rows of the same length.  (Two registers fewer: the loop has none to spare, and what lies in scratch
  // waits for the transfers ahead of it: 78 -> 60 us for the results of 8192 tokens x 32 heads in 8 pieces.)
  uint32_t off[2][2];
  TR::offsets(off[0], OUT ? p.ldq : p.ldk, LC - 1, wave, lane);
  TR::offsets(off[1], OUT ? p.ldk : p.ldv, LC - 1, wave, lane);
  const int steps = (c1 - c0) * heads;
  auto chunk_of = [&](int n) { return REV ? c1 - 1 - n : c0 + n; };
  constexpr int KT = 2 * TEAMS;  // tiles of LDS before K's
  int in = 0, ih = 0;  // of the step to transfer next
  auto issue = [&]() {
    const int chunk = chunk_of(in), slot_s = (in * heads + ih) & 1, slot_k = GROUPED ? slot_s : in & 1, last = min(LC, g.seq - chunk * LC) - 1, hkv = GROUPED ? hk * grp + ih : hk;
    const size_t row = t0 + (size_t)chunk * LC;
    if (OUT) TR::go(p.q + row * p.ldq + (size_t)(hk * grp + min(team * heads + ih, grp - 1)) * D, p.ldq, off[0], last, lds + (team * 2 + slot_s) * TR::TILE, wave, lane);
    if (GROUPED || ih == 0) {
      if (TEAMS == 1 || team == 0) TR::go(p.k + row * p.ldk + (size_t)hkv * D, p.ldk, off[OUT ? 1 : 0], last, lds + (KT + slot_k) * TR::TILE, wave, lane);
      if (TEAMS == 1 || team == 1) TR::go(p.v + row * p.ldv + (size_t)hkv * D, p.ldv, off[1], last, lds + (KT + 2 + slot_k) * TR::TILE, wave, lane);
    }
    if (++ih == heads) { ih = 0; in++; }
  };
  issue();
  LinFrag<D> fa;
  fa.init(lane, wave);
  f32x16 S[W];
  lin_state_load<D>(S, OUT && p.state && !lin_alone(l2) ? p.state + (((size_t)b * g.nkv + hk) * a.pieces + piece) * D * D : nullptr, p.transposed, wave, lane);
  LinPowers<REV> pw;
  if constexpr (OUT) pw.scores(l2, g.scale, lane);
  pw.chunk(LC, l2, g.scale, f_in, lane);
  int n = 0, h = 0;
  for (int s = 0; s < steps; s++) {
    // this step's tiles are here once the transfers before the last step's two stores are through
    if constexpr (OUT) { if (s > 0) dma_wait<2>(); else dma_wait<0>(); }
    else dma_wait<0>();
    __syncthreads();  // and every wave is done with the step before, whose slots the next one takes
    if (s + 1 < steps) issue();
    const int chunk = chunk_of(n), left = min(LC, g.seq - chunk * LC), slot_s = s & 1, slot_k = GROUPED ? slot_s : n & 1;
    const lds_char *Qt = sm + (team * 2 + slot_s) * TR::TILE, *Kt = sm + (KT + slot_k) * TR::TILE, *Vt = sm + (KT + 2 + slot_k) * TR::TILE;
    if (left != pw.left) pw.chunk(left, l2, g.scale, f_in, lane);
    LinValues v;
    LinRows<D> ahead[2];
    const bool last_head = GROUPED || h == heads - 1;
    v.load(Vt + fa.tr[0], Vt + fa.tr[1], D * 2);
    if constexpr (OUT) {
      bf16x8 qf[KS];
#pragma unroll
      for (int ks = 0; ks < KS; ks++) qf[ks] = lds_frag(Qt + fa.dir[ks], 0);
      v.look();
      f32x16 ot, st;
      lin_zero(ot);
      lin_zero(st);
#pragma unroll
      for (int ks = 0; ks < KS; ks++) ot = MFMA(pack_rows(S[ks >> 1], ks & 1), qf[ks], ot);
#pragma unroll
      for (int r = 0; r < 16; r++) ot[r] *= pw.read;
#pragma unroll
      for (int ks = 0; ks < KS; ks++) st = MFMA(lds_frag(Kt + fa.dir[ks], 0), qf[ks], st);
      lin_inside<REV>(ot, st, pw, v, lane);
      lin_out(ot, p.out + (t0 + (size_t)chunk * LC + l32) * p.ldo + (size_t)(hk * grp + min(team * heads + h, grp - 1)) * D + wave * 32, l32 < left, lane);
    } else {
      ahead[0].load(fa, Kt, 0);
      ahead[1].load(fa, Kt, 1);
      LIN_PIN();
    }
    if (last_head && !pw.alone) {
      if (!GROUPED || h == 0) {
#pragma unroll
        for (int dt = 0; dt < W; dt++)
#pragma unroll
          for (int r = 0; r < 16; r++) S[dt][r] *= pw.whole;
      }
      lin_into<D, EXACT ? 3 : 2, !OUT>(S, fa, Kt, ahead, v.all, pw.into);
    }
    if (++h == heads) { h = 0; n++; }
  }
  if constexpr (EXACT && !GROUPED) {  // (of R nothing is left)
    if (pw.alone) lin_state_alone<D>(S, sm + (KT + ((c1 - c0 - 1) & 1)) * TR::TILE, sm + (KT + 2 + ((c1 - c0 - 1) & 1)) * TR::TILE, pw.left - 1, wave);
  }
  if constexpr (EXACT) {
    if (p.sum && team == 0) lin_state_store<D>(S, p.sum + (OUT ? (size_t)b * g.nkv + hk : ((size_t)b * g.nkv + hk) * a.pieces + piece) * D * D, wave, lane);
  }
}

// dk and dv, from the row's end, over the group's heads.  Both are the same form: dv has the state R, rows of Q against keys, values of dO; dk has R's transpose, rows of dO against values, values
// of Q.  Half of a block's waves takes one of them each, off the same tiles, so that a SIMD has two waves: one that holds both states has it to itself and moves half of its registers to and from the
// accumulators' (2 x 4096 tokens on 32:8 heads, a training step: 285 -> 264 us).  Bound by the products' chains and the vector arithmetic between them; scores in two chains, or the state's products between
// the scores' and theirs, take registers that there are not (283 and 280 us).  LDS: two slots each of K, V, Q, dO tiles.
template <int D, bool EXACT>
__device__ __forceinline__ void lin_walk_kv(const LinArgs& a, const LinGrads& p, int piece, int hk, int b, char* smem) {
  using TR = LinTransfer<D>;
  constexpr int W = D / 32, KS = D / 16;
  const lds_char* sm = (const lds_char*)smem;
  const int lane = threadIdx.x & 63, both = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), is_dk = both >= W, wave = both - is_dk * W, l32 = lane & 31;
  const LinGeom& g = a.g;
  const int grp = g.nq / g.nkv, chunks = (g.seq + LC - 1) / LC, c0 = piece * a.per, c1 = min(chunks, c0 + a.per), ld = (g.nq + 2 * g.nkv) * D, ldo = g.nq * D, ldx = is_dk ? ldo : ld;
  const size_t t0 = (size_t)b * g.seq;
  const float l2 = g.log_decay[hk] * LOG2E;
  const uint32_t lds = lds_address(smem);
  uint32_t off[2][2];
  TR::offsets(off[0], ld, LC - 1, wave, lane);
  TR::offsets(off[1], ldx, LC - 1, wave, lane);
  const int steps = (c1 - c0) * grp, column = (g.nq + is_dk * g.nkv + hk) * D, to = (g.nq + (1 - is_dk) * g.nkv + hk) * D;
  int in = 0, ih = 0;
  auto issue = [&]() {  // each half the tiles that its products begin with
    const int chunk = c1 - 1 - in, slot_s = (in * grp + ih) & 1, slot_c = in & 1, last = min(LC, g.seq - chunk * LC) - 1;
    const size_t row = t0 + (size_t)chunk * LC;
    if (ih == 0) TR::go(p.qkv + row * ld + column, ld, off[0], last, lds + (2 * is_dk + slot_c) * TR::TILE, wave, lane);
    const bf16_t* x = is_dk ? p.dout + row * ldo : p.qkv + row * ld;
    TR::go(x + (size_t)(hk * grp + ih) * D, ldx, off[1], last, lds + (4 + 2 * is_dk + slot_s) * TR::TILE, wave, lane);
    if (++ih == grp) { ih = 0; in++; }
  };
  issue();
  LinFrag<D> fa;
  fa.init(lane, wave);
  f32x16 R[W];
  lin_state_load<D>(R, p.state ? p.state + (((size_t)b * g.nkv + hk) * a.pieces + piece) * D * D : nullptr, is_dk, wave, lane);
  LinPowers<true> pw;
  pw.scores(l2, g.scale, lane);
  pw.chunk(LC, l2, 1.f, g.scale, lane);
  f32x16 out;
  int n = 0, h = 0;
  for (int s = 0; s < steps; s++) {
    if (h == 0 && s > 0) dma_wait<2>(); else dma_wait<0>();  // the tiles stand before a chunk's two stores
    __syncthreads();
    if (s + 1 < steps) issue();
    const int chunk = c1 - 1 - n, left = min(LC, g.seq - chunk * LC);
    const lds_char *At = sm + (2 * is_dk + (n & 1)) * TR::TILE, *Xt = sm + (4 + 2 * is_dk + (s & 1)) * TR::TILE, *Yt = sm + (6 - 2 * is_dk + (s & 1)) * TR::TILE;
    if (left != pw.left) pw.chunk(left, l2, 1.f, g.scale, lane);
    LinValues y;
    y.load(Yt + fa.tr[0], Yt + fa.tr[1], D * 2);
    if (h == 0) {
      lin_zero(out);
#pragma unroll
      for (int ks = 0; ks < KS; ks++) out = MFMA(pack_rows(R[ks >> 1], ks & 1), lds_frag(At + fa.dir[ks], 0), out);
      const bool none = pw.alone && pw.read == 0.f;
#pragma unroll
      for (int r = 0; r < 16; r++) out[r] = none ? 0.f : out[r] * pw.read;
#pragma unroll
      for (int dt = 0; dt < W; dt++)
#pragma unroll
        for (int r = 0; r < 16; r++) R[dt][r] *= pw.whole;
    }
    y.look();
    f32x16 st;
    lin_zero(st);
#pragma unroll
    for (int ks = 0; ks < KS; ks++) st = MFMA(lds_frag(Xt + fa.dir[ks], 0), lds_frag(At + fa.dir[ks], 0), st);
    lin_inside<true>(out, st, pw, y, lane);
    LinRows<D> ahead[2];
    lin_into<D, EXACT ? 3 : 2, false>(R, fa, Xt, ahead, y.all, pw.into);
    if (++h < grp) continue;
    lin_out(out, p.dqkv + (t0 + (size_t)chunk * LC + l32) * ld + to + wave * 32, l32 < left, lane);
    if (pw.alone) {
#pragma unroll
      for (int dt = 0; dt < W; dt++) lin_zero(R[dt]);
    }
    h = 0;
    n++;
  }
  if constexpr (EXACT) {
    if (p.sum && !is_dk) lin_state_store<D>(R, p.sum + ((size_t)b * g.nkv + hk) * D * D, wave, lane);
  }
}

// The forward pass: OUT its results, otherwise the pieces' contributions to the states.  grid (pieces, nkv, batch)
template <int D, bool EXACT, bool OUT, int TEAMS>
__global__ __launch_bounds__(TEAMS * 2 * D, 2) void lin_fwd_kernel(const LinArgs a) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  lin_walk<D, false, false, EXACT, OUT, TEAMS>(a, a.pass[0], blockIdx.x, blockIdx.y, blockIdx.z, smem);
}
// The backward pass's dk and dv.  grid (pieces, nkv, batch)
template <int D, bool EXACT>
__global__ __launch_bounds__(4 * D, 2) void lin_bwd_kernel(const LinArgs a, const LinGrads k) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  lin_walk_kv<D, EXACT>(a, k, blockIdx.x, blockIdx.y, blockIdx.z, smem);
}
// The pieces' contributions to R (y < nkv) and to S.  grid (pieces, 2 * nkv, batch)
template <int D>
__global__ __launch_bounds__(2 * D, 2) void lin_bwd_sums_kernel(const LinArgs a) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const int nkv = a.g.nkv, y = blockIdx.y;
  if (y < nkv) lin_walk<D, true, true, true, false>(a, a.pass[1], blockIdx.x, y, blockIdx.z, smem);
  else lin_walk<D, false, false, true, false>(a, a.pass[0], blockIdx.x, y - nkv, blockIdx.z, smem);
}
// ------------------------------------------------------------------------------------ host side
// Pieces of a row: enough that the forward pass has a wave for each of the chip's 1024 SIMDs, and that dk and dv, whose blocks have twice the waves of which a unit of the chip holds one block, have a
// block for each unit (half of LIN_BB; the other half is for dq).  More pieces cost more states' way to memory and back.  us, 256 and 512: forward of 8192 tokens x 32 heads 100 and 106;
// training step of 2 x 4096 tokens on 32:8 heads, blocks of the backward pass, 256, 384, 512, 768 and 1024: 357, 300, 264, 315 and 286.
// Where rows are short for that, a piece holds two steps (a chunk of one head) at least: us, forward and backward, pieces from 1, 2 and 4 chunks on: 3092 tokens of 2:1 heads 26 and 48, 25 and 56, 31 and 70;
// 256 tokens of 8:2 17 and 41, 23 and 56, 33 and 86; 3 x 1999 of 8:8 heads of 64 26 and 43, 25 and 43, 27 and 48.  Rows of up to eight steps stay whole, without the launches of sums and carry:
// 192 tokens of 8:8 heads 13.4 and 31.8 whole, 15.5 and 34.5 cut; 256 17.1 and 40.3, and 17.1 and 37.5; 64 of 8:2 13.1 and 31.7, and 16.3 and 39.3; 96 18.3 and 44.2, and 16.4 and 39.6.
#define LIN_WHOLE 8
#define LIN_BF 256
#define LIN_BB 512
static LinCut lin_cut(const LinGeom& g, bool bwd) {
  const long long chunks = (g.seq + LC - 1) / LC, blocks = (long long)g.batch * g.nkv * (bwd ? 2 : 1), grp = g.nq / g.nkv;
  if (chunks * grp <= LIN_WHOLE) return {1, (int)chunks};
  const long long want = std::max(1ll, std::min(((bwd ? LIN_BB : LIN_BF) * (128 / g.d) + blocks - 1) / blocks, grp > 1 ? chunks : chunks / 2));
  const int per = (int)((chunks + want - 1) / want);
  return {(int)((chunks + per - 1) / per), per};
}
static size_t lin_states(const LinGeom& g, int pieces) { return (size_t)g.batch * g.nkv * pieces * g.d * g.d; }
size_t dh_linattn_bf16_ws_bytes(const LinGeom& g, bool bwd) {
  const LinCut c = lin_cut(g, bwd);
  return c.pieces == 1 ? 0 : (bwd ? 2 : 1) * lin_states(g, c.pieces) * sizeof(float);
}
// The forward pass's results.  From four heads of a group on two teams of waves share them and the tiles of keys and values, each with the state: us, one team and two, 2 x 4096 tokens of 32:8 heads 74.5 and
// 67.5, 64 of 8:2 13.2 and 10.9, 4 x 2048 of 32:8 heads of 64 38.7 and 32.4; but 8192 of 24:8 62.7 and 67.2, 3092 of 2:1 26.2 and 27.1, and dq, whose rows come from further away, gains nothing.
template <int D, bool EXACT>
static int lin_results(const LinArgs& a, hipStream_t s) {
  const dim3 grid(a.pieces, a.g.nkv, a.g.batch);
  if (a.g.nq / a.g.nkv >= 4) lin_fwd_kernel<D, EXACT, true, 2><<<grid, 4 * D, 8 * LC * D * 2, s>>>(a);
  else lin_fwd_kernel<D, EXACT, true, 1><<<grid, 2 * D, 6 * LC * D * 2, s>>>(a);
  DH_LAUNCH_CHECK();
  return DH_OK;
}
template <int D>
static int lin_fwd(const LinGeom& g, const bf16_t* qkv, const float* state_in, bf16_t* o, float* state_out, float* ws, hipStream_t s) {
  const int ld = (g.nq + 2 * g.nkv) * D;
  const LinCut c = lin_cut(g, false);
  LinArgs a = {g, c.pieces, c.per, {}};
  a.pass[0] = {qkv, qkv + (size_t)g.nq * D, qkv + (size_t)(g.nq + g.nkv) * D, o, ld, ld, ld, g.nq * D, state_in, state_out, 0};
  if (c.pieces > 1) {
    a.pass[0].state = nullptr;
    a.pass[0].sum = ws;
    lin_fwd_kernel<D, true, false, 1><<<dim3(c.pieces, g.nkv, g.batch), 2 * D, 6 * LC * D * 2, s>>>(a);
    DH_LAUNCH_CHECK();
    if (int rc = dh_launch_lin_carry(g, c.pieces, c.per * LC, {ws, state_in, state_out, 0}, nullptr, s)) return rc;
    a.pass[0].state = ws;
    return lin_results<D, false>(a, s);
  }
  return state_out ? lin_results<D, true>(a, s) : lin_results<D, false>(a, s);
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
  LinGrads kv = {qkv, dout, dqkv, dstate_out, dstate_in};
  const dim3 grid(c.pieces, g.nkv * 2, g.batch);
  if (c.pieces > 1) {
    float* R = ws + lin_states(g, c.pieces);
    LinArgs f = a;
    f.pass[0] = {nullptr, k, v, nullptr, 0, ld, ld, 0, nullptr, ws, 0};
    f.pass[1] = {nullptr, q, dout, nullptr, 0, ld, ldo, 0, nullptr, R, 0};
    lin_bwd_sums_kernel<D><<<grid, 2 * D, 6 * LC * D * 2, s>>>(f);
    DH_LAUNCH_CHECK();
    const LinCarry back = {R, dstate_out, dstate_in, 1};
    if (int rc = dh_launch_lin_carry(g, c.pieces, c.per * LC, {ws, state_in, nullptr, 0}, &back, s)) return rc;
    a.pass[0].state = ws;
    kv.state = R;
    kv.sum = nullptr;
  }
  const size_t lds = 8 * LC * D * 2;
  const dim3 one(c.pieces, g.nkv, g.batch);
  if (kv.sum) lin_bwd_kernel<D, true><<<one, 4 * D, lds, s>>>(a, kv);
  else lin_bwd_kernel<D, false><<<one, 4 * D, lds, s>>>(a, kv);
  DH_LAUNCH_CHECK();
  lin_fwd_kernel<D, false, true, 1><<<one, 2 * D, 6 * LC * D * 2, s>>>(a);
  DH_LAUNCH_CHECK();
  return DH_OK;
}
int dh_launch_linattn_bwd_bf16(const LinGeom& g, const bf16_t* qkv, const float* state_in, const bf16_t* dout, const float* dstate_out, bf16_t* dqkv, float* dstate_in, void* ws,
                               hipStream_t s) {
  return g.d == 128 ? lin_bwd<128>(g, qkv, state_in, dout, dstate_out, dqkv, dstate_in, (float*)ws, s) : lin_bwd<64>(g, qkv, state_in, dout, dstate_out, dqkv, dstate_in, (float*)ws, s);
}
