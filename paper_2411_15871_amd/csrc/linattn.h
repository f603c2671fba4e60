// Linear attention with a decay for each head: what its sources share.
#pragma once
#include "mixers.h"

struct LinGeom {
  int batch, seq, nq, nkv, d;
  float scale;
  const float* log_decay;
};
#define LC 32  // tokens of a chunk
// log2 of lambda may be minus infinity: then each token sees itself alone, and what others leave is not multiplied by zero (an infinity or a NaN would pass) but left out.
__device__ __forceinline__ bool lin_alone(float l2) { return __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, l2)) == (int)0xff800000; }
// lambda^m
__device__ __forceinline__ float lin_pow(float l2, int m) { return m == 0 ? 1.f : __builtin_amdgcn_exp2f(l2 * (float)m); }

// Pieces of a row, `per` chunks each, that run side by side.
struct LinCut { int pieces, per; };
// Carries the states along the pieces: each piece's contribution in sums [batch][nkv][pieces][d][d] gives place to the state before it, from `first` on (NULL: zeros); the one behind all of
// them goes to `last` (NULL: not wanted).  rev: from the row's end.
struct LinCarry { float* sums; const float* first; float* last; int rev; };
int dh_launch_lin_carry(const LinGeom& g, int pieces, int tokens, const LinCarry& c0, const LinCarry* c1, hipStream_t stream);  // tokens: of a piece

size_t dh_linattn_bf16_ws_bytes(const LinGeom& g, bool bwd);
int dh_launch_linattn_fwd_bf16(const LinGeom& g, const bf16_t* qkv, const float* state_in, bf16_t* o, float* state_out, void* ws, hipStream_t stream);
int dh_launch_linattn_bwd_bf16(const LinGeom& g, const bf16_t* qkv, const float* state_in, const bf16_t* dout, const float* dstate_out, bf16_t* dqkv, float* dstate_in, void* ws,
                               hipStream_t stream);
size_t dh_linattn_f32_ws_bytes(const LinGeom& g, bool bwd);
int dh_launch_linattn_fwd_f32(const LinGeom& g, const float* qkv, const float* state_in, float* o, float* state_out, void* ws, hipStream_t stream);
int dh_launch_linattn_bwd_f32(const LinGeom& g, const float* qkv, const float* state_in, const float* dout, const float* dstate_out, float* dqkv, float* dstate_in, void* ws,
                              hipStream_t stream);
