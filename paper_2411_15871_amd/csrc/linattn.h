// Linear attention with a decay for each head: what its sources share.
#pragma once
#include "mixers.h"

struct LinGeom {
  int batch, seq, nq, nkv, d;
  float scale;
  const float* log_decay;
};
size_t dh_linattn_bf16_ws_bytes(const LinGeom& g, bool bwd);
int dh_launch_linattn_fwd_bf16(const LinGeom& g, const bf16_t* qkv, const float* state_in, bf16_t* o, float* state_out, void* ws, hipStream_t stream);
int dh_launch_linattn_bwd_bf16(const LinGeom& g, const bf16_t* qkv, const float* state_in, const bf16_t* dout, const float* dstate_out, bf16_t* dqkv, float* dstate_in, void* ws,
                               hipStream_t stream);
