// linear_attn.h -- arguments shared by the linear-attention kernels and the
// C-ABI layer (not installed).
#pragma once

#include "sw_internal.h"

namespace sw {

// One (B, L, heads, width) operand, width contiguous; strides in elements.
struct HeadRows {
  const void* p = nullptr;
  int64_t sb = 0, sl = 0, sh = 0;
};

// One call of the chunked form, already validated.  cu == NULL: B sequences of
// L steps; else nseq sequences packed into one row (B == 1) of L steps,
// sequence n the steps cu[n] .. cu[n+1]-1.  g is (H) if g_head, else by the
// strides in gs.  States are (sequences, H, K, V) fp32.
struct LinAttnArgs {
  HeadRows q, k, v, dout;
  const float* g = nullptr;
  int64_t g_sb = 0, g_sl = 0, g_sh = 0;
  bool g_head = false;
  const int32_t* cu = nullptr;
  const float *h0 = nullptr, *dh_last = nullptr;
  void *o = nullptr, *dq = nullptr, *dk = nullptr, *dv = nullptr;
  float *h_last = nullptr, *dg = nullptr, *dh0 = nullptr;
  int64_t B = 0, L = 0, Hk = 0, H = 0, K = 0, V = 0, nseq = 0;
  bool bf16 = false;
  float scale = 1.0f;
  void* ws = nullptr;
  size_t ws_bytes = 0;
};
int linear_attn_fwd(const LinAttnArgs& a);
int linear_attn_bwd(const LinAttnArgs& a);
// Bytes of workspace (0: none needed); the pointers are not read.
int64_t linear_attn_fwd_workspace(const LinAttnArgs& a);
int64_t linear_attn_bwd_workspace(const LinAttnArgs& a);

// One step of B sequences: states (pool, H, K, V) fp32 in place, sequence b's
// at slots[b] (b if NULL); slots outside [0, pool) leave o zero and no state touched.
struct LinStepArgs {
  const void *q = nullptr, *k = nullptr, *v = nullptr;
  int64_t q_sb = 0, q_sh = 0, k_sb = 0, k_sh = 0, v_sb = 0, v_sh = 0;
  const float* g = nullptr;
  int64_t g_sb = 0, g_sh = 0;
  float* state = nullptr;
  const int32_t* slots = nullptr;
  void* o = nullptr;
  int64_t B = 0, Hk = 0, H = 0, K = 0, V = 0, pool = 0;
  bool bf16 = false;
  float scale = 1.0f;
};
int linear_attn_step(const LinStepArgs& a);

// The longest head widths the chunked kernels hold.
constexpr int64_t LINATTN_MAX_WIDTH = 256;

}  // namespace sw
