// block_norm.h -- arguments shared by the norm kernels and the C-ABI layer (not
// installed).
#pragma once

#include "sw_internal.h"

namespace sw {

// The norm before a block: R' = R + s x, y = w R' / rms(R').  Rows of D; x, R (and
// in the backward dy, dres, R') lie x_st ... elements apart, the others densely.
struct ResNormArgs {
  const void *x = nullptr, *res = nullptr, *dy = nullptr, *dres = nullptr;
  const void* stored = nullptr;  // backward: R' (x itself where there is no residual)
  const float *w = nullptr, *s = nullptr;
  void *y = nullptr, *res_out = nullptr, *dx = nullptr, *dr = nullptr;
  float *dw = nullptr, *ds = nullptr;
  int64_t M = 0, D = 0;
  int64_t x_st = 0, res_st = 0, dy_st = 0, dres_st = 0, stored_st = 0;
  bool bf16 = false, res_bf16 = false;
  float eps = 0.0f;
  void* ws = nullptr;
  size_t ws_bytes = 0;
};
int residual_norm_fwd(const ResNormArgs& a);
int residual_norm_bwd(const ResNormArgs& a);

// The norm after a block's mixer: rows of G groups of `group` columns, with the
// gate silu(z) before the norm or after it.
struct GatedNormArgs {
  const void *x = nullptr, *z = nullptr, *dy = nullptr;
  const float* w = nullptr;
  void *y = nullptr, *dx = nullptr, *dz = nullptr;
  float* dw = nullptr;
  int64_t M = 0, D = 0, group = 0;
  int64_t x_st = 0, z_st = 0, dy_st = 0;
  bool bf16 = false, after = false;
  float eps = 0.0f;
  void* ws = nullptr;
  size_t ws_bytes = 0;
};
int gated_norm_fwd(const GatedNormArgs& a);
int gated_norm_bwd(const GatedNormArgs& a);

// Bytes of the backward's workspace: partial sums of `grads` parameter gradients.
int64_t norm_bwd_workspace(int64_t M, int64_t D, int64_t width, int grads);

constexpr int64_t NORM_MAX_WIDTH = 16384;

}  // namespace sw
