// gated_scan.h -- arguments shared by the gated recurrence's kernels and the C-ABI
// layer (not installed).
#pragma once

#include "sw_internal.h"

namespace sw {

// Rows of D contiguous channels: element (b, l, d) lies at b * sb + l * sl + d.
struct StepRows {
  const void* p = nullptr;
  int64_t sb = 0, sl = 0;
};

struct GatedArgs {
  StepRows x, r, i, dh;
  const float *lam = nullptr, *h0 = nullptr, *dh_last = nullptr, *ckpt_in = nullptr;
  const int32_t* cu = nullptr;
  void *h = nullptr, *dx = nullptr, *dr = nullptr, *di = nullptr;
  float *h_last = nullptr, *ckpt = nullptr, *dlam = nullptr, *dh0 = nullptr;
  int64_t B = 0, L = 0, D = 0, nseq = 0;
  bool bf16 = false;
  float c = 0.0f;
  void* ws = nullptr;
  size_t ws_bytes = 0;
};
int gated_scan_fwd(const GatedArgs& a);
int64_t gated_scan_fwd_workspace(int64_t B, int64_t L, int64_t D);
int gated_scan_bwd(const GatedArgs& a);
int64_t gated_scan_bwd_workspace(int64_t B, int64_t L, int64_t D, bool ckpt);

struct GatedStepArgs {
  const void *x = nullptr, *r = nullptr, *i = nullptr;
  const float* lam = nullptr;
  float* state = nullptr;
  const int32_t* slots = nullptr;
  void* h = nullptr;
  int64_t B = 0, D = 0, pool = 0, x_st = 0, r_st = 0, i_st = 0;
  bool bf16 = false;
  float c = 0.0f;
};
int gated_scan_step(const GatedStepArgs& a);

}  // namespace sw
