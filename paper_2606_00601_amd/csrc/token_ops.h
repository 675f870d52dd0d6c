// token_ops.h -- arguments shared by the head norm's and the embedding's kernels and
// the C-ABI layer (not installed).
#pragma once

#include "sw_internal.h"

namespace sw {

constexpr int64_t HEAD_MAX_WIDTH = 256;

// Element (b, l, h, e) of a (B, L, H, K) tensor lies at b * sb + l * sl + h * sh + e.
struct Heads {
  const void* p = nullptr;
  int64_t sb = 0, sl = 0, sh = 0;
};

struct HeadNormArgs {
  Heads q, k, dyq, dyk;
  const float *wq = nullptr, *wk = nullptr, *inv_freq = nullptr;
  const void* pos = nullptr;
  int64_t pos_sb = 0, pos_sl = 0;
  void *yq = nullptr, *yk = nullptr;  // backward: dq, dk
  float *dwq = nullptr, *dwk = nullptr;
  int64_t B = 0, L = 0, H = 0, Hk = 0, K = 0, R = 0;
  bool bf16 = false, adjacent = false, pos64 = false;
  float eps = 0.0f;
  void* ws = nullptr;
  size_t ws_bytes = 0;
};
int head_norm_fwd(const HeadNormArgs& a);
int head_norm_bwd(const HeadNormArgs& a);
int64_t head_norm_bwd_workspace(int64_t T, int64_t H, int64_t Hk, int64_t K);

struct EmbedArgs {
  const void *tokens = nullptr, *table = nullptr, *dy = nullptr;
  void *y = nullptr, *dtable = nullptr;
  int64_t T = 0, V = 0, D = 0, dy_st = 0;
  bool wide = false, table_bf16 = false, y_bf16 = false;  // y_bf16: dy's type too
  float scale = 1.0f;
  void* ws = nullptr;
  size_t ws_bytes = 0;
};
int embedding_fwd(const EmbedArgs& a);
int embedding_bwd(const EmbedArgs& a);
int64_t embedding_bwd_workspace(int64_t T, int64_t V, int64_t D);

}  // namespace sw
