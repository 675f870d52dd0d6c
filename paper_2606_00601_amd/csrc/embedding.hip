// embedding.hip -- rows of a table by token.
#include "norm_rows.h"
#include "token_rows.h"

namespace sw {
namespace embed {
namespace {

using norm::load8;
using norm::store8;

// A wave's LPR lanes copy a row, 8 columns a lane at a time.  Bound by memory.
template <class E, class Y, int LPR>
__global__ __launch_bounds__(256) void fwd_kernel(EmbedArgs a, bool vec) {
  const int li = threadIdx.x % LPR;
  const int64_t rows = 256 / LPR * (int64_t)gridDim.x;
  for (int64_t t = blockIdx.x * (int64_t)(256 / LPR) + threadIdx.x / LPR; t < a.T; t += rows) {
    const uint32_t v = row_of(a, t);
    const E* src = (const E*)a.table + (int64_t)v * a.D;
    for (int64_t c = (blockIdx.y * (int64_t)LPR + li) * 8; c < a.D; c += gridDim.y * (int64_t)LPR * 8) {
      float x[8];
      load8(src + c, x, v < a.V ? a.D - c : 0, vec);
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = v < a.V ? x[j] * a.scale : 0.0f;
      store8((Y*)a.y + t * a.D + c, x, a.D - c, vec);
    }
  }
}

template <class E, class Y>
int fwd_typed(const EmbedArgs& a, bool vec, int cus, hipStream_t s) {
#define CALL(LPR)                                                                             \
  do {                                                                                        \
    const int64_t wgs = (a.T + 256 / LPR - 1) / (256 / LPR), most = 16 * (int64_t)cus;        \
    int64_t cols = 1; /* few rows: their columns over more workgroups */                      \
    while (wgs * cols < cus && cols * LPR * 8 < a.D) cols *= 2;                               \
    hipLaunchKernelGGL((fwd_kernel<E, Y, LPR>),                                               \
                       dim3((unsigned)(wgs < most ? wgs : most), (unsigned)cols), dim3(256), 0, s, a, vec); \
  } while (0)
  if (a.D <= 64)
    CALL(8);
  else if (a.D <= 128)
    CALL(16);
  else if (a.D <= 256)
    CALL(32);
  else
    CALL(64);
#undef CALL
  return check_launch("embedding fwd_kernel");
}

}  // namespace
}  // namespace embed

using namespace embed;

int embedding_fwd(const EmbedArgs& a) {
  int cus, st;
  if ((st = device_cus(&cus)) != SW_OK) return st;
  const bool vec = norm::vec_rows(a.table, a.D, a.D, a.table_bf16) && norm::vec_rows(a.y, a.D, a.D, a.y_bf16);
  const hipStream_t s = current_stream();
  if (a.table_bf16)
    return a.y_bf16 ? fwd_typed<uint16_t, uint16_t>(a, vec, cus, s) : fwd_typed<uint16_t, float>(a, vec, cus, s);
  return a.y_bf16 ? fwd_typed<float, uint16_t>(a, vec, cus, s) : fwd_typed<float, float>(a, vec, cus, s);
}

}  // namespace sw
