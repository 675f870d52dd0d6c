// residual_norm.hip -- the norm before a block, with the residual addition and
// its scale: R' = R + s x, y = w R' / sqrt(mean(R'^2) + eps), and its gradients.
#include "norm_rows.h"

namespace sw {
namespace norm {
namespace {

// R' is rounded to the residual stream's type first and y is the norm of what
// is stored, so that the backward, which reads R' back, meets the same numbers.
// s x and the sum are rounded to fp32 one after the other for the same reason.
// 16384 rows of 1536, bf16 with an fp32 stream: 59 us, 302 MB at 5.1 TB/s (a large
// copy's rate).
template <class E, class R, int LPR, int NV>
__global__ __launch_bounds__(threads_of(LPR)) void res_fwd_kernel(ResNormArgs a, bool vec) {
  constexpr int RPW = threads_of(LPR) / LPR;
  __shared__ RowSum<LPR, 1> sh;
  const int sub = threadIdx.x / LPR, li = threadIdx.x % LPR;
  int par = 0;
  float w[NV][8], s[NV][8];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int64_t c = (v * LPR + li) * 8;
    load8(a.w + c, w[v], a.D - c, vec);
    if (a.s) load8(a.s + c, s[v], a.D - c, vec);
  }
  for (int64_t m = blockIdx.x * (int64_t)RPW + sub; m < a.M; m += gridDim.x * (int64_t)RPW) {
    float x[NV][8];
    float sum[1] = {0.0f};
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int64_t c = (v * LPR + li) * 8;
      load8((const E*)a.x + m * a.x_st + c, x[v], a.D - c, vec);
      if (a.res) {
        float r[8];
        load8((const R*)a.res + m * a.res_st + c, r, a.D - c, vec);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float t = a.s ? __fmul_rn(s[v][j], x[v][j]) : x[v][j];
          x[v][j] = as_stored(__fadd_rn(r[j], t), (const R*)nullptr);
        }
        store8((R*)a.res_out + m * a.D + c, x[v], a.D - c, vec);
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) sum[0] = __builtin_fmaf(x[v][j], x[v][j], sum[0]);
    }
    row_sum<LPR, 1>(sum, sh, par);
    const float inv = rsqrtf(sum[0] / (float)a.D + a.eps);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int64_t c = (v * LPR + li) * 8;
#pragma unroll
      for (int j = 0; j < 8; ++j) x[v][j] *= inv * w[v][j];
      store8((E*)a.y + m * a.D + c, x[v], a.D - c, vec);
    }
  }
}

// dR' = dres + inv (w dy - n mean(w dy n)), n = R' inv; dx = s dR', dw = sum dy n,
// ds = sum x dR'.  Both sums of a row, of R'^2 and of w dy R', are of what the
// row's lanes hold, so one pass over memory gives everything.  16384 rows of 1536,
// bf16 with an fp32 stream and a scale: 96 us, 453 MB at 4.7 TB/s.  All of a row's
// loads are issued before its sums; as a branch in the kernel `vec` made each wait for
// the one before (102 us).
template <class E, class R, bool vec, int LPR, int NV>
__global__ __launch_bounds__(threads_of(LPR)) void res_bwd_kernel(ResNormArgs a, float* part) {
  constexpr int RPW = threads_of(LPR) / LPR;
  __shared__ RowSum<LPR, 2> sh;
  __shared__ float lds[partial_lds<LPR, NV>];
  const int sub = threadIdx.x / LPR, li = threadIdx.x % LPR;
  int par = 0;
  float dw[NV][8], ds[NV][8];
#pragma unroll
  for (int v = 0; v < NV; ++v)
#pragma unroll
    for (int j = 0; j < 8; ++j) dw[v][j] = ds[v][j] = 0.0f;
  for (int64_t m = blockIdx.x * (int64_t)RPW + sub; m < a.M; m += gridDim.x * (int64_t)RPW) {
    float r[NV][8], d[NV][8], w[NV][8], t[NV][8], x[NV][8];
    float sum[2] = {0.0f, 0.0f};
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int64_t c = (v * LPR + li) * 8;
      load8((const R*)a.stored + m * a.stored_st + c, r[v], a.D - c, vec);
      load8((const E*)a.dy + m * a.dy_st + c, d[v], a.D - c, vec);
      load8(a.w + c, w[v], a.D - c, vec);
      if (a.dres) load8((const R*)a.dres + m * a.dres_st + c, t[v], a.D - c, vec);
      if (a.s) load8((const E*)a.x + m * a.x_st + c, x[v], a.D - c, vec);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        sum[0] = __builtin_fmaf(r[v][j], r[v][j], sum[0]);
        sum[1] = __builtin_fmaf(w[v][j] * d[v][j], r[v][j], sum[1]);
      }
    }
    row_sum<LPR, 2>(sum, sh, par);
    const float inv = rsqrtf(sum[0] / (float)a.D + a.eps);
    const float mean = sum[1] * inv / (float)a.D;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int64_t c = (v * LPR + li) * 8;
      float dr[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float n = r[v][j] * inv;
        dw[v][j] = __builtin_fmaf(d[v][j], n, dw[v][j]);
        dr[j] = inv * (w[v][j] * d[v][j] - n * mean);
        if (a.dres) dr[j] += t[v][j];
      }
      if (a.dr) store8((R*)a.dr + m * a.D + c, dr, a.D - c, vec);
      if (a.s) {
        float s[8];
        load8(a.s + c, s, a.D - c, vec);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          ds[v][j] = __builtin_fmaf(x[v][j], dr[j], ds[v][j]);
          dr[j] *= s[j];
        }
      }
      if (a.dx) store8((E*)a.dx + m * a.D + c, dr, a.D - c, vec);
    }
  }
  put_partial<LPR, NV>(dw, lds, part + blockIdx.x * a.D, a.D);
  if (a.s) {
    __syncthreads();
    put_partial<LPR, NV>(ds, lds, part + ((int64_t)gridDim.x + blockIdx.x) * a.D, a.D);
  }
}

template <class E, class R>
int fwd_typed(const ResNormArgs& a, int64_t wgs, bool vec, hipStream_t s) {
#define CALL(LPR, NV)                                                                          \
  do {                                                                                         \
    const int64_t need = (a.M + threads_of(LPR) / LPR - 1) / (threads_of(LPR) / LPR);          \
    hipLaunchKernelGGL((res_fwd_kernel<E, R, LPR, NV>), dim3((unsigned)(need < wgs ? need : wgs)), \
                       dim3(threads_of(LPR)), 0, s, a, vec);                                   \
  } while (0)
  SW_NORM_PICK(a.D, CALL);
#undef CALL
  return check_launch("res_fwd_kernel");
}

template <class E, class R, bool VEC>
int bwd_vec(const ResNormArgs& a, float* part, int64_t blocks, hipStream_t s) {
#define CALL(LPR, NV)                                                              \
  hipLaunchKernelGGL((res_bwd_kernel<E, R, VEC, LPR, NV>), dim3((unsigned)blocks), \
                     dim3(threads_of(LPR)), 0, s, a, part)
  SW_NORM_PICK_BWD(a.D, CALL);
#undef CALL
  return check_launch("res_bwd_kernel");
}
template <class E, class R>
int bwd_typed(const ResNormArgs& a, float* part, int64_t blocks, bool vec, hipStream_t s) {
  return vec ? bwd_vec<E, R, true>(a, part, blocks, s) : bwd_vec<E, R, false>(a, part, blocks, s);
}

// Sums of the partial rows: 16 columns of one gradient, 16 rows at a time, added
// in a fixed order; of no rows zero.
struct Outs {
  float* p[2];
};
__global__ __launch_bounds__(256) void fold_partials_kernel(const float* __restrict__ part,
                                                            int64_t blocks, int64_t D, Outs outs) {
  __shared__ float sh[16][17];
  const int col = threadIdx.x & 15, row = threadIdx.x >> 4;
  const int64_t c = blockIdx.x * 16ll + col;
  const float* p = part + (int64_t)blockIdx.y * blocks * D + c;
  float s = 0.0f;
  if (c < D) {
    int64_t i = row;
    for (; i + 112 < blocks; i += 128) {
      float t[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) t[u] = p[(i + 16 * u) * D];
#pragma unroll
      for (int u = 0; u < 8; ++u) s += t[u];
    }
    for (; i < blocks; i += 16) s += p[i * D];
  }
  sh[row][col] = s;
  __syncthreads();
  if (row == 0 && c < D) {
    float t = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) t += sh[i][col];
    outs.p[blockIdx.y][c] = t;
  }
}

}  // namespace

int fold_partials(const float* part, int64_t blocks, int64_t D, float* const* outs, int nout,
                  hipStream_t s) {
  Outs o{};
  for (int i = 0; i < nout; ++i) o.p[i] = outs[i];
  hipLaunchKernelGGL(fold_partials_kernel, dim3((unsigned)((D + 15) / 16), (unsigned)nout), dim3(256),
                     0, s, part, blocks, D, o);
  return check_launch("fold_partials_kernel");
}

}  // namespace norm

using namespace norm;

int64_t norm_bwd_workspace(int64_t M, int64_t D, int64_t width, int grads) {
  int cus;
  if (device_cus(&cus) != SW_OK) return 0;
  return bwd_blocks(M, D, width, cus) * D * 4 * grads;
}

int residual_norm_fwd(const ResNormArgs& a) {
  int cus, st;
  if ((st = device_cus(&cus)) != SW_OK) return st;
  const bool vec = vec_rows(a.x, a.x_st, a.D, a.bf16) && vec_rows(a.w, 0, a.D, false) &&
                   vec_rows(a.s, 0, a.D, false) && vec_rows(a.res, a.res_st, a.D, a.res_bf16) &&
                   vec_rows(a.y, 0, a.D, a.bf16) && vec_rows(a.res_out, 0, a.D, a.res_bf16);
  const int64_t wgs = 8 * (int64_t)cus;
  const hipStream_t s = current_stream();
  if (!a.bf16) return fwd_typed<float, float>(a, wgs, vec, s);
  return a.res_bf16 ? fwd_typed<uint16_t, uint16_t>(a, wgs, vec, s)
                    : fwd_typed<uint16_t, float>(a, wgs, vec, s);
}

int residual_norm_bwd(const ResNormArgs& a) {
  int cus, st;
  if ((st = device_cus(&cus)) != SW_OK) return st;
  const hipStream_t s = current_stream();
  const int grads = a.s ? 2 : 1;
  float* outs[2] = {a.dw, a.ds};
  // no rows: sums of none, and inputs that may be NULL
  if (a.M == 0) return fold_partials(nullptr, 0, a.D, outs, grads, s);
  const int64_t blocks = bwd_blocks(a.M, a.D, a.D, cus);
  Partials part(s);
  if ((st = part.get(a.ws, a.ws_bytes, (size_t)(blocks * a.D * 4 * grads),
                     "sw_residual_norm_bwd")) != SW_OK)
    return st;
  const bool vec = vec_rows(a.x, a.x_st, a.D, a.bf16) && vec_rows(a.w, 0, a.D, false) &&
                   vec_rows(a.s, 0, a.D, false) && vec_rows(a.dy, a.dy_st, a.D, a.bf16) &&
                   vec_rows(a.dres, a.dres_st, a.D, a.res_bf16) &&
                   vec_rows(a.stored, a.stored_st, a.D, a.res_bf16) && vec_rows(a.dx, 0, a.D, a.bf16) &&
                   vec_rows(a.dr, 0, a.D, a.res_bf16);
  if (!a.bf16)
    st = bwd_typed<float, float>(a, part.p, blocks, vec, s);
  else if (a.res_bf16)
    st = bwd_typed<uint16_t, uint16_t>(a, part.p, blocks, vec, s);
  else
    st = bwd_typed<uint16_t, float>(a, part.p, blocks, vec, s);
  if (st != SW_OK) return st;
  return fold_partials(part.p, blocks, a.D, outs, grads, s);
}

}  // namespace sw
