// gated_norm.hip -- the norm after a block's mixer, with its gate, over groups
// of columns: y = w u / rms(u) with u = x silu(z), or y = w x / rms(x) silu(z),
// and its gradients.
#include "norm_rows.h"

namespace sw {
namespace norm {
namespace {

// 1 / (1 + e^-z) and, in rest, 1 minus it.  fp32 inputs: to fp32 rounding.  -z log2 e
// is rounded to h, which alone would cost 2^-24 |z| of the result; what that misses, r,
// multiplies 2^h by 1 + r ln 2.  z is held only where 2^h is 0 or infinite already: an
// infinite one would make r NaN.  bf16 inputs go without these (2^-18 at |z| = 64, beside
// results of 2^-9): with them the backward of 16384 rows of 12 groups of 128 took 54 us
// for 50.
template <class E>
__device__ __forceinline__ float sigmoid_f32(float z, float& rest) {
  constexpr float C = 1.4426950408889634f, REST = (float)(1.4426950408889634 - (double)C);
  if constexpr (sizeof(E) == 2) {
    const float s = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-z * C));
    rest = 1.0f - s;
    return s;
  } else {
    const float m = -__builtin_amdgcn_fmed3f(z, -200.0f, 200.0f);
    const float h = m * C;
    const float r = __builtin_fmaf(m, REST, __builtin_fmaf(m, C, -h));
    const float e = __builtin_amdgcn_exp2f(h) * __builtin_fmaf(r, 0.6931471805599453f, 1.0f);
    const float s = __builtin_amdgcn_rcpf(1.0f + e);
    rest = z > 0.0f ? e * s : 1.0f - s;
    return s;
  }
}

enum Gate { NONE, BEFORE, AFTER };

// Workgroup blockIdx.x takes group blockIdx.x % G of the rows of its block.  16384
// rows of 12 groups of 128, bf16: 27.6 us, 151 MB at a copy's rate.
template <class E, Gate GATE, int LPR, int NV>
__global__ __launch_bounds__(threads_of(LPR)) void gated_fwd_kernel(GatedNormArgs a, int groups,
                                                                    bool vec) {
  constexpr int RPW = threads_of(LPR) / LPR;
  __shared__ RowSum<LPR, 1> sh;
  const int sub = threadIdx.x / LPR, li = threadIdx.x % LPR;
  const int64_t g0 = (blockIdx.x % groups) * a.group;
  const int64_t blk = blockIdx.x / groups, blocks = gridDim.x / groups;
  int par = 0;
  float w[NV][8];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int64_t c = (v * LPR + li) * 8;
    load8(a.w + g0 + c, w[v], a.group - c, vec);
  }
  for (int64_t m = blk * RPW + sub; m < a.M; m += blocks * RPW) {
    float x[NV][8], gate[NV][8];
    float sum[1] = {0.0f};
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int64_t c = (v * LPR + li) * 8;
      load8((const E*)a.x + m * a.x_st + g0 + c, x[v], a.group - c, vec);
      if (GATE != NONE) {
        load8((const E*)a.z + m * a.z_st + g0 + c, gate[v], a.group - c, vec);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          float rest;
          gate[v][j] *= sigmoid_f32<E>(gate[v][j], rest);
          if (GATE == BEFORE) x[v][j] *= gate[v][j];
        }
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) sum[0] = __builtin_fmaf(x[v][j], x[v][j], sum[0]);
    }
    row_sum<LPR, 1>(sum, sh, par);
    const float inv = rsqrtf(sum[0] / (float)a.group + a.eps);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int64_t c = (v * LPR + li) * 8;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        x[v][j] *= inv * w[v][j];
        if (GATE == AFTER) x[v][j] *= gate[v][j];
      }
      store8((E*)a.y + m * a.D + g0 + c, x[v], a.group - c, vec);
    }
  }
}

// With the gate before: n = u inv, du = inv (w dy - n mean(w dy n)), dx = du silu(z),
// dz = du x silu'(z), dw = sum dy n.  After: the same with u = x and the gate's
// share of dy: dn = w dy silu(z), dz = w dy n silu'(z), dw = sum dy n silu(z).  The
// gate's place is a parameter of the kernel: as a branch it cost 72 us where this
// takes 65, and `vec` as one made each load wait for the one before: 51 us without
// (16384 rows of 12 groups of 128, bf16, 252 MB at 4.9 TB/s).
template <class E, Gate GATE, bool vec, int LPR, int NV>
__global__ __launch_bounds__(threads_of(LPR)) void gated_bwd_kernel(GatedNormArgs a, int groups,
                                                                    float* part) {
  constexpr int RPW = threads_of(LPR) / LPR;
  __shared__ RowSum<LPR, 2> sh;
  __shared__ float lds[partial_lds<LPR, NV>];
  const int sub = threadIdx.x / LPR, li = threadIdx.x % LPR;
  const int64_t g0 = (blockIdx.x % groups) * a.group;
  const int64_t blk = blockIdx.x / groups, blocks = gridDim.x / groups;
  int par = 0;
  float dw[NV][8], w[NV][8];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int64_t c = (v * LPR + li) * 8;
    load8(a.w + g0 + c, w[v], a.group - c, vec);
#pragma unroll
    for (int j = 0; j < 8; ++j) dw[v][j] = 0.0f;
  }
  for (int64_t m = blk * RPW + sub; m < a.M; m += blocks * RPW) {
    float x[NV][8], z[NV][8], slope[NV][8], d[NV][8];  // z becomes silu(z)
    float sum[2] = {0.0f, 0.0f};
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int64_t c = (v * LPR + li) * 8;
      load8((const E*)a.x + m * a.x_st + g0 + c, x[v], a.group - c, vec);
      load8((const E*)a.dy + m * a.dy_st + g0 + c, d[v], a.group - c, vec);
      if (GATE != NONE) load8((const E*)a.z + m * a.z_st + g0 + c, z[v], a.group - c, vec);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        float u = x[v][j], dn = w[v][j] * d[v][j];
        if (GATE != NONE) {
          float rest;
          const float sg = sigmoid_f32<E>(z[v][j], rest);
          slope[v][j] = sg * __builtin_fmaf(z[v][j], rest, 1.0f);
          z[v][j] *= sg;
          if (GATE == BEFORE) u *= z[v][j];
          if (GATE == AFTER) dn *= z[v][j];
        }
        sum[0] = __builtin_fmaf(u, u, sum[0]);
        sum[1] = __builtin_fmaf(dn, u, sum[1]);
      }
    }
    row_sum<LPR, 2>(sum, sh, par);
    const float inv = rsqrtf(sum[0] / (float)a.group + a.eps);
    const float mean = sum[1] * inv / (float)a.group;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int64_t c = (v * LPR + li) * 8;
      float dx[8], dz[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float gate = GATE == NONE ? 1.0f : z[v][j];
        const float n = (GATE == BEFORE ? x[v][j] * gate : x[v][j]) * inv;
        const float wd = w[v][j] * d[v][j];
        const float du = inv * ((GATE == AFTER ? wd * gate : wd) - n * mean);
        dw[v][j] = __builtin_fmaf(GATE == AFTER ? d[v][j] * gate : d[v][j], n, dw[v][j]);
        dx[j] = GATE == BEFORE ? du * gate : du;
        if (GATE != NONE) dz[j] = (GATE == AFTER ? wd * n : du * x[v][j]) * slope[v][j];
      }
      store8((E*)a.dx + m * a.D + g0 + c, dx, a.group - c, vec);
      if (GATE != NONE) store8((E*)a.dz + m * a.D + g0 + c, dz, a.group - c, vec);
    }
  }
  put_partial<LPR, NV>(dw, lds, part + blk * a.D + g0, a.group);
}

template <class E, Gate GATE>
int fwd_gated(const GatedNormArgs& a, int groups, int64_t wgs, bool vec, hipStream_t s) {
#define CALL(LPR, NV)                                                                             \
  do {                                                                                            \
    const int64_t need = (a.M + threads_of(LPR) / LPR - 1) / (threads_of(LPR) / LPR);             \
    int64_t n = (wgs + groups - 1) / groups;                                                      \
    if (n > need) n = need;                                                                       \
    hipLaunchKernelGGL((gated_fwd_kernel<E, GATE, LPR, NV>), dim3((unsigned)(n * groups)),              \
                       dim3(threads_of(LPR)), 0, s, a, groups, vec);                              \
  } while (0)
  SW_NORM_PICK(a.group, CALL);
#undef CALL
  return check_launch("gated_fwd_kernel");
}

template <class E, Gate GATE, bool VEC>
int bwd_vec(const GatedNormArgs& a, int groups, float* part, int64_t blocks, hipStream_t s) {
#define CALL(LPR, NV)                                                                              \
  hipLaunchKernelGGL((gated_bwd_kernel<E, GATE, VEC, LPR, NV>), dim3((unsigned)(blocks * groups)), \
                     dim3(threads_of(LPR)), 0, s, a, groups, part)
  SW_NORM_PICK_BWD(a.group, CALL);
#undef CALL
  return check_launch("gated_bwd_kernel");
}
template <class E, Gate GATE>
int bwd_gated(const GatedNormArgs& a, int groups, float* part, int64_t blocks, bool vec,
              hipStream_t s) {
  return vec ? bwd_vec<E, GATE, true>(a, groups, part, blocks, s)
             : bwd_vec<E, GATE, false>(a, groups, part, blocks, s);
}

template <class E>
int fwd_typed(const GatedNormArgs& a, int groups, int64_t wgs, bool vec, hipStream_t s) {
  return !a.z      ? fwd_gated<E, NONE>(a, groups, wgs, vec, s)
         : a.after ? fwd_gated<E, AFTER>(a, groups, wgs, vec, s)
                   : fwd_gated<E, BEFORE>(a, groups, wgs, vec, s);
}

template <class E>
int bwd_typed(const GatedNormArgs& a, int groups, float* part, int64_t blocks, bool vec,
              hipStream_t s) {
  return !a.z      ? bwd_gated<E, NONE>(a, groups, part, blocks, vec, s)
         : a.after ? bwd_gated<E, AFTER>(a, groups, part, blocks, vec, s)
                   : bwd_gated<E, BEFORE>(a, groups, part, blocks, vec, s);
}

}  // namespace
}  // namespace norm

using namespace norm;

int gated_norm_fwd(const GatedNormArgs& a) {
  int cus, st;
  if ((st = device_cus(&cus)) != SW_OK) return st;
  const bool vec = vec_rows(a.x, a.x_st, a.group, a.bf16) && vec_rows(a.z, a.z_st, a.group, a.bf16) &&
                   vec_rows(a.w, 0, a.group, false) && vec_rows(a.y, 0, a.group, a.bf16);
  const int groups = (int)(a.D / a.group);
  const hipStream_t s = current_stream();
  return a.bf16 ? fwd_typed<uint16_t>(a, groups, 8 * (int64_t)cus, vec, s)
                : fwd_typed<float>(a, groups, 8 * (int64_t)cus, vec, s);
}

int gated_norm_bwd(const GatedNormArgs& a) {
  int cus, st;
  if ((st = device_cus(&cus)) != SW_OK) return st;
  const hipStream_t s = current_stream();
  const int groups = (int)(a.D / a.group);
  float* outs[2] = {a.dw, nullptr};
  // no rows: a sum of none, and inputs that may be NULL
  if (a.M == 0) return fold_partials(nullptr, 0, a.D, outs, 1, s);
  const int64_t blocks = bwd_blocks(a.M, a.D, a.group, cus);
  Partials part(s);
  if ((st = part.get(a.ws, a.ws_bytes, (size_t)(blocks * a.D * 4), "sw_gated_norm_bwd")) != SW_OK)
    return st;
  const bool vec = vec_rows(a.x, a.x_st, a.group, a.bf16) && vec_rows(a.z, a.z_st, a.group, a.bf16) &&
                   vec_rows(a.w, 0, a.group, false) && vec_rows(a.dy, a.dy_st, a.group, a.bf16) &&
                   vec_rows(a.dx, 0, a.group, a.bf16) && vec_rows(a.dz, 0, a.group, a.bf16);
  st = a.bf16 ? bwd_typed<uint16_t>(a, groups, part.p, blocks, vec, s)
              : bwd_typed<float>(a, groups, part.p, blocks, vec, s);
  if (st != SW_OK) return st;
  return fold_partials(part.p, blocks, a.D, outs, 1, s);
}

}  // namespace sw
