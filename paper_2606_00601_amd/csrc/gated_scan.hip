// gated_scan.hip -- the gated linear recurrence: forward, backward and one step.
#include "gated_math.h"
#include "gated_scan.h"
#include "norm_rows.h"

namespace sw {
namespace gated {
namespace {

__device__ __forceinline__ float get(const StepRows& t, int64_t j, const float*) {
  return ((const float*)t.p)[j];
}
__device__ __forceinline__ float get(const StepRows& t, int64_t j, const uint16_t*) {
  return bf16_one(((const uint16_t*)t.p)[j]);
}
__device__ __forceinline__ void put(void* p, int64_t j, float v, const float*) { ((float*)p)[j] = v; }
__device__ __forceinline__ void put(void* p, int64_t j, float v, const uint16_t*) {
  ((uint16_t*)p)[j] = (uint16_t)bf16_rne(v);
}

// Steps [first, end) of sequence n, in row b.
struct Span {
  int64_t b, first, end;
};
__device__ __forceinline__ Span span_of(const GatedArgs& a, int64_t n) {
  if (!a.cu) return {n, 0, a.L};
  int64_t f = a.cu[n], e = a.cu[n + 1];
  f = f < 0 ? 0 : f > a.L ? a.L : f;
  e = e < f ? f : e > a.L ? a.L : e;
  return {0, f, e};
}

// A lane for each sequence and channel, step by step.
template <class E>
__global__ __launch_bounds__(64) void fwd_kernel(GatedArgs a, float* all) {
  const int64_t d = blockIdx.x * 64ll + threadIdx.x;
  if (d >= a.D) return;
  const E* type = nullptr;
  const int64_t nck = (a.L + SW_GATED_CKPT - 1) / SW_GATED_CKPT;
  const float k = a.B * a.L ? rate_of(a.lam[d], a.c) : 0.0f;
  for (int64_t n = blockIdx.y; n < a.nseq; n += gridDim.y) {
    const Span s = span_of(a, n);
    float h = a.h0 ? a.h0[n * a.D + d] : 0.0f;
    for (int64_t t = s.first; t < s.end; ++t) {
      if (a.ckpt && t % SW_GATED_CKPT == 0) a.ckpt[(s.b * nck + t / SW_GATED_CKPT) * a.D + d] = h;
      float f, u;
      pair_of<E>(get(a.x, s.b * a.x.sb + t * a.x.sl + d, type),
                 get(a.r, s.b * a.r.sb + t * a.r.sl + d, type),
                 get(a.i, s.b * a.i.sb + t * a.i.sl + d, type), k, f, u);
      h = __builtin_fmaf(f, h, u);
      if (all) all[(s.b * a.L + t) * a.D + d] = h;
      if (a.h) put(a.h, (s.b * a.L + t) * a.D + d, h, type);
    }
    if (a.h_last) a.h_last[n * a.D + d] = h;
  }
}

template <class E>
__global__ __launch_bounds__(64) void bwd_kernel(GatedArgs a, const float* all, float* part) {
  const int64_t d = blockIdx.x * 64ll + threadIdx.x;
  if (d >= a.D) return;
  const E* type = nullptr;
  const float k = a.B * a.L ? rate_of(a.lam[d], a.c) : 0.0f;
  float sum = 0.0f;
  for (int64_t n = blockIdx.y; n < a.nseq; n += gridDim.y) {
    const Span s = span_of(a, n);
    float g = a.dh_last ? a.dh_last[n * a.D + d] : 0.0f;
    const float h0 = a.h0 ? a.h0[n * a.D + d] : 0.0f;
    for (int64_t t = s.end - 1; t >= s.first; --t) {
      const float x = get(a.x, s.b * a.x.sb + t * a.x.sl + d, type);
      const Step p = step_of<E>(x, get(a.r, s.b * a.r.sb + t * a.r.sl + d, type),
                                get(a.i, s.b * a.i.sb + t * a.i.sl + d, type), k);
      const int64_t o = (s.b * a.L + t) * a.D + d;
      const float prev = t > s.first ? all[o - a.D] : h0;
      g += get(a.dh, s.b * a.dh.sb + t * a.dh.sl + d, type);
      const float gx = g * p.b * p.si;
      const float e = g * (p.q * p.si * x - (p.m < 1e3f ? p.m : 1e3f) * p.a * prev);
      put(a.dx, o, gx, type);
      put(a.di, o, gx * x * p.rest_i, type);
      put(a.dr, o, e * p.rest_r, type);
      sum += e;
      g *= p.a;
    }
    if (a.dh0) a.dh0[n * a.D + d] = g;
  }
  part[blockIdx.y * a.D + d] = sum * (a.B * a.L ? rate_slope(a.lam[d]) : 0.0f);
}

// Zero in up to three (L, D) arrays at the steps that no sequence covers.
template <class E>
__global__ __launch_bounds__(256) void uncovered_kernel(GatedArgs a, E* p, E* q, E* r) {
  int64_t f = a.cu[0], e = a.cu[a.nseq];
  f = f < 0 ? 0 : f > a.L ? a.L : f;
  e = e < f ? f : e > a.L ? a.L : e;
  for (int64_t t = blockIdx.x; t < a.L; t += gridDim.x) {
    if (t >= f && t < e) continue;
    for (int64_t d = threadIdx.x; d < a.D; d += 256) {
      if (p) p[t * a.D + d] = 0;
      if (q) q[t * a.D + d] = 0;
      if (r) r[t * a.D + d] = 0;
    }
  }
}

template <class E>
__global__ __launch_bounds__(256) void step_kernel(GatedStepArgs a) {
  const E* type = nullptr;
  const int64_t d = blockIdx.x * 256ll + threadIdx.x;
  if (d >= a.D) return;
  const float k = rate_of(a.lam[d], a.c);
  for (int64_t b = blockIdx.y; b < a.B; b += gridDim.y) {
    const int64_t slot = a.slots ? a.slots[b] : b;
    float h = 0.0f;
    if (slot >= 0 && slot < a.pool) {
      float f, u;
      pair_of<E>(get({a.x, 0, 0}, b * a.x_st + d, type), get({a.r, 0, 0}, b * a.r_st + d, type),
                 get({a.i, 0, 0}, b * a.i_st + d, type), k, f, u);
      float* s = a.state + slot * a.D + d;
      h = __builtin_fmaf(f, *s, u);
      *s = h;
    }
    put(a.h, b * a.D + d, h, type);
  }
}

constexpr int64_t ROWS = 256;
unsigned rows_of(int64_t n) { return (unsigned)(n < ROWS ? n : ROWS); }

template <class E>
int run_fwd(const GatedArgs& a, float* all, hipStream_t s) {
  hipLaunchKernelGGL(fwd_kernel<E>, dim3((unsigned)((a.D + 63) / 64), rows_of(a.nseq)), dim3(64), 0, s,
                     a, all);
  int st = check_launch("fwd_kernel");
  if (st == SW_OK && a.cu && a.h && a.L > 0) {
    hipLaunchKernelGGL(uncovered_kernel<E>, dim3((unsigned)(a.L < 1024 ? a.L : 1024)), dim3(256), 0,
                       s, a, (E*)a.h, (E*)nullptr, (E*)nullptr);
    st = check_launch("uncovered_kernel");
  }
  return st;
}

template <class E>
int run_bwd(const GatedArgs& a, float* ws, hipStream_t s) {
  int st;
  GatedArgs f = a;
  f.h_last = nullptr;
  if ((st = run_fwd<E>(f, ws, s)) != SW_OK) return st;
  float* part = ws + a.B * a.L * a.D;
  hipLaunchKernelGGL(bwd_kernel<E>, dim3((unsigned)((a.D + 63) / 64), rows_of(a.nseq)), dim3(64), 0, s,
                     a, ws, part);
  if ((st = check_launch("bwd_kernel")) != SW_OK) return st;
  if (a.cu && a.L > 0) {
    hipLaunchKernelGGL(uncovered_kernel<E>, dim3((unsigned)(a.L < 1024 ? a.L : 1024)), dim3(256), 0,
                       s, a, (E*)a.dx, (E*)a.dr, (E*)a.di);
    if ((st = check_launch("uncovered_kernel")) != SW_OK) return st;
  }
  float* outs[1] = {a.dlam};
  return norm::fold_partials(part, rows_of(a.nseq), a.D, outs, 1, s);
}

}  // namespace
}  // namespace gated

using namespace gated;

int64_t gated_scan_fwd_workspace(int64_t, int64_t, int64_t) { return 0; }
int64_t gated_scan_bwd_workspace(int64_t B, int64_t L, int64_t D, bool) {
  return (B * L + ROWS) * D * 4;
}

int gated_scan_fwd(const GatedArgs& a) {
  if (a.nseq == 0) return SW_OK;
  const hipStream_t s = current_stream();
  return a.bf16 ? run_fwd<uint16_t>(a, nullptr, s) : run_fwd<float>(a, nullptr, s);
}

int gated_scan_bwd(const GatedArgs& a) {
  const hipStream_t s = current_stream();
  float* outs[1] = {a.dlam};
  if (a.nseq == 0) return norm::fold_partials(nullptr, 0, a.D, outs, 1, s);
  norm::Partials ws(s);
  int st;
  if ((st = ws.get(a.ws, a.ws_bytes, (size_t)gated_scan_bwd_workspace(a.B, a.L, a.D, false), "sw_gated_scan_bwd")) != SW_OK)
    return st;
  return a.bf16 ? run_bwd<uint16_t>(a, ws.p, s) : run_bwd<float>(a, ws.p, s);
}

int gated_scan_step(const GatedStepArgs& a) {
  const hipStream_t s = current_stream();
  const dim3 grid((unsigned)((a.D + 255) / 256), rows_of(a.B));
  if (a.bf16)
    hipLaunchKernelGGL(step_kernel<uint16_t>, grid, dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL(step_kernel<float>, grid, dim3(256), 0, s, a);
  return check_launch("step_kernel");
}

}  // namespace sw
