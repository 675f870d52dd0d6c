// norm_api.hip -- the C ABI of the block norms: argument validation and dispatch.
// Declarations and the full contract are in include/scanweaver.h.
#include "block_norm.h"
#include "sw_check.h"

namespace sw {
namespace {

bool known(int dtype) { return dtype == SW_DTYPE_F32 || dtype == SW_DTYPE_BF16; }

// Sizes and strides shared by all: M rows of D columns, normed over `width`.
int check_rows(int64_t M, int64_t D, int64_t width, std::initializer_list<int64_t> strides) {
  if (M < 0 || D < 0) return fail(SW_ERR_INVALID_ARG, "negative size (M=%lld D=%lld)", (long long)M,
                                  (long long)D);
  if (width < 1 || width > NORM_MAX_WIDTH)
    return fail(SW_ERR_UNSUPPORTED, "norm over %lld columns, outside [1, %lld]", (long long)width,
                (long long)NORM_MAX_WIDTH);
  if (D % width != 0)
    return fail(SW_ERR_INVALID_ARG, "D=%lld is no multiple of the group's %lld columns", (long long)D,
                (long long)width);
  int64_t n;
  if (!mul_ok(M, D, &n) || !mul_ok(n, 4, &n) || !mul_ok(D, 1 << 16, &n))
    return fail(SW_ERR_UNSUPPORTED, "sizes overflow");
  if (D / width > SW_MAX_WGS / 4096)
    return fail(SW_ERR_UNSUPPORTED, "%lld groups exceed the launch limit", (long long)(D / width));
  for (int64_t s : strides) {
    if (s < 0) return fail(SW_ERR_INVALID_ARG, "negative stride");
    if (!mul_ok(M, s, &n) || !mul_ok(n, 4, &n))
      return fail(SW_ERR_UNSUPPORTED, "strides overflow");
  }
  return SW_OK;
}

// Bytes M rows of D elements of `es` bytes reach over.
size_t reach(int64_t M, int64_t D, int64_t st, size_t es) {
  return M == 0 ? 0 : (size_t)((M - 1) * st + D) * es;
}

struct In {
  const void* p;
  size_t align, bytes;
  const char* name;
  bool required;
};

// Inputs, then outputs: device memory, aligned, no output over another array.
int check_arrays(const In* ins, int nin, const In* outs, int nout) {
  int dev, st;
  if ((st = current_device(&dev)) != SW_OK) return st;
  Span is[8], os[8];
  for (int i = 0; i < nin; ++i) {
    if ((st = check_ptr(ins[i].p, ins[i].align, ins[i].name, ins[i].required, dev)) != SW_OK)
      return st;
    is[i] = {ins[i].p, ins[i].bytes, ins[i].name};
  }
  for (int i = 0; i < nout; ++i) {
    if ((st = check_ptr(outs[i].p, outs[i].align, outs[i].name, outs[i].required, dev)) != SW_OK)
      return st;
    os[i] = {outs[i].p, outs[i].bytes, outs[i].name};
  }
  return check_spans(os, nout, is, nin);
}

int res_fwd(const ResNormArgs& a) {
  int st;
  if ((st = check_rows(a.M, a.D, a.D, {a.x_st, a.res_st})) != SW_OK) return st;
  if (!a.res && (a.s || a.res_out))
    return fail(SW_ERR_INVALID_ARG, "res_scale and residual_out require residual");
  if (a.M == 0) return SW_OK;
  const size_t es = a.bf16 ? 2 : 4, rs = a.res_bf16 ? 2 : 4, d4 = (size_t)a.D * 4;
  const In ins[] = {{a.x, es, reach(a.M, a.D, a.x_st, es), "x", true},
                    {a.res, rs, reach(a.M, a.D, a.res_st, rs), "residual", false},
                    {a.w, 4, d4, "weight", true},
                    {a.s, 4, d4, "res_scale", false}};
  const In outs[] = {{a.y, es, reach(a.M, a.D, a.D, es), "y", true},
                     {a.res_out, rs, reach(a.M, a.D, a.D, rs), "residual_out", a.res != nullptr}};
  if ((st = check_arrays(ins, 4, outs, 2)) != SW_OK) return st;
  return residual_norm_fwd(a);
}

int res_bwd(const ResNormArgs& a) {
  int st;
  if ((st = check_rows(a.M, a.D, a.D, {a.x_st, a.dy_st, a.dres_st, a.stored_st})) != SW_OK) return st;
  if (a.ds && !a.s) return fail(SW_ERR_INVALID_ARG, "dres_scale requires res_scale");
  const bool any = a.M > 0;
  const size_t es = a.bf16 ? 2 : 4, rs = a.res_bf16 ? 2 : 4, d4 = (size_t)a.D * 4;
  const In ins[] = {{a.dy, es, reach(a.M, a.D, a.dy_st, es), "dy", any},
                    {a.dres, rs, reach(a.M, a.D, a.dres_st, rs), "dres", false},
                    {a.stored, rs, reach(a.M, a.D, a.stored_st, rs), "residual_out", any},
                    {a.w, 4, d4, "weight", any},
                    {a.x, es, reach(a.M, a.D, a.x_st, es), "x", any && a.s},
                    {a.s, 4, d4, "res_scale", false}};
  const In outs[] = {{a.dx, es, reach(a.M, a.D, a.D, es), "dx", false},
                     {a.dr, rs, reach(a.M, a.D, a.D, rs), "dresidual", false},
                     {a.dw, 4, d4, "dweight", true},
                     {a.ds, 4, d4, "dres_scale", a.s != nullptr},
                     {a.ws, 16, a.ws_bytes, "workspace", false}};
  if ((st = check_arrays(ins, 6, outs, 5)) != SW_OK) return st;
  return residual_norm_bwd(a);
}

int gated_fwd(const GatedNormArgs& a) {
  int st;
  if ((st = check_rows(a.M, a.D, a.group, {a.x_st, a.z_st})) != SW_OK) return st;
  if (a.M == 0 || a.D == 0) return SW_OK;
  const size_t es = a.bf16 ? 2 : 4;
  const In ins[] = {{a.x, es, reach(a.M, a.D, a.x_st, es), "x", true},
                    {a.z, es, reach(a.M, a.D, a.z_st, es), "z", false},
                    {a.w, 4, (size_t)a.D * 4, "weight", true}};
  const In outs[] = {{a.y, es, reach(a.M, a.D, a.D, es), "y", true}};
  if ((st = check_arrays(ins, 3, outs, 1)) != SW_OK) return st;
  return gated_norm_fwd(a);
}

int gated_bwd(const GatedNormArgs& a) {
  int st;
  if ((st = check_rows(a.M, a.D, a.group, {a.x_st, a.z_st, a.dy_st})) != SW_OK) return st;
  if (a.dz && !a.z) return fail(SW_ERR_INVALID_ARG, "dz requires z");
  if (a.D == 0) return SW_OK;
  const bool any = a.M > 0;
  const size_t es = a.bf16 ? 2 : 4;
  const In ins[] = {{a.dy, es, reach(a.M, a.D, a.dy_st, es), "dy", any},
                    {a.x, es, reach(a.M, a.D, a.x_st, es), "x", any},
                    {a.z, es, reach(a.M, a.D, a.z_st, es), "z", false},
                    {a.w, 4, (size_t)a.D * 4, "weight", any}};
  const In outs[] = {{a.dx, es, reach(a.M, a.D, a.D, es), "dx", any},
                     {a.dz, es, reach(a.M, a.D, a.D, es), "dz", any && a.z},
                     {a.dw, 4, (size_t)a.D * 4, "dweight", true},
                     {a.ws, 16, a.ws_bytes, "workspace", false}};
  if ((st = check_arrays(ins, 4, outs, 4)) != SW_OK) return st;
  return gated_norm_bwd(a);
}

}  // namespace
}  // namespace sw

SW_API int sw_residual_norm_fwd(const void* x, const void* residual, const float* weight,
                                const float* res_scale, void* y, void* residual_out, int64_t M,
                                int64_t D, int64_t x_stride, int64_t residual_stride, int dtype,
                                int res_dtype, float eps) {
  if (!sw::known(dtype) || !sw::known(res_dtype) ||
      (dtype == SW_DTYPE_F32 && res_dtype != SW_DTYPE_F32))
    return sw::fail(SW_ERR_INVALID_ARG, "unknown or unmatched dtypes (%d, residual %d)", dtype,
                    res_dtype);
  sw::ResNormArgs a;
  a.x = x;
  a.res = residual;
  a.w = weight;
  a.s = res_scale;
  a.y = y;
  a.res_out = residual_out;
  a.M = M;
  a.D = D;
  a.x_st = x_stride;
  a.res_st = residual_stride;
  a.bf16 = dtype == SW_DTYPE_BF16;
  a.res_bf16 = res_dtype == SW_DTYPE_BF16;
  a.eps = eps;
  return sw::res_fwd(a);
}

SW_API int sw_residual_norm_bwd(const void* dy, const void* dres, const void* residual_out,
                                const float* weight, const void* x, const float* res_scale,
                                void* dx, void* dresidual, float* dweight, float* dres_scale,
                                int64_t M, int64_t D, int64_t dy_stride, int64_t dres_stride,
                                int64_t residual_out_stride, int64_t x_stride, int dtype,
                                int res_dtype, float eps, void* workspace,
                                int64_t workspace_bytes) {
  if (!sw::known(dtype) || !sw::known(res_dtype) ||
      (dtype == SW_DTYPE_F32 && res_dtype != SW_DTYPE_F32))
    return sw::fail(SW_ERR_INVALID_ARG, "unknown or unmatched dtypes (%d, residual %d)", dtype,
                    res_dtype);
  if (workspace_bytes < 0) return sw::fail(SW_ERR_INVALID_ARG, "negative workspace size");
  sw::ResNormArgs a;
  a.dy = dy;
  a.dres = dres;
  a.stored = residual_out;
  a.w = weight;
  a.x = x;
  a.s = res_scale;
  a.dx = dx;
  a.dr = dresidual;
  a.dw = dweight;
  a.ds = dres_scale;
  a.M = M;
  a.D = D;
  a.dy_st = dy_stride;
  a.dres_st = dres_stride;
  a.stored_st = residual_out_stride;
  a.x_st = x_stride;
  a.bf16 = dtype == SW_DTYPE_BF16;
  a.res_bf16 = res_dtype == SW_DTYPE_BF16;
  a.eps = eps;
  a.ws = workspace;
  a.ws_bytes = workspace ? (size_t)workspace_bytes : 0;
  return sw::res_bwd(a);
}

SW_API int64_t sw_norm_bwd_workspace(int64_t M, int64_t D, int64_t width, int grads) {
  if (grads < 1 || grads > 2 || sw::check_rows(M, D, width, {}) != SW_OK) return 0;
  return sw::norm_bwd_workspace(M, D, width, grads);
}

SW_API int sw_gated_norm_fwd(const void* x, const void* z, const float* weight, void* y, int64_t M,
                             int64_t D, int64_t group, int64_t x_stride, int64_t z_stride,
                             int dtype, int flags, float eps) {
  if (!sw::known(dtype)) return sw::fail(SW_ERR_INVALID_ARG, "unknown dtype %d", dtype);
  if (flags & ~SW_GATE_AFTER)
    return sw::fail(SW_ERR_INVALID_ARG, "unknown flags 0x%x", (unsigned)flags);
  sw::GatedNormArgs a;
  a.x = x;
  a.z = z;
  a.w = weight;
  a.y = y;
  a.M = M;
  a.D = D;
  a.group = group;
  a.x_st = x_stride;
  a.z_st = z_stride;
  a.bf16 = dtype == SW_DTYPE_BF16;
  a.after = (flags & SW_GATE_AFTER) != 0;
  a.eps = eps;
  return sw::gated_fwd(a);
}

SW_API int sw_gated_norm_bwd(const void* dy, const void* x, const void* z, const float* weight,
                             void* dx, void* dz, float* dweight, int64_t M, int64_t D,
                             int64_t group, int64_t dy_stride, int64_t x_stride, int64_t z_stride,
                             int dtype, int flags, float eps, void* workspace,
                             int64_t workspace_bytes) {
  if (!sw::known(dtype)) return sw::fail(SW_ERR_INVALID_ARG, "unknown dtype %d", dtype);
  if (flags & ~SW_GATE_AFTER)
    return sw::fail(SW_ERR_INVALID_ARG, "unknown flags 0x%x", (unsigned)flags);
  if (workspace_bytes < 0) return sw::fail(SW_ERR_INVALID_ARG, "negative workspace size");
  sw::GatedNormArgs a;
  a.dy = dy;
  a.x = x;
  a.z = z;
  a.w = weight;
  a.dx = dx;
  a.dz = dz;
  a.dw = dweight;
  a.M = M;
  a.D = D;
  a.group = group;
  a.dy_st = dy_stride;
  a.x_st = x_stride;
  a.z_st = z_stride;
  a.bf16 = dtype == SW_DTYPE_BF16;
  a.after = (flags & SW_GATE_AFTER) != 0;
  a.eps = eps;
  a.ws = workspace;
  a.ws_bytes = workspace ? (size_t)workspace_bytes : 0;
  return sw::gated_bwd(a);
}
