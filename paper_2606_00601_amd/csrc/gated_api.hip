// gated_api.hip -- the C ABI of the gated recurrence: argument validation and
// dispatch.  Declarations and the full contract are in include/scanweaver.h.
#include <math.h>

#include "gated_scan.h"
#include "sw_check.h"

namespace sw {
namespace {

bool known(int dtype) { return dtype == SW_DTYPE_F32 || dtype == SW_DTYPE_BF16; }

bool is_rate(float c) { return c > 0.0f && isfinite(c); }

// Bytes that rows of these strides reach over; false on overflow.
bool reach(const StepRows& x, int64_t B, int64_t L, int64_t D, int64_t es, size_t* bytes) {
  int64_t n = D, t;
  if (B == 0 || L == 0 || D == 0) {
    *bytes = 0;
    return true;
  }
  if (!mul_ok(B - 1, x.sb, &t) || __builtin_add_overflow(n, t, &n) || !mul_ok(L - 1, x.sl, &t) ||
      __builtin_add_overflow(n, t, &n) || !mul_ok(n, es, &n))
    return false;
  *bytes = (size_t)n;
  return true;
}

int check_sizes(const GatedArgs& a) {
  if (a.B < 0 || a.L < 0 || a.D < 0 || a.nseq < 0)
    return fail(SW_ERR_INVALID_ARG, "negative size (B=%lld L=%lld D=%lld nseq=%lld)", (long long)a.B,
                (long long)a.L, (long long)a.D, (long long)a.nseq);
  if (!is_rate(a.c)) return fail(SW_ERR_INVALID_ARG, "c=%g is not positive and finite", (double)a.c);
  if (a.cu ? a.B != 1 || a.nseq < 1 : a.nseq != a.B)
    return fail(SW_ERR_INVALID_ARG, a.cu ? "packed sequences need B=1 and nseq>=1 (B=%lld nseq=%lld)"
                                         : "nseq must be B without cu_seqlens (B=%lld nseq=%lld)",
                (long long)a.B, (long long)a.nseq);
  if (a.L >= ((int64_t)1 << 31) - 1024)
    return fail(SW_ERR_UNSUPPORTED, "L=%lld steps", (long long)a.L);
  if (a.D >= (int64_t)1 << 28) return fail(SW_ERR_UNSUPPORTED, "D=%lld channels", (long long)a.D);
  int64_t n;
  // the largest workspace holds 24 bytes a channel for every 64 steps begun, of groups of 64
  // channels: words of 16, a partial sum and a state
  if (!mul_ok(a.B, a.L + 1, &n) || !mul_ok(n, a.D + 64, &n) || !mul_ok(n, 32, &n) ||
      !mul_ok(a.nseq, a.D, &n) || !mul_ok(n, 16, &n))
    return fail(SW_ERR_UNSUPPORTED, "sizes overflow");
  for (const StepRows* x : {&a.x, &a.r, &a.i, &a.dh})
    if (x->sb < 0 || x->sl < 0) return fail(SW_ERR_INVALID_ARG, "negative stride");
  return SW_OK;
}

int64_t ckpt_rows(const GatedArgs& a) { return a.B * ((a.L + SW_GATED_CKPT - 1) / SW_GATED_CKPT); }

int fwd(const GatedArgs& a) {
  int st;
  if ((st = check_sizes(a)) != SW_OK) return st;
  const bool any = a.B * a.L * a.D > 0;
  if (!any && !(a.nseq * a.D > 0 && a.h_last)) return SW_OK;
  const size_t es = a.bf16 ? 2 : 4, d4 = (size_t)a.D * 4;
  size_t nx, nr, ni;
  if (!reach(a.x, a.B, a.L, a.D, (int64_t)es, &nx) || !reach(a.r, a.B, a.L, a.D, (int64_t)es, &nr) ||
      !reach(a.i, a.B, a.L, a.D, (int64_t)es, &ni))
    return fail(SW_ERR_UNSUPPORTED, "strides overflow");
  const In ins[] = {{a.x.p, es, nx, "x", any},
                    {a.r.p, es, nr, "r", any},
                    {a.i.p, es, ni, "i", any},
                    {a.lam, 4, d4, "lam", any},
                    {a.h0, 4, (size_t)a.nseq * d4, "h0", false},
                    {a.cu, 4, (size_t)(a.nseq + 1) * 4, "cu_seqlens", false}};
  const In outs[] = {{a.h, es, (size_t)(a.B * a.L * a.D) * es, "h", false},
                     {a.h_last, 4, (size_t)a.nseq * d4, "h_last", false},
                     {a.ckpt, 4, (size_t)ckpt_rows(a) * d4, "ckpt", false},
                     {a.ws, 16, a.ws_bytes, "workspace", false}};
  if ((st = check_arrays(ins, 6, outs, 4)) != SW_OK) return st;
  return gated_scan_fwd(a);
}

int bwd(const GatedArgs& a) {
  int st;
  if ((st = check_sizes(a)) != SW_OK) return st;
  if (a.D == 0) return SW_OK;
  const bool any = a.B * a.L > 0;
  const size_t es = a.bf16 ? 2 : 4, d4 = (size_t)a.D * 4;
  size_t nx, nr, ni, nd;
  if (!reach(a.x, a.B, a.L, a.D, (int64_t)es, &nx) || !reach(a.r, a.B, a.L, a.D, (int64_t)es, &nr) ||
      !reach(a.i, a.B, a.L, a.D, (int64_t)es, &ni) || !reach(a.dh, a.B, a.L, a.D, (int64_t)es, &nd))
    return fail(SW_ERR_UNSUPPORTED, "strides overflow");
  const size_t ng = (size_t)(a.B * a.L * a.D) * es, ns = (size_t)a.nseq * d4;
  const In ins[] = {{a.x.p, es, nx, "x", any},
                    {a.r.p, es, nr, "r", any},
                    {a.i.p, es, ni, "i", any},
                    {a.lam, 4, d4, "lam", any},
                    {a.h0, 4, ns, "h0", false},
                    {a.cu, 4, (size_t)(a.nseq + 1) * 4, "cu_seqlens", false},
                    {a.ckpt_in, 4, (size_t)ckpt_rows(a) * d4, "ckpt", false},
                    {a.dh.p, es, nd, "dh", any},
                    {a.dh_last, 4, ns, "dh_last", false}};
  const In outs[] = {{a.dx, es, ng, "dx", any},
                     {a.dr, es, ng, "dr", any},
                     {a.di, es, ng, "di", any},
                     {a.dlam, 4, d4, "dlam", true},
                     {a.dh0, 4, ns, "dh0", false},
                     {a.ws, 16, a.ws_bytes, "workspace", false}};
  if ((st = check_arrays(ins, 9, outs, 6)) != SW_OK) return st;
  return gated_scan_bwd(a);
}

int step(const GatedStepArgs& a) {
  if (a.B < 0 || a.D < 0 || a.pool < 0)
    return fail(SW_ERR_INVALID_ARG, "negative size (B=%lld D=%lld pool=%lld)", (long long)a.B,
                (long long)a.D, (long long)a.pool);
  if (!is_rate(a.c)) return fail(SW_ERR_INVALID_ARG, "c=%g is not positive and finite", (double)a.c);
  if (!a.slots && a.pool < a.B)
    return fail(SW_ERR_INVALID_ARG, "pool=%lld states for B=%lld sequences", (long long)a.pool,
                (long long)a.B);
  int64_t n;
  if (!mul_ok(a.B, a.D, &n) || !mul_ok(n, 8, &n) || !mul_ok(a.pool, a.D, &n) || !mul_ok(n, 8, &n))
    return fail(SW_ERR_UNSUPPORTED, "sizes overflow");
  if (a.D >= (int64_t)1 << 28) return fail(SW_ERR_UNSUPPORTED, "D=%lld channels", (long long)a.D);
  if (a.x_st < 0 || a.r_st < 0 || a.i_st < 0) return fail(SW_ERR_INVALID_ARG, "negative stride");
  if (a.B == 0 || a.D == 0) return SW_OK;
  const size_t es = a.bf16 ? 2 : 4;
  size_t nx, nr, ni;
  if (!reach({nullptr, a.x_st, 0}, a.B, 1, a.D, (int64_t)es, &nx) ||
      !reach({nullptr, a.r_st, 0}, a.B, 1, a.D, (int64_t)es, &nr) ||
      !reach({nullptr, a.i_st, 0}, a.B, 1, a.D, (int64_t)es, &ni))
    return fail(SW_ERR_UNSUPPORTED, "strides overflow");
  const In ins[] = {{a.x, es, nx, "x", true},
                    {a.r, es, nr, "r", true},
                    {a.i, es, ni, "i", true},
                    {a.lam, 4, (size_t)a.D * 4, "lam", true},
                    {a.slots, 4, (size_t)a.B * 4, "slots", false}};
  const In outs[] = {{a.state, 4, (size_t)(a.pool * a.D) * 4, "state", a.pool > 0},
                     {a.h, es, (size_t)(a.B * a.D) * es, "h", true}};
  int st;
  if ((st = check_arrays(ins, 5, outs, 2)) != SW_OK) return st;
  return gated_scan_step(a);
}

GatedArgs common(const void* x, const void* r, const void* i, const float* lam, const float* h0,
                 const int32_t* cu, int64_t B, int64_t L, int64_t D, int64_t nseq,
                 const int64_t* st, int dtype, float c, void* ws, int64_t ws_bytes) {
  GatedArgs a;
  a.x = {x, st[0], st[1]};
  a.r = {r, st[2], st[3]};
  a.i = {i, st[4], st[5]};
  a.lam = lam;
  a.h0 = h0;
  a.cu = cu;
  a.B = B;
  a.L = L;
  a.D = D;
  a.nseq = nseq;
  a.bf16 = dtype == SW_DTYPE_BF16;
  a.c = c;
  a.ws = ws;
  a.ws_bytes = ws ? (size_t)ws_bytes : 0;
  return a;
}

int check_call(const int64_t* strides, int dtype, int64_t ws_bytes) {
  if (!known(dtype)) return fail(SW_ERR_INVALID_ARG, "unknown dtype %d", dtype);
  if (!strides) return fail(SW_ERR_INVALID_ARG, "strides is NULL");
  if (ws_bytes < 0) return fail(SW_ERR_INVALID_ARG, "negative workspace size");
  return SW_OK;
}

// Sizes a workspace query answers for.
bool sane(int64_t B, int64_t L, int64_t D) {
  GatedArgs a;
  a.B = a.nseq = B;
  a.L = L;
  a.D = D;
  a.c = 1.0f;
  return check_sizes(a) == SW_OK && B * L * D > 0;
}

}  // namespace
}  // namespace sw

SW_API int sw_gated_scan_fwd(const void* x, const void* r, const void* i, const float* lam,
                             const float* h0, const int32_t* cu_seqlens, void* h, float* h_last,
                             float* ckpt, int64_t B, int64_t L, int64_t D, int64_t nseq,
                             const int64_t* strides, int dtype, float c, void* workspace,
                             int64_t workspace_bytes) {
  int st;
  if ((st = sw::check_call(strides, dtype, workspace_bytes)) != SW_OK) return st;
  sw::GatedArgs a = sw::common(x, r, i, lam, h0, cu_seqlens, B, L, D, nseq, strides, dtype, c,
                               workspace, workspace_bytes);
  a.h = h;
  a.h_last = h_last;
  a.ckpt = ckpt;
  return sw::fwd(a);
}

SW_API int64_t sw_gated_scan_fwd_workspace(int64_t B, int64_t L, int64_t D) {
  return sw::sane(B, L, D) ? sw::gated_scan_fwd_workspace(B, L, D) : 0;
}

SW_API int sw_gated_scan_bwd(const void* x, const void* r, const void* i, const float* lam,
                             const float* h0, const int32_t* cu_seqlens, const float* ckpt,
                             const void* dh, const float* dh_last, void* dx, void* dr, void* di,
                             float* dlam, float* dh0, int64_t B, int64_t L, int64_t D, int64_t nseq,
                             const int64_t* strides, int dtype, float c, void* workspace,
                             int64_t workspace_bytes) {
  int st;
  if ((st = sw::check_call(strides, dtype, workspace_bytes)) != SW_OK) return st;
  sw::GatedArgs a = sw::common(x, r, i, lam, h0, cu_seqlens, B, L, D, nseq, strides, dtype, c,
                               workspace, workspace_bytes);
  a.dh = {dh, strides[6], strides[7]};
  a.ckpt_in = ckpt;
  a.dh_last = dh_last;
  a.dx = dx;
  a.dr = dr;
  a.di = di;
  a.dlam = dlam;
  a.dh0 = dh0;
  return sw::bwd(a);
}

SW_API int64_t sw_gated_scan_bwd_workspace(int64_t B, int64_t L, int64_t D, int ckpt) {
  return sw::sane(B, L, D) ? sw::gated_scan_bwd_workspace(B, L, D, ckpt != 0) : 0;
}

SW_API int sw_gated_scan_step(const void* x, const void* r, const void* i, const float* lam,
                              float* state, const int32_t* slots, void* h, int64_t B, int64_t D,
                              int64_t pool, const int64_t* strides, int dtype, float c) {
  int st;
  if ((st = sw::check_call(strides, dtype, 0)) != SW_OK) return st;
  sw::GatedStepArgs a;
  a.x = x;
  a.r = r;
  a.i = i;
  a.lam = lam;
  a.state = state;
  a.slots = slots;
  a.h = h;
  a.B = B;
  a.D = D;
  a.pool = pool;
  a.x_st = strides[0];
  a.r_st = strides[1];
  a.i_st = strides[2];
  a.bf16 = dtype == SW_DTYPE_BF16;
  a.c = c;
  return sw::step(a);
}
