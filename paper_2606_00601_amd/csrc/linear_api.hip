// linear_api.hip -- the C ABI of linear attention: argument validation and
// dispatch.  Declarations and the full contract are in include/scanweaver.h.
#include "linear_attn.h"
#include "sw_check.h"

namespace sw {
namespace {

// Elements an operand of these strides reaches over; false on overflow.
bool extent(const HeadRows& x, int64_t B, int64_t L, int64_t H, int64_t W, int64_t* n) {
  if (B == 0 || L == 0 || H == 0) {
    *n = 0;
    return true;
  }
  int64_t t, s = W;
  const int64_t st[3] = {x.sb, x.sl, x.sh}, c[3] = {B, L, H};
  for (int i = 0; i < 3; ++i)
    if (!mul_ok(c[i] - 1, st[i], &t) || __builtin_add_overflow(s, t, &s)) return false;
  *n = s;
  return mul_ok(s, 4, &t);
}

int check_sizes(const LinAttnArgs& a) {
  if (a.B < 0 || a.L < 0 || a.Hk < 0 || a.H < 0 || a.K < 0 || a.V < 0 || a.nseq < 0)
    return fail(SW_ERR_INVALID_ARG,
                "negative size (B=%lld L=%lld Hk=%lld H=%lld K=%lld V=%lld nseq=%lld)",
                (long long)a.B, (long long)a.L, (long long)a.Hk, (long long)a.H, (long long)a.K,
                (long long)a.V, (long long)a.nseq);
  if (a.K < 1 || a.K > LINATTN_MAX_WIDTH || a.V < 1 || a.V > LINATTN_MAX_WIDTH)
    return fail(SW_ERR_UNSUPPORTED, "head widths K=%lld, V=%lld outside [1, %lld]", (long long)a.K,
                (long long)a.V, (long long)LINATTN_MAX_WIDTH);
  if (a.H > 0 && (a.Hk == 0 || a.H % a.Hk != 0))
    return fail(SW_ERR_INVALID_ARG, "H=%lld is no multiple of Hk=%lld", (long long)a.H,
                (long long)a.Hk);
  if (a.cu ? a.B != 1 || a.nseq < 1 : a.nseq != a.B)
    return fail(SW_ERR_INVALID_ARG, a.cu ? "packed sequences need B=1 and nseq>=1 (B=%lld nseq=%lld)"
                                         : "nseq must be B without cu_seqlens (B=%lld nseq=%lld)",
                (long long)a.B, (long long)a.nseq);
  if (a.L >= ((int64_t)1 << 31) - 1024)
    return fail(SW_ERR_UNSUPPORTED, "L=%lld steps", (long long)a.L);
  int64_t T, n;
  const int64_t width = a.K > a.V ? a.K : a.V;
  if (!mul_ok(a.B, a.L, &T) || !mul_ok(T, a.H, &n) || !mul_ok(n, width, &n) ||
      !mul_ok(n, 16, &n) || !mul_ok(a.nseq + T / 64 + 1, a.H, &n) ||
      !mul_ok(n, a.K * a.V, &n) || !mul_ok(n, 32, &n))
    return fail(SW_ERR_UNSUPPORTED, "sizes overflow");
  for (const HeadRows* x : {&a.q, &a.k, &a.v, &a.dout})
    if (x->sb < 0 || x->sl < 0 || x->sh < 0)
      return fail(SW_ERR_INVALID_ARG, "negative stride");
  if (a.g_sb < 0 || a.g_sl < 0 || a.g_sh < 0) return fail(SW_ERR_INVALID_ARG, "negative stride");
  return SW_OK;
}

// Checks shared by the forward and the backward: the inputs' spans.
int check_inputs(const LinAttnArgs& a, int dev, bool bwd, Span* ins, int* nin) {
  int st;
  const size_t es = a.bf16 ? 2 : 4;
  const bool any = a.B * a.L * a.H > 0;
  int64_t nq, nk, nv, nd = 0, ng, tmp;
  HeadRows gr;
  gr.sb = a.g_head ? 0 : a.g_sb;
  gr.sl = a.g_head ? 0 : a.g_sl;
  gr.sh = a.g_sh;
  if (!extent(a.q, a.B, a.L, a.Hk, a.K, &nq) || !extent(a.k, a.B, a.L, a.Hk, a.K, &nk) ||
      !extent(a.v, a.B, a.L, a.H, a.V, &nv) || !extent(gr, a.B, a.L, a.H, 1, &ng) ||
      (bwd && !extent(a.dout, a.B, a.L, a.H, a.V, &nd)) || !mul_ok(nq, 4, &tmp))
    return fail(SW_ERR_UNSUPPORTED, "strides overflow");
  if ((st = check_ptr(a.q.p, es, "q", any, dev)) != SW_OK) return st;
  if ((st = check_ptr(a.k.p, es, "k", any, dev)) != SW_OK) return st;
  if ((st = check_ptr(a.v.p, es, "v", any, dev)) != SW_OK) return st;
  if ((st = check_ptr(a.g, 4, "g", any, dev)) != SW_OK) return st;
  if ((st = check_ptr(a.h0, 4, "h0", false, dev)) != SW_OK) return st;
  if ((st = check_ptr(a.cu, 4, "cu_seqlens", false, dev)) != SW_OK) return st;
  if ((st = check_ptr(a.ws, 16, "workspace", false, dev)) != SW_OK) return st;
  const size_t nh = (size_t)(a.nseq * a.H * a.K * a.V) * 4;
  int i = 0;
  ins[i++] = {a.q.p, (size_t)nq * es, "q"};
  ins[i++] = {a.k.p, (size_t)nk * es, "k"};
  ins[i++] = {a.v.p, (size_t)nv * es, "v"};
  ins[i++] = {a.g, (size_t)ng * 4, "g"};
  ins[i++] = {a.h0, nh, "h0"};
  ins[i++] = {a.cu, (size_t)(a.nseq + 1) * 4, "cu_seqlens"};
  if (bwd) {
    if ((st = check_ptr(a.dout.p, es, "dout", any, dev)) != SW_OK) return st;
    if ((st = check_ptr(a.dh_last, 4, "dh_last", false, dev)) != SW_OK) return st;
    ins[i++] = {a.dout.p, (size_t)nd * es, "dout"};
    ins[i++] = {a.dh_last, nh, "dh_last"};
  }
  *nin = i;
  return SW_OK;
}

int fwd_common(const LinAttnArgs& a) {
  int st, dev, nin;
  if ((st = check_sizes(a)) != SW_OK) return st;
  const bool any = a.B * a.L * a.H > 0, states = a.nseq * a.H > 0 && a.h_last;
  if (!any && !states) return SW_OK;
  if ((st = current_device(&dev)) != SW_OK) return st;
  Span ins[8];
  if ((st = check_inputs(a, dev, false, ins, &nin)) != SW_OK) return st;
  const size_t es = a.bf16 ? 2 : 4, nh = (size_t)(a.nseq * a.H * a.K * a.V) * 4;
  if ((st = check_ptr(a.o, es, "o", any, dev)) != SW_OK) return st;
  if ((st = check_ptr(a.h_last, 4, "h_last", false, dev)) != SW_OK) return st;
  Span outs[] = {{a.o, (size_t)(a.B * a.L * a.H * a.V) * es, "o"},
                 {a.h_last, nh, "h_last"},
                 {a.ws, a.ws_bytes, "workspace"}};
  if ((st = check_spans(outs, 3, ins, nin)) != SW_OK) return st;
  return linear_attn_fwd(a);
}

int bwd_common(const LinAttnArgs& a) {
  int st, dev, nin;
  if ((st = check_sizes(a)) != SW_OK) return st;
  const int64_t T = a.B * a.L;
  // without heads only dq and dk hold anything: sums over none
  const bool any = T > 0 && (a.H > 0 || a.Hk > 0), states = a.nseq * a.H > 0 && a.dh0;
  if (!any && !states && !(a.g_head && a.H > 0)) return SW_OK;
  if ((st = current_device(&dev)) != SW_OK) return st;
  Span ins[8];
  if ((st = check_inputs(a, dev, true, ins, &nin)) != SW_OK) return st;
  const size_t es = a.bf16 ? 2 : 4, nh = (size_t)(a.nseq * a.H * a.K * a.V) * 4;
  if ((st = check_ptr(a.dq, es, "dq", any, dev)) != SW_OK) return st;
  if ((st = check_ptr(a.dk, es, "dk", any, dev)) != SW_OK) return st;
  if ((st = check_ptr(a.dv, es, "dv", any && a.H > 0, dev)) != SW_OK) return st;
  if ((st = check_ptr(a.dg, 4, "dg", (any || a.g_head) && a.H > 0, dev)) != SW_OK) return st;
  if ((st = check_ptr(a.dh0, 4, "dh0", false, dev)) != SW_OK) return st;
  Span outs[] = {{a.dq, (size_t)(T * a.Hk * a.K) * es, "dq"},
                 {a.dk, (size_t)(T * a.Hk * a.K) * es, "dk"},
                 {a.dv, (size_t)(T * a.H * a.V) * es, "dv"},
                 {a.dg, (size_t)(a.g_head ? a.H : T * a.H) * 4, "dg"},
                 {a.dh0, nh, "dh0"},
                 {a.ws, a.ws_bytes, "workspace"}};
  if ((st = check_spans(outs, 6, ins, nin)) != SW_OK) return st;
  return linear_attn_bwd(a);
}

int step_common(const LinStepArgs& a) {
  if (a.B < 0 || a.Hk < 0 || a.H < 0 || a.K < 0 || a.V < 0 || a.pool < 0)
    return fail(SW_ERR_INVALID_ARG, "negative size (B=%lld Hk=%lld H=%lld K=%lld V=%lld pool=%lld)",
                (long long)a.B, (long long)a.Hk, (long long)a.H, (long long)a.K, (long long)a.V,
                (long long)a.pool);
  if (a.K < 1 || a.K > LINATTN_MAX_WIDTH || a.V < 1 || a.V > LINATTN_MAX_WIDTH)
    return fail(SW_ERR_UNSUPPORTED, "head widths K=%lld, V=%lld outside [1, %lld]", (long long)a.K,
                (long long)a.V, (long long)LINATTN_MAX_WIDTH);
  if (a.H > 0 && (a.Hk == 0 || a.H % a.Hk != 0))
    return fail(SW_ERR_INVALID_ARG, "H=%lld is no multiple of Hk=%lld", (long long)a.H,
                (long long)a.Hk);
  if (!a.slots && a.pool < a.B)
    return fail(SW_ERR_INVALID_ARG, "%lld states for %lld sequences", (long long)a.pool,
                (long long)a.B);
  for (int64_t s : {a.q_sb, a.q_sh, a.k_sb, a.k_sh, a.v_sb, a.v_sh, a.g_sb, a.g_sh})
    if (s < 0) return fail(SW_ERR_INVALID_ARG, "negative stride");
  int64_t n, ns;
  if (!mul_ok(a.B, a.H, &n) || !mul_ok(n, a.V, &n) || !mul_ok(n, 4, &n) ||
      !mul_ok(a.pool, a.H, &ns) || !mul_ok(ns, a.K * a.V, &ns) || !mul_ok(ns, 4, &ns))
    return fail(SW_ERR_UNSUPPORTED, "sizes overflow");
  if (a.B == 0 || a.H == 0) return SW_OK;
  const HeadRows q{a.q, a.q_sb, 0, a.q_sh}, k{a.k, a.k_sb, 0, a.k_sh}, v{a.v, a.v_sb, 0, a.v_sh},
      g{a.g, a.g_sb, 0, a.g_sh};
  int64_t nq, nk, nv, ng;
  if (!extent(q, a.B, 1, a.Hk, a.K, &nq) || !extent(k, a.B, 1, a.Hk, a.K, &nk) ||
      !extent(v, a.B, 1, a.H, a.V, &nv) || !extent(g, a.B, 1, a.H, 1, &ng))
    return fail(SW_ERR_UNSUPPORTED, "strides overflow");
  int dev, st;
  if ((st = current_device(&dev)) != SW_OK) return st;
  const size_t es = a.bf16 ? 2 : 4;
  if ((st = check_ptr(a.q, es, "q", true, dev)) != SW_OK) return st;
  if ((st = check_ptr(a.k, es, "k", true, dev)) != SW_OK) return st;
  if ((st = check_ptr(a.v, es, "v", true, dev)) != SW_OK) return st;
  if ((st = check_ptr(a.g, 4, "g", true, dev)) != SW_OK) return st;
  if ((st = check_ptr(a.state, 4, "state", a.pool > 0, dev)) != SW_OK) return st;
  if ((st = check_ptr(a.slots, 4, "slots", false, dev)) != SW_OK) return st;
  if ((st = check_ptr(a.o, es, "o", true, dev)) != SW_OK) return st;
  Span outs[] = {{a.o, (size_t)(a.B * a.H * a.V) * es, "o"}, {a.state, (size_t)ns, "state"}};
  Span ins[] = {{a.q, (size_t)nq * es, "q"},
                {a.k, (size_t)nk * es, "k"},
                {a.v, (size_t)nv * es, "v"},
                {a.g, (size_t)ng * 4, "g"},
                {a.slots, (size_t)a.B * 4, "slots"}};
  if ((st = check_spans(outs, 2, ins, 5)) != SW_OK) return st;
  return linear_attn_step(a);
}

int check_kind(int dtype, int flags) {
  if (dtype != SW_DTYPE_F32 && dtype != SW_DTYPE_BF16)
    return fail(SW_ERR_INVALID_ARG, "unknown dtype %d", dtype);
  if (flags & ~SW_LINEAR_G_HEAD)
    return fail(SW_ERR_INVALID_ARG, "unknown flags 0x%x", (unsigned)flags);
  return SW_OK;
}

LinAttnArgs sizes(int64_t B, int64_t L, int64_t Hk, int64_t H, int64_t K, int64_t V, int64_t nseq,
                  int dtype, int flags) {
  LinAttnArgs a;
  a.B = B;
  a.L = L;
  a.Hk = Hk;
  a.H = H;
  a.K = K;
  a.V = V;
  a.nseq = nseq;
  a.bf16 = dtype == SW_DTYPE_BF16;
  a.g_head = (flags & SW_LINEAR_G_HEAD) != 0;
  return a;
}

void operands(LinAttnArgs& a, const void* q, const void* k, const void* v, const float* g,
              const int64_t* st) {
  a.q = {q, st[0], st[1], st[2]};
  a.k = {k, st[3], st[4], st[5]};
  a.v = {v, st[6], st[7], st[8]};
  a.g = g;
  a.g_sb = st[9];
  a.g_sl = st[10];
  a.g_sh = st[11];
}

// The workspace of a call of these sizes, packed (nseq sequences) or not.
int64_t workspace(int64_t B, int64_t L, int64_t Hk, int64_t H, int64_t K, int64_t V, int64_t nseq,
                  int dtype, int flags, int packed, bool bwd) {
  static const int32_t stand_in[2] = {0, 0};  // tells packed from not, and is never read
  LinAttnArgs a = sizes(B, L, Hk, H, K, V, nseq, dtype, flags);
  if (packed) a.cu = stand_in;
  if (check_kind(dtype, flags) != SW_OK || check_sizes(a) != SW_OK || nseq * H == 0) return 0;
  return bwd ? linear_attn_bwd_workspace(a) : linear_attn_fwd_workspace(a);
}

}  // namespace
}  // namespace sw

SW_API int sw_linear_attn_fwd(const void* q, const void* k, const void* v, const float* g,
                              const float* h0, const int32_t* cu_seqlens, void* o, float* h_last,
                              int64_t B, int64_t L, int64_t Hk, int64_t H, int64_t K, int64_t V,
                              int64_t nseq, const int64_t* strides, int dtype, int flags,
                              float scale, void* workspace, int64_t workspace_bytes) {
  int st;
  if ((st = sw::check_kind(dtype, flags)) != SW_OK) return st;
  if (!strides) return sw::fail(SW_ERR_INVALID_ARG, "strides is NULL");
  if (workspace_bytes < 0) return sw::fail(SW_ERR_INVALID_ARG, "negative workspace size");
  sw::LinAttnArgs a = sw::sizes(B, L, Hk, H, K, V, nseq, dtype, flags);
  sw::operands(a, q, k, v, g, strides);
  a.h0 = h0;
  a.cu = cu_seqlens;
  a.o = o;
  a.h_last = h_last;
  a.scale = scale;
  a.ws = workspace;
  a.ws_bytes = workspace ? (size_t)workspace_bytes : 0;
  return sw::fwd_common(a);
}

SW_API int64_t sw_linear_attn_fwd_workspace(int64_t B, int64_t L, int64_t Hk, int64_t H, int64_t K,
                                            int64_t V, int64_t nseq, int dtype, int flags,
                                            int packed) {
  return sw::workspace(B, L, Hk, H, K, V, nseq, dtype, flags, packed, false);
}

SW_API int sw_linear_attn_bwd(const void* q, const void* k, const void* v, const float* g,
                              const float* h0, const int32_t* cu_seqlens, const void* dout,
                              const float* dh_last, void* dq, void* dk, void* dv, float* dg,
                              float* dh0, int64_t B, int64_t L, int64_t Hk, int64_t H, int64_t K,
                              int64_t V, int64_t nseq, const int64_t* strides, int dtype, int flags,
                              float scale, void* workspace, int64_t workspace_bytes) {
  int st;
  if ((st = sw::check_kind(dtype, flags)) != SW_OK) return st;
  if (!strides) return sw::fail(SW_ERR_INVALID_ARG, "strides is NULL");
  if (workspace_bytes < 0) return sw::fail(SW_ERR_INVALID_ARG, "negative workspace size");
  sw::LinAttnArgs a = sw::sizes(B, L, Hk, H, K, V, nseq, dtype, flags);
  sw::operands(a, q, k, v, g, strides);
  a.dout = {dout, strides[12], strides[13], strides[14]};
  a.h0 = h0;
  a.cu = cu_seqlens;
  a.dh_last = dh_last;
  a.dq = dq;
  a.dk = dk;
  a.dv = dv;
  a.dg = dg;
  a.dh0 = dh0;
  a.scale = scale;
  a.ws = workspace;
  a.ws_bytes = workspace ? (size_t)workspace_bytes : 0;
  return sw::bwd_common(a);
}

SW_API int64_t sw_linear_attn_bwd_workspace(int64_t B, int64_t L, int64_t Hk, int64_t H, int64_t K,
                                            int64_t V, int64_t nseq, int dtype, int flags,
                                            int packed) {
  return sw::workspace(B, L, Hk, H, K, V, nseq, dtype, flags, packed, true);
}

SW_API int sw_linear_attn_step(const void* q, const void* k, const void* v, const float* g,
                               float* state, const int32_t* slots, void* o, int64_t B, int64_t Hk,
                               int64_t H, int64_t K, int64_t V, int64_t pool,
                               const int64_t* strides, int dtype, int flags, float scale) {
  int st;
  if ((st = sw::check_kind(dtype, flags)) != SW_OK) return st;
  if (!strides) return sw::fail(SW_ERR_INVALID_ARG, "strides is NULL");
  sw::LinStepArgs a;
  a.q = q;
  a.k = k;
  a.v = v;
  a.g = g;
  a.q_sb = strides[0];
  a.q_sh = strides[1];
  a.k_sb = strides[2];
  a.k_sh = strides[3];
  a.v_sb = strides[4];
  a.v_sh = strides[5];
  a.g_sb = flags & SW_LINEAR_G_HEAD ? 0 : strides[6];
  a.g_sh = strides[7];
  a.state = state;
  a.slots = slots;
  a.o = o;
  a.B = B;
  a.Hk = Hk;
  a.H = H;
  a.K = K;
  a.V = V;
  a.pool = pool;
  a.bf16 = dtype == SW_DTYPE_BF16;
  a.scale = scale;
  return sw::step_common(a);
}
