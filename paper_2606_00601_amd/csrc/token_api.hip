// token_api.hip -- the C ABI of the head norm and the embedding: argument validation
// and dispatch.  Declarations and the full contract are in include/scanweaver.h.
#include "sw_check.h"
#include "token_ops.h"

namespace sw {
namespace {

bool known(int dtype) { return dtype == SW_DTYPE_F32 || dtype == SW_DTYPE_BF16; }

// Bytes a (B, L, H, W) array of these strides reaches over; false on overflow.
bool reach(const Heads& x, int64_t B, int64_t L, int64_t H, int64_t W, int64_t es, size_t* bytes) {
  *bytes = 0;
  if (B == 0 || L == 0 || H == 0 || W == 0) return true;
  int64_t n = W, t;
  const int64_t st[3] = {x.sb, x.sl, x.sh}, c[3] = {B, L, H};
  for (int i = 0; i < 3; ++i)
    if (!mul_ok(c[i] - 1, st[i], &t) || __builtin_add_overflow(n, t, &n)) return false;
  if (!mul_ok(n, es, &n)) return false;
  *bytes = (size_t)n;
  return true;
}

int check_head(const HeadNormArgs& a) {
  if (a.B < 0 || a.L < 0 || a.H < 0 || a.Hk < 0 || a.K < 0 || a.R < 0)
    return fail(SW_ERR_INVALID_ARG, "negative size (B=%lld L=%lld H=%lld Hk=%lld K=%lld R=%lld)",
                (long long)a.B, (long long)a.L, (long long)a.H, (long long)a.Hk, (long long)a.K,
                (long long)a.R);
  if (a.K < 1 || a.K > HEAD_MAX_WIDTH)
    return fail(SW_ERR_UNSUPPORTED, "head width K=%lld outside [1, %lld]", (long long)a.K,
                (long long)HEAD_MAX_WIDTH);
  if (a.R > a.K || a.R % 2 != 0)
    return fail(SW_ERR_INVALID_ARG, "R=%lld is not an even number of the K=%lld columns",
                (long long)a.R, (long long)a.K);
  int64_t n, T;
  if (!mul_ok(a.B, a.L, &T) || __builtin_add_overflow(a.H, a.Hk, &n) || !mul_ok(T, n, &n) ||
      !mul_ok(n, a.K * 8, &n))
    return fail(SW_ERR_UNSUPPORTED, "sizes overflow");
  // a workgroup takes 8 tokens or more of a call that fills the card
  if (T > SW_MAX_WGS * 8 || a.H + a.Hk >= ((int64_t)1 << 31))
    return fail(SW_ERR_UNSUPPORTED, "%lld tokens of %lld heads exceed the launch limit", (long long)T,
                (long long)(a.H + a.Hk));
  for (const Heads* x : {&a.q, &a.k, &a.dyq, &a.dyk})
    if (x->sb < 0 || x->sl < 0 || x->sh < 0) return fail(SW_ERR_INVALID_ARG, "negative stride");
  if (a.pos_sb < 0 || a.pos_sl < 0) return fail(SW_ERR_INVALID_ARG, "negative stride");
  return SW_OK;
}

int head(const HeadNormArgs& a, bool bwd) {
  int st;
  if ((st = check_head(a)) != SW_OK) return st;
  if (bwd && !a.dwq != !a.dwk)
    return fail(SW_ERR_INVALID_ARG, "dwq and dwk are both given or neither");
  const int64_t T = a.B * a.L;
  const bool q = T * a.H > 0, k = T * a.Hk > 0;
  if (!q && !k && !a.dwq) return SW_OK;
  const int64_t es = a.bf16 ? 2 : 4, ps = a.pos64 ? 8 : 4;
  const size_t k4 = (size_t)a.K * 4, nyq = (size_t)(T * a.H * a.K * es),
               nyk = (size_t)(T * a.Hk * a.K * es);
  size_t nq, nk, ndq = 0, ndk = 0, np;
  if (!reach(a.q, a.B, a.L, a.H, a.K, es, &nq) || !reach(a.k, a.B, a.L, a.Hk, a.K, es, &nk) ||
      !reach({nullptr, a.pos_sb, a.pos_sl, 0}, a.B, a.L, 1, 1, ps, &np) ||
      (bwd && (!reach(a.dyq, a.B, a.L, a.H, a.K, es, &ndq) ||
               !reach(a.dyk, a.B, a.L, a.Hk, a.K, es, &ndk))))
    return fail(SW_ERR_UNSUPPORTED, "strides overflow");
  const size_t ea = (size_t)es;
  const In ins[] = {{a.q.p, ea, nq, "q", q},
                    {a.k.p, ea, nk, "k", k},
                    {a.wq, 4, k4, "wq", false},
                    {a.wk, 4, k4, "wk", false},
                    {a.pos, (size_t)ps, np, "positions", false},
                    {a.inv_freq, 4, (size_t)a.R * 2, "inv_freq", a.R > 0 && (q || k)},
                    {a.dyq.p, ea, ndq, "dyq", bwd && q},
                    {a.dyk.p, ea, ndk, "dyk", bwd && k}};
  const In outs[] = {{a.yq, ea, nyq, bwd ? "dq" : "yq", q},
                     {a.yk, ea, nyk, bwd ? "dk" : "yk", k},
                     {a.dwq, 4, k4, "dwq", false},
                     {a.dwk, 4, k4, "dwk", false},
                     {a.ws, 16, a.ws_bytes, "workspace", false}};
  if ((st = check_arrays(ins, 8, outs, 5)) != SW_OK) return st;
  return bwd ? head_norm_bwd(a) : head_norm_fwd(a);
}

int check_embed(const EmbedArgs& a) {
  if (a.T < 0 || a.V < 0 || a.D < 0)
    return fail(SW_ERR_INVALID_ARG, "negative size (T=%lld V=%lld D=%lld)", (long long)a.T,
                (long long)a.V, (long long)a.D);
  if (a.dy_st < 0) return fail(SW_ERR_INVALID_ARG, "negative stride");
  int64_t n;
  if (!mul_ok(a.T, a.D, &n) || !mul_ok(n, 8, &n) || !mul_ok(a.V, a.D, &n) || !mul_ok(n, 8, &n) ||
      !mul_ok(a.T, a.dy_st, &n) || !mul_ok(n, 4, &n))
    return fail(SW_ERR_UNSUPPORTED, "sizes overflow");
  if (a.T >= (int64_t)1 << 31 || a.V >= (int64_t)1 << 31 || a.D >= (int64_t)1 << 24)
    return fail(SW_ERR_UNSUPPORTED, "T=%lld, V=%lld (below 2^31) or D=%lld (below 2^24)",
                (long long)a.T, (long long)a.V, (long long)a.D);
  return SW_OK;
}

int embed_fwd(const EmbedArgs& a) {
  int st;
  if ((st = check_embed(a)) != SW_OK) return st;
  if (a.T == 0 || a.D == 0) return SW_OK;
  const size_t ts = a.table_bf16 ? 2 : 4, ys = a.y_bf16 ? 2 : 4, ks = a.wide ? 8 : 4;
  const In ins[] = {{a.tokens, ks, (size_t)a.T * ks, "tokens", true},
                    {a.table, ts, (size_t)(a.V * a.D) * ts, "table", a.V > 0}};
  const In outs[] = {{a.y, ys, (size_t)(a.T * a.D) * ys, "y", true}};
  if ((st = check_arrays(ins, 2, outs, 1)) != SW_OK) return st;
  return embedding_fwd(a);
}

int embed_bwd(const EmbedArgs& a) {
  int st;
  if ((st = check_embed(a)) != SW_OK) return st;
  if (a.V == 0 || a.D == 0) return SW_OK;
  const size_t ts = a.table_bf16 ? 2 : 4, ys = a.y_bf16 ? 2 : 4, ks = a.wide ? 8 : 4;
  const size_t ny = a.T ? (size_t)((a.T - 1) * a.dy_st + a.D) * ys : 0;
  const In ins[] = {{a.tokens, ks, (size_t)a.T * ks, "tokens", a.T > 0},
                    {a.dy, ys, ny, "dy", a.T > 0}};
  const In outs[] = {{a.dtable, ts, (size_t)(a.V * a.D) * ts, "dtable", true},
                     {a.ws, 16, a.ws_bytes, "workspace", false}};
  if ((st = check_arrays(ins, 2, outs, 2)) != SW_OK) return st;
  return embedding_bwd(a);
}

int head_call(HeadNormArgs* a, const int64_t* strides, int dtype, int flags) {
  if (!known(dtype)) return fail(SW_ERR_INVALID_ARG, "unknown dtype %d", dtype);
  if (flags & ~(SW_HEAD_ADJACENT | SW_HEAD_POS_I64))
    return fail(SW_ERR_INVALID_ARG, "unknown flags 0x%x", (unsigned)flags);
  if (!strides) return fail(SW_ERR_INVALID_ARG, "strides is NULL");
  a->bf16 = dtype == SW_DTYPE_BF16;
  a->adjacent = (flags & SW_HEAD_ADJACENT) != 0;
  a->pos64 = (flags & SW_HEAD_POS_I64) != 0;
  return SW_OK;
}

int embed_call(EmbedArgs* a, int table_dtype, int y_dtype, int flags) {
  if (!known(table_dtype) || !known(y_dtype))
    return fail(SW_ERR_INVALID_ARG, "unknown dtype %d or %d", table_dtype, y_dtype);
  if (flags & ~SW_EMBED_TOKENS_I64)
    return fail(SW_ERR_INVALID_ARG, "unknown flags 0x%x", (unsigned)flags);
  a->table_bf16 = table_dtype == SW_DTYPE_BF16;
  a->y_bf16 = y_dtype == SW_DTYPE_BF16;
  a->wide = (flags & SW_EMBED_TOKENS_I64) != 0;
  return SW_OK;
}

}  // namespace
}  // namespace sw

SW_API int sw_head_norm_fwd(const void* q, const void* k, const float* wq, const float* wk,
                            const void* positions, const float* inv_freq, void* yq, void* yk,
                            int64_t B, int64_t L, int64_t H, int64_t Hk, int64_t K, int64_t R,
                            const int64_t* strides, int dtype, int flags, float eps) {
  sw::HeadNormArgs a;
  int st;
  if ((st = sw::head_call(&a, strides, dtype, flags)) != SW_OK) return st;
  a.q = {q, strides[0], strides[1], strides[2]};
  a.k = {k, strides[3], strides[4], strides[5]};
  a.pos = positions;
  a.pos_sb = strides[6];
  a.pos_sl = strides[7];
  a.wq = wq;
  a.wk = wk;
  a.inv_freq = inv_freq;
  a.yq = yq;
  a.yk = yk;
  a.B = B;
  a.L = L;
  a.H = H;
  a.Hk = Hk;
  a.K = K;
  a.R = R;
  a.eps = eps;
  return sw::head(a, false);
}

SW_API int sw_head_norm_bwd(const void* dyq, const void* dyk, const void* q, const void* k,
                            const float* wq, const float* wk, const void* positions,
                            const float* inv_freq, void* dq, void* dk, float* dwq, float* dwk,
                            int64_t B, int64_t L, int64_t H, int64_t Hk, int64_t K, int64_t R,
                            const int64_t* strides, int dtype, int flags, float eps,
                            void* workspace, int64_t workspace_bytes) {
  sw::HeadNormArgs a;
  int st;
  if ((st = sw::head_call(&a, strides, dtype, flags)) != SW_OK) return st;
  if (workspace_bytes < 0) return sw::fail(SW_ERR_INVALID_ARG, "negative workspace size");
  a.dyq = {dyq, strides[0], strides[1], strides[2]};
  a.dyk = {dyk, strides[3], strides[4], strides[5]};
  a.q = {q, strides[6], strides[7], strides[8]};
  a.k = {k, strides[9], strides[10], strides[11]};
  a.pos = positions;
  a.pos_sb = strides[12];
  a.pos_sl = strides[13];
  a.wq = wq;
  a.wk = wk;
  a.inv_freq = inv_freq;
  a.yq = dq;
  a.yk = dk;
  a.dwq = dwq;
  a.dwk = dwk;
  a.B = B;
  a.L = L;
  a.H = H;
  a.Hk = Hk;
  a.K = K;
  a.R = R;
  a.eps = eps;
  a.ws = workspace;
  a.ws_bytes = workspace ? (size_t)workspace_bytes : 0;
  return sw::head(a, true);
}

SW_API int64_t sw_head_norm_bwd_workspace(int64_t B, int64_t L, int64_t H, int64_t Hk, int64_t K) {
  sw::HeadNormArgs a;
  a.B = B;
  a.L = L;
  a.H = H;
  a.Hk = Hk;
  a.K = K;
  if (sw::check_head(a) != SW_OK) return 0;
  return sw::head_norm_bwd_workspace(B * L, H, Hk, K);
}

SW_API int sw_embedding_fwd(const void* tokens, const void* table, void* y, int64_t T, int64_t V,
                            int64_t D, int table_dtype, int y_dtype, int flags, float scale) {
  sw::EmbedArgs a;
  int st;
  if ((st = sw::embed_call(&a, table_dtype, y_dtype, flags)) != SW_OK) return st;
  a.tokens = tokens;
  a.table = table;
  a.y = y;
  a.T = T;
  a.V = V;
  a.D = D;
  a.scale = scale;
  return sw::embed_fwd(a);
}

SW_API int sw_embedding_bwd(const void* tokens, const void* dy, void* dtable, int64_t T, int64_t V,
                            int64_t D, int64_t dy_stride, int dy_dtype, int table_dtype, int flags,
                            float scale, void* workspace, int64_t workspace_bytes) {
  sw::EmbedArgs a;
  int st;
  if ((st = sw::embed_call(&a, table_dtype, dy_dtype, flags)) != SW_OK) return st;
  if (workspace_bytes < 0) return sw::fail(SW_ERR_INVALID_ARG, "negative workspace size");
  a.tokens = tokens;
  a.dy = dy;
  a.dtable = dtable;
  a.T = T;
  a.V = V;
  a.D = D;
  a.dy_st = dy_stride;
  a.scale = scale;
  a.ws = workspace;
  a.ws_bytes = workspace ? (size_t)workspace_bytes : 0;
  return sw::embed_bwd(a);
}

SW_API int64_t sw_embedding_bwd_workspace(int64_t T, int64_t V, int64_t D) {
  sw::EmbedArgs a;
  a.T = T;
  a.V = V;
  a.D = D;
  if (sw::check_embed(a) != SW_OK || T == 0 || V == 0 || D == 0) return 0;
  return sw::embedding_bwd_workspace(T, V, D);
}
