// head_norm.hip -- the norm of each head's query and key with the rotation by the
// token's position, u = w x / rms(x), y = R(position) u, and its gradients.
//
// LPH lanes hold a head, 16 columns each as two vectors of 8 which hold both members
// of every pair they turn: (8 j .. , R/2 + 8 j ..) for halves, (16 j ..) for
// neighbours; columns that are not turned go to the lanes behind.  So the turn needs
// no exchange and the norm a sum over LPH lanes.  A workgroup forms its tokens' angles once,
// in LDS; a lane keeps its pairs' of one token and steps through its heads.  Bound by
// memory: a value is read once and written once.
#include "norm_rows.h"
#include "token_ops.h"

// Which products are fused is written out: the same in every instance, whatever its loads.
#pragma clang fp contract(off)

namespace sw {
namespace head {
namespace {

using norm::load8;
using norm::store8;

// Where a lane's two vectors lie in a head and how many of their 8 columns are there.
struct Lane {
  int o1, o2, n1, n2;
  int pair;  // first of its 8 pairs, or -1
};
__device__ __forceinline__ int cut8(int n) { return n < 0 ? 0 : n > 8 ? 8 : n; }
__device__ __forceinline__ Lane lane_of(const HeadNormArgs& a, int j) {
  const int K = (int)a.K, R = (int)a.R, half = R / 2, turned = (half + 7) / 8;
  Lane l;
  if (j < turned) {
    l.pair = 8 * j;
    l.o1 = a.adjacent ? 16 * j : 8 * j;
    l.o2 = a.adjacent ? 16 * j + 8 : half + 8 * j;
    l.n1 = a.adjacent ? cut8(R - l.o1) : cut8(half - l.o1);
    l.n2 = a.adjacent ? cut8(R - l.o2) : l.n1;
  } else {
    l.pair = -1;
    l.o1 = R + 16 * (j - turned);
    l.o2 = l.o1 + 8;
    l.n1 = cut8(K - l.o1);
    l.n2 = cut8(K - l.o2);
  }
  return l;
}

// cos and sin of position * freq.  The angle is counted in quarter turns in 64 bits; its
// nearest whole number picks the quadrant and what is left, within 1/2, is rounded to
// 32 bits, where Taylor's series to the 9th and 10th power are off by less than 2^-28.
__device__ __forceinline__ void angle(double pos, float freq, float& c, float& s) {
  const double turns = pos * ((double)freq * 0.15915494309189533577);
  const double part = 4.0 * (turns - rint(turns));
  const double quad = rint(part);
  const float x = (float)(part - quad) * 1.57079632679489661923f;
  const float x2 = x * x;
  float sn = __builtin_fmaf(x2, 1.0f / 362880.0f, -1.0f / 5040.0f);
  sn = __builtin_fmaf(x2, sn, 1.0f / 120.0f);
  sn = __builtin_fmaf(x2, sn, -1.0f / 6.0f);
  sn = __builtin_fmaf(x * x2, sn, x);
  float cs = __builtin_fmaf(x2, -1.0f / 3628800.0f, 1.0f / 40320.0f);
  cs = __builtin_fmaf(x2, cs, -1.0f / 720.0f);
  cs = __builtin_fmaf(x2, cs, 1.0f / 24.0f);
  cs = __builtin_fmaf(x2, cs, -0.5f);
  cs = __builtin_fmaf(x2, cs, 1.0f);
  const int n = (int)quad & 3;  // -2 .. 2
  c = n & 1 ? sn : cs;
  s = n & 1 ? cs : sn;
  if (n == 1 || n == 2) c = -c;
  if (n >= 2) s = -s;
}

struct Angles {
  float c[8], s[8];
};
// The angles of `tokens` tokens from m0 on, 256 threads one each at a time: sh[token * R / 2 +
// pair].
__device__ __forceinline__ void form_angles(const HeadNormArgs& a, int64_t m0, int tokens, float2* sh) {
  const int half = (int)a.R / 2;
  const int64_t T = a.B * a.L;
  for (int j = threadIdx.x; j < tokens * half; j += 256) {
    const int64_t m = m0 + j / half;
    if (m >= T) break;
    const int64_t at = m / a.L * a.pos_sb + m % a.L * a.pos_sl;
    const double pos = !a.pos   ? (double)(m % a.L)
                       : a.pos64 ? (double)((const int64_t*)a.pos)[at]
                                 : (double)((const int32_t*)a.pos)[at];
    angle(pos, a.inv_freq[j % half], sh[j].x, sh[j].y);
  }
}
__device__ __forceinline__ void load_angles(const HeadNormArgs& a, const Lane& l, const float2* sh,
                                            Angles& g) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const bool there = l.pair >= 0 && l.pair + j < (int)a.R / 2;
    const float2 v = there ? sh[l.pair + j] : make_float2(1.0f, 0.0f);
    g.c[j] = v.x;
    g.s[j] = v.y;
  }
}

// The lane's pairs turned by their angles, or back by them (sign -1).  A lane of columns that
// are not turned has none: a turn by nothing, p 1 - q 0, would hand on a q that is not finite.
template <bool ADJ>
__device__ __forceinline__ void turn(const Lane& l, float* x, const Angles& g, float sign) {
  if (l.pair < 0) return;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    float& p = x[ADJ ? 2 * j : j];
    float& q = x[ADJ ? 2 * j + 1 : 8 + j];
    const float s = sign * g.s[j], pp = __builtin_fmaf(p, g.c[j], -(q * s));
    q = __builtin_fmaf(q, g.c[j], p * s);
    p = pp;
  }
}

template <bool VEC, class E>
__device__ __forceinline__ void load_head(const E* p, const Lane& l, float* x) {
  load8(p + l.o1, x, l.n1, VEC);
  load8(p + l.o2, x + 8, l.n2, VEC);
}
template <bool VEC, class E>
__device__ __forceinline__ void store_head(E* p, const Lane& l, const float* x) {
  store8(p + l.o1, x, l.n1, VEC);
  store8(p + l.o2, x + 8, l.n2, VEC);
}
// The head's weights; zero where there is no column.
__device__ __forceinline__ void load_weights(const float* w, const Lane& l, float* x) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    x[j] = j < l.n1 ? (w ? w[l.o1 + j] : 1.0f) : 0.0f;
    x[8 + j] = j < l.n2 ? (w ? w[l.o2 + j] : 1.0f) : 0.0f;
  }
}

template <int LPH, int N>
__device__ __forceinline__ void head_sum(float* v) {
#pragma unroll
  for (int d = LPH / 2; d > 0; d >>= 1)
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += __shfl_xor(v[i], d);
}

template <class E, int LPH, bool ADJ, bool VEC>
__device__ __forceinline__ void fwd_heads(const HeadNormArgs& a, const Heads& x, const float* w, void* y,
                                          int64_t heads, int64_t first, int64_t step, int64_t b, int64_t t,
                                          const Lane& l, const Angles& g) {
  if (first >= heads) return;
  float wt[16];
  load_weights(w, l, wt);
  const E* src = (const E*)x.p + b * x.sb + t * x.sl;
  E* dst = (E*)y + (b * a.L + t) * heads * a.K;
  for (int64_t h = first; h < heads; h += step) {
    float v[16];
    load_head<VEC>(src + h * x.sh, l, v);
    float sum[1] = {0.0f};
#pragma unroll
    for (int j = 0; j < 16; ++j) sum[0] = __builtin_fmaf(v[j], v[j], sum[0]);
    head_sum<LPH, 1>(sum);
    const float inv = rsqrtf(sum[0] / (float)a.K + a.eps);
#pragma unroll
    for (int j = 0; j < 16; ++j) v[j] *= inv * wt[j];
    turn<ADJ>(l, v, g, 1.0f);
    store_head<VEC>(dst + h * a.K, l, v);
  }
}

// Lanes: (token, one of `per` places of it, lane of the head); queries first, then keys.
// 16384 tokens of 12 + 12 heads of 128, bf16: 41 us, 201 MB at 4.9 TB/s; fp32 87 us, 4.6; heads
// of 100, R = 50, an element a load, bf16 133 us, 157 MB at 1.2 TB/s.
template <class E, int LPH, bool ADJ, bool VEC>
__global__ __launch_bounds__(256) void fwd_kernel(HeadNormArgs a, int per) {
  extern __shared__ float2 angles[];
  const int j = threadIdx.x % LPH, place = threadIdx.x / LPH, tokens = 256 / LPH / per;
  const int64_t m0 = blockIdx.x * (int64_t)tokens, m = m0 + place / per;
  if (a.R) {
    form_angles(a, m0, tokens, angles);
    __syncthreads();
  }
  if (m >= a.B * a.L) return;  // whole heads' lanes leave together
  const int64_t b = m / a.L, t = m % a.L;
  const Lane l = lane_of(a, j);
  Angles g;
  load_angles(a, l, angles + (place / per) * (a.R / 2), g);
  const int64_t first = place % per;
  fwd_heads<E, LPH, ADJ, VEC>(a, a.q, a.wq, a.yq, a.H, first, per, b, t, l, g);
  const int64_t done = first >= a.H ? first : first + (a.H - first + per - 1) / per * per;
  fwd_heads<E, LPH, ADJ, VEC>(a, a.k, a.wk, a.yk, a.Hk, done - a.H, per, b, t, l, g);
}

// The backward takes queries and keys in workgroups of their own: one's weights and sums fit
// 128 registers (both at once took 201 and ran 132 us at the shape below).
struct Side {
  Heads x, dy;
  const float* w;
  void* dx;
  float* part;   // (blocks, K) partial sums, or NULL
  int64_t heads, blocks;
  int per;
};

// A workgroup's sums of a weight's gradient: a wave's lanes of the same columns by
// exchanges, then the four waves in order.
template <int LPH>
__device__ __forceinline__ void put_partial(const Lane& l, float* dw, float* lds, float* out) {
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
#pragma unroll
  for (int d = 32; d >= LPH; d >>= 1)
#pragma unroll
    for (int e = 0; e < 16; ++e) dw[e] += __shfl_xor(dw[e], d);
  if (lane < LPH)
#pragma unroll
    for (int e = 0; e < 16; ++e) lds[(wave * 16 + e) * LPH + lane] = dw[e];
  __syncthreads();
  if (threadIdx.x < LPH) {
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      float t = 0.0f;
#pragma unroll
      for (int w = 0; w < 4; ++w) t += lds[(w * 16 + e) * LPH + lane];
      if (e < 8 ? e < l.n1 : e - 8 < l.n2) out[e < 8 ? l.o1 + e : l.o2 + e - 8] = t;
    }
  }
}

// dx = inv (w g - n mean(w g n)), n = x inv, with g the gradient turned back; dw += g n.
// At the shape above 69 us, 302 MB at 4.4 TB/s; fp32 128 us, 4.7; heads of 100 181 us, 1.3.
template <class E, int LPH, bool ADJ, bool VEC>
__global__ __launch_bounds__(256, 4) void bwd_kernel(HeadNormArgs a, Side q, Side k) {
  extern __shared__ float2 angles[];
  __shared__ float lds[4 * 16 * LPH];
  const bool keys = blockIdx.x >= q.blocks;
  const Side s = keys ? k : q;
  const int64_t block = blockIdx.x - (keys ? q.blocks : 0);
  const int j = threadIdx.x % LPH, place = threadIdx.x / LPH, tokens = 256 / LPH / s.per;
  const int64_t T = a.B * a.L;
  const Lane l = lane_of(a, j);
  float wt[16], dw[16];
  load_weights(s.w, l, wt);
#pragma unroll
  for (int e = 0; e < 16; ++e) dw[e] = 0.0f;
  for (int64_t m0 = block * tokens; m0 < T; m0 += s.blocks * tokens) {
    if (a.R) {
      __syncthreads();
      form_angles(a, m0, tokens, angles);
      __syncthreads();
    }
    const int64_t m = m0 + place / s.per;
    if (m >= T) continue;
    const int64_t b = m / a.L, t = m % a.L;
    Angles g;
    load_angles(a, l, angles + (place / s.per) * (a.R / 2), g);
    const E* src = (const E*)s.x.p + b * s.x.sb + t * s.x.sl;
    const E* up = (const E*)s.dy.p + b * s.dy.sb + t * s.dy.sl;
    E* dst = (E*)s.dx + m * s.heads * a.K;
    for (int64_t h = place % s.per; h < s.heads; h += s.per) {
      float v[16], d[16];
      load_head<VEC>(src + h * s.x.sh, l, v);
      load_head<VEC>(up + h * s.dy.sh, l, d);
      turn<ADJ>(l, d, g, -1.0f);
      float sum[2] = {0.0f, 0.0f};
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        sum[0] = __builtin_fmaf(v[e], v[e], sum[0]);
        sum[1] = __builtin_fmaf(wt[e] * d[e], v[e], sum[1]);
      }
      head_sum<LPH, 2>(sum);
      const float inv = rsqrtf(sum[0] / (float)a.K + a.eps);
      const float mean = sum[1] * inv / (float)a.K;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const float n = v[e] * inv;
        dw[e] = __builtin_fmaf(d[e], n, dw[e]);
        v[e] = inv * __builtin_fmaf(wt[e], d[e], -(n * mean));
      }
      store_head<VEC>(dst + h * a.K, l, v);
    }
  }
  if (s.part) put_partial<LPH>(l, dw, lds, s.part + block * a.K);
}

int lanes_of(int64_t K, int64_t R) {
  const int64_t n = (R / 2 + 7) / 8 + (K - R + 15) / 16;
  int lph = 1;
  while (lph < n) lph *= 2;
  return lph;  // at most 32: 256 columns are 16 lanes, and one more where R is cut
}

// Places of a token that work side by side: enough for 1024 lanes a compute unit, but of
// three heads each at least, over which a lane's weights and angles serve (two places of 16384
// tokens of 24 heads of 128 bf16 41 us, one 46; of 2048 tokens of 20 + 4 heads four 18 us
// backward, eight 20, sixteen 24); and of fewer where the card would lie idle, in decoding.
int places_of(int64_t T, int64_t heads, int lph, int cus) {
  int per = 1;
  while (per < heads && per * lph < 256 && T * per * lph < (int64_t)cus * 1024 &&
         (per * 6 <= heads || T * per * lph < (int64_t)cus * 128))
    per *= 2;
  return per;
}

bool vec_heads(const HeadNormArgs& a, const Heads& x, bool dense) {
  const int64_t m = a.bf16 ? 8 : 4;
  return (uintptr_t)x.p % 16 == 0 && (dense || (x.sb % m == 0 && x.sl % m == 0 && x.sh % m == 0));
}
bool vec_of(const HeadNormArgs& a, bool bwd) {
  return a.K % 8 == 0 && a.R % 16 == 0 && vec_heads(a, a.q, false) && vec_heads(a, a.k, false) &&
         vec_heads(a, {a.yq}, true) && vec_heads(a, {a.yk}, true) &&
         (!bwd || (vec_heads(a, a.dyq, false) && vec_heads(a, a.dyk, false)));
}

// Workgroups of one side of the backward: four for each compute unit, shared by the sides'
// heads, and no more than its tokens fill.
int64_t bwd_blocks(int64_t T, int64_t heads, int64_t all, int lph, int per, int cus) {
  if (T * heads == 0) return 0;
  const int64_t tokens = 256 / lph / per, need = (T + tokens - 1) / tokens;
  const int64_t most = (4 * (int64_t)cus * heads + all - 1) / all;
  return need < most ? need : most;
}

#define SW_HEAD_PICK(lph, CALL)   \
  do {                            \
    switch (lph) {                \
      case 1: CALL(1); break;     \
      case 2: CALL(2); break;     \
      case 4: CALL(4); break;     \
      case 8: CALL(8); break;     \
      case 16: CALL(16); break;   \
      default: CALL(32); break;   \
    }                             \
  } while (0)

template <class E, bool ADJ, bool VEC>
int fwd_typed(const HeadNormArgs& a, int cus, hipStream_t s) {
  const int64_t T = a.B * a.L;
  const int lph = lanes_of(a.K, a.R), per = places_of(T, a.H + a.Hk, lph, cus);
  const int64_t tokens = 256 / lph / per;
  const size_t lds = (size_t)(tokens * (a.R / 2)) * sizeof(float2);
#define CALL(LPH)                                                                                     \
  hipLaunchKernelGGL((fwd_kernel<E, LPH, ADJ, VEC>), dim3((unsigned)((T + tokens - 1) / tokens)), dim3(256), \
                     lds, s, a, per)
  SW_HEAD_PICK(lph, CALL);
#undef CALL
  return check_launch("head fwd_kernel");
}

template <class E, bool ADJ, bool VEC>
int bwd_typed(const HeadNormArgs& a, const Side& q, const Side& k, int lph, hipStream_t s) {
  const int per = q.blocks && (!k.blocks || q.per < k.per) ? q.per : k.per;
  const size_t lds = (size_t)(256 / lph / per * (a.R / 2)) * sizeof(float2);
#define CALL(LPH)                                                                                        \
  hipLaunchKernelGGL((bwd_kernel<E, LPH, ADJ, VEC>), dim3((unsigned)(q.blocks + k.blocks)), dim3(256), lds, s, \
                     a, q, k)
  SW_HEAD_PICK(lph, CALL);
#undef CALL
  return check_launch("head bwd_kernel");
}

}  // namespace
}  // namespace head

using namespace head;

int64_t head_norm_bwd_workspace(int64_t T, int64_t H, int64_t Hk, int64_t K) {
  int cus;
  if (device_cus(&cus) != SW_OK) return 0;
  // of any R: as many blocks as one token each would be
  return (bwd_blocks(T, H, H + Hk, 32, 8, cus) + bwd_blocks(T, Hk, H + Hk, 32, 8, cus)) * K * 4;
}

int head_norm_fwd(const HeadNormArgs& a) {
  int cus, st;
  if ((st = device_cus(&cus)) != SW_OK) return st;
  const hipStream_t s = current_stream();
  const bool vec = vec_of(a, false);
#define CALL(E)                                                                                     \
  (a.adjacent ? vec ? fwd_typed<E, true, true>(a, cus, s) : fwd_typed<E, true, false>(a, cus, s)    \
              : vec ? fwd_typed<E, false, true>(a, cus, s) : fwd_typed<E, false, false>(a, cus, s))
  return a.bf16 ? CALL(uint16_t) : CALL(float);
#undef CALL
}

int head_norm_bwd(const HeadNormArgs& a) {
  int cus, st;
  if ((st = device_cus(&cus)) != SW_OK) return st;
  const hipStream_t s = current_stream();
  const int64_t T = a.B * a.L;
  const int lph = lanes_of(a.K, a.R);
  Side q = {a.q, a.dyq, a.wq, a.yq, nullptr, a.H, 0, 1}, k = {a.k, a.dyk, a.wk, a.yk, nullptr, a.Hk, 0, 1};
  for (Side* x : {&q, &k}) {
    x->per = places_of(T, x->heads, lph, cus);
    x->blocks = bwd_blocks(T, x->heads, a.H + a.Hk, lph, x->per, cus);
  }
  norm::Partials part(s);
  const int64_t rows = q.blocks + k.blocks;
  if (a.dwq && rows) {
    if ((st = part.get(a.ws, a.ws_bytes, (size_t)(rows * a.K * 4), "sw_head_norm_bwd")) != SW_OK) return st;
    q.part = part.p;
    k.part = part.p + q.blocks * a.K;
  }
  const bool vec = vec_of(a, true);
#define CALL(E)                                                                                           \
  (a.adjacent ? vec ? bwd_typed<E, true, true>(a, q, k, lph, s) : bwd_typed<E, true, false>(a, q, k, lph, s) \
              : vec ? bwd_typed<E, false, true>(a, q, k, lph, s) : bwd_typed<E, false, false>(a, q, k, lph, s))
  if (rows && (st = a.bf16 ? CALL(uint16_t) : CALL(float)) != SW_OK) return st;
#undef CALL
  if (!a.dwq) return SW_OK;
  const int64_t blocks[2] = {q.blocks, k.blocks};
  float* outs[2] = {a.dwq, a.dwk};
  return norm::fold_partial_rows(part.p, blocks, a.K, outs, 2, s);
}

}  // namespace sw
