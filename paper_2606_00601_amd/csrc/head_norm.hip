// head_norm.hip -- the norm of each head's query and key with the rotation by the
// token's position, u = w x / rms(x), y = R(position) u, and its gradients.
//
// LPH lanes hold a head, 16 columns each as two vectors of 8 which hold both members
// of every pair they turn: (8 j .. , R/2 + 8 j ..) for halves, (16 j ..) for
// neighbours; columns that are not turned go to the lanes behind.  So the turn needs
// no exchange and the norm a sum over LPH lanes.  A lane keeps one token's angles and
// steps through its heads, queries first, then keys.  Bound by memory: a value is read
// once and written once.
#include "norm_rows.h"
#include "token_ops.h"

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
__device__ __forceinline__ void angles_of(const HeadNormArgs& a, const Lane& l, int64_t b, int64_t t,
                                          Angles& g) {
  const int64_t at = b * a.pos_sb + t * a.pos_sl;
  const double pos = !a.pos   ? (double)t
                     : a.pos64 ? (double)((const int64_t*)a.pos)[at]
                               : (double)((const int32_t*)a.pos)[at];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    g.c[j] = 1.0f;
    g.s[j] = 0.0f;
    if (l.pair >= 0 && l.pair + j < (int)a.R / 2) angle(pos, a.inv_freq[l.pair + j], g.c[j], g.s[j]);
  }
}

// The lane's pairs turned by their angles, or back by them (sign -1).
template <bool ADJ>
__device__ __forceinline__ void turn(float* x, const Angles& g, float sign) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    float& p = x[ADJ ? 2 * j : j];
    float& q = x[ADJ ? 2 * j + 1 : 8 + j];
    const float s = sign * g.s[j], pp = p * g.c[j] - q * s;
    q = q * g.c[j] + p * s;
    p = pp;
  }
}

template <class E>
__device__ __forceinline__ void load_head(const E* p, const Lane& l, float* x, bool vec) {
  load8(p + l.o1, x, l.n1, vec);
  load8(p + l.o2, x + 8, l.n2, vec);
}
template <class E>
__device__ __forceinline__ void store_head(E* p, const Lane& l, const float* x, bool vec) {
  store8(p + l.o1, x, l.n1, vec);
  store8(p + l.o2, x + 8, l.n2, vec);
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

template <class E, int LPH, bool ADJ>
__device__ __forceinline__ void fwd_heads(const HeadNormArgs& a, const Heads& x, const float* w, void* y,
                                          int64_t heads, int64_t first, int64_t step, int64_t b, int64_t t,
                                          const Lane& l, const Angles& g, bool vec) {
  if (first >= heads) return;
  float wt[16];
  load_weights(w, l, wt);
  const E* src = (const E*)x.p + b * x.sb + t * x.sl;
  E* dst = (E*)y + (b * a.L + t) * heads * a.K;
  for (int64_t h = first; h < heads; h += step) {
    float v[16];
    load_head(src + h * x.sh, l, v, vec);
    float sum[1] = {0.0f};
#pragma unroll
    for (int j = 0; j < 16; ++j) sum[0] = __builtin_fmaf(v[j], v[j], sum[0]);
    head_sum<LPH, 1>(sum);
    const float inv = rsqrtf(sum[0] / (float)a.K + a.eps);
#pragma unroll
    for (int j = 0; j < 16; ++j) v[j] *= inv * wt[j];
    if (a.R) turn<ADJ>(v, g, 1.0f);
    store_head(dst + h * a.K, l, v, vec);
  }
}

// Lanes: (token, one of `per` places of it, lane of the head).
template <class E, int LPH, bool ADJ>
__global__ __launch_bounds__(256) void fwd_kernel(HeadNormArgs a, int per, bool vec) {
  const int j = threadIdx.x % LPH, place = threadIdx.x / LPH;
  const int64_t T = a.B * a.L;
  const int64_t m = blockIdx.x * (int64_t)(256 / LPH / per) + place / per;
  if (m >= T) return;  // whole heads' lanes leave together
  const int64_t b = m / a.L, t = m % a.L;
  const Lane l = lane_of(a, j);
  Angles g;
  angles_of(a, l, b, t, g);
  const int64_t first = place % per;
  fwd_heads<E, LPH, ADJ>(a, a.q, a.wq, a.yq, a.H, first, per, b, t, l, g, vec);
  const int64_t done = first >= a.H ? first : first + (a.H - first + per - 1) / per * per;
  fwd_heads<E, LPH, ADJ>(a, a.k, a.wk, a.yk, a.Hk, done - a.H, per, b, t, l, g, vec);
}

// dx = inv (w g - n mean(w g n)), n = x inv, with g the gradient turned back; dw += g n.
template <class E, int LPH, bool ADJ>
__device__ __forceinline__ void bwd_heads(const HeadNormArgs& a, const Heads& x, const Heads& dy,
                                          const float* w, void* dx, float* dw, int64_t heads,
                                          int64_t first, int64_t step, int64_t b, int64_t t,
                                          const Lane& l, const Angles& g, bool vec) {
  if (first >= heads) return;
  float wt[16];
  load_weights(w, l, wt);
  const E* src = (const E*)x.p + b * x.sb + t * x.sl;
  const E* up = (const E*)dy.p + b * dy.sb + t * dy.sl;
  E* dst = (E*)dx + (b * a.L + t) * heads * a.K;
  for (int64_t h = first; h < heads; h += step) {
    float v[16], d[16];
    load_head(src + h * x.sh, l, v, vec);
    load_head(up + h * dy.sh, l, d, vec);
    if (a.R) turn<ADJ>(d, g, -1.0f);
    float sum[2] = {0.0f, 0.0f};
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      sum[0] = __builtin_fmaf(v[j], v[j], sum[0]);
      sum[1] = __builtin_fmaf(wt[j] * d[j], v[j], sum[1]);
    }
    head_sum<LPH, 2>(sum);
    const float inv = rsqrtf(sum[0] / (float)a.K + a.eps);
    const float mean = sum[1] * inv / (float)a.K;
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      const float n = v[j] * inv;
      dw[j] = __builtin_fmaf(d[j], n, dw[j]);
      v[j] = inv * (wt[j] * d[j] - n * mean);
    }
    store_head(dst + h * a.K, l, v, vec);
  }
}

// A workgroup's sums of the weights' gradients, over its 256 / LPH heads in order.
template <int LPH>
__device__ __forceinline__ void put_partial(const HeadNormArgs& a, const Lane& l, const float* dw,
                                            float* lds, float* out) {
  const int j = threadIdx.x % LPH, place = threadIdx.x / LPH;
  for (int i = 0; i < 256 / LPH; ++i) {
    __syncthreads();
    if (place == i)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        float* p = lds + e * LPH + j;
        *p = i ? *p + dw[e] : dw[e];
      }
  }
  __syncthreads();
  if (place == 0) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (e < l.n1) out[l.o1 + e] = lds[e * LPH + j];
      if (e < l.n2) out[l.o2 + e] = lds[(8 + e) * LPH + j];
    }
  }
}

template <class E, int LPH, bool ADJ>
__global__ __launch_bounds__(256) void bwd_kernel(HeadNormArgs a, float* part, int per, bool vec) {
  __shared__ float lds[16 * LPH];
  const int j = threadIdx.x % LPH, place = threadIdx.x / LPH;
  const int64_t T = a.B * a.L, tokens = 256 / LPH / per;
  const Lane l = lane_of(a, j);
  float dq[16], dk[16];
#pragma unroll
  for (int e = 0; e < 16; ++e) dq[e] = dk[e] = 0.0f;
  const int64_t first = place % per;
  const int64_t done = first >= a.H ? first : first + (a.H - first + per - 1) / per * per;
  for (int64_t m = blockIdx.x * tokens + place / per; m < T; m += gridDim.x * tokens) {
    const int64_t b = m / a.L, t = m % a.L;
    Angles g;
    angles_of(a, l, b, t, g);
    bwd_heads<E, LPH, ADJ>(a, a.q, a.dyq, a.wq, a.yq, dq, a.H, first, per, b, t, l, g, vec);
    bwd_heads<E, LPH, ADJ>(a, a.k, a.dyk, a.wk, a.yk, dk, a.Hk, done - a.H, per, b, t, l, g, vec);
  }
  if (part) {
    put_partial<LPH>(a, l, dq, lds, part + blockIdx.x * a.K);
    __syncthreads();
    put_partial<LPH>(a, l, dk, lds, part + ((int64_t)gridDim.x + blockIdx.x) * a.K);
  }
}

int lanes_of(int64_t K, int64_t R) {
  const int64_t n = (R / 2 + 7) / 8 + (K - R + 15) / 16;
  int lph = 1;
  while (lph < n) lph *= 2;
  return lph;  // at most 32: 256 columns are 16 lanes, and one more where R is cut
}

// Places of a token that work side by side: as few as fill the card, since each
// forms the token's angles again, and no more than there are heads.
int places_of(int64_t T, int64_t heads, int lph, int cus) {
  int per = 1;
  while (per < heads && per * lph < 256 && T * per * lph < (int64_t)cus * 1024) per *= 2;
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

int64_t bwd_blocks(int64_t T, int64_t heads, int lph, int cus) {
  const int64_t tokens = 256 / lph / places_of(T, heads, lph, cus);
  const int64_t need = (T + tokens - 1) / tokens, most = 4 * (int64_t)cus;
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

template <class E, bool ADJ>
int fwd_typed(const HeadNormArgs& a, int cus, hipStream_t s) {
  const int64_t T = a.B * a.L;
  const int lph = lanes_of(a.K, a.R), per = places_of(T, a.H + a.Hk, lph, cus);
  const int64_t tokens = 256 / lph / per;
  const bool vec = vec_of(a, false);
#define CALL(LPH)                                                                                 \
  hipLaunchKernelGGL((fwd_kernel<E, LPH, ADJ>), dim3((unsigned)((T + tokens - 1) / tokens)), dim3(256), 0, \
                     s, a, per, vec)
  SW_HEAD_PICK(lph, CALL);
#undef CALL
  return check_launch("head fwd_kernel");
}

template <class E, bool ADJ>
int bwd_typed(const HeadNormArgs& a, float* part, int64_t blocks, int cus, hipStream_t s) {
  const int lph = lanes_of(a.K, a.R), per = places_of(a.B * a.L, a.H + a.Hk, lph, cus);
  const bool vec = vec_of(a, true);
#define CALL(LPH)                                                                             \
  hipLaunchKernelGGL((bwd_kernel<E, LPH, ADJ>), dim3((unsigned)blocks), dim3(256), 0, s, a, part, per, vec)
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
  // the most blocks any R asks for: one token each
  const int64_t most = 4 * (int64_t)cus;
  return (H + Hk) * T == 0 ? 0 : (T < most ? T : most) * K * 8;
}

int head_norm_fwd(const HeadNormArgs& a) {
  int cus, st;
  if ((st = device_cus(&cus)) != SW_OK) return st;
  const hipStream_t s = current_stream();
  if (a.bf16)
    return a.adjacent ? fwd_typed<uint16_t, true>(a, cus, s) : fwd_typed<uint16_t, false>(a, cus, s);
  return a.adjacent ? fwd_typed<float, true>(a, cus, s) : fwd_typed<float, false>(a, cus, s);
}

int head_norm_bwd(const HeadNormArgs& a) {
  int cus, st;
  if ((st = device_cus(&cus)) != SW_OK) return st;
  const hipStream_t s = current_stream();
  const int64_t T = a.B * a.L;
  float* outs[2] = {a.dwq, a.dwk};
  if (T * (a.H + a.Hk) == 0) return norm::fold_partials(nullptr, 0, a.K, outs, 2, s);
  const int64_t blocks = bwd_blocks(T, a.H + a.Hk, lanes_of(a.K, a.R), cus);
  norm::Partials part(s);
  if (a.dwq && (st = part.get(a.ws, a.ws_bytes, (size_t)(blocks * a.K * 8), "sw_head_norm_bwd")) != SW_OK)
    return st;
  if (a.bf16)
    st = a.adjacent ? bwd_typed<uint16_t, true>(a, part.p, blocks, cus, s)
                    : bwd_typed<uint16_t, false>(a, part.p, blocks, cus, s);
  else
    st = a.adjacent ? bwd_typed<float, true>(a, part.p, blocks, cus, s)
                    : bwd_typed<float, false>(a, part.p, blocks, cus, s);
  if (st != SW_OK || !a.dwq) return st;
  return norm::fold_partials(part.p, blocks, a.K, outs, 2, s);
}

}  // namespace sw
