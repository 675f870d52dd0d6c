// gated_scan.hip -- the gated linear recurrence: forward and one step.
#include "gated_walk.h"

namespace sw {
namespace gated {
namespace {

// A chunk of 16 S steps of 64 channels.  Between memory and vector issue, some 45 slots a value
// of which the six transcendental instructions take 24: B=1 L=65536 D=5120 bf16 541 us, 2.68 GB
// at 5.0 TB/s (a copy reaches 5.1); B=8 L=2048 D=1536, one and a half rounds of workgroups,
// 53 us, 3.8 TB/s, and 91 with a channel a load (D=1537).  Looking back is a fourteenth of the
// latter shape (49 us without it) and a third at B=1 L=65536 D=256 (38 us without, 56 with).
template <class E, Mode MODE, bool PACKED, int S>
__global__ __launch_bounds__(THREADS, S == 16 ? 4 : 6) void fwd_kernel(GatedArgs a, Words k, int64_t chunks) {
  using G = FwdShape;
  constexpr int N = G::N, LANES = G::LANES, SLOTS = G::SLOTS, GROUP = G::GROUP, STEPS = SLOTS * S;
  __shared__ Pairs<N> sh[WAVES][LANES], back[LOOK][LANES];
  __shared__ Sequences<PACKED ? STEPS : 1> sq;
  __shared__ float rates[GROUP];
  __shared__ uint32_t ticket;
  const int slot = threadIdx.x / LANES, lane = threadIdx.x % LANES;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / 64);
  const bool second = slot & 1;
  uint32_t work = blockIdx.x;
  if (chunks > 1) {
    if (threadIdx.x == 0) ticket = atomicAdd(k.ticket, 1u);
    __syncthreads();
    work = (uint32_t)__builtin_amdgcn_readfirstlane((int)ticket) - k.base;
  }
  const uint32_t chunk = work / k.groups, group = work % k.groups;
  const int64_t b = group / k.per, base = (int64_t)(group % k.per) * GROUP, c0 = base + lane * N;
  const int64_t t0 = (int64_t)chunk * STEPS, left = a.L - t0;
  const int steps = (int)(left < STEPS ? left : STEPS), first = slot * S;
  const float lam = threadIdx.x < GROUP && base + threadIdx.x < a.D && a.L > 0 ? a.lam[base + threadIdx.x] : 0.0f;
  float start[N], in[N];
#pragma unroll
  for (int c = 0; c < N; ++c)
    start[c] = !PACKED && a.h0 && c0 + c < a.D ? a.h0[b * a.D + c0 + c] : 0.0f;
  if constexpr (PACKED) find_sequences(a, t0, sq);

  Rows<E, MODE, N> x, r, i;
  x.init(a.x.p, b * a.x.sb + t0 * a.x.sl, a.x.sl, steps, a.D, first, c0);
  r.init(a.r.p, b * a.r.sb + t0 * a.r.sl, a.r.sl, steps, a.D, first, c0);
  i.init(a.i.p, b * a.i.sb + t0 * a.i.sl, a.i.sl, steps, a.D, first, c0);

  // pairs of this lane's steps; past the row's end they do not matter
  float A[S][N], U[S][N], rate[N];
  Pairs<N> own = identity<N>();
  constexpr int BATCH = 8;  // steps whose loads are in flight together
#pragma unroll
  for (int j0 = 0; j0 < S; j0 += BATCH) {
    Raw<E, N> xw[BATCH], rw[BATCH], iw[BATCH];
#pragma unroll
    for (int j = 0; j < BATCH; ++j) {
      xw[j] = x.get(j0 + j);
      rw[j] = r.get(j0 + j);
      iw[j] = i.get(j0 + j);
    }
    if (j0 == 0) {
      if (threadIdx.x < GROUP) rates[threadIdx.x] = rate_of(lam, a.c);
      __syncthreads();
#pragma unroll
      for (int c = 0; c < N; ++c) rate[c] = rates[lane * N + c];
    }
#pragma unroll
    for (int j = 0; j < BATCH; ++j) {
      const int n = PACKED ? sq.seq[first + j0 + j] : 0;
      const bool starts = PACKED && sq.first(first + j0 + j);
#pragma unroll
      for (int c = 0; c < N; ++c) {
        float f, u;
        pair_of<E>(xw[j].get(c), rw[j].get(c), iw[j].get(c), rate[c], f, u);
        if constexpr (PACKED) {
          if (n < 0) {
            f = -1.0f;
            u = 0.0f;
          } else if (starts) {
            if (a.h0 && c0 + c < a.D) u = __builtin_fmaf(f, a.h0[n * a.D + c0 + c], u);
            f = -1.0f;
          }
        }
        A[j0 + j][c] = f;
        U[j0 + j][c] = u;
        own.U[c] = apply<PACKED>(f, u, own.U[c]);
        own.A[c] = PACKED && (f < 0.0f || own.A[c] < 0.0f) ? -1.0f : own.A[c] * f;
      }
    }
  }
  // what lies before a slot: a wave's halves exchange pairs by lanes, waves by LDS
  Pairs<N> other;
#pragma unroll
  for (int c = 0; c < N; ++c) {
    other.A[c] = __shfl_xor(own.A[c], 32);
    other.U[c] = __shfl_xor(own.U[c], 32);
  }
  if (!second) {
    Pairs<N> both = own;
    after<PACKED>(both, other);
    sh[wave][lane] = both;
  }
  __syncthreads();
  Pairs<N> before = first_of<PACKED, false, 4>(sh, wave, lane);
  if (second) after<PACKED>(before, other);

  if (chunks > 1) {
    Pairs<N> all = before;
    unsigned long long* w = word_at<G>(k, chunk, group, lane);
    bool end[N];
    const bool publishes = slot == SLOTS - 1 && chunk + 1 < chunks;
    if (publishes) {
      after<PACKED>(all, own);
#pragma unroll
      for (int c = 0; c < N; ++c) {
        end[c] = chunk == 0 || all.A[c] < 0.0f;
        if (chunk == 0) all.U[c] = apply<PACKED>(all.A[c], all.U[c], start[c]);
      }
      publish<G>(w, k.epoch, all, end);
    }
    look_back<G>(k, chunk, group, slot, lane, start, back, in);
    if (publishes)
#pragma unroll
      for (int c = 0; c < N; ++c)
        if (!end[c])
          carry_put(w + c, carry_status(k.epoch, CARRY_INC),
                    __float_as_uint(__builtin_fmaf(all.A[c], in[c], all.U[c])));
  } else {
#pragma unroll
    for (int c = 0; c < N; ++c) in[c] = start[c];
  }

  float h[N];
#pragma unroll
  for (int c = 0; c < N; ++c) h[c] = apply<PACKED>(before.A[c], before.U[c], in[c]);
  if (a.ckpt && first % BWD_STEPS == 0 && first < steps) {
    const int64_t row = b * ((a.L + BWD_STEPS - 1) / BWD_STEPS) + (t0 + first) / BWD_STEPS;
#pragma unroll
    for (int c = 0; c < N; ++c)
      if (c0 + c < a.D) a.ckpt[row * a.D + c0 + c] = h[c];
  }
  Rows<E, MODE, N> out;
  out.init_out(a.h, (b * a.L + t0) * a.D, a.h ? steps : 0, a.D, first, c0);
#pragma unroll
  for (int j = 0; j < S; ++j) {
#pragma unroll
    for (int c = 0; c < N; ++c) h[c] = apply<PACKED>(A[j][c], U[j][c], h[c]);
    out.put(j, h);
    if (a.h_last && (PACKED ? sq.last(first + j) : t0 + first + j == a.L - 1)) {
      const int64_t n = PACKED ? sq.seq[first + j] : b;
#pragma unroll
      for (int c = 0; c < N; ++c)
        if (c0 + c < a.D) a.h_last[n * a.D + c0 + c] = h[c];
    }
  }
  // sequences of no steps
  if (a.h_last) {
    if constexpr (PACKED) {
      for (int64_t n = chunk + (int64_t)slot * chunks; n < a.nseq; n += chunks * SLOTS)
        if (edge(a, n) >= edge(a, n + 1))
#pragma unroll
          for (int c = 0; c < N; ++c)
            if (c0 + c < a.D) a.h_last[n * a.D + c0 + c] = a.h0 ? a.h0[n * a.D + c0 + c] : 0.0f;
    } else if (a.L == 0 && slot == 0) {
#pragma unroll
      for (int c = 0; c < N; ++c)
        if (c0 + c < a.D) a.h_last[b * a.D + c0 + c] = start[c];
    }
  }
}

// A token of each sequence: bound by memory, or by the launch.
template <class E>
__global__ __launch_bounds__(256) void step_kernel(GatedStepArgs a) {
  const int64_t d = blockIdx.x * 256ll + threadIdx.x;
  if (d >= a.D) return;
  const float k = rate_of(a.lam[d], a.c);
  const auto value = [](const void* p, int64_t j) {
    if constexpr (sizeof(E) == 4)
      return ((const float*)p)[j];
    else
      return bf16_one(((const uint16_t*)p)[j]);
  };
  for (int64_t b = blockIdx.y; b < a.B; b += gridDim.y) {
    const int64_t slot = a.slots ? a.slots[b] : b;
    float h = 0.0f;
    if (slot >= 0 && slot < a.pool) {
      float f, u;
      pair_of<E>(value(a.x, b * a.x_st + d), value(a.r, b * a.r_st + d), value(a.i, b * a.i_st + d), k,
                 f, u);
      float* s = a.state + slot * a.D + d;
      h = __builtin_fmaf(f, *s, u);
      *s = h;
    }
    if constexpr (sizeof(E) == 4)
      ((float*)a.h)[b * a.D + d] = h;
    else
      ((uint16_t*)a.h)[b * a.D + d] = (uint16_t)bf16_rne(h);
  }
}

}  // namespace

// Steps of a lane: 8 where they hold the row.  (Two chunks for one of 16 are slower in bf16, B=8
// L=2048 D=1536 65 us for 52, B=1 L=65536 D=256 108 for 57, and no faster in fp32, 91 for 90.)
int fwd_s(const GatedArgs& a) { return a.L <= FwdShape::SLOTS * FWD_SHORT_S ? FWD_SHORT_S : FWD_S; }

int64_t fwd_words(const GatedArgs& a) {
  return words_bytes(chunks_of(a.L, FwdShape::SLOTS * fwd_s(a)), groups_of(a, FwdShape::GROUP), FwdShape::GROUP);
}

int run_fwd(const GatedArgs& a, void* ws, size_t ws_bytes, hipStream_t s) {
  const int S = fwd_s(a), steps = FwdShape::SLOTS * S;
  const int64_t chunks = chunks_of(a.L, steps), groups = groups_of(a, FwdShape::GROUP);
  if (chunks * groups > SW_MAX_WGS / 2)
    return fail(SW_ERR_UNSUPPORTED, "%lld chunks of the recurrence exceed the launch limit",
                (long long)(chunks * groups));
  int st;
  LaunchWords words(s);
  if ((st = words.get(ws, ws_bytes, chunks, groups, FwdShape::GROUP, a.B, s, "sw_gated_scan_fwd")) != SW_OK)
    return st;
  const Words& k = words.k;
  const Mode mode = mode_of(a, steps, FwdShape::N, {&a.x, &a.r, &a.i}, {a.h});
  const dim3 grid((unsigned)(chunks * groups));
#define LAUNCH(E, MODE, PACKED, S) \
  hipLaunchKernelGGL((fwd_kernel<E, MODE, PACKED, S>), grid, dim3(THREADS), 0, s, a, k, chunks)
#define CALL(E, MODE)                       \
  do {                                      \
    if (S == FWD_S && a.cu)                 \
      LAUNCH(E, MODE, true, FWD_S);         \
    else if (S == FWD_S)                    \
      LAUNCH(E, MODE, false, FWD_S);        \
    else if (a.cu)                          \
      LAUNCH(E, MODE, true, FWD_SHORT_S);   \
    else                                    \
      LAUNCH(E, MODE, false, FWD_SHORT_S);  \
  } while (0)
#define TYPED(E)          \
  do {                    \
    if (mode == NEAR)     \
      CALL(E, NEAR);      \
    else if (mode == SPLIT) \
      CALL(E, SPLIT);     \
    else                  \
      CALL(E, FAR);       \
  } while (0)
  if (a.bf16)
    TYPED(uint16_t);
  else
    TYPED(float);
#undef TYPED
#undef CALL
#undef LAUNCH
  return words.done(check_launch("gated fwd_kernel"));
}

}  // namespace gated

using namespace gated;

int64_t gated_scan_fwd_workspace(int64_t B, int64_t L, int64_t D) {
  GatedArgs a;
  a.B = B;
  a.L = L;
  a.D = D;
  return fwd_words(a);
}

int gated_scan_fwd(const GatedArgs& a) {
  if (a.nseq == 0) return SW_OK;
  return run_fwd(a, a.ws, a.ws_bytes, current_stream());
}

int gated_scan_step(const GatedStepArgs& a) {
  const hipStream_t s = current_stream();
  const int64_t cols = (a.D + 255) / 256;
  int64_t rows = SW_MAX_WGS / cols;  // the kernel steps through the others
  rows = a.B < rows ? a.B : rows;
  const dim3 grid((unsigned)cols, (unsigned)(rows < 65535 ? rows : 65535));
  if (a.bf16)
    hipLaunchKernelGGL(step_kernel<uint16_t>, grid, dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL(step_kernel<float>, grid, dim3(256), 0, s, a);
  return check_launch("gated step_kernel");
}

}  // namespace sw
