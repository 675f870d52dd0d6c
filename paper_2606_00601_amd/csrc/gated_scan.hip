// gated_scan.hip -- the gated linear recurrence: forward and one step.
#include "gated_walk.h"
#include "norm_rows.h"

namespace sw {
namespace gated {
namespace {

// A chunk of 256 steps of a group of channels.
template <class E, Mode MODE, bool PACKED>
__global__ __launch_bounds__(THREADS, 4) void fwd_kernel(GatedArgs a, Words k, int64_t chunks) {
  using G = FwdShape<E>;
  constexpr int N = G::N, S = FWD_S, LANES = G::LANES, SLOTS = G::SLOTS;
  __shared__ Pairs<N> sh[SLOTS][LANES], back[LOOK][LANES];
  __shared__ Sequences<PACKED ? FWD_STEPS : 1> sq;
  __shared__ float rates[G::GROUP];
  __shared__ uint32_t ticket;
  const int slot = threadIdx.x / LANES, lane = threadIdx.x % LANES;
  uint32_t work = blockIdx.x;
  if (chunks > 1) {
    if (threadIdx.x == 0) ticket = atomicAdd(k.ticket, 1u);
    __syncthreads();
    work = ticket;
  }
  const int64_t chunk = work / (uint32_t)k.groups, group = work % (uint32_t)k.groups;
  const int64_t per = (a.D + G::GROUP - 1) / G::GROUP;
  const int64_t b = group / per, c0 = group % per * G::GROUP + lane * N;
  const int64_t t0 = chunk * FWD_STEPS, left = a.L - t0, steps = left < FWD_STEPS ? left : FWD_STEPS;
  const int first = slot * S;
  if constexpr (PACKED) find_sequences(a, t0, sq);

  Rows<E, MODE, N> x, r, i;
  x.init(a.x.p, b * a.x.sb + t0 * a.x.sl, a.x.sl, steps, a.D, first, c0);
  r.init(a.r.p, b * a.r.sb + t0 * a.r.sl, a.r.sl, steps, a.D, first, c0);
  i.init(a.i.p, b * a.i.sb + t0 * a.i.sl, a.i.sl, steps, a.D, first, c0);
  const int nrate = (int)(a.D - (c0 - lane * N) < G::GROUP ? a.D - (c0 - lane * N) : G::GROUP);
  if (threadIdx.x < G::GROUP)
    rates[threadIdx.x] =
        (int)threadIdx.x < nrate && a.L > 0 ? rate_of(a.lam[c0 - lane * N + threadIdx.x], a.c) : 0.0f;
  // pairs of this lane's steps; past the row's end they do not matter
  float A[S][N], U[S][N];
  Pairs<N> own;
#pragma unroll
  for (int c = 0; c < N; ++c) {
    own.A[c] = 1.0f;
    own.U[c] = 0.0f;
  }
  constexpr int BATCH = 8;  // steps whose loads are in flight together
  float rate[N];
#pragma unroll
  for (int j0 = 0; j0 < S; j0 += BATCH) {
    uint32_t xw[BATCH], rw[BATCH], iw[BATCH];
#pragma unroll
    for (int j = 0; j < BATCH; ++j) {
      xw[j] = x.get(j0 + j);
      rw[j] = r.get(j0 + j);
      iw[j] = i.get(j0 + j);
    }
    if (j0 == 0) {
      __syncthreads();
#pragma unroll
      for (int c = 0; c < N; ++c) rate[c] = rates[lane * N + c];
    }
#pragma unroll
    for (int j = 0; j < BATCH; ++j) {
#pragma unroll
      for (int c = 0; c < N; ++c) {
        float f, u;
        pair_of<E>(channel<E>(xw[j], c), channel<E>(rw[j], c), channel<E>(iw[j], c), rate[c], f, u);
        if constexpr (PACKED) {
          const int n = sq.seq[first + j0 + j];
          if (n < 0) {
            f = -1.0f;
            u = 0.0f;
          } else if (sq.first(first + j0 + j)) {
            if (a.h0 && c0 + c < a.D) u = __builtin_fmaf(f, a.h0[n * a.D + c0 + c], u);
            f = -1.0f;
          }
        }
        A[j0 + j][c] = f;
        U[j0 + j][c] = u;
        own.U[c] = apply<PACKED>(f, u, own.U[c]);
        if constexpr (PACKED)
          own.A[c] = f < 0.0f || own.A[c] < 0.0f ? -1.0f : own.A[c] * f;
        else
          own.A[c] *= f;
      }
    }
  }
  sh[slot][lane] = own;
  __syncthreads();
  Pairs<N> before;  // the chunk's steps before this slot
#pragma unroll
  for (int c = 0; c < N; ++c) {
    before.A[c] = 1.0f;
    before.U[c] = 0.0f;
  }
  for (int s = 0; s < slot; ++s) after<PACKED>(before, sh[s][lane]);

  float start[N], in[N];
#pragma unroll
  for (int c = 0; c < N; ++c)
    start[c] = !PACKED && a.h0 && c0 + c < a.D ? a.h0[b * a.D + c0 + c] : 0.0f;
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
      publish<G>(w, all, end);
    }
    look_back<G>(k, chunk, group, slot, lane, start, back, in);
    if (publishes)
#pragma unroll
      for (int c = 0; c < N; ++c)
        if (!end[c]) carry_put(w + c, CARRY_INC, __float_as_uint(__builtin_fmaf(all.A[c], in[c], all.U[c])));
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
    if (PACKED ? sq.last(first + j) && a.h_last : a.h_last && t0 + first + j == a.L - 1) {
      const int64_t n = PACKED ? sq.seq[first + j] : b;
#pragma unroll
      for (int c = 0; c < N; ++c)
        if (c0 + c < a.D) a.h_last[n * a.D + c0 + c] = h[c];
    }
  }
  // sequences of no steps
  if (a.h_last) {
    if constexpr (PACKED) {
      for (int64_t n = chunk + slot * chunks; n < a.nseq; n += chunks * SLOTS)
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

constexpr int group_of(bool bf16) { return bf16 ? FwdShape<uint16_t>::GROUP : FwdShape<float>::GROUP; }

int64_t fwd_words(const GatedArgs& a) {
  const int g = group_of(a.bf16);
  return words_bytes(chunks_of(a.L, FWD_STEPS), groups_of(a.B, a.D, g), g);
}

int run_fwd(const GatedArgs& a, void* ws, hipStream_t s) {
  const int64_t chunks = chunks_of(a.L, FWD_STEPS), groups = groups_of(a.B, a.D, group_of(a.bf16));
  if (chunks * groups > SW_MAX_WGS / 2)
    return fail(SW_ERR_UNSUPPORTED, "%lld chunks of the recurrence exceed the launch limit",
                (long long)(chunks * groups));
  int st;
  if (chunks > 1 && (st = zero_words((uint32_t*)ws, (size_t)fwd_words(a) / 4, s)) != SW_OK) return st;
  const Words k = {(uint32_t*)ws, (unsigned long long*)((char*)ws + 64), groups};
  // pairs of bf16 channels go in words where every row begins on one
  const StepRows* rows[3] = {&a.x, &a.r, &a.i};
  bool whole = a.D % 2 == 0 && (uintptr_t)a.h % 4 == 0;
  for (const StepRows* x : rows)
    whole = whole && (uintptr_t)x->p % 4 == 0 && x->sl % 2 == 0 && x->sb % 2 == 0;
  const Mode mode = !near_rows(a, rows, 3, FWD_STEPS) ? FAR : whole || !a.bf16 ? NEAR : SPLIT;
  const dim3 grid((unsigned)(chunks * groups));
#define CALL(E, MODE)                                                                                  \
  do {                                                                                                 \
    if (a.cu)                                                                                          \
      hipLaunchKernelGGL((fwd_kernel<E, MODE, true>), grid, dim3(THREADS), 0, s, a, k, chunks);        \
    else                                                                                               \
      hipLaunchKernelGGL((fwd_kernel<E, MODE, false>), grid, dim3(THREADS), 0, s, a, k, chunks);       \
  } while (0)
  if (a.bf16) {
    if (mode == NEAR)
      CALL(uint16_t, NEAR);
    else if (mode == SPLIT)
      CALL(uint16_t, SPLIT);
    else
      CALL(uint16_t, FAR);
  } else if (mode == NEAR) {
    CALL(float, NEAR);
  } else {
    CALL(float, FAR);
  }
#undef CALL
  return check_launch("gated fwd_kernel");
}

}  // namespace gated

using namespace gated;

int64_t gated_scan_fwd_workspace(int64_t B, int64_t L, int64_t D) {
  GatedArgs a;
  a.B = B;
  a.L = L;
  a.D = D;
  const int64_t f = fwd_words(a);
  a.bf16 = true;
  const int64_t h = fwd_words(a);
  return f > h ? f : h;
}

int gated_scan_fwd(const GatedArgs& a) {
  if (a.nseq == 0) return SW_OK;
  const hipStream_t s = current_stream();
  norm::Partials ws(s);
  int st;
  const int64_t need = fwd_words(a);
  if (need > 0 && (st = ws.get(a.ws, a.ws_bytes, (size_t)need, "sw_gated_scan_fwd")) != SW_OK) return st;
  return run_fwd(a, ws.p, s);
}

int gated_scan_step(const GatedStepArgs& a) {
  const hipStream_t s = current_stream();
  const dim3 grid((unsigned)((a.D + 255) / 256), (unsigned)(a.B < 65535 ? a.B : 65535));
  if (a.bf16)
    hipLaunchKernelGGL(step_kernel<uint16_t>, grid, dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL(step_kernel<float>, grid, dim3(256), 0, s, a);
  return check_launch("gated step_kernel");
}

}  // namespace sw
