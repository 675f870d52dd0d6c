// gated_bwd.hip -- the gated linear recurrence: backward.
//
// The states before the backward's chunks of 128 steps are what a training forward kept, so
// a chunk's own are formed from its registers alone.  The gradient's recurrence runs the
// other way, over v_t = a_t g_t, what step t hands to the one before it:
//   v_t = a_t (dh_t + v_{t+1}),
// an affine pair again, composed in slots and between workgroups from the last chunk on.
#include "gated_walk.h"
#include "norm_rows.h"

namespace sw {
namespace gated {
namespace {

template <class E, Mode MODE, bool PACKED>
__global__ __launch_bounds__(THREADS, sizeof(E) == 4 ? 4 : 2) void bwd_kernel(GatedArgs a, const float* ckpt, float* part,
                                                         Words k, int64_t chunks) {
  constexpr int N = VC<E>, S = BWD_S;
  __shared__ Pairs<N> sh[SLOTS][LANES], sg[SLOTS][LANES];
  __shared__ Sequences<PACKED ? BWD_STEPS : 1> sq;
  __shared__ float rates[GROUP<E>];
  __shared__ uint32_t ticket;
  const int slot = threadIdx.x / LANES, lane = threadIdx.x % LANES;
  uint32_t work = blockIdx.x;
  if (chunks > 1) {
    if (threadIdx.x == 0) ticket = atomicAdd(k.ticket, 1u);
    __syncthreads();
    work = ticket;
  }
  // `turn` counts the chunks from the last one on
  const int64_t turn = work / (uint32_t)k.groups, group = work % (uint32_t)k.groups;
  const int64_t chunk = chunks - 1 - turn;
  const int64_t per = (a.D + GROUP<E> - 1) / GROUP<E>;
  const int64_t b = group / per, base = group % per * GROUP<E>, c0 = base + lane * N;
  const int64_t t0 = chunk * BWD_STEPS, left = a.L - t0, steps = left < BWD_STEPS ? left : BWD_STEPS;
  const int first = slot * S;
  if constexpr (PACKED) find_sequences(a, t0, sq);

  Rows<E, MODE> x, r, i, d;
  x.init(a.x.p, b * a.x.sb + t0 * a.x.sl, a.x.sl, steps, a.D, first, c0);
  r.init(a.r.p, b * a.r.sb + t0 * a.r.sl, a.r.sl, steps, a.D, first, c0);
  i.init(a.i.p, b * a.i.sb + t0 * a.i.sl, a.i.sl, steps, a.D, first, c0);
  d.init(a.dh.p, b * a.dh.sb + t0 * a.dh.sl, a.dh.sl, steps, a.D, first, c0);
  uint32_t xw[S], rw[S], iw[S], dw[S];
#pragma unroll
  for (int j = 0; j < S; ++j) {
    xw[j] = x.get(j);
    rw[j] = r.get(j);
    iw[j] = i.get(j);
    dw[j] = d.get(j);
  }
  float start[N], in[N], tail[N];
#pragma unroll
  for (int c = 0; c < N; ++c) {
    const bool there = c0 + c < a.D;
    start[c] = there ? ckpt[(b * chunks + chunk) * a.D + c0 + c] : 0.0f;
    tail[c] = !PACKED && a.dh_last && there ? a.dh_last[b * a.D + c0 + c] : 0.0f;
  }
  if (threadIdx.x < GROUP<E>)
    rates[threadIdx.x] = base + threadIdx.x < a.D ? rate_of(a.lam[base + threadIdx.x], a.c) : 0.0f;
  __syncthreads();

  // of each step: a, b s, (m / b) a^2 s x, m a, 1 - sigmoid(r), (1 - s) x, dh
  float A[S][N], bs[S][N], q[S][N], ma[S][N], rest[S][N], xi[S][N], dh[S][N];
  float h0[PACKED ? S : 1][N];  // PACKED: the state before a sequence's first step
  uint32_t none = 0, starts = 0, ends = 0;  // PACKED: steps of no sequence, first and last ones
  Pairs<N> fwd, bwd;
#pragma unroll
  for (int c = 0; c < N; ++c) {
    fwd.A[c] = bwd.A[c] = 1.0f;
    fwd.U[c] = bwd.U[c] = 0.0f;
  }
#pragma unroll
  for (int j = 0; j < S; ++j) {
    int n = 0;
    if constexpr (PACKED) {
      n = sq.seq[first + j];
      none |= (uint32_t)(n < 0) << j;
      starts |= (uint32_t)sq.first[first + j] << j;
      ends |= (uint32_t)sq.last[first + j] << j;
    }
#pragma unroll
    for (int c = 0; c < N; ++c) {
      const float xv = channel<E>(xw[j], c);
      const Step s = step_of<E>(xv, channel<E>(rw[j], c), channel<E>(iw[j], c), rates[lane * N + c]);
      A[j][c] = s.a;
      bs[j][c] = s.b * s.si;
      q[j][c] = s.q * s.si * xv;
      ma[j][c] = (s.m < 1e3f ? s.m : 1e3f) * s.a;
      rest[j][c] = s.rest_r;
      xi[j][c] = xv * s.rest_i;
      dh[j][c] = channel<E>(dw[j], c);
      float f = s.a, u = s.u;
      if constexpr (PACKED) {
        const bool there = c0 + c < a.D;
        h0[j][c] = 0.0f;
        if (n < 0) {
          f = -1.0f;
          u = 0.0f;
          A[j][c] = bs[j][c] = q[j][c] = ma[j][c] = rest[j][c] = xi[j][c] = dh[j][c] = 0.0f;
        } else {
          if (starts >> j & 1) {
            if (a.h0 && there) h0[j][c] = a.h0[n * a.D + c0 + c];
            u = __builtin_fmaf(f, h0[j][c], u);
            f = -1.0f;
          }
          if ((ends >> j & 1) && a.dh_last && there) dh[j][c] += a.dh_last[n * a.D + c0 + c];
        }
      } else {
        // past the row's end (rows of stride 0 are read there again) nothing is added, and
        // what comes in passes through
        if (first + j >= steps) {
          f = A[j][c] = 1.0f;
          dh[j][c] = 0.0f;
        }
      }
      fwd.U[c] = apply<PACKED>(f, u, fwd.U[c]);
      fwd.A[c] = PACKED && (f < 0.0f || fwd.A[c] < 0.0f) ? -1.0f : fwd.A[c] * f;
    }
  }
#pragma unroll
  for (int j = S - 1; j >= 0; --j)
#pragma unroll
    for (int c = 0; c < N; ++c) {
      const bool cut = PACKED && ((ends | none) >> j & 1);
      bwd.U[c] = A[j][c] * (dh[j][c] + (cut ? 0.0f : bwd.U[c]));
      bwd.A[c] = cut || (PACKED && bwd.A[c] < 0.0f) ? -1.0f : bwd.A[c] * A[j][c];
    }
  sh[slot][lane] = fwd;
  sg[slot][lane] = bwd;
  __syncthreads();
  Pairs<N> before, behind;
#pragma unroll
  for (int c = 0; c < N; ++c) {
    before.A[c] = behind.A[c] = 1.0f;
    before.U[c] = behind.U[c] = 0.0f;
  }
  for (int s = 0; s < slot; ++s) after<PACKED>(before, sh[s][lane]);
  for (int s = SLOTS - 1; s > slot; --s) after<PACKED>(behind, sg[s][lane]);
  // the states before the steps go into what a step's dr is of its g: f = q - m a h
  float h[N];
#pragma unroll
  for (int c = 0; c < N; ++c) h[c] = apply<PACKED>(before.A[c], before.U[c], start[c]);
#pragma unroll
  for (int j = 0; j < S; ++j)
#pragma unroll
    for (int c = 0; c < N; ++c) {
      if (PACKED && (starts >> j & 1)) h[c] = h0[j][c];
      const float xv = channel<E>(xw[j], c);
      q[j][c] = __builtin_fmaf(-ma[j][c], h[c], q[j][c]);
      h[c] = __builtin_fmaf(A[j][c], h[c], bs[j][c] * xv);
      if (PACKED && (none >> j & 1)) h[c] = q[j][c] = 0.0f;
    }

  if (chunks > 1) {
    Pairs<N> all = behind;
    unsigned long long* w = word_at<E>(k, turn, group, lane);
    bool end[N];
    const bool publishes = slot == 0 && chunk > 0;
    if (publishes) {
      after<PACKED>(all, bwd);
#pragma unroll
      for (int c = 0; c < N; ++c) {
        end[c] = turn == 0 || all.A[c] < 0.0f;
        if (turn == 0) all.U[c] = apply<PACKED>(all.A[c], all.U[c], tail[c]);
      }
      publish<E>(w, all, end);
    }
    look_back<E>(k, turn, group, slot, lane, tail, sh, in);
    if (publishes)
#pragma unroll
      for (int c = 0; c < N; ++c)
        if (!end[c]) carry_put(w + c, CARRY_INC, __float_as_uint(__builtin_fmaf(all.A[c], in[c], all.U[c])));
  } else {
#pragma unroll
    for (int c = 0; c < N; ++c) in[c] = tail[c];
  }

  Rows<E, MODE> dx, dr, di;
  dx.init_out(a.dx, (b * a.L + t0) * a.D, steps, a.D, first, c0);
  dr.init_out(a.dr, (b * a.L + t0) * a.D, steps, a.D, first, c0);
  di.init_out(a.di, (b * a.L + t0) * a.D, steps, a.D, first, c0);
  float v[N], sum[N];
#pragma unroll
  for (int c = 0; c < N; ++c) {
    v[c] = apply<PACKED>(behind.A[c], behind.U[c], in[c]);
    sum[c] = 0.0f;
  }
#pragma unroll
  for (int j = S - 1; j >= 0; --j) {
    float ox[N], oi[N], orr[N];
#pragma unroll
    for (int c = 0; c < N; ++c) {
      const bool cut = PACKED && ((ends | none) >> j & 1);
      const float g = dh[j][c] + (cut ? 0.0f : v[c]);
      const float e = g * q[j][c];
      ox[c] = g * bs[j][c];
      oi[c] = ox[c] * xi[j][c];
      orr[c] = e * rest[j][c];
      sum[c] += PACKED || first + j < steps ? e : 0.0f;
      v[c] = A[j][c] * g;
    }
    dx.put(j, ox);
    di.put(j, oi);
    dr.put(j, orr);
    if (a.dh0 && (PACKED ? starts >> j & 1 : t0 + first + j == 0)) {
      const int64_t n = PACKED ? sq.seq[first + j] : b;
#pragma unroll
      for (int c = 0; c < N; ++c)
        if (c0 + c < a.D) a.dh0[n * a.D + c0 + c] = v[c];
    }
  }
  if constexpr (PACKED) {
    if (a.dh0)  // sequences of no steps
      for (int64_t n = chunk + slot * chunks; n < a.nseq; n += chunks * SLOTS)
        if (edge(a, n) >= edge(a, n + 1))
#pragma unroll
          for (int c = 0; c < N; ++c)
            if (c0 + c < a.D) a.dh0[n * a.D + c0 + c] = a.dh_last ? a.dh_last[n * a.D + c0 + c] : 0.0f;
  }
  // lam's gradient: the slots' sums in order, then a row of the partial sums for each chunk
  __syncthreads();
  float(*fold)[GROUP<E>] = (float(*)[GROUP<E>])&sg[0][0];
#pragma unroll
  for (int c = 0; c < N; ++c) fold[slot][lane * N + c] = sum[c];
  __syncthreads();
  if (threadIdx.x < GROUP<E> && base + threadIdx.x < a.D) {
    float t = 0.0f;
    for (int s = 0; s < SLOTS; ++s) t += fold[s][threadIdx.x];
    part[(b * chunks + chunk) * a.D + base + threadIdx.x] = t * rate_slope(a.lam[base + threadIdx.x]);
  }
}

// Of no steps: dh0 = dh_last.
__global__ __launch_bounds__(256) void no_steps_kernel(float* dh0, const float* dh_last, int64_t n) {
  for (int64_t j = blockIdx.x * 256ll + threadIdx.x; j < n; j += gridDim.x * 256ll)
    dh0[j] = dh_last ? dh_last[j] : 0.0f;
}

int64_t align64(int64_t n) { return (n + 63) / 64 * 64; }

// The workspace: words (the forward's before the backward's, if states are formed again),
// partial sums, states.
struct Layout {
  int64_t chunks, words, part, states, total;
};
Layout layout_of(int64_t B, int64_t L, int64_t D, bool bf16, bool ckpt) {
  Layout l;
  l.chunks = chunks_of(L, BWD_STEPS);
  const int64_t w = words_bytes(B, D, l.chunks, bf16);
  const int64_t f = ckpt ? 0 : words_bytes(B, D, chunks_of(L, FWD_STEPS), bf16);
  l.words = align64(w > f ? w : f);
  l.part = align64(B * l.chunks * D * 4);
  l.states = ckpt ? 0 : l.part;
  l.total = l.words + l.part + l.states;
  return l;
}

}  // namespace
}  // namespace gated

using namespace gated;

int64_t gated_scan_bwd_workspace(int64_t B, int64_t L, int64_t D, bool ckpt) {
  const int64_t f = layout_of(B, L, D, false, ckpt).total, h = layout_of(B, L, D, true, ckpt).total;
  return f > h ? f : h;
}

int gated_scan_bwd(const GatedArgs& a) {
  const hipStream_t s = current_stream();
  float* outs[1] = {a.dlam};
  int st;
  if (a.B * a.L == 0) {
    const int64_t n = a.nseq * a.D;
    if (a.dh0 && n > 0) {
      hipLaunchKernelGGL(no_steps_kernel, dim3((unsigned)((n + 255) / 256 < 4096 ? (n + 255) / 256 : 4096)),
                         dim3(256), 0, s, a.dh0, a.dh_last, n);
      if ((st = check_launch("no_steps_kernel")) != SW_OK) return st;
    }
    return norm::fold_partials(nullptr, 0, a.D, outs, 1, s);
  }
  const Layout l = layout_of(a.B, a.L, a.D, a.bf16, a.ckpt_in != nullptr);
  const int64_t groups = groups_of(a.B, a.D, a.bf16);
  if (l.chunks * groups > SW_MAX_WGS / 2)
    return fail(SW_ERR_UNSUPPORTED, "%lld chunks of the recurrence exceed the launch limit",
                (long long)(l.chunks * groups));
  norm::Partials mem(s);
  if ((st = mem.get(a.ws, a.ws_bytes, (size_t)l.total, "sw_gated_scan_bwd")) != SW_OK) return st;
  char* ws = (char*)mem.p;
  float* part = (float*)(ws + l.words);
  const float* ckpt = a.ckpt_in;
  if (!ckpt) {
    GatedArgs f = a;
    f.h = nullptr;
    f.h_last = nullptr;
    f.ckpt = (float*)(ws + l.words + l.part);
    if ((st = run_fwd(f, ws, s)) != SW_OK) return st;
    ckpt = f.ckpt;
  }
  if (l.chunks > 1 &&
      (st = zero_words((uint32_t*)ws, (size_t)words_bytes(a.B, a.D, l.chunks, a.bf16) / 4, s)) != SW_OK)
    return st;
  const Words k = {(uint32_t*)ws, (unsigned long long*)(ws + 64), groups};
  const StepRows* rows[4] = {&a.x, &a.r, &a.i, &a.dh};
  const void* grads[3] = {a.dx, a.dr, a.di};
  const Mode mode = mode_of(a, rows, 4, grads, 3);
#define CALL(MODE, PACKED)                                                                          \
  do {                                                                                              \
    if (a.bf16)                                                                                     \
      hipLaunchKernelGGL((bwd_kernel<uint16_t, MODE, PACKED>), dim3((unsigned)(l.chunks * groups)), \
                         dim3(THREADS), 0, s, a, ckpt, part, k, l.chunks);                          \
    else                                                                                            \
      hipLaunchKernelGGL((bwd_kernel<float, MODE, PACKED>), dim3((unsigned)(l.chunks * groups)),    \
                         dim3(THREADS), 0, s, a, ckpt, part, k, l.chunks);                          \
  } while (0)
  SW_GATED_PICK(mode, a.cu != nullptr, CALL);
#undef CALL
  if ((st = check_launch("gated bwd_kernel")) != SW_OK) return st;
  return norm::fold_partials(part, a.B * l.chunks, a.D, outs, 1, s);
}

}  // namespace sw
