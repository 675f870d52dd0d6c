// gated_bwd.hip -- the gated linear recurrence: backward.
//
// The states before the backward's chunks of 64 steps are what a training forward kept, so
// a chunk's own are formed from its registers alone.  The gradient's recurrence runs the
// other way, over v_t = a_t g_t, what step t hands to the one before it:
//   v_t = a_t (dh_t + v_{t+1}),
// an affine pair again, composed in slots and between workgroups from the last chunk on.
//
// Seven values are moved for each, against some 84 vector instructions: B=8 L=2048 D=1536
// bf16 107 us, 353 MB at 3.3 TB/s with vector issue in 62% of the busy cycles; fp32, packed,
// 11003 x 2048 144 us, 631 MB at 4.4 TB/s.  A lane's 8 values of one channel take 126
// registers.  Tried at the first shape, with the same waits: two channels and 4 steps a lane
// 117 us for 114 in all, two and 8 steps with values aside in LDS 127 (15 registers spilled),
// six waves a SIMD on 80 registers 118 (7 spilled; fp32 155 for 151).
#include "gated_walk.h"

namespace sw {
namespace gated {
namespace {

template <class E, Mode MODE, bool PACKED>
__global__ __launch_bounds__(THREADS, 4) void bwd_kernel(GatedArgs a, const float* ckpt, float* part,
                                                         Words k, int64_t chunks) {
  using G = BwdShape;
  constexpr int S = BWD_S, SLOTS = G::SLOTS;
  __shared__ Pairs<1> sh[LOOK][G::LANES], sg[SLOTS][G::LANES];
  __shared__ Sequences<PACKED ? BWD_STEPS : 1> sq;
  __shared__ float rates[G::GROUP];
  __shared__ uint32_t ticket;
  const int slot = __builtin_amdgcn_readfirstlane((int)threadIdx.x / G::LANES);
  const int lane = threadIdx.x % G::LANES;
  uint32_t work = blockIdx.x;
  if (chunks > 1) {
    if (threadIdx.x == 0) ticket = atomicAdd(k.ticket, 1u);
    __syncthreads();
    work = (uint32_t)__builtin_amdgcn_readfirstlane((int)ticket) - k.base;
  }
  // `turn` counts the chunks from the last one on
  const uint32_t turn = work / k.groups, group = work % k.groups;
  const int64_t chunk = chunks - 1 - turn;
  const int64_t b = group / k.per, base = (int64_t)(group % k.per) * G::GROUP, c0 = base + lane;
  const int64_t t0 = chunk * BWD_STEPS, left = a.L - t0;
  const int steps = (int)(left < BWD_STEPS ? left : BWD_STEPS), first = slot * S;
  const bool there = c0 < a.D;
  if constexpr (PACKED) find_sequences(a, t0, sq);

  Rows<E, MODE, 1> x, r, i, d;
  x.init(a.x.p, b * a.x.sb + t0 * a.x.sl, a.x.sl, steps, a.D, first, c0);
  r.init(a.r.p, b * a.r.sb + t0 * a.r.sl, a.r.sl, steps, a.D, first, c0);
  i.init(a.i.p, b * a.i.sb + t0 * a.i.sl, a.i.sl, steps, a.D, first, c0);
  d.init(a.dh.p, b * a.dh.sb + t0 * a.dh.sl, a.dh.sl, steps, a.D, first, c0);
  const float lam = there ? a.lam[c0] : 0.0f;
  const float start = there ? ckpt[(b * chunks + chunk) * a.D + c0] : 0.0f;
  const float tail = !PACKED && a.dh_last && there ? a.dh_last[b * a.D + c0] : 0.0f;
  Raw<E, 1> xw[S], rw[S], iw[S], dw[S];
#pragma unroll
  for (int j = 0; j < S; ++j) {
    xw[j] = x.get(j);
    rw[j] = r.get(j);
    iw[j] = i.get(j);
    dw[j] = d.get(j);
  }
  if (slot == 0) rates[lane] = there ? rate_of(lam, a.c) : 0.0f;
  __syncthreads();
  const float rate = rates[lane];

  // of each step: a, b s, (m / b) a^2 s x, m a, 1 - sigmoid(r), (1 - s) x, u, dh
  float A[S], bs[S], q[S], ma[S], rest[S], xi[S], u[S], dh[S];
  uint32_t none = 0, starts = 0, ends = 0;  // PACKED: steps of no sequence, first and last ones
  Pairs<1> fwd = identity<1>(), bwd = fwd;
#pragma unroll
  for (int j = 0; j < S; ++j) {
    const float xv = xw[j].get(0);
    const Step s = step_of<E>(xv, rw[j].get(0), iw[j].get(0), rate);
    A[j] = s.a;
    bs[j] = s.bs;
    q[j] = s.q;
    ma[j] = s.ma;
    rest[j] = s.rest_r;
    xi[j] = xv * s.rest_i;
    u[j] = s.bs * xv;
    dh[j] = dw[j].get(0);
    float f = s.a;
    if constexpr (PACKED) {
      const int n = __builtin_amdgcn_readfirstlane(sq.seq[first + j]);
      if (n < 0) {
        none |= 1u << j;
        f = -1.0f;
        A[j] = bs[j] = q[j] = ma[j] = rest[j] = xi[j] = u[j] = dh[j] = 0.0f;
      } else {
        const int at = __builtin_amdgcn_readfirstlane((int)sq.ends[first + j]);
        if (at & 1) {
          starts |= 1u << j;
          // the state before is known: what it adds is a constant
          u[j] = __builtin_fmaf(f, a.h0 && there ? a.h0[n * a.D + c0] : 0.0f, u[j]);
          f = -1.0f;
        }
        if (at & 2) {
          ends |= 1u << j;
          if (a.dh_last && there) dh[j] += a.dh_last[n * a.D + c0];
        }
      }
    } else if (first + j >= steps) {
      // past the row's end (rows of stride 0 are read there again) nothing is added, and
      // what comes in passes through
      f = A[j] = 1.0f;
      dh[j] = 0.0f;
    }
    fwd.U[0] = apply<PACKED>(f, u[j], fwd.U[0]);
    fwd.A[0] = PACKED && (f < 0.0f || fwd.A[0] < 0.0f) ? -1.0f : fwd.A[0] * f;
  }
#pragma unroll
  for (int j = S - 1; j >= 0; --j) {
    const bool cut = PACKED && ((ends | none) >> j & 1);
    bwd.U[0] = A[j] * (dh[j] + (cut ? 0.0f : bwd.U[0]));
    bwd.A[0] = cut || (PACKED && bwd.A[0] < 0.0f) ? -1.0f : bwd.A[0] * A[j];
  }
  sh[slot][lane] = fwd;
  sg[slot][lane] = bwd;
  __syncthreads();
  const Pairs<1> before = first_of<PACKED, false, 4>(sh, slot, lane);
  const Pairs<1> behind = first_of<PACKED, true, 4>(sg, SLOTS - 1 - slot, lane);

  float in = tail;
  Pairs<1> all = behind;
  unsigned long long* w = word_at<G>(k, turn, group, lane);
  bool end = true;
  const bool publishes = slot == 0 && chunk > 0;
  if (publishes) {
    after<PACKED>(all, bwd);
    end = turn == 0 || all.A[0] < 0.0f;
    if (turn == 0) all.U[0] = apply<PACKED>(all.A[0], all.U[0], tail);
    publish<G>(w, k.epoch, all, &end);
  }
  // the states before the steps go into what a step's dr is of its g: q - m a h
  float h = apply<PACKED>(before.A[0], before.U[0], start);
#pragma unroll
  for (int j = 0; j < S; ++j) {
    if (PACKED && (starts >> j & 1)) {
      h = a.h0 && there ? a.h0[sq.seq[first + j] * a.D + c0] : 0.0f;
      q[j] = __builtin_fmaf(-ma[j], h, q[j]);
      h = u[j];
    } else if (PACKED && (none >> j & 1)) {
      h = q[j] = 0.0f;
    } else {
      q[j] = __builtin_fmaf(-ma[j], h, q[j]);
      h = __builtin_fmaf(A[j], h, u[j]);
      if (!PACKED && first + j >= steps) q[j] = 0.0f;
    }
  }
  if (chunks > 1) {
    look_back<G>(k, turn, group, slot, lane, &tail, sh, &in);
    if (publishes && !end)
      carry_put(w, carry_status(k.epoch, CARRY_INC),
                __float_as_uint(__builtin_fmaf(all.A[0], in, all.U[0])));
  }

  Rows<E, MODE, 1> dx, dr, di;
  dx.init_out(a.dx, (b * a.L + t0) * a.D, steps, a.D, first, c0);
  dr.init_out(a.dr, (b * a.L + t0) * a.D, steps, a.D, first, c0);
  di.init_out(a.di, (b * a.L + t0) * a.D, steps, a.D, first, c0);
  float v = apply<PACKED>(behind.A[0], behind.U[0], in), sum = 0.0f;
#pragma unroll
  for (int j = S - 1; j >= 0; --j) {
    const bool cut = PACKED && ((ends | none) >> j & 1);
    const float g = dh[j] + (cut ? 0.0f : v);
    const float e = g * q[j], gx = g * bs[j], gi = gx * xi[j], gr = e * rest[j];
    sum += e;
    v = A[j] * g;
    dx.put(j, &gx);
    di.put(j, &gi);
    dr.put(j, &gr);
    if (a.dh0 && there && (PACKED ? starts >> j & 1 : t0 + first + j == 0))
      a.dh0[(PACKED ? sq.seq[first + j] : b) * a.D + c0] = v;
  }
  if constexpr (PACKED) {
    if (a.dh0 && there)  // sequences of no steps
      for (int64_t n = chunk + slot * chunks; n < a.nseq; n += chunks * SLOTS)
        if (edge(a, n) >= edge(a, n + 1)) a.dh0[n * a.D + c0] = a.dh_last ? a.dh_last[n * a.D + c0] : 0.0f;
  }
  // lam's gradient: the slots' sums in order, then a row of the partial sums for each chunk
  __syncthreads();
  float(*fold)[G::GROUP] = (float(*)[G::GROUP])&sg[0][0];
  fold[slot][lane] = sum;
  __syncthreads();
  if (slot == 0 && there) {
    float t = 0.0f;
#pragma unroll
    for (int s = 0; s < SLOTS; ++s) t += fold[s][lane];
    part[(b * chunks + chunk) * a.D + c0] = t * rate_slope(lam);
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
  int group;
  int64_t chunks, groups, words, part, states, total;
};
Layout layout_of(const GatedArgs& a, bool ckpt) {
  Layout l;
  l.chunks = chunks_of(a.L, BWD_STEPS);
  l.group = BwdShape::GROUP;
  l.groups = groups_of(a, l.group);
  const int64_t w = words_bytes(l.chunks, l.groups, l.group), f = ckpt ? 0 : fwd_words(a);
  l.words = align64(w > f ? w : f);
  l.part = align64(a.B * l.chunks * a.D * 4);
  l.states = ckpt ? 0 : l.part;
  l.total = l.words + l.part + l.states;
  return l;
}

}  // namespace
}  // namespace gated

using namespace gated;

int64_t gated_scan_bwd_workspace(int64_t B, int64_t L, int64_t D, bool ckpt) {
  GatedArgs a;
  a.B = B;
  a.L = L;
  a.D = D;
  return layout_of(a, ckpt).total;
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
  const Layout l = layout_of(a, a.ckpt_in != nullptr);
  const int64_t wgs = l.chunks * l.groups;
  if (wgs > SW_MAX_WGS / 2)
    return fail(SW_ERR_UNSUPPORTED, "%lld chunks of the recurrence exceed the launch limit", (long long)wgs);
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
    if ((st = run_fwd(f, ws, (size_t)l.words, s)) != SW_OK) return st;
    ckpt = f.ckpt;
  }
  LaunchWords words(s);
  if ((st = words.get(ws, (size_t)l.words, l.chunks, l.groups, l.group, a.B, s, "sw_gated_scan_bwd")) != SW_OK)
    return st;
  const Words& k = words.k;
  const bool near = mode_of(a, BWD_STEPS, 1, {&a.x, &a.r, &a.i, &a.dh}, {}) == NEAR;
#define CALL(E, MODE)                                                                                   \
  do {                                                                                                  \
    if (a.cu)                                                                                           \
      hipLaunchKernelGGL((bwd_kernel<E, MODE, true>), dim3((unsigned)wgs), dim3(THREADS), 0, s, a, ckpt, \
                         part, k, l.chunks);                                                            \
    else                                                                                                \
      hipLaunchKernelGGL((bwd_kernel<E, MODE, false>), dim3((unsigned)wgs), dim3(THREADS), 0, s, a, ckpt, \
                         part, k, l.chunks);                                                            \
  } while (0)
  if (a.bf16) {
    if (near)
      CALL(uint16_t, NEAR);
    else
      CALL(uint16_t, FAR);
  } else if (near) {
    CALL(float, NEAR);
  } else {
    CALL(float, FAR);
  }
#undef CALL
  if ((st = words.done(check_launch("gated bwd_kernel"))) != SW_OK) return st;
  return norm::fold_partials(part, a.B * l.chunks, a.D, outs, 1, s);
}

}  // namespace sw
