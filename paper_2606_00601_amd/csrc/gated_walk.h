// gated_walk.h -- what the gated recurrence's walks share (device code).
//
// A workgroup of 8 waves holds a chunk of steps of one group of channels in registers: slots
// of a few steps, each some lanes of one or two channels.  A slot's steps are one affine pair;
// the pairs before a slot are composed in LDS, and the chunk's from what the chunks before it
// have published, so each input is read once.
//
// Between workgroups: a chunk publishes its own pair as soon as it has it (AGG), and the
// state at its end once it knows it (INC), as 64-bit words of a status and a value.  To find
// its incoming state a workgroup looks at the 4 to 16 chunks before it at once until one of
// them has its end's state.  Chunks are handed out in their order by a ticket, a chunk publishes
// AGG without waiting, and the first knows its end, so every wait ends.
#pragma once

#include <initializer_list>

#include "gated_math.h"
#include "gated_scan.h"
#include "norm_rows.h"
#include "selective_common.h"

namespace sw {
namespace gated {

constexpr int THREADS = 512, WAVES = THREADS / 64, LOOK = 16;
template <int N_, int LANES_>
struct Shape {
  static constexpr int N = N_, LANES = LANES_, SLOTS = THREADS / LANES_, GROUP = N_ * LANES_;
};
// The forward keeps two values of a step: half a wave is a slot, and chunks are long, which
// makes few of them (16 steps a lane; 8 for short rows).
using FwdShape = Shape<2, 32>;
constexpr int FWD_S = 16, FWD_SHORT_S = 8;
// The backward keeps more of each value, so a lane takes one channel; a wave is a slot, and
// what depends on the step alone is scalar.
using BwdShape = Shape<1, 64>;
constexpr int BWD_S = 8, BWD_STEPS = THREADS / 64 * BWD_S;
static_assert(BWD_STEPS == SW_GATED_CKPT && FwdShape::SLOTS * FWD_SHORT_S % BWD_STEPS == 0,
              "a state for each chunk of the backward");

// How rows are loaded: NEAR, a lane's two channels a load from a buffer over the chunk's
// rows (out of range reads as zero); SPLIT, the same, a channel a load (odd widths, strides or
// addresses); FAR, by 64-bit addresses (a chunk's rows reach over 2^31 bytes).
enum Mode { NEAR, SPLIT, FAR };

// A lane's channels of a step as loaded.
template <class E, int N>
struct Raw {
  uint32_t w[(sizeof(E) * N + 3) / 4];
  __device__ __forceinline__ float get(int c) const {
    if constexpr (sizeof(E) == 4)
      return __uint_as_float(w[c]);
    else
      return c ? bf16_hi(w[0]) : bf16_lo(w[0]);
  }
};

template <class E, Mode MODE, int N>
struct Rows {
  __amdgpu_buffer_rsrc_t rs;
  const char* p;
  uint32_t off;
  int64_t step;
  int left, chan;  // steps (FAR) and channels from here on

  // steps first .. of `steps` in the chunk whose first row begins at element p0, channels from c
  __device__ __forceinline__ void init(const void* base, int64_t p0, int64_t sl, int steps, int64_t D,
                                       int first, int64_t c) {
    step = sl * (int64_t)sizeof(E);
    chan = (int)(D - c < N ? D - c : N);
    const char* b = (const char*)base + p0 * (int64_t)sizeof(E);
    if constexpr (MODE == FAR) {
      p = b + first * step + c * (int64_t)sizeof(E);
      left = steps - first;
    } else {
      rs = buffer_rsrc(b, steps > 0 ? (uint32_t)((steps - 1) * step + D * (int64_t)sizeof(E)) : 0u);
      off = (uint32_t)first * (uint32_t)step + (uint32_t)c * (uint32_t)sizeof(E);
    }
  }
  // an output: lanes whose channels are past D store outside the buffer
  __device__ __forceinline__ void init_out(void* base, int64_t p0, int steps, int64_t D, int first,
                                           int64_t c) {
    init(base, p0, D, steps, D, first, c);
    if constexpr (MODE != FAR) {
      if (chan <= 0) off = 0x80000000u;
    }
  }
  __device__ __forceinline__ Raw<E, N> get(int j) const {
    Raw<E, N> r = {};
    const int o = (int)(off + (uint32_t)j * (uint32_t)step);
    if constexpr (MODE == FAR) {
      if (j < left) {
        const E* q = (const E*)(p + j * step);
        if constexpr (sizeof(E) == 4) {
#pragma unroll
          for (int c = 0; c < N; ++c)
            if (c < chan) r.w[c] = __float_as_uint(q[c]);
        } else {
          if (chan > 0) r.w[0] = q[0];
          if (N > 1 && chan > 1) r.w[0] |= (uint32_t)q[1] << 16;
        }
      }
    } else if constexpr (sizeof(E) == 4) {
      if constexpr (N == 1) {
        r.w[0] = (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(rs, o, 0, 0);
      } else if constexpr (MODE == NEAR) {
        const uint2 v = __builtin_bit_cast(uint2, __builtin_amdgcn_raw_buffer_load_b64(rs, o, 0, 0));
        r.w[0] = v.x;
        r.w[1] = v.y;
      } else {
        r.w[0] = (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(rs, o, 0, 0);
        r.w[1] = (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(rs, o + 4, 0, 0);
      }
    } else if constexpr (N == 1) {
      r.w[0] = (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(rs, o, 0, 0);
    } else if constexpr (MODE == NEAR) {
      r.w[0] = (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(rs, o, 0, 0);
    } else {
      const uint32_t lo = (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(rs, o, 0, 0);
      r.w[0] = lo | (uint32_t)(uint16_t)__builtin_amdgcn_raw_buffer_load_b16(rs, o + 2, 0, 0) << 16;
    }
    return r;
  }
  __device__ __forceinline__ void put(int j, const float* v) const {
    const int o = (int)(off + (uint32_t)j * (uint32_t)step);
    if constexpr (MODE == FAR) {
      if (j < left) {
        E* q = (E*)(p + j * step);
#pragma unroll
        for (int c = 0; c < N; ++c)
          if (c < chan) {
            if constexpr (sizeof(E) == 4)
              q[c] = v[c];
            else
              q[c] = (uint16_t)bf16_rne(v[c]);
          }
      }
    } else if constexpr (sizeof(E) == 4) {
      if constexpr (N == 1) {
        __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(v[0]), rs, o, 0, 0);
      } else if constexpr (MODE == NEAR) {
        const sw_u32x2 w = {__float_as_uint(v[0]), __float_as_uint(v[1])};
        __builtin_amdgcn_raw_buffer_store_b64(w, rs, o, 0, 0);
      } else {
        __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(v[0]), rs, o, 0, 0);
        if (chan > 1) __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(v[1]), rs, o + 4, 0, 0);
      }
    } else if constexpr (N == 1) {
      __builtin_amdgcn_raw_buffer_store_b16((uint16_t)bf16_rne(v[0]), rs, o, 0, 0);
    } else {
      const uint32_t w = bf16x2_rne(v[0], v[1]);
      if constexpr (MODE == NEAR) {
        __builtin_amdgcn_raw_buffer_store_b32(w, rs, o, 0, 0);
      } else {
        __builtin_amdgcn_raw_buffer_store_b16((uint16_t)w, rs, o, 0, 0);
        if (chan > 1) __builtin_amdgcn_raw_buffer_store_b16((uint16_t)(w >> 16), rs, o + 2, 0, 0);
      }
    }
  }
};

// An affine pair: v -> A v + U, or, with A below zero, the constant U (a sequence begins
// inside: what came before does not reach its end, were it infinite).
template <int N>
struct Pairs {
  float A[N], U[N];
};
template <int N>
__device__ __forceinline__ Pairs<N> identity() {
  Pairs<N> p;
#pragma unroll
  for (int c = 0; c < N; ++c) {
    p.A[c] = 1.0f;
    p.U[c] = 0.0f;
  }
  return p;
}
template <bool PACKED, int N>
__device__ __forceinline__ void after(Pairs<N>& p, const Pairs<N>& later) {
#pragma unroll
  for (int c = 0; c < N; ++c) {
    const float u = __builtin_fmaf(later.A[c], p.U[c], later.U[c]);
    const float a = later.A[c] * p.A[c];
    if constexpr (PACKED) {
      p.U[c] = later.A[c] < 0.0f ? later.U[c] : u;
      p.A[c] = later.A[c] < 0.0f || p.A[c] < 0.0f ? -1.0f : a;
    } else {
      p.U[c] = u;
      p.A[c] = a;
    }
  }
}
template <bool PACKED>
__device__ __forceinline__ float apply(float A, float U, float v) {
  const float r = __builtin_fmaf(A, v, U);
  return PACKED && A < 0.0f ? U : r;
}

// The composition of the first n of 8 pairs in LDS, from the last one back if TURNED.
template <bool PACKED, bool TURNED, int DEPTH, int N, int LANES>
__device__ __forceinline__ Pairs<N> first_of(const Pairs<N> (*sh)[LANES], int n, int lane) {
  Pairs<N> p = identity<N>();
#pragma unroll
  for (int w0 = 0; w0 < 8; w0 += DEPTH) {  // DEPTH in flight at a time
    Pairs<N> q[DEPTH];
#pragma unroll
    for (int e = 0; e < DEPTH; ++e) q[e] = sh[TURNED ? 7 - (w0 + e) : w0 + e][lane];
#pragma unroll
    for (int e = 0; e < DEPTH; ++e)
      if (w0 + e < n) after<PACKED>(p, q[e]);
  }
  return p;
}

// Where the words between workgroups lie: one for each channel of a group's chunk, values,
// then factors.
struct Words {
  uint32_t* ticket;
  unsigned long long* w;
  uint32_t groups, per;  // groups of channels in all, and of one row of the batch
  int look;              // chunks a workgroup looks back over at once
  uint32_t base, epoch;  // the ticket this launch starts from, and the tag of its words
};
template <class G>
__device__ __forceinline__ unsigned long long* word_at(const Words& k, int64_t chunk, uint32_t group,
                                                       int lane) {
  return k.w + (chunk * (int64_t)k.groups + group) * (2 * G::GROUP) + lane * G::N;
}
template <class G>
__device__ __forceinline__ void publish(unsigned long long* w, uint32_t epoch, const Pairs<G::N>& p,
                                        const bool* end) {
#pragma unroll
  for (int c = 0; c < G::N; ++c) {
    if (!end[c]) carry_put(w + G::GROUP + c, carry_status(epoch, CARRY_AGG), __float_as_uint(p.A[c]));
    carry_put(w + c, carry_status(epoch, end[c] ? CARRY_INC : CARRY_AGG), __float_as_uint(p.U[c]));
  }
}

// The value that reaches `chunk` from those before it (chunk - 1, chunk - 2 .. in the walk's
// order; before the first, `first`): the latest known end, taken through the pairs behind it
// one after the other, exactly as those chunks take it through their own.  So its bits do
// not depend on which ends were known.  All of the workgroup take part.
template <class G>
__device__ __forceinline__ void look_back(const Words& k, int64_t chunk, uint32_t group, int slot, int lane,
                                          const float* first, Pairs<G::N> (*sh)[G::LANES], float* value) {
  constexpr int N = G::N;
  const uint32_t agg = carry_status(k.epoch, CARRY_AGG), inc = carry_status(k.epoch, CARRY_INC);
  bool open;
  do {
    __syncthreads();
    for (int at = slot; at < k.look; at += G::SLOTS) {
      const int64_t mine = chunk - 1 - at;
      Pairs<N> p;  // A < 0: U is the end's value
#pragma unroll
      for (int c = 0; c < N; ++c) {
        p.A[c] = -1.0f;
        p.U[c] = first[c];
      }
      if (mine >= 0) {
        // all words at once: one after the other each would wait for the one before
        const unsigned long long* w = word_at<G>(k, mine, group, lane);
        unsigned long long u[N], f[N];
        bool there;
        do {
#pragma unroll
          for (int c = 0; c < N; ++c) {
            u[c] = carry_get(w + c);
            f[c] = carry_get(w + G::GROUP + c);
          }
          there = true;
#pragma unroll
          for (int c = 0; c < N; ++c)
            there = there && (u[c] >> 32 == inc || (u[c] >> 32 == agg && f[c] >> 32 == agg));
          if (!there) __builtin_amdgcn_s_sleep(1);
        } while (!there);
#pragma unroll
        for (int c = 0; c < N; ++c) {
          p.U[c] = __uint_as_float((uint32_t)u[c]);
          if (u[c] >> 32 == agg) p.A[c] = __uint_as_float((uint32_t)f[c]);
        }
      }
      sh[at][lane] = p;
    }
    __syncthreads();
    // from the farthest on: an end found on the way replaces what was made up before it
    bool known[N];
#pragma unroll
    for (int c = 0; c < N; ++c) {
      value[c] = 0.0f;
      known[c] = false;
    }
    for (int s = k.look - 4; s >= 0; s -= 4) {
      Pairs<N> q[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) q[e] = sh[s + e][lane];
#pragma unroll
      for (int e = 3; e >= 0; --e)
#pragma unroll
        for (int c = 0; c < N; ++c) {
          const bool is = q[e].A[c] < 0.0f;
          value[c] = is ? q[e].U[c] : __builtin_fmaf(q[e].A[c], value[c], q[e].U[c]);
          known[c] = known[c] || is;
        }
    }
    open = false;
#pragma unroll
    for (int c = 0; c < N; ++c) open = open || !known[c];
  } while (__any(open));  // a wave's lanes hold all of the group's channels: all waves agree
}

// The sequence a packed row's step belongs to (-1: none) and whether it is its first or
// last, for the steps of a chunk.
template <int STEPS>
struct Sequences {
  int seq[STEPS];
  uint8_t ends[STEPS];  // bit 0: first, bit 1: last
  __device__ __forceinline__ bool first(int j) const { return ends[j] & 1; }
  __device__ __forceinline__ bool last(int j) const { return ends[j] >> 1; }
};
__device__ __forceinline__ int64_t edge(const GatedArgs& a, int64_t n) {
  const int64_t e = a.cu[n];
  return e < 0 ? 0 : e > a.L ? a.L : e;
}
template <int STEPS>
__device__ __forceinline__ void find_sequences(const GatedArgs& a, int64_t t0, Sequences<STEPS>& sh) {
  for (int j = threadIdx.x; j < STEPS; j += THREADS) {
    const int64_t t = t0 + j;
    int64_t lo = 0, hi = a.nseq;  // the last edge at or before t is in [lo, hi]
    while (lo < hi) {
      const int64_t mid = (lo + hi + 1) / 2;
      if (edge(a, mid) <= t)
        lo = mid;
      else
        hi = mid - 1;
    }
    const int64_t e0 = edge(a, lo), e1 = lo < a.nseq ? edge(a, lo + 1) : 0;
    const bool in = t < a.L && lo < a.nseq && e0 <= t && t < e1;
    sh.seq[j] = in ? (int)lo : -1;
    sh.ends[j] = (uint8_t)((in && t == e0) | (in && t + 1 == e1) << 1);
  }
  __syncthreads();
}

inline int64_t chunks_of(int64_t L, int steps) { return L > steps ? (L + steps - 1) / steps : 1; }
inline int64_t groups_of(const GatedArgs& a, int group) { return a.B * ((a.D + group - 1) / group); }
// Few groups have many chunks under way at once, so they look further back: 4 chunks, or up
// to 16 where that leaves fewer than 128 for all groups.  (bf16 at 4, 8, 16 chunks: B=1 L=65536
// D=256 forward 95, 67, 56 us, backward 235, 148, 105; D=1024 134, 131, 134 and 322, 286, 307;
// D=5120 forward 551, 563, 587; B=8 L=2048 D=1536 52, 53, 54 and 107, 106, 112.)
constexpr int64_t LOOK_ALL = 128;

// Bytes of the words of a walk, its ticket before them.
inline int64_t words_bytes(int64_t chunks, int64_t groups, int group) {
  return chunks > 1 ? 64 + chunks * groups * group * 16 : 0;
}

// The words of a launch of chunks x groups workgroups, held until it is enqueued: of the
// stream's scratch, whose words of earlier launches carry other epochs, or of a workspace that
// is cleared first (a launch and a wait, 4 us) where the stream is capturing or the words
// pass SCRATCH_MOST bytes, which the scratch would keep.
constexpr int64_t SCRATCH_MOST = (int64_t)16 << 20;
struct LaunchWords {
  Words k = {};
  ScratchSession scratch;
  norm::Partials own;
  bool shared = false;
  explicit LaunchWords(hipStream_t s) : own(s) {}
  int get(void* ws, size_t have, int64_t chunks, int64_t groups, int group, int64_t B, hipStream_t s,
          const char* what) {
    k.groups = (uint32_t)groups;
    k.per = (uint32_t)(groups / B);
    k.look = 4;
    while (k.look < LOOK && k.look * groups < LOOK_ALL) k.look *= 2;
    if (chunks <= 1) return SW_OK;
    const int64_t bytes = words_bytes(chunks, groups, group);
    int st;
    hipStreamCaptureStatus cs = hipStreamCaptureStatusNone;
    if (bytes <= SCRATCH_MOST && hipStreamIsCapturing(s, &cs) == hipSuccess &&
        cs == hipStreamCaptureStatusNone) {
      if ((st = scratch.reserve((size_t)(bytes - 64) / 8, (uint32_t)(chunks * groups), s)) != SW_OK) return st;
      shared = true;
      k.ticket = scratch.ticket;
      k.w = scratch.carry;
      k.base = scratch.ticket_base;
      k.epoch = scratch.epoch;
      return SW_OK;
    }
    if ((st = own.get(ws, have, (size_t)bytes, what)) != SW_OK) return st;
    k.ticket = (uint32_t*)own.p;
    k.w = (unsigned long long*)((char*)own.p + 64);
    k.epoch = 1;
    return zero_words(k.ticket, (size_t)bytes / 4, s);
  }
  // after the launch
  int done(int st) {
    if (st != SW_OK && shared) scratch.invalidate();
    return st;
  }
};

// The mode of a walk of `steps` a chunk, `n` channels a lane, over these rows and dense results.
inline Mode mode_of(const GatedArgs& a, int steps, int n, std::initializer_list<const StepRows*> rows,
                    std::initializer_list<const void*> outs) {
  const int64_t es = a.bf16 ? 2 : 4, most = (int64_t)1 << 31;
  bool near = (steps + 1) * a.D * es < most, pairs = n == 1 || a.D % 2 == 0;
  for (const StepRows* x : rows) {
    near = near && x->sl < most && steps * x->sl * es + a.D * es < most;
    // bf16 pairs are words
    if (a.bf16 && n > 1) pairs = pairs && (uintptr_t)x->p % 4 == 0 && x->sl % 2 == 0 && x->sb % 2 == 0;
  }
  for (const void* p : outs)
    if (a.bf16 && n > 1) pairs = pairs && (uintptr_t)p % 4 == 0;
  return !near ? FAR : pairs ? NEAR : SPLIT;
}

int64_t fwd_words(const GatedArgs& a);
int run_fwd(const GatedArgs& a, void* ws, size_t ws_bytes, hipStream_t s);

}  // namespace gated
}  // namespace sw
