// gated_walk.h -- what the gated recurrence's walks share (device code).
//
// A workgroup of 8 waves holds a chunk of steps of one group of channels in registers: slots
// of a few steps, each some lanes of N channels.  A slot's steps are one affine pair; the
// pairs before a slot are composed from LDS, and the chunk's from what the chunks before it
// have published, so each input is read once.
//
// Between workgroups: a chunk publishes its own pair as soon as it has it (AGG), and the
// state at its end once it knows it (INC), as 64-bit words of a status and a value.  To find
// its incoming state a workgroup looks at the 16 chunks before it at once until one of them
// has its end's state.  Chunks are handed out in their order by a ticket, a chunk publishes
// AGG without waiting, and the first knows its end, so every wait ends.
#pragma once

#include "gated_math.h"
#include "gated_scan.h"
#include "selective_common.h"

namespace sw {
namespace gated {

constexpr int THREADS = 512, LOOK = 16;
template <int N_, int LANES_>
struct Shape {
  static constexpr int N = N_, LANES = LANES_, SLOTS = THREADS / LANES_, GROUP = N_ * LANES_;
};
// The forward: 32 lanes of four bytes each, a row of 128 bytes, 16 slots of 16 steps.
template <class E>
using FwdShape = Shape<4 / (int)sizeof(E), 32>;
// The backward holds more of each value, so a lane takes one channel and 8 steps of it: a
// wave is a slot.  (Two bf16 channels a lane, 16 values, took 183 us at B=8 L=2048 D=1536
// with 42 of 128 registers spilled, and 161 with 256 registers and one workgroup a compute
// unit.)
using BwdShape = Shape<1, 64>;
constexpr int FWD_S = 16, BWD_S = 8;
constexpr int FWD_STEPS = 16 * FWD_S, BWD_STEPS = BwdShape::SLOTS * BWD_S;
static_assert(BWD_STEPS == SW_GATED_CKPT && FWD_STEPS % BWD_STEPS == 0, "a state for each chunk of the backward");

// How rows are loaded: NEAR, a lane's channels a load from a buffer over the chunk's rows (out of
// range reads as zero); SPLIT, the same, a channel a load (odd widths, strides or addresses);
// FAR, by 64-bit addresses (a chunk's rows reach over 2^31 bytes).
enum Mode { NEAR, SPLIT, FAR };

template <class E, Mode MODE, int N>
struct Rows {
  static_assert(N == 1 || sizeof(E) * N == 4, "a word or an element");
  __amdgpu_buffer_rsrc_t rs;
  const char* p;
  uint32_t off;
  int64_t step;
  int left, chan;  // FAR: steps and channels from here on

  // steps first .. of `steps` in the chunk at row base p0, channels from c
  __device__ __forceinline__ void init(const void* base, int64_t p0, int64_t sl, int64_t steps, int64_t D,
                                       int first, int64_t c) {
    step = sl * (int64_t)sizeof(E);
    const char* b = (const char*)base + p0 * (int64_t)sizeof(E);
    if constexpr (MODE == FAR) {
      p = b + first * step + c * (int64_t)sizeof(E);
      left = (int)(steps - first);
      chan = (int)(D - c < N ? D - c : N);
    } else {
      rs = buffer_rsrc(b, steps > 0 ? (uint32_t)((steps - 1) * step + D * (int64_t)sizeof(E)) : 0u);
      off = (uint32_t)(first * (uint32_t)step + (uint32_t)c * sizeof(E));
    }
  }
  // step first + j as raw bits: bf16, both channels in one word
  __device__ __forceinline__ uint32_t get(int j) const {
    if constexpr (MODE == FAR) {
      uint32_t w = 0;
      if (j < left) {
        const E* q = (const E*)(p + j * step);
        if constexpr (sizeof(E) == 4) {
          if (chan > 0) w = __float_as_uint(q[0]);
        } else {
          if (chan > 0) w = q[0];
          if (N > 1 && chan > 1) w |= (uint32_t)q[1] << 16;
        }
      }
      return w;
    } else {
      const int o = (int)(off + (uint32_t)j * (uint32_t)step);
      if constexpr (sizeof(E) * N == 4 && (MODE == NEAR || N == 1)) {
        return (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(rs, o, 0, 0);
      } else if constexpr (N == 1) {
        return (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(rs, o, 0, 0);
      } else {
        const uint32_t lo = (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(rs, o, 0, 0);
        return lo | (uint32_t)(uint16_t)__builtin_amdgcn_raw_buffer_load_b16(rs, o + 2, 0, 0) << 16;
      }
    }
  }
  // the lane's channels of an output's step; those past D go nowhere
  __device__ __forceinline__ void put(int j, const float* v) const {
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
    } else {
      const int o = (int)(off + (uint32_t)j * (uint32_t)step);
      if constexpr (sizeof(E) == 4) {
        __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(v[0]), rs, o, 0, 0);
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
  }
  // an output: lanes whose channels are past D store outside the buffer
  __device__ __forceinline__ void init_out(void* base, int64_t p0, int64_t steps, int64_t D, int first,
                                           int64_t c) {
    init(base, p0, D, steps, D, first, c);
    chan = (int)(D - c < N ? D - c : N);
    if constexpr (MODE != FAR) {
      if (chan <= 0) off = 0x80000000u;
    }
  }
};

template <class E>
__device__ __forceinline__ float channel(uint32_t w, int c) {
  if constexpr (sizeof(E) == 4) {
    return __uint_as_float(w);
  } else {
    return c ? bf16_hi(w) : bf16_lo(w);
  }
}

// An affine pair: v -> A v + U, or, with A below zero, the constant U (a sequence begins
// inside: what came before does not reach its end, were it infinite).
template <int N>
struct Pairs {
  float A[N], U[N];
};
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

// Where the words between workgroups lie: one for each channel of a group's chunk, values,
// then factors.
struct Words {
  uint32_t* ticket;
  unsigned long long* w;
  int64_t groups;
};
template <class G>
__device__ __forceinline__ unsigned long long* word_at(const Words& k, int64_t chunk, int64_t group,
                                                       int lane) {
  return k.w + (chunk * k.groups + group) * (2 * G::GROUP) + lane * G::N;
}
template <class G>
__device__ __forceinline__ void publish(unsigned long long* w, const Pairs<G::N>& p, const bool* end) {
#pragma unroll
  for (int c = 0; c < G::N; ++c) {
    if (!end[c]) carry_put(w + G::GROUP + c, CARRY_AGG, __float_as_uint(p.A[c]));
    carry_put(w + c, end[c] ? CARRY_INC : CARRY_AGG, __float_as_uint(p.U[c]));
  }
}

// The value that reaches `chunk` from those before it (chunk - 1, chunk - 2 .. in the walk's
// order; before the first, `first`): the latest known end, taken through the pairs behind it
// one after the other, exactly as those chunks take it through their own.  So its bits do
// not depend on which ends were known.  All of the workgroup take part.
template <class G>
__device__ __forceinline__ void look_back(const Words& k, int64_t chunk, int64_t group, int slot, int lane,
                                          const float* first, Pairs<G::N> (*sh)[G::LANES], float* value) {
  constexpr int N = G::N, EACH = LOOK / G::SLOTS;  // chunks a slot looks at
  bool open;
  do {
    Pairs<N> p[EACH];  // A < 0: U is the end's value
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
      const int64_t mine = chunk - 1 - (e * G::SLOTS + slot);
      const unsigned long long* w = word_at<G>(k, mine < 0 ? 0 : mine, group, lane);
#pragma unroll
      for (int c = 0; c < N; ++c) {
        p[e].A[c] = -1.0f;
        p[e].U[c] = first[c];
        if (mine >= 0) {
          unsigned long long v;
          while ((v = carry_get(w + c)) >> 32 == CARRY_EMPTY) __builtin_amdgcn_s_sleep(1);
          p[e].U[c] = __uint_as_float((uint32_t)v);
          if (v >> 32 == CARRY_AGG) {
            while ((v = carry_get(w + G::GROUP + c)) >> 32 == CARRY_EMPTY) __builtin_amdgcn_s_sleep(1);
            p[e].A[c] = __uint_as_float((uint32_t)v);
          }
        }
      }
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < EACH; ++e) sh[e * G::SLOTS + slot][lane] = p[e];
    __syncthreads();
    open = false;
#pragma unroll
    for (int c = 0; c < N; ++c) {
      int s = 0;
      while (s < LOOK - 1 && !(sh[s][lane].A[c] < 0.0f)) ++s;
      open |= !(sh[s][lane].A[c] < 0.0f);
      value[c] = sh[s][lane].U[c];
      while (--s >= 0) value[c] = __builtin_fmaf(sh[s][lane].A[c], value[c], sh[s][lane].U[c]);
    }
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
inline int64_t groups_of(int64_t B, int64_t D, int group) { return B * ((D + group - 1) / group); }
// Bytes of the words of a walk, its ticket before them.
inline int64_t words_bytes(int64_t chunks, int64_t groups, int group) {
  return chunks > 1 ? 64 + chunks * groups * group * 16 : 0;
}
// Whether the rows of a chunk reach over less than 2^31 bytes.
inline bool near_rows(const GatedArgs& a, const StepRows* const* rows, int n, int steps) {
  const int64_t es = a.bf16 ? 2 : 4, most = (int64_t)1 << 31;
  bool near = (steps + 1) * a.D * es < most;
  for (int j = 0; j < n; ++j)
    near = near && rows[j]->sl < most && steps * rows[j]->sl * es + a.D * es < most;
  return near;
}

int run_fwd(const GatedArgs& a, void* words, hipStream_t s);
int64_t fwd_words(const GatedArgs& a);

}  // namespace gated
}  // namespace sw
