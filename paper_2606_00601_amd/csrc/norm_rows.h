// norm_rows.h -- what the norm kernels share (device code).
//
// A norm reads a row once, keeps it in registers, sums over the lanes that
// hold it, and writes what follows from the sums: bound by memory, every
// tensor read or written once.  LPR lanes share one row (of one group), NV
// vectors of 8 columns each; the smallest that holds the row is taken, so that
// short groups fill waves with several rows.  A workgroup keeps one group's
// columns while it steps through the rows, so the weights stay in registers
// and the parameters' gradients accumulate there, in fp32.
#pragma once

#include "block_norm.h"

namespace sw {
namespace norm {

typedef float f4 __attribute__((ext_vector_type(4)));

// Eight columns from p, `left` of them in the row; vec: whole 16-byte vectors.
__device__ __forceinline__ void load8(const uint16_t* p, float* x, int64_t left, bool vec) {
  if (vec) {
    uint4 u = make_uint4(0, 0, 0, 0);
    if (left > 0) u = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      x[2 * j] = bf16_lo(w[j]);
      x[2 * j + 1] = bf16_hi(w[j]);
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = j < left ? bf16_one(p[j]) : 0.0f;
  }
}
__device__ __forceinline__ void load8(const float* p, float* x, int64_t left, bool vec) {
  if (vec) {
    f4 a = {0.f, 0.f, 0.f, 0.f}, b = a;
    if (left > 0) {
      a = *reinterpret_cast<const f4*>(p);
      b = *reinterpret_cast<const f4*>(p + 4);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      x[j] = a[j];
      x[4 + j] = b[j];
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = j < left ? p[j] : 0.0f;
  }
}
__device__ __forceinline__ void store8(uint16_t* p, const float* x, int64_t left, bool vec) {
  uint32_t w[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) w[j] = bf16x2_rne(x[2 * j], x[2 * j + 1]);
  if (vec) {
    if (left > 0) *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < left) p[j] = (uint16_t)(w[j / 2] >> (16 * (j & 1)));
  }
}
__device__ __forceinline__ void store8(float* p, const float* x, int64_t left, bool vec) {
  if (vec) {
    if (left > 0) {
      *reinterpret_cast<f4*>(p) = f4{x[0], x[1], x[2], x[3]};
      *reinterpret_cast<f4*>(p + 4) = f4{x[4], x[5], x[6], x[7]};
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < left) p[j] = x[j];
  }
}
// The value as stored in E.
__device__ __forceinline__ float as_stored(float x, const uint16_t*) {
  return bf16_one((uint16_t)bf16_rne(x));
}
__device__ __forceinline__ float as_stored(float x, const float*) { return x; }

constexpr int threads_of(int lpr) { return lpr > 64 ? lpr : 256; }  // whole rows

// N sums over the LPR lanes of a row; `par` alternates from call to call, so
// that one barrier each suffices where a row spans waves.
template <int LPR, int N>
struct RowSum {
  float part[2][LPR > 64 ? LPR / 64 : 1][N];
};
template <int LPR, int N>
__device__ __forceinline__ void row_sum(float* v, RowSum<LPR, N>& sh, int& par) {
#pragma unroll
  for (int d = (LPR < 64 ? LPR : 64) / 2; d > 0; d >>= 1)
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += __shfl_xor(v[i], d);
  if constexpr (LPR > 64) {
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int i = 0; i < N; ++i) sh.part[par][wave][i] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      v[i] = 0.0f;
#pragma unroll
      for (int q = 0; q < LPR / 64; ++q) v[i] += sh.part[par][q][i];
    }
    par ^= 1;
  }
}

// A workgroup's gradient of its group's columns: its rows' accumulators added in
// order in LDS, then written to its row of the partial sums.
template <int LPR, int NV>
__device__ __forceinline__ void put_partial(const float (*acc)[8], float* lds, float* out,
                                            int64_t width) {
  constexpr int RPW = threads_of(LPR) / LPR;
  const int sub = threadIdx.x / LPR, li = threadIdx.x % LPR;
  if constexpr (RPW > 1) {
    for (int i = 0; i < RPW; ++i) {
      __syncthreads();
      if (sub == i) {
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            float* p = lds + (v * 8 + j) * LPR + li;
            *p = i ? *p + acc[v][j] : acc[v][j];
          }
      }
    }
    __syncthreads();
    if (sub != 0) return;
  }
#pragma unroll
  for (int v = 0; v < NV; ++v)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int64_t c = (v * LPR + li) * 8 + j;
      if (c < width) out[c] = RPW > 1 ? lds[(v * 8 + j) * LPR + li] : acc[v][j];
    }
}
template <int LPR, int NV>
constexpr int partial_lds = threads_of(LPR) / LPR > 1 ? LPR * NV * 8 : 1;

// Whether rows of this type, address, stride and width go in whole vectors of
// 8 columns (a group's start included: the width is a multiple of 8).
inline bool vec_rows(const void* p, int64_t st, int64_t width, bool bf16) {
  return (uintptr_t)p % 16 == 0 && st % (bf16 ? 8 : 4) == 0 && width % 8 == 0;
}

// Row blocks of a backward: the workgroups' partial sums are this many rows.
// Four workgroups for each compute unit run side by side.
inline int64_t bwd_blocks(int64_t M, int64_t D, int64_t width, int cus) {
  const int64_t groups = D / width;
  int64_t n = (4 * (int64_t)cus + groups - 1) / groups;
  if (n > M) n = M;
  return n < 1 ? 1 : n;
}

// CALL(LPR, NV) for the smallest that holds a row of `width`; a wave for each row
// of up to 1536 columns needs no barrier.  A backward's registers hold more of each column, so a row takes more lanes: at
// 16384 rows of 1536 (residual norm, fp32 stream) 64 lanes of three vectors ran two
// waves per SIMD and 121 us, 192 lanes of one four waves and 96.  Rows over 8192
// spill some of theirs.
#define SW_NORM_PICK_BWD(width, CALL)           \
  do {                                          \
    if ((width) <= 64) { CALL(8, 1); }          \
    else if ((width) <= 128) { CALL(16, 1); }   \
    else if ((width) <= 256) { CALL(32, 1); }   \
    else if ((width) <= 512) { CALL(64, 1); }   \
    else if ((width) <= 1024) { CALL(128, 1); } \
    else if ((width) <= 1536) { CALL(192, 1); } \
    else if ((width) <= 2048) { CALL(256, 1); } \
    else if ((width) <= 4096) { CALL(512, 1); } \
    else if ((width) <= 8192) { CALL(1024, 1); } \
    else { CALL(1024, 2); }                     \
  } while (0)
#define SW_NORM_PICK(width, CALL)              \
  do {                                         \
    if ((width) <= 64) { CALL(8, 1); }         \
    else if ((width) <= 128) { CALL(16, 1); }  \
    else if ((width) <= 256) { CALL(32, 1); }  \
    else if ((width) <= 512) { CALL(64, 1); }  \
    else if ((width) <= 1024) { CALL(64, 2); } \
    else if ((width) <= 1536) { CALL(64, 3); } \
    else if ((width) <= 2048) { CALL(256, 1); } \
    else if ((width) <= 4096) { CALL(256, 2); } \
    else if ((width) <= 6144) { CALL(256, 3); } \
    else if ((width) <= 8192) { CALL(256, 4); } \
    else { CALL(512, 4); }                     \
  } while (0)

int fold_partials(const float* part, int64_t blocks, int64_t D, float* const* outs, int nout,
                  hipStream_t s);

// The backward's partial sums: the caller's workspace or the pool's.
struct Partials {
  float* p = nullptr;
  bool own = false;
  hipStream_t s;
  explicit Partials(hipStream_t st) : s(st) {}
  ~Partials() {
    if (own) workspace_free(p, s);
  }
  int get(void* ws, size_t have, size_t need, const char* what) {
    if (ws) {
      if (have < need)
        return fail(SW_ERR_INVALID_ARG, "workspace of %zu bytes, %zu needed", have, need);
      p = (float*)ws;
      return SW_OK;
    }
    int st = refuse_capture(s, what);
    if (st != SW_OK) return st;
    void* v = nullptr;
    if ((st = workspace_alloc(&v, need, s)) != SW_OK) return st;
    p = (float*)v;
    own = true;
    return SW_OK;
  }
};

}  // namespace norm
}  // namespace sw
