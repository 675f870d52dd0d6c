// linear_walk.h -- the chunked walk of linear attention (device code and its
// launch), included by one source file per element type so that they compile
// side by side.
//
// With roles X (read-out), Y (key), Z (value) and log decays g, one walk
// evaluates, over the steps of a sequence in the walk's order,
//     S_i = e^{g_i} S_{i-1} + w Y_i Z_i^T,     out_i = S_i^T X_i
// and so serves the forward (q, k, v) and, with the roles exchanged, every
// gradient: dq walks forward with (do, v, k), dk backwards with (v, do, q),
// dv backwards with (k, q, do).  Backwards, the decay between a step and the
// one walked before it is that of the later step in time.
//
// C steps at a time (G_i: the decays' running sum inside the chunk):
//     P_ts = (X_t . Y_s) e^{G_t - G_s}  for s <= t, else 0
//     out  = P Z + e^G X S        S <- e^{G_C} S + (e^{G_C - G} Z)^T-weighted Y^T
// All four products run on the matrix cores.  A workgroup of four waves walks
// one (sequence, segment, head, tile of Z's columns); a wave owns 16 NT
// columns and keeps its part of S in accumulators, fp32, from the first step
// to the last.  The lane that holds an accumulator's column is the lane that
// the next product wants as an operand's row, and the contraction order is
// free, so S and the weighted Z go from accumulators to operands without
// moving between lanes.
//
// Rounding (bf16): products of inputs are exact in fp32 accumulators.  The
// weighted Z is split in three bf16 parts whose sum is the fp32 value, so S
// keeps fp32 accuracy whatever the number of chunks.  P and S are split in two as
// operands of an output: 2^-17 of its terms beside its own rounding of 2^-9, so that
// every output is rounded to bf16 once, at its end, in calls of any size (one part
// each made 1.41 times that error and took 72 us for o's walk at B=8 L=2048 H=12
// K=V=128 where two take 76).  For dq and dk S is split in three, since its products
// make dg too.  fp32 inputs run on the fp32 matrix instructions throughout.
#pragma once

#include "linear_attn.h"

namespace sw {
namespace lin {

constexpr int CHUNK = 64;      // steps between the places where walks may start or stop
constexpr float G_MIN = -104.0f;  // e^g is zero in fp32 here: the lowest that counts

struct Job {
  HeadRows X, Y, Z, A;   // A: in the gradients' walks the input of which out is the gradient
  int xdiv, ydiv, zdiv, adiv;  // head h reads head h / div
  bool xvec, yvec, zvec, avec;  // rows are 16-byte aligned whole vectors
  bool ovec, orows;             // out's rows: whole fours of columns; and 16-byte granules
  void* out;
  int64_t ob, ol, oh;
  bool out_f32;
  bool reverse;
  const float* init;     // (sequences, H, K, V): the state before the first step, or NULL
  float* last;           // the state after the last step, or NULL
  float* carry;          // (slots, H, K, V): carries written, or initial states read, or NULL
  float* decay;          // (slots, H): the segments' decays (written with the carries)
  // dg: dk's walk writes its rows' sums and its states between chunks, dq's reads them
  float* sums;           // [tile][H][B * L]
  float* kept;           // (chunk ends inside sequences, H, K, V)
  const float* dlast;    // (sequences, H, K, V): the state after the last step, or NULL
  bool dvec;             // it lies on 16 bytes
  float* dg;             // dg of step i, head h and tile q at dg[i dg_st + h dg_sh + q dg_sq], or NULL
  int64_t dg_st, dg_sh, dg_sq;
  double* by_slot;       // (slots, tiles, H): dg's sums over the segment's steps, or NULL
  int64_t skk, svv;      // where state element (Y's column, Z's column) lies in (K, V)
  // scales of P (its absolute value and log2), of the state's increments and of the
  // read-out; neg: out changes its sign
  float pabs, wscale, rscale;
  double plog;
  bool neg;
};

struct WalkArgs {
  Job job[2];
  const float* g;
  int64_t g_sb, g_sl, g_sh;
  const int32_t* cu;
  int64_t B, L, nseq, H;
  int KK, VV;            // widths: of X and Y, of Z and out
  int64_t KV;            // K * V
  int64_t lseg;          // steps of a segment, a multiple of CHUNK
  int64_t per_seq;       // segments of a sequence (cu == NULL)
  int64_t slots;
  int tiles, njobs;
};

// Where slot `slot` of width `w` steps lies: packed sequence n's slots start at
// cu[n] / w + n, which leaves room for each one's ceil(length / w).
struct Place {
  int64_t n, first, len, part, parts;  // sequence, its first step, length, which slot of how many
  bool valid;
};

__device__ __forceinline__ int64_t cu_at(const int32_t* cu, int64_t i, int64_t L) {
  const int64_t c = cu[i];
  return c < 0 ? 0 : c > L ? L : c;  // never outside the row, whatever cu holds
}

__device__ __forceinline__ Place place_of(const int32_t* cu, int64_t slot, int64_t w,
                                          int64_t per_seq, int64_t nseq, int64_t L) {
  Place p;
  if (!cu) {
    p.n = slot / per_seq;
    p.part = slot - p.n * per_seq;
    p.first = 0;
    p.len = L;
  } else {
    int64_t lo = 0, hi = nseq - 1;
    while (lo < hi) {
      const int64_t mid = (lo + hi + 1) / 2;
      if (cu_at(cu, mid, L) / w + mid <= slot) lo = mid; else hi = mid - 1;
    }
    p.n = lo;
    p.first = cu_at(cu, lo, L);
    const int64_t end = cu_at(cu, lo + 1, L);
    p.len = end > p.first ? end - p.first : 0;
    p.part = slot - (p.first / w + lo);
  }
  p.parts = p.len > 0 ? (p.len + w - 1) / w : 1;
  p.valid = p.n < nseq && p.part >= 0 && p.part < p.parts;
  return p;
}

// e^g of a decay as the walks use it.
__device__ __forceinline__ float clamp_g(float g) { return g < G_MIN ? G_MIN : g; }

// One step of an inclusive sum over a wave's lanes: v plus that of the lane the
// control names, where it has one.
template <int CTRL, int ROW_MASK>
__device__ __forceinline__ double add_from(double v) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo =
      (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)u, CTRL, ROW_MASK, 0xf, false);
  const uint32_t hi =
      (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(u >> 32), CTRL, ROW_MASK, 0xf, false);
  return v + __builtin_bit_cast(double, ((uint64_t)hi << 32) | lo);
}
// Inclusive sums over the 64 lanes; all: the last lane's, on every lane.
__device__ __forceinline__ double wave_running_sum(double v, double* all) {
  v = add_from<DPP_ROW_SHR1, 0xf>(v);
  v = add_from<DPP_ROW_SHR2, 0xf>(v);
  v = add_from<DPP_ROW_SHR4, 0xf>(v);
  v = add_from<DPP_ROW_SHR8, 0xf>(v);
  v = add_from<DPP_ROW_BCAST15, 0xa>(v);
  v = add_from<DPP_ROW_BCAST31, 0xc>(v);
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)u, 63);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(u >> 32), 63);
  *all = __builtin_bit_cast(double, ((uint64_t)hi << 32) | lo);
  return v;
}

// The sum over the 16 lanes of a lane's row, on each of them.
__device__ __forceinline__ float row_sum16(float v) {
  v += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x128, 0xf, 0xf, false));
  v += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x124, 0xf, 0xf, false));
  v += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x122, 0xf, 0xf, false));
  v += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x121, 0xf, 0xf, false));
  return v;
}

// 2^x of a double, to fp32 rounding.
__device__ __forceinline__ float exp2_of(double x) {
  const double n = rint(x);
  const float f = __builtin_amdgcn_exp2f((float)(x - n));
  const float e = (float)n;
  return e < -300.0f ? 0.0f : e > 300.0f ? INFINITY : ldexpf(f, (int)e);
}

typedef float f4 __attribute__((ext_vector_type(4)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef short s4 __attribute__((ext_vector_type(4)));
typedef short s8 __attribute__((ext_vector_type(8)));
typedef __bf16 b8 __attribute__((ext_vector_type(8)));

struct Bf16 {
  typedef uint16_t E;
  static constexpr int C = 64, G = 8, GB = 3;  // steps of a chunk; elements of 16 bytes
  static constexpr int NW = 3;                 // parts of the weighted Z
  static constexpr bool SPLIT = true;
};
struct F32 {
  typedef float E;
  static constexpr int C = 32, G = 4, GB = 2;
  static constexpr int NW = 1;
  static constexpr bool SPLIT = false;
};

// An operand fragment of a 16 x 16 product over 32 contraction indices: lane
// (g = lane / 16, r = lane % 16) holds row r at indices 8 g .. 8 g + 7.
template <class T> struct Frag;
template <> struct Frag<Bf16> { s8 v; };
template <> struct Frag<F32> { float v[8]; };

__device__ __forceinline__ f4 mma(const Frag<Bf16>& a, const Frag<Bf16>& b, f4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(b8, a.v),
                                                 __builtin_bit_cast(b8, b.v), c, 0, 0, 0);
}
__device__ __forceinline__ f4 mma(const Frag<F32>& a, const Frag<F32>& b, f4 c) {
#pragma unroll
  for (int j = 0; j < 8; ++j)
    c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.v[j], b.v[j], c, 0, 0, 0);
  return c;
}

// Tiles in LDS.  The contraction over steps runs in blocks of 32, whose place
// (lane group g, element j) is step 4 g + j (j < 4) or 16 + 4 g + j - 4; that over
// columns in blocks of 32, whose (g, j) is column 8 g + j.  An accumulator's rows
// then are an operand's places, X's fragments are one read, and transposed reads
// take four neighbouring rows a group.
// Rows have 32 bytes of padding: 32 bytes of each of eight neighbouring rows lie
// in different banks.  In Y (bf16), 16-byte granules of odd pairs have their halves
// exchanged: a transposed read takes the same half of four granules, and so meets
// all of those 32 bytes.  By the conflict counter the reads of X's, Y's and Z's
// fragments take the cycles that their bytes need.
template <class T, int W>
constexpr int ROW = W + 2 * T::G;

// Step s's place in its chunk.
__device__ __forceinline__ int place_in(int s) {
  return (s & ~31) + 8 * ((s >> 2) & 3) + 4 * ((s >> 4) & 1) + (s & 3);
}

// Eight columns of a row of X or Y.
__device__ __forceinline__ Frag<Bf16> row_frag(const uint16_t* t) {
  return {*reinterpret_cast<const s8*>(t)};
}
__device__ __forceinline__ Frag<F32> row_frag(const float* t) {
  Frag<F32> f;
  *reinterpret_cast<f4*>(f.v) = *reinterpret_cast<const f4*>(t);
  *reinterpret_cast<f4*>(f.v + 4) = *reinterpret_cast<const f4*>(t + 4);
  return f;
}
// The same of a row in memory, `left` columns of it from p on (vec: whole 16-byte granules).
__device__ __forceinline__ void load_frag(Frag<Bf16>& f, const uint16_t* p, int left, bool vec) {
  f.v = s8{0, 0, 0, 0, 0, 0, 0, 0};
  if (vec) {
    if (left > 0) f.v = *reinterpret_cast<const s8*>(p);
  } else if (left > 0) {  // in flight together: past the row its last one, not used
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const short x = (short)p[min(j, left - 1)];
      f.v[j] = j < left ? x : (short)0;
    }
  }
}
__device__ __forceinline__ void load_frag(Frag<F32>& f, const float* p, int left, bool vec) {
#pragma unroll
  for (int j = 0; j < 8; ++j) f.v[j] = 0.0f;
  if (vec) {
    if (left > 0) *reinterpret_cast<f4*>(f.v) = *reinterpret_cast<const f4*>(p);
    if (left > 4) *reinterpret_cast<f4*>(f.v + 4) = *reinterpret_cast<const f4*>(p + 4);
  } else if (left > 0) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float x = p[min(j, left - 1)];
      f.v[j] = j < left ? x : 0.0f;
    }
  }
}
// X's fragment in the order of Y's.
__device__ __forceinline__ Frag<Bf16> as_y(const Frag<Bf16>& f, int g) {
  const u4 u = __builtin_bit_cast(u4, f.v);
  return {__builtin_bit_cast(s8, g & 2 ? u4{u[2], u[3], u[0], u[1]} : u)};
}
__device__ __forceinline__ Frag<F32> as_y(const Frag<F32>& f, int) { return f; }

// P's rows hold what lies on and below the diagonal's blocks: of 64 steps, the
// first 32 rows one block of 32 places and the others two.  16-byte granule c of
// row t is at c ^ pswz(t) of its row.
template <class T>
__device__ __forceinline__ int p_row(int t) {  // the row's first element
  return T::C == 32 || t >= 32 ? t * T::C - (T::C == 64 ? 32 * 32 : 0) : t * 32;
}
template <class T>
__device__ __forceinline__ int pswz(int t) {
  return T::C == 32 || t >= 32 ? t & 7 : 2 * ((t >> 2) & 1);
}
template <class T>
constexpr int P_SIZE = T::C == 64 ? 64 * 64 - 32 * 32 : 32 * 32;
// A lane's eight places 8 g .. + 7 of block sb.
__device__ __forceinline__ Frag<Bf16> p_frag(const uint16_t* p, int t, int sb, int g) {
  return {*reinterpret_cast<const s8*>(p + p_row<Bf16>(t) + ((4 * sb + g) ^ pswz<Bf16>(t)) * 8)};
}
__device__ __forceinline__ Frag<F32> p_frag(const float* p, int t, int, int g) {
  Frag<F32> f;
  const int m = pswz<F32>(t);
  const float* row = p + p_row<F32>(t);
  *reinterpret_cast<f4*>(f.v) = *reinterpret_cast<const f4*>(row + ((2 * g) ^ m) * 4);
  *reinterpret_cast<f4*>(f.v + 4) = *reinterpret_cast<const f4*>(row + ((2 * g + 1) ^ m) * 4);
  return f;
}

// The transposed fragment of 32 steps: lane (g, r) holds a column at its group's
// places: of Z, column r of 16 (z_base); of Y, column 8 (r / 4) + 4 half + r % 4 of
// 32 (y_base; half: 0 or 1).  Both give the lane's address for the block's first
// step and the columns' first.
template <int W>
__device__ __forceinline__ const uint16_t* z_base(const uint16_t* t, int g, int r) {
  return t + (4 * g + (r >> 2)) * ROW<Bf16, W> + 4 * (r & 3);
}
template <int W>
__device__ __forceinline__ const float* z_base(const float* t, int g, int r) {
  return t + 4 * g * ROW<F32, W> + r;
}
template <int W>
__device__ __forceinline__ const uint16_t* y_base(const uint16_t* t, int g, int r, int half) {
  return t + (4 * g + (r >> 2)) * ROW<Bf16, W> + 8 * (r & 3) + 4 * (half ^ ((r >> 1) & 1));
}
template <int W>
__device__ __forceinline__ const float* y_base(const float* t, int g, int r, int half) {
  return t + 4 * g * ROW<F32, W> + 8 * (r >> 2) + 4 * half + (r & 3);
}
template <int W>
__device__ __forceinline__ Frag<Bf16> col_frag(const uint16_t* t) {
  typedef __attribute__((address_space(3))) s4* lds_s4;
  const s4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4)t);
  const s4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4)(t + 16 * ROW<Bf16, W>));
  return {s8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]}};
}
template <int W>
__device__ __forceinline__ Frag<F32> col_frag(const float* t) {
  Frag<F32> f;
#pragma unroll
  for (int j = 0; j < 8; ++j) f.v[j] = t[(j + (j < 4 ? 0 : 12)) * ROW<F32, W>];
  return f;
}

__device__ __forceinline__ s8 pack8(const float* x) {
  uint4 u;
  u.x = bf16x2_rne(x[0], x[1]);
  u.y = bf16x2_rne(x[2], x[3]);
  u.z = bf16x2_rne(x[4], x[5]);
  u.w = bf16x2_rne(x[6], x[7]);
  return __builtin_bit_cast(s8, u);
}
// x minus its bf16 rounding h (exact).
__device__ __forceinline__ void take_off(float* x, s8 h) {
  const uint4 u = __builtin_bit_cast(uint4, h);
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int j = 0; j < 8; ++j) x[j] -= j & 1 ? bf16_hi(w[j / 2]) : bf16_lo(w[j / 2]);
}
// Eight fp32 values as N operand parts.
template <int N>
__device__ __forceinline__ void parts_of(const float* x, Frag<Bf16>* f) {
  float t[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) t[j] = x[j];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    f[i].v = pack8(t);
    if (i + 1 < N) take_off(t, f[i].v);
  }
}
template <int N>
__device__ __forceinline__ void parts_of(const float* x, Frag<F32>* f) {
#pragma unroll
  for (int j = 0; j < 8; ++j) f[0].v[j] = x[j];
}
__device__ __forceinline__ float widen1(uint16_t e) { return bf16_one(e); }
__device__ __forceinline__ float widen1(float e) { return e; }

// Adds zero times each element of a granule to acc: NaN once one is not finite.
__device__ __forceinline__ float check_finite(u4 u, float acc, Bf16*) {
  typedef __bf16 b2 __attribute__((ext_vector_type(2)));
  const b2 zero = {(__bf16)0.0f, (__bf16)0.0f};
#pragma unroll
  for (int j = 0; j < 4; ++j)
    acc = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(b2, (uint32_t)u[j]), zero, acc, false);
  return acc;
}
__device__ __forceinline__ float check_finite(u4 u, float acc, F32*) {
#pragma unroll
  for (int j = 0; j < 4; ++j) acc = __builtin_fmaf(__uint_as_float(u[j]), 0.0f, acc);
  return acc;
}

// One thread's granules of a C x W tile of rows `step` elements apart, `rows` the
// one lowest in memory: row i of the tile is row i there (rev: row n - 1 - i),
// rows from n and columns from width are zero.
// VEC: 16-byte buffer loads without a branch, so that they stay in flight until
// the granules are stored.  What lies outside the tile has an offset past the
// buffer's end (rows from n do since a row is no longer than a step; backwards
// their offsets are negative) and reads zero.
template <class T, int W, int THREADS, bool VEC>
struct Tile {
  static constexpr int NG = W / T::G, RPG = THREADS / NG, PER = RPG < T::C ? T::C / RPG : 1;
  static_assert(THREADS % NG == 0 && (RPG >= T::C || T::C % RPG == 0), "whole rows at a time");
  typedef typename T::E E;
  u4 u[PER];
  __device__ __forceinline__ void load(const E* rows, int64_t step, int n, bool rev, int width,
                                       int tid) {
    asm volatile("" : "+v"(tid));  // offsets worked out here, not kept across the walk
    const int row = (unsigned)tid / NG, col = (unsigned)tid % NG * T::G;
    if constexpr (VEC) {
      const int st = (int)step * (int)sizeof(E);
      const int end = max((n - 1) * st + min(width, W) * (int)sizeof(E), 0);  // none: n = 0
      const auto rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)rows, 0, end, 0x00020000);
      uint32_t off = (uint32_t)((rev ? n - 1 - row : row) * st) +
                     (col < width ? col * (uint32_t)sizeof(E) : 0x40000000u);
      const int next = (rev ? -RPG : RPG) * st;
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        u[i] = __builtin_amdgcn_raw_buffer_load_b128(rsrc, off, 0, 0);
        off += next;
      }
    } else {
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const int r = row + i * RPG;
        const E* p = rows + (rev ? n - 1 - r : r) * step + col;
        E e[T::G];
#pragma unroll
        for (int j = 0; j < T::G; ++j) e[j] = r < n && col + j < width ? p[j] : (E)0;
        __builtin_memcpy(&u[i], e, 16);
      }
    }
  }
  // To the tile's rows (SWAP: as Y's).
  template <bool SWAP>
  __device__ __forceinline__ void store(E* lds, int tid) const {
    E* p = lds + tid / NG * ROW<T, W> + tid % NG * T::G;
    const bool swap = SWAP && T::SPLIT && (tid & 2);  // NG is a multiple of 4
#pragma unroll
    for (int i = 0; i < PER; ++i)
      if (RPG <= T::C || tid / NG < T::C)
        *reinterpret_cast<u4*>(p + i * RPG * ROW<T, W>) =
            swap ? u4{u[i][2], u[i][3], u[i][0], u[i][1]} : u[i];
  }
  // Zero, or NaN if an element is not finite.
  __device__ __forceinline__ float finite() const {
    float acc = 0.0f;
#pragma unroll
    for (int i = 0; i < PER; ++i) acc = check_finite(u[i], acc, (T*)nullptr);
    return acc;
  }
};

// What a walk is for: the segments' carries; an output; dk, and dq, with their parts
// of dg.
//
// dg_t = e^{g_t} <dS_t, S_{t-1}> is the sum over the pairs of a step s < t and a step
// t' >= t of scale (q_t' . k_s) (do_t' . v_s) e^{G_t' - G_s} (and h0's and dh_last's
// with them).  A difference of what q . dq and k . dk sum to is shorter, but keeps
// only the digits of its largest terms: where a step forgets much, dg_t is far
// smaller than they are (at decays of e^-16 nothing of it was left).  So the pairs are
// added up as they are, those of one chunk and head as
//   dg_t = D + sum_{t' >= t} a_t' + sum_{s < t} b_s + sum_{t' >= t, s < t} M_t's
//   M_t's = P_t's (q_t' . k_s)                       both steps in the chunk
//   a_t' = q_t' . (dq's part from the state before)  s before the chunk
//   b_s  = k_s . (dk's part from the state after)    t' after it
//   D    = e^{G_C} <S before, dS after>              the one before, the other after
// with no difference anywhere.  dk's walk runs first: it leaves b, and its state at
// each chunk's end, decayed by the step after it.  dq's walk has S before each chunk
// in its accumulators.  The states' traffic is 8 K V bytes a chunk and head; keeping
// both and multiplying them apart would be twice that.
enum Mode { CARRY, OUT, GRAD_K, GRAD_Q };
constexpr bool is_grad(Mode m) { return m >= GRAD_K; }

template <class T, int KP, int NT, Mode MODE>
struct Shared {
  static constexpr int VT = 64 * NT, C = T::C;
  // Parts of S, which makes a and b too, of fp32 accuracy; and of P
  static constexpr int NS = !T::SPLIT ? 1 : is_grad(MODE) ? 3 : 2;
  static constexpr int NP = T::SPLIT ? 2 : 1;
  static constexpr bool XS = MODE != CARRY;
  typename T::E y[C * ROW<T, KP>];
  typename T::E z[C * ROW<T, VT>];
  typename T::E x[XS ? C * ROW<T, KP> : 8];
  typename T::E p[XS ? NP * P_SIZE<T> : 8];
  // A chunk's decays, of this chunk and the next.
  struct alignas(16) Decays {  // read in fours
    float gs[C], gsl[C];  // by step s: the running log2 decay, high and low parts
    float gt[C], gtl[C];  // by step t: the same with log2 |pscale|
    float er[C];                     // by step: rscale 2^G
    float g1[C];                     // by step: its own decay
    float ew[C];                     // by place: wscale 2^(G_C - G)
    float ec;                        // 2^G_C
  } dec[2];
  // bf16 outputs leave as whole rows: a wave's columns are 32 or 64 bytes of each step's
  static constexpr bool ROWS = MODE == OUT && T::SPLIT;
  static constexpr bool IN_X = ROWS && KP >= VT;  // x is read by then
  typename T::E o[ROWS && !IN_X ? C * VT : 8];  // granule c of row t at c ^ oswz(t)
  float dots[is_grad(MODE) ? 4 * C : 4];       // a or b: each wave's columns' part
  alignas(16) float pairs[MODE == GRAD_Q ? 4 * C : 4];     // by wave and step s: M summed for dg of step s + 1
  float rows[MODE == GRAD_Q && C == 32 ? 16 : 4];  // steps 16 ..: M summed over the steps before 16
  float ends[4];                               // <S, dS>: each wave's part
  uint32_t bad[2];                // the chunk (of odd or even number) holds what is not finite
};

template <int VT>
__device__ __forceinline__ int oswz(int t) {
  return VT == 128 ? t & 15 : (t >> 1) & 7;
}

template <int N>
struct Count {
  static constexpr int value = N;
};

// Keeps what follows from moving before what precedes: a product, a few vector
// instructions that run beside it, the next product.
__device__ __forceinline__ void in_order() { __builtin_amdgcn_sched_barrier(0); }

// Two values of an operand fragment on their way into bf16 parts, one part a call.
struct Pair {
  float a, b;
  __device__ __forceinline__ uint32_t part(bool last) {
    const uint32_t u = bf16x2_rne(a, b);
    if (!last) {
      a -= bf16_lo(u);
      b -= bf16_hi(u);
    }
    return u;
  }
};
template <int N>
struct Parts {  // of one fragment: its pairs' N parts
  Pair x[4];
  u4 u[N];
  __device__ __forceinline__ Frag<Bf16> frag(int q) const {
    return {__builtin_bit_cast(s8, u[q])};
  }
};

// The lane's place in a fragment, worked out anew: what is derived from it (each
// phase's addresses in LDS) is not kept in registers across the walk.
struct LanePlace {
  int g, r;
};
__device__ __forceinline__ LanePlace lane_place(int tid) {
  asm volatile("" : "+v"(tid));
  return {(tid >> 4) & 3, tid & 15};
}

// Waves per SIMD, as the accumulators of S and out (16 NT + KP NT / 2 registers) and
// the loads in flight leave room for.  Wider tiles a wave (NT = 2) read each
// fragment of X, Y and P for twice the products: with eight waves of 16 columns
// instead, LDS reads doubled and set the pace.
constexpr int walk_waves(int KP, int NT, Mode m) {
  return KP >= 256 ? 1 : NT == 2 || KP == 128 ? 2 : m != CARRY ? 3 : 4;
}

template <class T, int KP, int NT, Mode MODE, bool VEC>
__global__ __launch_bounds__(256, walk_waves(KP, NT, MODE)) void walk_kernel(WalkArgs a) {
  typedef typename T::E E;
  typedef Shared<T, KP, NT, MODE> Sh;
  constexpr bool XS = MODE != CARRY;
  constexpr bool GRAD = is_grad(MODE);
  constexpr int C = T::C, KT = KP / 16, VT = 64 * NT, SB = C / 32, TT = C / 16, NS = Sh::NS;
  constexpr int THREADS = 256;
  constexpr int KR = ROW<T, KP>, VR = ROW<T, VT>, G = T::G;
  __shared__ __align__(16) Sh sh;

  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 4, r = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  uint32_t w = xcd_contiguous(blockIdx.x, gridDim.x);
  const int tile = w % (uint32_t)a.tiles;
  w /= (uint32_t)a.tiles;
  const int h = w % (uint32_t)a.H;
  w /= (uint32_t)a.H;
  const int64_t slot = w % (uint32_t)a.slots;
  const Job& job = a.job[w / (uint32_t)a.slots];
  const Place pl = place_of(a.cu, slot, a.lseg, a.per_seq, a.nseq, a.L);
  if (!pl.valid) {
    if (MODE == GRAD_Q && job.by_slot && tid == 0) job.by_slot[(slot * a.tiles + tile) * a.H + h] = 0.0;
    return;
  }
  const bool rev = job.reverse;
  // the last segment in the walk's order hands nothing on
  const bool final_seg = rev ? pl.part == 0 : pl.part == pl.parts - 1;
  if (MODE == CARRY && final_seg) return;
  const int64_t b = a.cu ? 0 : pl.n;
  const int v0 = tile * VT, vb = wave * 16 * NT;  // the tile's first column; the wave's in it

  // steps [lo, hi) of the sequence, in chunks of at most C
  const int len = (int)pl.len, lo = (int)(pl.part * a.lseg);
  const int hi = len - lo < a.lseg ? len : lo + (int)a.lseg;
  const int nch = hi > lo ? (hi - lo + C - 1) / C : 0;

  // the rows of the sequence's first step
  const E* X = nullptr;
  if (XS) X = (const E*)job.X.p + b * job.X.sb + pl.first * job.X.sl + h / job.xdiv * job.X.sh;
  const E* Y = (const E*)job.Y.p + b * job.Y.sb + pl.first * job.Y.sl + h / job.ydiv * job.Y.sh;
  const E* Z = (const E*)job.Z.p + b * job.Z.sb + pl.first * job.Z.sl + h / job.zdiv * job.Z.sh + v0;
  const float* gp = a.g + b * a.g_sb + pl.first * a.g_sl + h * a.g_sh;

  f4 S[KT][NT];
  // state element of accumulator (kt, nt, i): Y's column 32 (kt / 2) + 8 g + 4 (kt % 2) + i,
  // Z's v0 + vb + 16 nt + r
  auto each_state = [&](auto fn) __attribute__((always_inline)) {
    int kk = 8 * g, vv = v0 + vb + r;
    asm volatile("" : "+v"(kk), "+v"(vv));  // worked out here, not kept across the walk
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
      if (vv + 16 * nt < a.VV) {
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int k = kk + 32 * (kt >> 1) + 4 * (kt & 1) + i;
            if (k < a.KK) fn(kt, nt, i, k * job.skk + (vv + 16 * nt) * job.svv);
          }
      }
  };
  auto store_state = [&](float* p, float f) __attribute__((always_inline)) {
    each_state([&](int kt, int nt, int i, int64_t at)
                   __attribute__((always_inline)) { p[at] = S[kt][nt][i] * f; });
  };
  // The gradients' walks have Y's columns side by side in a state (skk == 1): fn of each
  // accumulator's four of them, which the address is of and of which `left` are there.
  auto each_four = [&](auto* p, auto fn) __attribute__((always_inline)) {
    int kk = 8 * g, vv = v0 + vb + r;
    asm volatile("" : "+v"(kk), "+v"(vv));
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
      if (vv + 16 * nt < a.VV) {
        auto* row = p + (int64_t)(vv + 16 * nt) * job.svv + kk;
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) {
          const int k = 32 * (kt >> 1) + 4 * (kt & 1);
          if (kk + k < a.KK) fn(kt, nt, row + k, a.KK - kk - k);
        }
      }
  };
  // dS at the end of a chunk, before the sequence's step t
  auto kept_at = [&](int t) {
    const int64_t base = a.cu ? pl.first / C : pl.n * ((a.L - 1) / C);
    return job.kept + ((base + t / C - 1) * a.H + h) * a.KV;
  };
#pragma unroll
  for (int kt = 0; kt < KT; ++kt)
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) S[kt][nt] = f4{0.f, 0.f, 0.f, 0.f};
  if (XS) {
    const float* p = job.carry ? job.carry + (slot * a.H + h) * a.KV
                     : job.init ? job.init + (pl.n * a.H + h) * a.KV
                                : nullptr;
    if (p)
      each_state([&](int kt, int nt, int i, int64_t at)
                     __attribute__((always_inline)) { S[kt][nt][i] = p[at]; });
  }
  float seg_decay = 1.0f;
  E* const orow = Sh::IN_X ? sh.x : sh.o;
  double dg_sum = 0.0;

  Tile<T, KP, THREADS, VEC> tx, ty;
  Tile<T, VT, THREADS, VEC> tz;
  float tg = 0.0f;
  int t0 = 0, n = 0;  // a chunk's steps: t0 .. t0 + n - 1; its row i is the walk's i-th of them
  auto load_chunk = [&](int c) __attribute__((always_inline)) {  // c = nch: nothing
    t0 = lo + (rev ? nch - 1 - c : c) * C;
    n = c >= nch ? 0 : hi - t0 < C ? hi - t0 : C;
    const int64_t t = c >= nch ? lo : t0;
    if (XS) tx.load(X + t * job.X.sl, job.X.sl, n, rev, a.KK, tid);
    ty.load(Y + t * job.Y.sl, job.Y.sl, n, rev, a.KK, tid);
    tz.load(Z + t * job.Z.sl, job.Z.sl, n, rev, a.VV - v0, tid);
  };
  // The first wave works out a chunk's decays while the others still multiply for
  // the chunk before (it has the least to do above P's diagonal); their g is on its
  // way a chunk earlier still.
  auto cnt_of = [&](int c) {
    const int c0 = lo + (rev ? nch - 1 - c : c) * C;
    return c >= nch ? 0 : hi - c0 < C ? hi - c0 : C;
  };
  auto load_decays = [&](int c) __attribute__((always_inline)) {
    const int c0 = lo + (rev ? nch - 1 - c : c) * C, cn = cnt_of(c);
    // backwards, a step's decay is that of the step after it in time; none at the end
    const int s = rev ? c0 + cn - lane : c0 + lane;
    tg = lane < cn && s < len ? gp[s * a.g_sl] : 0.0f;
  };
  auto put_decays = [&](int c) __attribute__((always_inline)) {
    typename Sh::Decays& d = sh.dec[c & 1];
    const double g1 = (double)clamp_g(tg) * 1.4426950408889634;
    double GC;
    const double G = wave_running_sum(lane < cnt_of(c) ? g1 : 0.0, &GC);
    if (lane < C) {
      if (XS) {
        const double Gt = G + job.plog;
        const float s_ = (float)G, t_ = (float)Gt;
        d.gs[lane] = s_;
        d.gt[lane] = t_;
        d.gsl[lane] = (float)(G - (double)s_);
        d.gtl[lane] = job.plog > -1.0e30 ? (float)(Gt - (double)t_) : 0.0f;
        d.er[lane] = exp2_of(G) * job.rscale;
      }
      d.ew[place_in(lane)] = exp2_of(GC - G) * job.wscale;
      d.g1[lane] = exp2_of(g1);
    }
    if (lane == 0) d.ec = exp2_of(GC);
  };

  const int64_t ob = b * job.ob + pl.first * job.ol + h * job.oh;
  const E* ap = nullptr;
  if (GRAD)
    ap = (const E*)job.A.p + b * job.A.sb + pl.first * job.A.sl + h / job.adiv * job.A.sh;

  if (tid < 2) sh.bad[tid] = 0;
  if (nch > 0) {
    load_chunk(0);
    if (wave == 0) {
      load_decays(0);
      put_decays(0);
      load_decays(1);
    }
    __syncthreads();
  }
  for (int c = 0; c < nch; ++c) {
    // what is not finite in X and Y meets its own steps and columns only; in Z, zero
    // weights too
    const float fin = tz.finite();
    tz.template store<false>(sh.z, tid);
    ty.template store<true>(sh.y, tid);
    if (XS) tx.template store<false>(sh.x, tid);
    if (fin != fin) sh.bad[c & 1] = 1;
    __syncthreads();
    const bool bad = sh.bad[c & 1];
    const typename Sh::Decays& dec = sh.dec[c & 1];
    if (tid == 0) sh.bad[(c + 1) & 1] = 0;

    // rows of this chunk: cnt, the first of them step tfirst, the next tstep on
    const int cnt = n, tfirst = rev ? t0 + n - 1 : t0, tstep = rev ? -1 : 1;
    const int tend = t0 + n;  // the step after the chunk's last in time

    if constexpr (MODE == GRAD_K) {
      if (tend < len) {
        const float g1 = dec.g1[0];  // of step tend
        each_four(kept_at(tend), [&](int kt, int nt, float* p, int left) __attribute__((always_inline)) {
          const f4 x = S[kt][nt] * g1;
          if (VEC) {
            *reinterpret_cast<f4*>(p) = x;
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (i < left) p[i] = x[i];
          }
        });
      }
    }
    // dg: what one wave adds up at the chunk's end is on its way from here on
    float later = 0.0f, own_g = 0.0f;
    f4 after[MODE == GRAD_Q ? KT : 1][NT];  // dS
    if constexpr (MODE == GRAD_Q) {
      if (wave == 1 && lane < cnt) {
        const int64_t at = ((int64_t)tile * a.H + h) * (a.B * a.L) + b * a.L + pl.first + tfirst + lane;
        if (lane > 0) later = job.sums[at - 1];
        own_g = gp[(int64_t)(tfirst + lane) * a.g_sl];
      }
#pragma unroll
      for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) after[kt][nt] = f4{0.f, 0.f, 0.f, 0.f};
      const float* p = tend < len  ? kept_at(tend)
                       : job.dlast ? job.dlast + (pl.n * a.H + h) * a.KV
                                   : nullptr;
      if (p)
        each_four(p, [&](int kt, int nt, const float* q, int left) __attribute__((always_inline)) {
          if (VEC) {
            after[kt][nt] = *reinterpret_cast<const f4*>(q);
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float x = q[min(i, left - 1)];
              after[kt][nt][i] = i < left ? x : 0.0f;
            }
          }
        });
    }

    if (XS && (MODE == GRAD_Q || !bad)) {
      // P^T = Y X^T: a wave has 16 steps t (columns) and of the tiles of 16 steps s
      // (rows) those up to the diagonal's; the pair that holds it is filled with zeros
      const LanePlace me = lane_place(tid);
      const int g = me.g, r = me.r;
      const int tt = wave & (TT - 1), t = tt * 16 + r;
      const int first = C == 32 ? wave >> 1 : 0;  // its first tile of steps s
      Frag<T> xf[KP / 32];
      const E* const xr = sh.x + t * KR + 8 * g;
#pragma unroll
      for (int p = 0; p < KP / 32; ++p) xf[p] = as_y(row_frag(xr + 32 * p), g);
      // A's row of step t, for the products of the pairs
      Frag<T> af[MODE == GRAD_Q ? VT / 32 : 1];
      if constexpr (MODE == GRAD_Q) {
        const E* const ar = ap + (int64_t)(tfirst + t) * job.A.sl + v0 + 8 * g;
#pragma unroll
        for (int p = 0; p < VT / 32; ++p)
          load_frag(af[p], ar + 32 * p, t < cnt ? a.VV - v0 - 8 * g - 32 * p : 0, VEC);
      }
      const float gt = dec.gt[t], gtl = dec.gtl[t];
      E* const pw = sh.p + p_row<T>(t);
      const int m = pswz<T>(t);
      // N tiles from `first`, the last of them the diagonal's if `diag`
      auto weigh = [&](auto count, bool diag) __attribute__((always_inline)) {
        constexpr int N = decltype(count)::value;
        f4 acc[N];
#pragma unroll
        for (int i = 0; i < N; ++i) acc[i] = f4{0.f, 0.f, 0.f, 0.f};
        const E* const yr = sh.y + (16 * first + r) * KR + 8 * g;
#pragma unroll
        for (int p = 0; p < KP / 32; ++p)
#pragma unroll
          for (int i = 0; i < N; ++i)
            acc[i] = mma(row_frag(yr + 16 * i * KR + 32 * p), xf[p], acc[i]);
        float pv[4 * (N + (N & 1))];
#pragma unroll
        for (int i = 0; i < N + (N & 1); ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) pv[4 * i + j] = 0.0f;
#pragma unroll
        for (int i = 0; i < N; ++i) {
          f4 d = gt - *reinterpret_cast<const f4*>(dec.gs + 16 * (first + i) + 4 * g);
          d += gtl - *reinterpret_cast<const f4*>(dec.gsl + 16 * (first + i) + 4 * g);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float e = acc[i][j] * __builtin_amdgcn_exp2f(d[j]);
            pv[4 * i + j] = i == N - 1 && diag && 4 * g + j > r ? 0.0f : e;
          }
        }
        if constexpr (T::SPLIT) {
#pragma unroll
          for (int i = 0; i < (N + 1) / 2; ++i) {  // places 32 i + 8 g .. + 7
            Frag<T> f[Sh::NP];
            parts_of<Sh::NP>(pv + 8 * i, f);
#pragma unroll
            for (int q = 0; q < Sh::NP; ++q)
              *reinterpret_cast<s8*>(pw + q * P_SIZE<T> + ((4 * i + g) ^ m) * 8) = f[q].v;
          }
        } else {  // places 8 g + 4 first .. + 3
          *reinterpret_cast<f4*>(pw + ((2 * g + first) ^ m) * 4) = f4{pv[0], pv[1], pv[2], pv[3]};
        }
        if constexpr (MODE == GRAD_Q) {
          // M: this lane's step t = t', its rows s.  Summed over s up to each, then over t'.
          f4 kq[N];
#pragma unroll
          for (int i = 0; i < N; ++i) kq[i] = f4{0.f, 0.f, 0.f, 0.f};
          const E* const zr = sh.z + (16 * first + r) * VR + 8 * g;
#pragma unroll
          for (int p = 0; p < VT / 32; ++p)
#pragma unroll
            for (int i = 0; i < N; ++i)
              kq[i] = mma(row_frag(zr + 16 * i * VR + 32 * p), af[p], kq[i]);
          float upto = 0.0f;
#pragma unroll
          for (int i = 0; i < N; ++i) {
            const bool whole = i < N - 1 || !diag;
            f4 c;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const float x = whole || 4 * g + j < r ? pv[4 * i + j] * kq[i][j] : 0.0f;
              c[j] = j ? c[j ? j - 1 : 0] + x : x;
            }
            const float other = __shfl_xor(c[3], 16), two = c[3] + other, far = __shfl_xor(two, 32);
            const float before = upto + ((g & 1 ? other : 0.0f) + (g & 2 ? far : 0.0f));
#pragma unroll
            for (int j = 0; j < 4; ++j)
              c[j] = row_sum16(whole || 4 * g + j < r ? before + c[j] : 0.0f);
            if (r == 0) *reinterpret_cast<f4*>(sh.pairs + wave * C + 16 * (first + i) + 4 * g) = c;
            upto += two + far;
          }
          if (C == 32 && !diag && g == 0) sh.rows[r] = upto;
        }
      };
      if constexpr (C == 64) {
        if (tt == 0) weigh(Count<1>(), true);
        else if (tt == 1) weigh(Count<2>(), true);
        else if (tt == 2) weigh(Count<3>(), true);
        else weigh(Count<4>(), true);
      } else if (first <= tt) {
        weigh(Count<1>(), first == tt);
      } else {
        *reinterpret_cast<f4*>(pw + ((2 * g + first) ^ m) * 4) = f4{0.f, 0.f, 0.f, 0.f};
      }
    }
    if constexpr (MODE == GRAD_Q) {
      f4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int i = 0; i < 4; ++i) sum[i] = __builtin_fmaf(S[kt][nt][i], after[kt][nt][i], sum[i]);
      float d = (sum[0] + sum[1]) + (sum[2] + sum[3]);
#pragma unroll
      for (int q = 1; q < 64; q <<= 1) d += __shfl_xor(d, q);
      if (lane == 0) sh.ends[wave] = d;
    }

    if (__builtin_expect(bad, 0)) {
      if constexpr (GRAD) {  // a or b, of the state that the chunk starts from
#pragma unroll 1
        for (int i = 0; i < cnt; ++i) {
          int vc = v0 + vb + r, kg = 8 * g;
          asm volatile("" : "+v"(vc), "+v"(kg));
          float d = 0.0f, acc[NT];
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) acc[nt] = 0.0f;
#pragma unroll
          for (int kt = 0; kt < KT; ++kt)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const int kk = kg + 32 * (kt >> 1) + 4 * (kt & 1) + j;
              if (kk < a.KK) {
                const float x = widen1(sh.x[i * KR + kk]);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) acc[nt] = __builtin_fmaf(x, S[kt][nt][j], acc[nt]);
              }
            }
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
            if (vc + 16 * nt < a.VV)
              d += acc[nt] * widen1(ap[(int64_t)(tfirst + tstep * i) * job.A.sl + vc + 16 * nt]);
          d *= job.neg ? -dec.er[i] : dec.er[i];
#pragma unroll
          for (int q = 1; q < 64; q <<= 1) d += __shfl_xor(d, q);
          if (lane == 0) sh.dots[wave * C + i] = d;
        }
      }
      // A zero weight does not silence an infinity or a NaN in a product: such a
      // chunk goes step by step, as the recurrence says, on plain arithmetic.
#pragma unroll 1
      for (int i = 0; i < cnt; ++i) {
        const float a1 = dec.g1[i];
        int vc = v0 + vb + r, kg = 8 * g;
        asm volatile("" : "+v"(vc), "+v"(kg));  // worked out here, not kept across the walk
        float xy = 0.0f, acc[NT], z[NT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          acc[nt] = 0.0f;
          z[nt] = widen1(sh.z[i * VR + vc - v0 + 16 * nt]);
        }
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int kk = kg + 32 * (kt >> 1) + 4 * (kt & 1) + j;
            if (kk < a.KK) {
              const float y = widen1(sh.y[i * KR + (T::SPLIT && (kk & 16) ? kk ^ 4 : kk)]);
              const float x = XS ? widen1(sh.x[i * KR + kk]) : 0.0f;
              xy = __builtin_fmaf(x, y, xy);
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) {
                acc[nt] = __builtin_fmaf(x, S[kt][nt][j], acc[nt]);
                S[kt][nt][j] = __builtin_fmaf(y, job.wscale * z[nt], a1 * S[kt][nt][j]);
              }
            }
          }
        if (MODE == CARRY) seg_decay *= a1;
        if (XS) {
          const int64_t t = tfirst + tstep * i;
          xy += __shfl_xor(xy, 16);
          xy += __shfl_xor(xy, 32);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            acc[nt] += __shfl_xor(acc[nt], 16);
            acc[nt] += __shfl_xor(acc[nt], 32);
            float y = a1 * job.rscale * acc[nt] + job.pabs * xy * z[nt];
            if (job.neg) y = -y;
            if (g == 0 && vc + 16 * nt < a.VV) {
              const int64_t off = ob + t * job.ol + vc + 16 * nt;
              if (T::SPLIT && !job.out_f32)
                ((uint16_t*)job.out)[off] = (uint16_t)bf16_rne(y);
              else
                ((float*)job.out)[off] = y;
            }
          }
        }
      }
      load_chunk(c + 1);
      if (wave == 0) {
        put_decays(c + 1);
        load_decays(c + 2);
      }
    } else {
      f4 O[TT][NT];
      if (wave == 0) {
        put_decays(c + 1);
        load_decays(c + 2);
      }
      // the next chunk's loads fly during the products (after X S where its operands' parts
      // leave no room for them)
      constexpr bool LATE = GRAD && NT == 2;
      if (!LATE) load_chunk(c + 1);

      // From here to the barrier the products and the vector instructions that make
      // their operands alternate, so that both units work: while the products of
      // one block run, the next one's parts are worked out.
      const LanePlace me = lane_place(tid);
      const int g = me.g, r = me.r;
      const E* const zcol = z_base<VT>(sh.z, g, r) + vb;
      const E* const ycol[2] = {y_base<KP>(sh.y, g, r, 0), y_base<KP>(sh.y, g, r, 1)};
      const E* const xrow = sh.x + r * KR + 8 * g;
      const float ec = dec.ec;
      if (MODE == CARRY) seg_decay *= ec;
      if (XS) {
#pragma unroll
        for (int i = 0; i < TT; ++i)
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) O[i][nt] = f4{0.f, 0.f, 0.f, 0.f};
      }
      if constexpr (T::SPLIT) {
        constexpr int NP = KP / 32, NW = T::NW;
        // the weighted Z of block sb: NT fragments of four pairs, each weighed (a step) and
        // split (NW steps)
        Parts<NW> wz[NT];
        Frag<T> zf[NT];
        f4 ew[2];
        constexpr int WSTEPS = NT * 4 * (NW + 1);
        auto begin_z = [&](int sb) __attribute__((always_inline)) {
          ew[0] = *reinterpret_cast<const f4*>(dec.ew + 32 * sb + 8 * g);
          ew[1] = *reinterpret_cast<const f4*>(dec.ew + 32 * sb + 8 * g + 4);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) zf[nt] = col_frag<VT>(zcol + 32 * sb * VR + 16 * nt);
        };
        auto z_steps = [&](int from, int to) __attribute__((always_inline)) {
#pragma unroll
          for (int i = from; i < to; ++i) {
            const int nt = i / (4 * (NW + 1)), j = i / (NW + 1) % 4, q = i % (NW + 1);
            if (q == 0) {
              const u4 u = __builtin_bit_cast(u4, zf[nt].v);
              wz[nt].x[j] = {bf16_lo(u[j]) * ew[j / 2][2 * (j & 1)],
                             bf16_hi(u[j]) * ew[j / 2][2 * (j & 1) + 1]};
            } else {
              wz[nt].u[q - 1][j] = wz[nt].x[j].part(q == NW);
            }
          }
        };
        begin_z(0);
        if constexpr (XS) {  // X S
          Parts<NS> sp[2][NT];  // S's rows of this block of columns and the next
          constexpr int SSTEPS = NT * 4 * NS;
          auto s_steps = [&](int p, int from, int to) __attribute__((always_inline)) {
#pragma unroll
            for (int i = from; i < to; ++i) {
              const int nt = i / (4 * NS), j = i / NS % 4, q = i % NS;
              Parts<NS>& t = sp[p & 1][nt];
              if (q == 0) t.x[j] = {S[2 * p + j / 2][nt][2 * (j & 1)], S[2 * p + j / 2][nt][2 * (j & 1) + 1]};
              t.u[q][j] = t.x[j].part(q == NS - 1);
            }
          };
          Frag<T> xf[2][TT];
#pragma unroll
          for (int i = 0; i < TT; ++i) xf[0][i] = row_frag(xrow + i * 16 * KR);
          s_steps(0, 0, SSTEPS);
          in_order();
          constexpr int M = NS * TT * NT;  // products of a block of columns
#pragma unroll
          for (int p = 0; p < NP; ++p) {
            if (p + 1 < NP)
#pragma unroll
              for (int i = 0; i < TT; ++i) xf[(p + 1) & 1][i] = row_frag(xrow + i * 16 * KR + 32 * (p + 1));
#pragma unroll
            for (int m = 0; m < M; ++m) {
              const int q = NS - 1 - m / (TT * NT), i = m / NT % TT, nt = m % NT;
              O[i][nt] = mma(sp[p & 1][nt].frag(q), xf[p & 1][i], O[i][nt]);
              if (p + 1 < NP) s_steps(p + 1, m * SSTEPS / M, (m + 1) * SSTEPS / M);
              z_steps((p * M + m) * WSTEPS / (NP * M), (p * M + m + 1) * WSTEPS / (NP * M));
              in_order();
            }
          }
        } else {
          z_steps(0, WSTEPS);
        }

        if (LATE) load_chunk(c + 1);
        // S <- e^{G_C} S + Y^T (weighted Z)
        constexpr int M = KT * NT * NW;  // products of a block of steps
        auto scale = [&](int k, int nt) __attribute__((always_inline)) { S[k][nt] *= ec; };
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          scale(0, nt);
          scale(1, nt);
        }
        Frag<T> yf[2][2];
        auto load_y = [&](int at) __attribute__((always_inline)) {  // at: sb * KT / 2 + k / 2
          const int sb = at / (KT / 2), k2 = at % (KT / 2);
#pragma unroll
          for (int k = 0; k < 2; ++k) yf[at & 1][k] = col_frag<KP>(ycol[k] + 32 * sb * KR + 32 * k2);
        };
        load_y(0);
#pragma unroll
        for (int sb = 0; sb < SB; ++sb) {
          Frag<T> wf[NT][NW];
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int q = 0; q < NW; ++q) wf[nt][q] = wz[nt].frag(q);
          if (sb + 1 < SB) begin_z(sb + 1);
          float er[TT];
          if (XS && sb + 1 == SB)
#pragma unroll
            for (int i = 0; i < TT; ++i) er[i] = dec.er[i * 16 + r];
          in_order();
#pragma unroll
          for (int k2 = 0; k2 < KT / 2; ++k2) {
            const int at = sb * (KT / 2) + k2;
            if (at + 1 < SB * (KT / 2)) load_y(at + 1);
            constexpr int MK = 2 * NT * NW;
#pragma unroll
            for (int m = 0; m < MK; ++m) {
              const int q = NW - 1 - m / (2 * NT), k = m / NT % 2, nt = m % NT;
              S[2 * k2 + k][nt] = mma(yf[at & 1][k], wf[nt][q], S[2 * k2 + k][nt]);
              const int done = k2 * MK + m;
              if (sb + 1 < SB) z_steps(done * WSTEPS / M, (done + 1) * WSTEPS / M);
              // the next rows of S, before their first product
              if (sb == 0 && k2 + 1 < KT / 2)
#pragma unroll
                for (int i = m * 2 * NT / MK; i < (m + 1) * 2 * NT / MK; ++i)
                  scale(2 * (k2 + 1) + i / NT, i % NT);
              if (XS && sb + 1 == SB)
#pragma unroll
                for (int i = done * TT * NT / M; i < (done + 1) * TT * NT / M; ++i)
                  O[i / NT][i % NT] *= er[i / NT];
              in_order();
            }
          }
        }
      } else {
        if (XS) {  // X S
#pragma unroll
          for (int p = 0; p < KP / 32; ++p) {
            Frag<T> sf[NT];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                sf[nt].v[i] = S[2 * p][nt][i];
                sf[nt].v[4 + i] = S[2 * p + 1][nt][i];
              }
#pragma unroll
            for (int i = 0; i < TT; ++i) {
              const Frag<T> xf = row_frag(xrow + i * 16 * KR + 32 * p);
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) O[i][nt] = mma(sf[nt], xf, O[i][nt]);
            }
          }
#pragma unroll
          for (int i = 0; i < TT; ++i) {
            const float er = dec.er[i * 16 + r];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) O[i][nt] *= er;
          }
        }
        if (LATE) load_chunk(c + 1);
        // S <- e^{G_C} S + Y^T (weighted Z)
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) S[kt][nt] *= ec;
        Frag<T> wf[NT];
        float ew[8];
        *reinterpret_cast<f4*>(ew) = *reinterpret_cast<const f4*>(dec.ew + 8 * g);
        *reinterpret_cast<f4*>(ew + 4) = *reinterpret_cast<const f4*>(dec.ew + 8 * g + 4);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          wf[nt] = col_frag<VT>(zcol + 16 * nt);
#pragma unroll
          for (int j = 0; j < 8; ++j) wf[nt].v[j] *= ew[j];
        }
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) {
          const Frag<T> yf = col_frag<KP>(ycol[kt & 1] + 32 * (kt >> 1));
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) S[kt][nt] = mma(yf, wf[nt], S[kt][nt]);
        }
      }

      if constexpr (GRAD) {  // a or b: O is the state's part yet
        const LanePlace me = lane_place(tid);
        const int g = me.g, r = me.r;
        const int vc = v0 + vb + 4 * g;
#pragma unroll
        for (int i = 0; i < TT; ++i) {
          const int row = i * 16 + r;
          const E* const p = ap + (int64_t)(tfirst + tstep * row) * job.A.sl + vc;
          float d = 0.0f;
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
            if (row < cnt && vc + 16 * nt < a.VV) {
              if (VEC) {
                E e[4];
                __builtin_memcpy(e, __builtin_assume_aligned(p + 16 * nt, 4 * sizeof(E)), sizeof(e));
#pragma unroll
                for (int j = 0; j < 4; ++j) d = __builtin_fmaf(O[i][nt][j], widen1(e[j]), d);
              } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                  const int last = a.VV - 1 - vc - 16 * nt;
                  const float x = widen1(p[16 * nt + min(j, last)]);
                  d = __builtin_fmaf(O[i][nt][j], j <= last ? x : 0.0f, d);
                }
              }
            }
          d += __shfl_xor(d, 16);
          d += __shfl_xor(d, 32);
          if (g == 0) sh.dots[wave * C + row] = job.neg ? -d : d;
        }
      }

      if (XS) {
        __syncthreads();  // P is whole
        const LanePlace me = lane_place(tid);
        const int g = me.g, r = me.r;
        const E* const zcol = z_base<VT>(sh.z, g, r) + vb;
#pragma unroll
        for (int sb = 0; sb < SB; ++sb) {
          Frag<T> zf[NT];
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) zf[nt] = col_frag<VT>(zcol + 32 * sb * VR + 16 * nt);
#pragma unroll
          for (int q = Sh::NP - 1; q >= 0; --q)
#pragma unroll
            for (int i = 2 * sb; i < TT; ++i) {  // steps t before the block have no weight in it
              const Frag<T> pf = p_frag(sh.p + q * P_SIZE<T>, i * 16 + r, sb, g);
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) O[i][nt] = mma(zf[nt], pf, O[i][nt]);
            }
        }

        if (job.neg) {
#pragma unroll
          for (int i = 0; i < TT; ++i)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) O[i][nt] = -O[i][nt];
        }
        // this lane: rows i * 16 + r of the chunk, columns vc + 16 nt .. + 3
        const int vc = v0 + vb + 4 * g;
#pragma unroll
        for (int i = 0; i < TT; ++i) {
          const int row = i * 16 + r;
          const int64_t t = tfirst + tstep * row;
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            const int v = vc + 16 * nt;
            const bool live = row < cnt && v < a.VV;
            if constexpr (Sh::ROWS) {
              if (job.orows) {
                const int c = 2 * (NT * wave + nt) + (g >> 1);  // its granule
                *reinterpret_cast<uint2*>(orow + row * VT + (c ^ oswz<VT>(row)) * 8 + 4 * (g & 1)) =
                    make_uint2(bf16x2_rne(O[i][nt][0], O[i][nt][1]),
                               bf16x2_rne(O[i][nt][2], O[i][nt][3]));
                continue;
              }
            }
            if (live) {
              const int64_t off = ob + t * job.ol + v;
              if (T::SPLIT && !job.out_f32) {
                uint16_t* op = (uint16_t*)job.out + off;
                const uint32_t u[2] = {bf16x2_rne(O[i][nt][0], O[i][nt][1]),
                                       bf16x2_rne(O[i][nt][2], O[i][nt][3])};
                if (job.ovec) {
                  *reinterpret_cast<uint2*>(op) = make_uint2(u[0], u[1]);
                } else {
#pragma unroll
                  for (int j = 0; j < 4; ++j)
                    if (v + j < a.VV) op[j] = (uint16_t)(u[j / 2] >> (16 * (j & 1)));
                }
              } else {
                float* op = (float*)job.out + off;
                if (job.ovec) {
                  *reinterpret_cast<f4*>(op) = O[i][nt];
                } else {
#pragma unroll
                  for (int j = 0; j < 4; ++j)
                    if (v + j < a.VV) op[j] = O[i][nt][j];
                }
              }
            }
          }
        }
      }
    }
    __syncthreads();  // the tiles are free
    if constexpr (Sh::ROWS) {
      if (job.orows && !bad) {
        constexpr int NG = VT / G;
        int id = tid;
        asm volatile("" : "+v"(id));
        const int col = id % NG * G;
#pragma unroll
        for (int i = 0; i < C * NG / THREADS; ++i) {
          const int row = id / NG + i * (THREADS / NG);
          if (row < cnt && v0 + col < a.VV)
            *reinterpret_cast<u4*>((E*)job.out + ob + (tfirst + tstep * row) * job.ol + v0 + col) =
                *reinterpret_cast<const u4*>(orow + row * VT + (col / G ^ oswz<VT>(row)) * G);
        }
        if (Sh::IN_X) __syncthreads();  // x is free
      }
    }
    if constexpr (MODE == GRAD_K) {
      if (wave == 0 && lane < cnt) {
        float d = 0.0f;
#pragma unroll
        for (int q = 0; q < 4; ++q) d += sh.dots[q * C + lane];
        job.sums[((int64_t)tile * a.H + h) * (a.B * a.L) + b * a.L + pl.first + tfirst -
                 lane] = d;
      }
    }
    if constexpr (MODE == GRAD_Q) {
      if (wave == 1) {  // lane t: step t of the chunk; its sums in 64 bits
        const int back = C - 1 - lane;  // the running sum over the steps from the last on
        double x = 0.0, y = 0.0, all, pairs = 0.0;
        if (back >= 0 && back < cnt)
          x = ((double)sh.dots[back] + sh.dots[C + back]) + ((double)sh.dots[2 * C + back] + sh.dots[3 * C + back]);
        x = wave_running_sum(x, &all);
        double v = __shfl(x, back & 63);
        if (lane > 0 && lane < cnt) {
          const int s = lane - 1;
          if (C == 64) {
            for (int q = 0; q < 4; ++q)
              if (q >= s >> 4) pairs += sh.pairs[q * C + s];
          } else if (s < 16) {
            pairs = (double)sh.pairs[s] + sh.pairs[C + s];
          } else {
            pairs = sh.pairs[3 * C + s];
          }
        }
        if constexpr (C == 32) {  // pairs of the steps before 16 and from 16 on
          if (back >= 16 && back < cnt) y = sh.rows[back - 16];
          y = wave_running_sum(y, &all);
          y = __shfl(y, back & 63);
          if (lane > 16) pairs += y;
        }
        v += job.neg ? -pairs : pairs;
        v += wave_running_sum(later, &all);
        v += ((double)sh.ends[0] + sh.ends[1] + sh.ends[2] + sh.ends[3]) * dec.ec;
        // where e^g is held at zero its derivative is zero too
        if (lane >= cnt || own_g < G_MIN) v = 0.0;
        if (job.dg && lane < cnt)
          job.dg[(b * a.L + pl.first + tfirst + lane) * job.dg_st + h * job.dg_sh + tile * job.dg_sq] =
              (float)v;
        dg_sum += v;
      }
    }
  }

  if (MODE == CARRY) {
    store_state(job.carry + (slot * a.H + h) * a.KV, 1.0f);
    if (tile == 0 && tid == 0) job.decay[slot * a.H + h] = seg_decay;
  } else if (final_seg) {
    // backwards, the initial state reaches the first step through its decay
    if (job.last)
      store_state(job.last + (pl.n * a.H + h) * a.KV,
                  rev && len > 0 ? exp2_of((double)clamp_g(gp[0]) * 1.4426950408889634) : 1.0f);
  }
  if constexpr (MODE == GRAD_Q) {
    if (job.by_slot && wave == 1) {
#pragma unroll
      for (int q = 32; q > 0; q >>= 1) dg_sum += __shfl_xor(dg_sum, q);
      if (lane == 0) job.by_slot[(slot * a.tiles + tile) * a.H + h] = dg_sum;
    }
  }
}

template <class T, int KP, int NT, bool VEC>
int launch_walk_at(const WalkArgs& a, Mode m, int64_t wgs, hipStream_t st) {
  const dim3 grid((unsigned)wgs), block(256);
  if (m == CARRY)
    hipLaunchKernelGGL((walk_kernel<T, KP, NT, CARRY, VEC>), grid, block, 0, st, a);
  else if (m == GRAD_K)
    hipLaunchKernelGGL((walk_kernel<T, KP, NT, GRAD_K, VEC>), grid, block, 0, st, a);
  else if (m == GRAD_Q)
    hipLaunchKernelGGL((walk_kernel<T, KP, NT, GRAD_Q, VEC>), grid, block, 0, st, a);
  else
    hipLaunchKernelGGL((walk_kernel<T, KP, NT, OUT, VEC>), grid, block, 0, st, a);
  return check_launch("walk_kernel");
}

// The instance: X's and Y's columns rounded up to 32, 64, 128 or 256; tiles of
// 64 nt of Z's columns (nt = 1 above 128 columns of Y: the state's registers).
template <class T, bool VEC>
int launch_walk_vec(const WalkArgs& a, Mode m, int nt, int64_t wgs, hipStream_t st) {
#define SW_WALK(KP)                                             \
  return nt == 1 ? launch_walk_at<T, KP, 1, VEC>(a, m, wgs, st) \
                 : launch_walk_at<T, KP, 2, VEC>(a, m, wgs, st)
  if (a.KK <= 32) SW_WALK(32);
  if (a.KK <= 64) SW_WALK(64);
  if (a.KK <= 128) SW_WALK(128);
  return launch_walk_at<T, 256, 1, VEC>(a, m, wgs, st);
#undef SW_WALK
}

template <class T>
int launch_walk(const WalkArgs& a, Mode m, int nt, hipStream_t st) {
  const int64_t wgs = a.slots * a.H * a.tiles * a.njobs;
  if (wgs == 0) return SW_OK;
  bool vec = true;
  for (int i = 0; i < a.njobs; ++i)
    vec = vec && (m == CARRY || a.job[i].xvec) && a.job[i].yvec && a.job[i].zvec &&
          (!is_grad(m) || a.job[i].avec) && (m != GRAD_Q || a.job[i].dvec);
  return vec ? launch_walk_vec<T, true>(a, m, nt, wgs, st)
             : launch_walk_vec<T, false>(a, m, nt, wgs, st);
}

int launch_walk_bf16(const WalkArgs& a, Mode m, int nt, hipStream_t st);
int launch_walk_f32(const WalkArgs& a, Mode m, int nt, hipStream_t st);

}  // namespace lin
}  // namespace sw
