// embedding_bwd.hip -- the gradient of an embedding's table: dtable[v] = scale * sum of
// dy_t over the t whose token is v.
//
// The steps are sorted by token, stably (few by counting, in one launch; many by a radix sort
// of (token, t), 11 bits a pass at most), so that a row's terms lie next to each other in the
// order of t; then every wave adds a piece of P sorted steps in fp32 and writes the rows that
// lie in it whole.  A row that crosses pieces leaves partial sums, which a last launch adds in
// order.  No atomics on sums: the same call gives the same bits.
//
// Bound by memory: dy is read once, the whole table written once.  The sort moves 8 bytes a
// step and waits on itself, so its launches carry the table's zeros beside it.
#include "norm_rows.h"
#include "token_rows.h"

namespace sw {
namespace embed {
namespace {

using norm::load8;
using norm::store8;

constexpr int MAX_BITS = 11, MAX_BINS = 1 << MAX_BITS;
constexpr int TILE = 1024, MAX_TILES = 128;  // steps a workgroup ranks at a time; workgroups
constexpr int FIX = 4;                       // pieces a workgroup of the last launch looks at

struct Entry {
  uint32_t row, t;
};

// What of the table this launch clears: 16-byte words [first, end), and in one launch the
// bytes before and behind them.
struct Clear {
  uint4* words;
  int64_t first, end;
  char *head, *tail;
  int nhead, ntail;
};
__device__ __forceinline__ void clear(const Clear& z, int64_t wg, int64_t wgs) {
  for (int64_t j = z.first + wg * blockDim.x + threadIdx.x; j < z.end; j += wgs * blockDim.x)
    z.words[j] = make_uint4(0, 0, 0, 0);
  if (wg == 0 && (int)threadIdx.x < z.nhead) z.head[threadIdx.x] = 0;
  if (wg == 0 && (int)threadIdx.x < z.ntail) z.tail[threadIdx.x] = 0;
}

struct Sort {
  Entry *in, *out;  // in NULL: the tokens themselves
  uint32_t* hist;   // (tiles, bins)
  int64_t tile;     // steps a workgroup holds, a multiple of TILE
  int tiles, shift, bits;
};

__device__ __forceinline__ Entry entry_at(const EmbedArgs& a, const Sort& s, int64_t t) {
  return s.in ? s.in[t] : Entry{row_of(a, t), (uint32_t)t};
}

// The sort of a few steps in one launch: a step's place is how many steps come before it,
// those of lower rows and the earlier ones of its own.  A workgroup holds all rows in LDS and
// places 64 steps, a lane each; its waves count over a share of the rows each.  T^2 compares,
// so only up to RANK_MOST steps for each pass of the radix sort that it spares.  (The whole
// gradient at D=256 with this sort and with the other: V=256, one pass, T=600 15 us and 19,
// 2000 17 and 20, 4096 21 and 20; V=20000, two passes, 600 15 and 29, 8192 33 and 34, 16384 54
// and 39.)
constexpr int RANK_MOST = 4096, RANK_WAVES = 8;
__global__ __launch_bounds__(RANK_WAVES * 64) void rank_kernel(EmbedArgs a, Entry* out, int share, int wgs,
                                                               Clear z) {
  if ((int)blockIdx.x >= wgs) return clear(z, blockIdx.x - wgs, gridDim.x - wgs);
  extern __shared__ uint4 rows4[];  // RANK_WAVES * share rows, those behind the last above every row
  __shared__ uint32_t counts[RANK_WAVES][64];
  uint32_t* rows = (uint32_t*)rows4;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / 64), lane = tid % 64;
  for (int j = tid; j < RANK_WAVES * share; j += RANK_WAVES * 64 * 8) {
    uint32_t r[8];  // loads in flight
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int at = j + u * RANK_WAVES * 64;
      r[u] = row_of(a, at < a.T ? at : a.T - 1);
    }
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int at = j + u * RANK_WAVES * 64;
      if (at < RANK_WAVES * share) rows[at] = at < a.T ? r[u] : ~0u;
    }
  }
  __syncthreads();
  const int t0 = blockIdx.x * 64, t = t0 + lane, first = wave * share, end = first + share;
  const uint32_t mine = t < a.T ? rows[t] : 0;
  uint32_t n = 0;
  const auto below = [&](int from, int to, uint32_t bound) {
#pragma unroll 4
    for (int j = from; j < to; j += 4) {
      const uint4 r = rows4[j / 4];
      n += (r.x < bound) + (r.y < bound) + (r.z < bound) + (r.w < bound);
    }
  };
  const int mid = min(max(t0, first), end), hi = min(max(t0 + 64, first), end);
  below(first, mid, mine + 1);
  for (int j = mid; j < hi; ++j) n += rows[j] < mine + (j < t);
  below(hi, end, mine);
  counts[wave][lane] = n;
  __syncthreads();
  if (wave == 0 && t < a.T) {
    uint32_t at = 0;
#pragma unroll
    for (int w = 0; w < RANK_WAVES; ++w) at += counts[w][lane];
    out[at] = Entry{mine, (uint32_t)t};
  }
}

// How many of a workgroup's steps have each digit.
__global__ __launch_bounds__(256) void count_kernel(EmbedArgs a, Sort s, Clear z) {
  if ((int)blockIdx.x >= s.tiles) return clear(z, blockIdx.x - s.tiles, gridDim.x - s.tiles);
  __shared__ uint32_t n[MAX_BINS];
  const int bins = 1 << s.bits;
  for (int d = threadIdx.x; d < bins; d += 256) n[d] = 0;
  __syncthreads();
  const int64_t t0 = blockIdx.x * s.tile, t1 = t0 + s.tile < a.T ? t0 + s.tile : a.T;
  for (int64_t t = t0 + threadIdx.x; t < t1; t += 256)
    atomicAdd(&n[entry_at(a, s, t).row >> s.shift & (bins - 1)], 1u);
  __syncthreads();
  for (int d = threadIdx.x; d < bins; d += 256) s.hist[(int64_t)blockIdx.x * bins + d] = n[d];
}

// Each step to its place: behind those of lower digits, of the same digit in earlier
// workgroups, in earlier waves and in earlier lanes.
__global__ __launch_bounds__(256) void place_kernel(EmbedArgs a, Sort s, Clear z) {
  if ((int)blockIdx.x >= s.tiles) return clear(z, blockIdx.x - s.tiles, gridDim.x - s.tiles);
  __shared__ uint32_t base[MAX_BINS], wave_n[4][MAX_BINS], sums[4];
  const int bins = 1 << s.bits, tid = threadIdx.x, wave = tid / 64, lane = tid % 64;
  // thread tid's bins are next to each other: their totals, then a scan over the threads
  const int per = bins > 256 ? bins / 256 : 1;
  uint32_t mine = 0;
  for (int k0 = 0; k0 < per; k0 += 2) {
    uint32_t total[2] = {}, before[2] = {};
    const int d = tid * per + k0;
    for (int q = 0; q < s.tiles; q += 32) {  // 64 counts in flight
      uint32_t n[32][2];
#pragma unroll
      for (int u = 0; u < 32; ++u)
#pragma unroll
        for (int k = 0; k < 2; ++k)
          n[u][k] = q + u < s.tiles && k0 + k < per && d + k < bins ? s.hist[(int64_t)(q + u) * bins + d + k] : 0;
#pragma unroll
      for (int u = 0; u < 32; ++u)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          total[k] += n[u][k];
          before[k] += q + u < (int)blockIdx.x ? n[u][k] : 0;
        }
    }
#pragma unroll
    for (int k = 0; k < 2; ++k)
      if (k0 + k < per && d + k < bins) {
        base[d + k] = mine + before[k];
        mine += total[k];
      }
  }
  uint32_t upto = mine;  // of the wave's threads up to this one
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const uint32_t n = __shfl_up(upto, d);
    upto += lane >= d ? n : 0;
  }
  if (lane == 63) sums[wave] = upto;
  __syncthreads();
  for (int w = 0; w < wave; ++w) upto += sums[w];
  for (int d = tid * per; d < (tid + 1) * per && d < bins; ++d) base[d] += upto - mine;

  const int64_t t0 = blockIdx.x * s.tile, t1 = t0 + s.tile < a.T ? t0 + s.tile : a.T;
  for (int64_t u = t0; u < t1; u += TILE) {
    for (int d = tid; d < 4 * bins; d += 256) wave_n[d / bins][d % bins] = 0;
    __syncthreads();
    Entry e[TILE / 256];
    uint32_t digit[TILE / 256], rank[TILE / 256];
#pragma unroll
    for (int j = 0; j < TILE / 256; ++j) {
      const int64_t t = u + wave * (TILE / 4) + j * 64 + lane;
      if (t < t1) e[j] = entry_at(a, s, t);
    }
#pragma unroll
    for (int j = 0; j < TILE / 256; ++j) {
      const bool there = u + wave * (TILE / 4) + j * 64 + lane < t1;
      digit[j] = there ? e[j].row >> s.shift & (bins - 1) : 0;
      uint64_t same = __ballot(there);
      for (int k = 0; k < s.bits; ++k) {
        const uint64_t set = __ballot(digit[j] >> k & 1);
        same &= digit[j] >> k & 1 ? set : ~set;
      }
      const uint32_t below = __popcll(same & (((uint64_t)1 << lane) - 1));
      // a wave's LDS accesses keep their order: all read before the first of them adds
      volatile uint32_t* n = &wave_n[wave][digit[j]];
      const uint32_t had = *n;
      if (there && below == 0) *n = had + (uint32_t)__popcll(same);
      rank[j] = had + below;
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < TILE / 256; ++j)
      if (u + wave * (TILE / 4) + j * 64 + lane < t1) {
        uint32_t at = base[digit[j]] + rank[j];
        for (int w = 0; w < wave; ++w) at += wave_n[w][digit[j]];
        s.out[at] = e[j];
      }
    __syncthreads();
    for (int d = tid; d < bins; d += 256)
      base[d] += wave_n[0][d] + wave_n[1][d] + wave_n[2][d] + wave_n[3][d];
    __syncthreads();
  }
}

// Where a row that crosses pieces leaves its sum: [piece][0] one that comes from the piece
// before, [piece][1] one that begins here and goes on.
__device__ __forceinline__ float* part_of(float* part, int64_t piece, int which, int64_t D) {
  return part + (piece * 2 + which) * D;
}

// LPR lanes add 8 columns each of a piece's steps.
template <class E, class Y, int LPR, bool VEC>
__global__ __launch_bounds__(256) void sum_kernel(EmbedArgs a, const Entry* sorted, float* part, int P,
                                                  int64_t pieces) {
  constexpr int U = 8;  // rows in flight
  const int li = threadIdx.x % LPR;
  const int64_t piece = blockIdx.x * (int64_t)(256 / LPR) + threadIdx.x / LPR;
  if (piece >= pieces) return;
  const int64_t c = (blockIdx.y * (int64_t)LPR + li) * 8, left = a.D - c;
  const int64_t i0 = piece * P, i1 = i0 + P < a.T ? i0 + P : a.T;
  const uint32_t V = (uint32_t)a.V;
  uint32_t row = sorted[i0].row;
  bool from = i0 > 0 && sorted[i0 - 1].row == row;
  float acc[8] = {};
  const auto flush = [&](bool on) {
    if (row == V) return;
    if (from || on) {
      store8(part_of(part, piece, from ? 0 : 1, a.D) + c, acc, left, VEC);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[j] *= a.scale;
      store8((E*)a.dtable + (int64_t)row * a.D + c, acc, left, VEC);
    }
  };
  Entry next = {};
  for (int64_t i = i0; i < i1 && row != V; i += U) {
    Entry e[U];
    float v[U][8];
    if (LPR == 64 && (i - i0) % 64 == 0) next = sorted[i + li < i1 ? i + li : i1 - 1];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if constexpr (LPR == 64) {  // a wave's piece: 64 entries in one load
        const int at = (int)(i - i0) % 64 + u;
        e[u].row = (uint32_t)__builtin_amdgcn_readlane((int)next.row, at);
        e[u].t = (uint32_t)__builtin_amdgcn_readlane((int)next.t, at);
      } else {
        e[u] = sorted[i + u < i1 ? i + u : i1 - 1];
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      load8((const Y*)a.dy + (int64_t)e[u].t * a.dy_st + c, v[u], i + u < i1 && e[u].row != V ? left : 0, VEC);
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (i + u < i1 && row != V) {
        if (e[u].row != row) {
          flush(false);
          row = e[u].row;
          from = false;
#pragma unroll
          for (int j = 0; j < 8; ++j) acc[j] = 0.0f;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[j] += v[u][j];
      }
  }
  flush(row != V && i1 < a.T && sorted[i1].row == row);
}

// The rows that begin in one piece and end in a later one: the first piece's sum and then, in
// order, those of the pieces they reach.  Each quarter of a workgroup takes a piece and 512
// columns; a row over more than SHORT pieces is left to the whole workgroup, whose 16 waves
// add every 16th piece and then their sums in order.
constexpr int SHORT = 32;
template <class E>
__device__ __forceinline__ void put_row(const EmbedArgs& a, uint32_t row, int64_t c, float v) {
  v *= a.scale;
  if constexpr (sizeof(E) == 4)
    ((float*)a.dtable)[(int64_t)row * a.D + c] = v;
  else
    ((uint16_t*)a.dtable)[(int64_t)row * a.D + c] = (uint16_t)bf16_rne(v);
}
template <class E>
__global__ __launch_bounds__(1024) void join_kernel(EmbedArgs a, const Entry* sorted, float* part, int P,
                                                    int64_t pieces) {
  __shared__ float sh[16][512];
  __shared__ int64_t lengths[FIX];  // of the rows left to all; else 0
  const int tid = threadIdx.x, wave = tid / 64, lane = tid % 64;
  const int64_t p0 = blockIdx.x * (int64_t)FIX, c0 = blockIdx.y * 512ll;
  {
    const int mine = __builtin_amdgcn_readfirstlane(tid / 256);
    const int64_t p = p0 + mine, i0 = p * P, i1 = i0 + P;
    int64_t n = 0;  // the pieces that go on with the row follow one another
    uint32_t row = 0;
    if (i1 < a.T) {
      row = sorted[i1 - 1].row;
      if (row != (uint32_t)a.V && sorted[i1].row == row &&
          (sorted[i0].row != row || i0 == 0 || sorted[i0 - 1].row != row)) {
        uint64_t more;
        do {
          const int64_t q = p + 1 + n + lane;
          more = __ballot(q < pieces && sorted[q * P].row == row);
          n += __popcll(more);
        } while (more == ~(uint64_t)0);
      }
    }
    if (tid % 256 == 0) lengths[mine] = n > SHORT ? n : 0;
    if (n > 0 && n <= SHORT) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int64_t c = c0 + k * 256 + tid % 256;
        if (c < a.D) {
          float t = part_of(part, p, 1, a.D)[c];
          for (int64_t q = 0; q < n; q += 8) {
            float v[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) v[u] = q + u < n ? part_of(part, p + 1 + q + u, 0, a.D)[c] : 0.0f;
#pragma unroll
            for (int u = 0; u < 8; ++u) t += v[u];
          }
          put_row<E>(a, row, c, t);
        }
      }
    }
  }
  __syncthreads();
  const bool vec = a.D % 8 == 0;
  for (int k = 0; k < FIX; ++k) {
    const int64_t n = lengths[k], p = p0 + k;
    if (n == 0) continue;
    float acc[8] = {};
    const int64_t c = c0 + lane * 8;
    for (int64_t q = wave; q < n; q += 16 * 8) {
      float v[8][8];
#pragma unroll
      for (int u = 0; u < 8; ++u)
        load8(part_of(part, p + 1 + q + 16 * u, 0, a.D) + c, v[u], q + 16 * u < n ? a.D - c : 0, vec);
#pragma unroll
      for (int u = 0; u < 8; ++u)
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[j] += v[u][j];
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) sh[wave][lane * 8 + j] = acc[j];
    __syncthreads();
    if (tid < 512 && c0 + tid < a.D) {
      float t = part_of(part, p, 1, a.D)[c0 + tid];
#pragma unroll
      for (int w = 0; w < 16; ++w) t += sh[w][tid];
      put_row<E>(a, sorted[(p + 1) * P - 1].row, c0 + tid, t);
    }
    __syncthreads();
  }
}

__global__ __launch_bounds__(256) void clear_kernel(Clear z) { clear(z, blockIdx.x, gridDim.x); }

struct Plan {
  int bits, passes, tiles, P;
  int64_t tile, pieces, cols;  // cols: blocks of 512 columns
  int64_t entries, hist, part, total;
};
int64_t align64(int64_t n) { return (n + 63) / 64 * 64; }
Plan plan_of(int64_t T, int64_t V, int64_t D) {
  Plan p;
  int bits = 1;
  while (V >> bits) ++bits;  // rows 0 .. V
  p.passes = (bits + MAX_BITS - 1) / MAX_BITS;
  p.bits = (bits + p.passes - 1) / p.passes;
  p.tile = (T + (int64_t)TILE * MAX_TILES - 1) / ((int64_t)TILE * MAX_TILES) * TILE;
  p.tiles = (int)((T + p.tile - 1) / p.tile);
  p.cols = (D + 511) / 512;
  // 32 steps, or pieces for some 4096 waves; where those are fewer than 1024 waves, 16 or 8.
  // (T=65536 V=256 D=512 fp32 69, 59, 57 us at 16, 32, 64 steps; T=131072 V=32000 D=256 95, 83, 87;
  // T=7800 V=17000 D=5120 121, 117, 123; the whole gradient at V=256 D=256 at 8 and 32 steps T=600
  // 19 and 26 us, 8192 20 and 25.)
  p.P = 8;
  while (p.P < 32 && T * p.cols > (int64_t)p.P * 1024) p.P *= 2;
  while (p.P >= 32 && p.P < 256 && T * p.cols > (int64_t)p.P * 4096) p.P *= 2;
  p.pieces = (T + p.P - 1) / p.P;
  p.entries = align64(T * (int64_t)sizeof(Entry));
  p.hist = align64((int64_t)p.tiles << (p.bits + 2));
  p.part = align64(p.pieces * 2 * D * 4);
  p.total = 2 * p.entries + p.hist + p.part;
  return p;
}

template <class E, class Y>
int sum_typed(const EmbedArgs& a, const Entry* sorted, float* part, const Plan& p, bool vec, hipStream_t s) {
#define CALL(LPR, VEC)                                                                                  \
  hipLaunchKernelGGL((sum_kernel<E, Y, LPR, VEC>),                                                      \
                     dim3((unsigned)((p.pieces + 256 / LPR - 1) / (256 / LPR)),                         \
                          (unsigned)((a.D + LPR * 8 - 1) / (LPR * 8))),                                 \
                     dim3(256), 0, s, a, sorted, part, p.P, p.pieces)
#define WIDTH(VEC)      \
  do {                  \
    if (a.D <= 64)      \
      CALL(8, VEC);     \
    else if (a.D <= 128) \
      CALL(16, VEC);    \
    else if (a.D <= 256) \
      CALL(32, VEC);    \
    else                \
      CALL(64, VEC);    \
  } while (0)
  if (vec)
    WIDTH(true);
  else
    WIDTH(false);
#undef WIDTH
#undef CALL
  return check_launch("embedding sum_kernel");
}

}  // namespace
}  // namespace embed

using namespace embed;

int64_t embedding_bwd_workspace(int64_t T, int64_t V, int64_t D) { return plan_of(T, V, D).total; }

int embedding_bwd(const EmbedArgs& a) {
  const hipStream_t s = current_stream();
  int cus, st;
  if ((st = device_cus(&cus)) != SW_OK) return st;
  const int64_t bytes = a.V * a.D * (a.table_bf16 ? 2 : 4);
  Clear whole = {};
  whole.head = (char*)a.dtable;
  whole.nhead = (int)(-(intptr_t)a.dtable & 15);
  if (whole.nhead > bytes) whole.nhead = (int)bytes;
  whole.words = (uint4*)(whole.head + whole.nhead);
  whole.end = (bytes - whole.nhead) / 16;
  whole.tail = (char*)(whole.words + whole.end);
  whole.ntail = (int)((bytes - whole.nhead) % 16);
  if (a.T == 0) {
    hipLaunchKernelGGL(clear_kernel, dim3(8 * cus), dim3(256), 0, s, whole);
    return check_launch("clear_kernel");
  }
  const Plan p = plan_of(a.T, a.V, a.D);
  norm::Partials mem(s);
  if ((st = mem.get(a.ws, a.ws_bytes, (size_t)p.total, "sw_embedding_bwd")) != SW_OK) return st;
  char* ws = (char*)mem.p;
  Entry* buf[2] = {(Entry*)ws, (Entry*)(ws + p.entries)};
  uint32_t* hist = (uint32_t*)(ws + 2 * p.entries);
  float* part = (float*)(ws + 2 * p.entries + p.hist);
  const bool rank = a.T <= (int64_t)RANK_MOST * p.passes;
  const int launches = rank ? 1 : 2 * p.passes;
  // each launch clears its share of the table beside its step of the sort
  const auto share = [&](int j) {
    Clear z = whole;
    z.first = whole.end * j / launches;
    z.end = whole.end * (j + 1) / launches;
    if (j) z.nhead = z.ntail = 0;
    return z;
  };
  int64_t wgs = (whole.end / launches + 1023) / 1024;
  wgs = wgs < 1 ? 1 : wgs > 8 * cus ? 8 * cus : wgs;
  const dim3 grid((unsigned)(p.tiles + wgs));
  const Entry* sorted = nullptr;
  if (rank) {
    const int steps = (int)((a.T + 63) / 64), share = (int)((a.T + RANK_WAVES * 4 - 1) / (RANK_WAVES * 4)) * 4;
    hipLaunchKernelGGL(rank_kernel, dim3((unsigned)(steps + wgs)), dim3(RANK_WAVES * 64),
                       (size_t)(RANK_WAVES * share) * 4, s, a, buf[0], share, steps, whole);
    if ((st = check_launch("rank_kernel")) != SW_OK) return st;
    sorted = buf[0];
  }
  for (int j = 0; j < (rank ? 0 : p.passes); ++j) {
    const Sort so = {j ? buf[(j + 1) % 2] : nullptr, buf[j % 2], hist, p.tile, p.tiles, j * p.bits, p.bits};
    hipLaunchKernelGGL(count_kernel, grid, dim3(256), 0, s, a, so, share(2 * j));
    if ((st = check_launch("count_kernel")) != SW_OK) return st;
    hipLaunchKernelGGL(place_kernel, grid, dim3(256), 0, s, a, so, share(2 * j + 1));
    if ((st = check_launch("place_kernel")) != SW_OK) return st;
    sorted = so.out;
  }
  const bool vec = norm::vec_rows(a.dy, a.dy_st, a.D, a.y_bf16) && norm::vec_rows(a.dtable, a.D, a.D, a.table_bf16);
  if (a.table_bf16)
    st = a.y_bf16 ? sum_typed<uint16_t, uint16_t>(a, sorted, part, p, vec, s)
                  : sum_typed<uint16_t, float>(a, sorted, part, p, vec, s);
  else
    st = a.y_bf16 ? sum_typed<float, uint16_t>(a, sorted, part, p, vec, s)
                  : sum_typed<float, float>(a, sorted, part, p, vec, s);
  if (st != SW_OK || p.pieces == 1) return st;
  const dim3 joins((unsigned)((p.pieces + FIX - 1) / FIX), (unsigned)p.cols);
  if (a.table_bf16)
    hipLaunchKernelGGL(join_kernel<uint16_t>, joins, dim3(1024), 0, s, a, sorted, part, p.P, p.pieces);
  else
    hipLaunchKernelGGL(join_kernel<float>, joins, dim3(1024), 0, s, a, sorted, part, p.P, p.pieces);
  return check_launch("join_kernel");
}

}  // namespace sw
