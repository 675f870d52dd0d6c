// linear_attn.hip -- linear attention with a log decay for each head: plans
// the chunked walks of linear_walk.h, composes their segments, forms the
// decays' gradient and the sums over shared heads; and the one-step form.
#include <math.h>

#include "linear_walk.h"

namespace sw {
namespace lin {
namespace {

// Segments composed: carry (slots, H, KV) holds what each segment adds to a
// zero state, and gets each segment's initial state; 1024 elements of one
// (sequence, head) per workgroup, the segments in the walk's order.
struct FoldArgs {
  struct {
    float* carry;
    const float *decay, *init;
    bool reverse;
  } job[2];
  const int32_t* cu;
  int64_t L, nseq, H, KV, lseg, per_seq, blocks;
};

__global__ __launch_bounds__(256) void fold_kernel(FoldArgs a) {
  int64_t w = blockIdx.x;
  const int64_t blk = w % a.blocks;
  w /= a.blocks;
  const int64_t h = w % a.H;
  w /= a.H;
  const int64_t n = w % a.nseq;
  const auto& job = a.job[w / a.nseq];
  int64_t first, parts;
  if (a.cu) {
    const int64_t c0 = cu_at(a.cu, n, a.L), c1 = cu_at(a.cu, n + 1, a.L);
    first = c0 / a.lseg + n;
    parts = c1 > c0 ? (c1 - c0 + a.lseg - 1) / a.lseg : 1;
  } else {
    first = n * a.per_seq;
    parts = a.per_seq;
  }
  constexpr int U = 4;  // elements of a thread
  const int KV = (int)a.KV, e0 = (int)blk * (256 * U) + (int)threadIdx.x;
  float s[U];
  uint32_t e[U];  // past the state: its last element, read and left alone
#pragma unroll
  for (int u = 0; u < U; ++u) {
    e[u] = e0 + 256 * u < KV ? e0 + 256 * u : KV - 1;
    s[u] = job.init ? (job.init + (n * a.H + h) * a.KV)[e[u]] : 0.0f;
  }
  float* const carry = job.carry;
  const float* const decay = job.decay;
  const bool reverse = job.reverse;
  auto place = [&](int64_t j) { return (first + (reverse ? parts - 1 - j : j)) * a.H + h; };
  auto put = [&](int64_t j) __attribute__((always_inline)) {  // segment j's initial state
    float* const p = carry + place(j) * a.KV;
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (e0 + 256 * u < KV) p[e[u]] = s[u];
  };
  // The carries of N segments in flight at once, read without a branch: where few
  // heads make few workgroups, the reads' latency is what this costs (H=1 L=32996
  // K=16 V=128, 172 segments: 125 us with 4 of them, 74 with 16).  Where few are
  // left, four: 64 reads for a sequence of one or two segments took 5 us of 95.
  auto compose = [&](auto count, int64_t j0) __attribute__((always_inline)) {
    constexpr int N = decltype(count)::value;
    float c[N][U], dec[N];
#pragma unroll
    for (int d = 0; d < N; ++d) {
      const int64_t at = place(j0 + d < parts - 1 ? j0 + d : parts - 2);  // past them: not used
      dec[d] = decay[at];
      const float* const p = carry + at * a.KV;
#pragma unroll
      for (int u = 0; u < U; ++u) c[d][u] = p[e[u]];
    }
#pragma unroll
    for (int d = 0; d < N; ++d) {
      if (j0 + d >= parts - 1) break;
      put(j0 + d);
#pragma unroll
      for (int u = 0; u < U; ++u) s[u] = __builtin_fmaf(dec[d], s[u], c[d][u]);
    }
  };
  for (int64_t j = 0; j < parts - 1;) {  // the last segment hands nothing on
    if (parts - 1 - j > 4) {
      compose(Count<16>(), j);
      j += 16;
    } else {
      compose(Count<4>(), j);
      j += 4;
    }
  }
  put(parts - 1);
}

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
  return v;
}

// dg where a head's columns of q and k are several tiles: each tile's share (tile, H,
// B L) added up in order, to (B, L, H).
__global__ __launch_bounds__(256) void dg_tiles_kernel(const float* share, float* dg, int tiles,
                                                       int64_t H, int64_t T) {
  const int64_t n = H * T;
  for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < n; i += gridDim.x * 256ll) {
    double v = 0.0;
    for (int q = 0; q < tiles; ++q) v += share[q * n + i];
    const int64_t h = i / T;
    dg[(i - h * T) * H + h] = (float)v;
  }
}

// The gradient of a decay per head: the sums of segments and tiles, in a fixed order.
__global__ __launch_bounds__(64) void dg_head_kernel(const double* by_slot, float* dg,
                                                     int64_t slots, int64_t H) {
  const int64_t h = blockIdx.x;
  double s = 0.0;
  for (int64_t i = threadIdx.x; i < slots; i += 64) s += by_slot[i * H + h];
  s = wave_sum(s);
  if (threadIdx.x == 0) dg[h] = (float)s;
}

// Gradients of shared heads: rows of r * W fp32 values, summed over the r heads
// of a group in order and rounded once; dq and dk in one launch.  N columns of a
// thread: 4 where W allows (98 MB of rows: 19 us, a copy's rate; a column each 39).
struct ShareArgs {
  const float* part[2];
  void* out[2];
  int64_t groups;
  int r, W;
};
template <bool BF16, int N>
__global__ __launch_bounds__(256) void share_kernel(ShareArgs a) {
  typedef float fn __attribute__((ext_vector_type(N)));
  const float* __restrict__ part = a.part[blockIdx.y];
  const uint32_t per = (uint32_t)(a.W / N);
  const int64_t n = a.groups * per;
  for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < n; i += gridDim.x * 256ll) {
    const int64_t gi = n <= 0xffffffffll ? (int64_t)((uint32_t)i / per) : i / per;
    const int64_t c = (i - gi * per) * N;
    const float* p = part + gi * a.r * a.W + c;
    fn s = 0.0f;
    for (int j = 0; j < a.r; ++j) s += *reinterpret_cast<const fn*>(p + (int64_t)j * a.W);
    if constexpr (BF16) {
      uint16_t* o = (uint16_t*)a.out[blockIdx.y] + gi * a.W + c;
#pragma unroll
      for (int j = 0; j < N; ++j) o[j] = (uint16_t)bf16_rne(s[j]);
    } else {
      *reinterpret_cast<fn*>((float*)a.out[blockIdx.y] + gi * a.W + c) = s;
    }
  }
}

// Zeros at the steps of a packed row that no sequence covers (a row padded to a
// fixed length): before cu[0] and from cu[nseq] on, `per[i]` units of `unit` bytes a
// step of each output.  The range is known on the device only, so the launch is made
// for every packed call; where all steps are covered it ends at once.  cu == NULL:
// all L steps.
struct ClearArgs {
  void* out[4];
  int64_t per[4];
  int unit[4];
  const int32_t* cu;
  int64_t nseq, L;
};
template <class U>
__device__ __forceinline__ void clear_units(void* out, int64_t first, int64_t end) {
  U* const p = (U*)out;
  for (int64_t i = first + blockIdx.x * 256ll + threadIdx.x; i < end; i += gridDim.x * 256ll)
    p[i] = U{};
}
__global__ __launch_bounds__(256) void clear_kernel(ClearArgs a) {
  const int64_t c0 = a.cu ? cu_at(a.cu, 0, a.L) : a.L;
  const int64_t cn = a.cu ? cu_at(a.cu, a.nseq, a.L) : a.L;
  const int64_t per = a.per[blockIdx.y];
  const int unit = a.unit[blockIdx.y];
  void* const out = a.out[blockIdx.y];
  const int64_t spans[2][2] = {{0, c0}, {cn > c0 ? cn : c0, a.L}};
  for (const auto& s : spans) {
    if (unit == 16)
      clear_units<u4>(out, s[0] * per, s[1] * per);
    else if (unit == 4)
      clear_units<uint32_t>(out, s[0] * per, s[1] * per);
    else
      clear_units<uint16_t>(out, s[0] * per, s[1] * per);
  }
}

// -------------------------------------------------------------- planning

struct Plan {
  int nt_v = 1, nt_k = 1;          // tiles of 64 nt columns: of V (fwd, dv), of K (dq, dk)
  int64_t tiles_v = 1, tiles_k = 1;
  int64_t lseg = CHUNK, per_seq = 1, slots = 0;  // segments
  bool cut = false;                // some sequence may have several
  int64_t kept = 0;                // chunk ends inside sequences: dS is kept there for dg
};

// What a chunk of a walk takes, in units of one alone, where `wgs` workgroups are
// spread over the compute units: how many share one (registers and LDS), and what
// each beside the first adds.  Two side by side finish in 1.5; narrow fp32 walks,
// whose chunks are half as long and wait for one product after another, in 1.3.
double pace(int64_t wgs, int cus, int64_t contracted, int nt, bool bf16) {
  const bool narrow = contracted <= 64 && nt == 1;
  const int res = contracted > 128 ? 1 : !narrow ? 2 : bf16 ? 3 : 4;
  const double more = narrow && !bf16 ? 0.3 : 0.5;
  const int64_t load = (wgs + cus - 1) / cus;  // of the fullest compute unit
  const int64_t rounds = load / res, rest = load % res;
  return rounds * (1.0 + more * (res - 1)) + (rest ? 1.0 + more * (rest - 1) : 0.0);
}

// Segments: the count with the lowest price.  Prices in us, of a chunk of a walk
// alone on its compute unit (K = V = 128, bf16): output 5.5, carries 3, dk and dq
// with their parts of dg 22 together; a workgroup's start and end are worth one
// chunk of the kernel's (half of one for fp32), the two launches more 20 us and 0.2 for
// each segment.  Over 44 forwards and 44 backwards of all widths, lengths and both
// types, timed at every count, the count so priced took 2.8% and 1.6% more than the
// best (geometric mean): starts of two chunks, no segment below two and 12 us took 5.7%
// and 6.4%.  At B=8 L=2048 H=12 K=V=128 forward and backward take 1010 us with the
// backward's sequences whole and 612 in the parts chosen.
Plan make_plan(const LinAttnArgs& a, bool bwd, int cus) {
  Plan p;
  p.nt_v = a.V <= 64 || a.K > 128 ? 1 : 2;
  p.nt_k = a.K <= 64 || a.V > 128 ? 1 : 2;
  p.tiles_v = (a.V + 64 * p.nt_v - 1) / (64 * p.nt_v);
  p.tiles_k = (a.K + 64 * p.nt_k - 1) / (64 * p.nt_k);
  const int64_t longest = a.L, chunks = (longest + CHUNK - 1) / CHUNK;
  const int64_t rows = a.B * a.H;
  int64_t parts = 1;
  double best = 0.0;
  for (int64_t n = 1; n <= 256 && (n == 1 || n <= chunks); ++n) {
    const double len = (double)((chunks + n - 1) / n) + (a.bf16 ? 1.0 : 0.5);
    // packed: sequences end inside a segment
    const int64_t segs = a.cu ? a.H * n + 3 * a.H * a.nseq / 4 : rows * n;
    double us;
    if (bwd) {
      us = len * ((n > 1 ? 3.0 * pace(2 * segs * p.tiles_k, cus, a.V, p.nt_k, a.bf16) : 0.0) +
                  22.0 * pace(segs * p.tiles_k, cus, a.V, p.nt_k, a.bf16) +
                  5.5 * pace(segs * p.tiles_v, cus, a.K, p.nt_v, a.bf16));
    } else {
      us = len * pace(segs * p.tiles_v, cus, a.K, p.nt_v, a.bf16) * (n > 1 ? 8.5 : 5.5);
    }
    if (n > 1) us += 20.0 + 0.2 * (double)n;
    if (n == 1 || us < best) {
      best = us;
      parts = n;
    }
  }
  int64_t lseg = (chunks + parts - 1) / parts * CHUNK;
  if (lseg < CHUNK) lseg = CHUNK;
  p.lseg = lseg;
  p.cut = lseg < longest;
  p.per_seq = longest > 0 ? (longest + lseg - 1) / lseg : 1;
  p.slots = a.cu ? a.L / lseg + a.nseq : a.B * p.per_seq;
  const int64_t step = a.bf16 ? Bf16::C : F32::C;
  p.kept = !bwd || a.L == 0 ? 0 : a.cu ? a.L / step : a.B * ((a.L - 1) / step);
  return p;
}

// The workspace's parts, in bytes from its start; every one 256-byte aligned.
struct Layout {
  size_t carry[2] = {0, 0}, decay[2] = {0, 0}, kept = 0, sums = 0, share = 0, dq = 0, dk = 0,
         by_slot = 0, bytes = 0;
};

Layout make_layout(const LinAttnArgs& a, const Plan& p, bool bwd) {
  Layout l;
  auto take = [&](size_t n) {
    const size_t at = l.bytes;
    l.bytes += (n + 255) / 256 * 256;
    return at;
  };
  const size_t HKV = (size_t)(a.H * a.K * a.V), T = (size_t)(a.B * a.L);
  if (p.cut)
    for (int i = 0; i < (bwd ? 2 : 1); ++i) {
      l.carry[i] = take((size_t)p.slots * HKV * 4);
      l.decay[i] = take((size_t)(p.slots * a.H) * 4);
    }
  if (bwd) {
    const size_t rows = (size_t)(p.tiles_k * a.H) * T * 4;
    l.kept = take((size_t)p.kept * HKV * 4);
    l.sums = take(rows);
    if (p.tiles_k > 1 && !a.g_head) l.share = take(rows);
    if (a.H != a.Hk) {
      l.dq = take(T * (size_t)(a.H * a.K) * 4);
      l.dk = take(T * (size_t)(a.H * a.K) * 4);
    }
    if (a.g_head) l.by_slot = take((size_t)(p.slots * p.tiles_k * a.H) * 8);
  }
  return l;
}

// Whole 16-byte granules: the address, the strides and the width allow them, and
// a chunk's rows follow each other within a buffer load's offsets.
bool rows_vec(const HeadRows& x, int64_t width, bool bf16) {
  const int64_t G = bf16 ? 8 : 4;
  return (uintptr_t)x.p % 16 == 0 && x.sb % G == 0 && x.sl % G == 0 && x.sh % G == 0 &&
         width % G == 0 && x.sl >= width && x.sl < ((int64_t)1 << 22);
}

WalkArgs walk_args(const LinAttnArgs& a, const Plan& p) {
  WalkArgs w{};
  w.g = a.g;
  w.g_sb = a.g_head ? 0 : a.g_sb;
  w.g_sl = a.g_head ? 0 : a.g_sl;
  w.g_sh = a.g_sh;
  w.cu = a.cu;
  w.B = a.B;
  w.L = a.L;
  w.nseq = a.nseq;
  w.H = a.H;
  w.KV = a.K * a.V;
  w.lseg = p.lseg;
  w.per_seq = p.per_seq;
  w.slots = p.slots;
  w.njobs = 1;
  return w;
}

struct Role {
  HeadRows rows;
  int div;
};

// The roles of one job; `swapped`: the walk's state is (V, K).
Job make_job(const LinAttnArgs& a, const Role& X, const Role& Y, const Role& Z, bool swapped) {
  Job j{};
  const int64_t cw = swapped ? a.V : a.K, zw = swapped ? a.K : a.V;
  j.X = X.rows;
  j.Y = Y.rows;
  j.Z = Z.rows;
  if (a.L <= 1) {  // the only step's stride says nothing
    j.X.sl = j.Y.sl = cw;
    j.Z.sl = zw;
  }
  j.xdiv = X.div;
  j.ydiv = Y.div;
  j.zdiv = Z.div;
  j.adiv = 1;
  j.xvec = rows_vec(j.X, cw, a.bf16);
  j.yvec = rows_vec(j.Y, cw, a.bf16);
  j.zvec = rows_vec(j.Z, zw, a.bf16);
  j.skk = swapped ? 1 : a.V;
  j.svv = swapped ? a.V : 1;
  j.pabs = fabsf(a.scale);
  j.plog = log2((double)j.pabs);
  j.neg = a.scale < 0.0f;
  j.wscale = 1.0f;
  j.rscale = 1.0f;
  return j;
}

void set_out(Job& j, const LinAttnArgs& a, void* out, int64_t heads, int64_t width, bool f32) {
  j.out = out;
  j.oh = width;
  j.ol = heads * width;
  j.ob = a.L * j.ol;
  j.out_f32 = f32;
  j.ovec = (uintptr_t)out % 16 == 0 && width % 4 == 0;  // a lane's four columns
  j.orows = (uintptr_t)out % 16 == 0 && width % 8 == 0 && a.bf16 && !f32;
}

int launch_walk_any(const LinAttnArgs& a, WalkArgs& w, Mode m, int64_t KK, int64_t VV,
                    int nt, int64_t tiles, hipStream_t st) {
  w.KK = (int)KK;
  w.VV = (int)VV;
  w.tiles = (int)tiles;
  return a.bf16 ? launch_walk_bf16(w, m, nt, st) : launch_walk_f32(w, m, nt, st);
}

int launch_fold(const LinAttnArgs& a, const Plan& p, FoldArgs& f, int njobs, hipStream_t s) {
  f.cu = a.cu;
  f.L = a.L;
  f.nseq = a.nseq;
  f.H = a.H;
  f.KV = a.K * a.V;
  f.lseg = p.lseg;
  f.per_seq = p.per_seq;
  f.blocks = (f.KV + 1023) / 1024;
  hipLaunchKernelGGL(fold_kernel, dim3((unsigned)(f.blocks * a.H * a.nseq * njobs)), dim3(256), 0, s,
                     f);
  return check_launch("fold_kernel");
}

// An output of rows of `row` bytes a step for the next clearing launch.
void add_clear(ClearArgs& c, int* n, void* out, int64_t row) {
  const uintptr_t at = (uintptr_t)out | (uintptr_t)row;
  c.unit[*n] = at % 16 == 0 ? 16 : at % 4 == 0 ? 4 : 2;
  c.per[*n] = row / c.unit[*n];
  c.out[(*n)++] = out;
}

int launch_clear(const LinAttnArgs& a, ClearArgs& c, int n, hipStream_t s) {
  c.cu = a.H > 0 ? a.cu : nullptr;
  c.nseq = a.nseq;
  c.L = a.H > 0 ? a.L : a.B * a.L;
  hipLaunchKernelGGL(clear_kernel, dim3(256, (unsigned)n), dim3(256), 0, s, c);
  return check_launch("clear_kernel");
}

// Every launch of the call keeps within the limit.
int check_grid(const LinAttnArgs& a, const Plan& p, bool bwd) {
  const int64_t jobs = bwd ? 2 : 1, blocks = (a.K * a.V + 1023) / 1024;
  const int64_t grids[][2] = {
      {p.slots * a.H, p.tiles_v},                            // o, or dv
      {p.slots * a.H, bwd ? jobs * p.tiles_k : 0},           // dq and dk's carries
      {p.cut ? a.nseq * a.H : 0, jobs * blocks},             // the composition
  };
  for (const auto& g : grids) {
    int64_t n;
    if (__builtin_mul_overflow(g[0], g[1], &n) || n > SW_MAX_WGS)
      return fail(SW_ERR_UNSUPPORTED, "%lld segments of %lld heads exceed the launch limit",
                  (long long)p.slots, (long long)a.H);
  }
  return SW_OK;
}

// The call's workspace: the caller's, or the pool's for the call.
struct Workspace {
  char* p = nullptr;
  bool own = false;
  hipStream_t s;
  explicit Workspace(hipStream_t st) : s(st) {}
  ~Workspace() {
    if (own) workspace_free(p, s);
  }
  int get(const LinAttnArgs& a, size_t bytes, const char* what) {
    if (bytes == 0) return SW_OK;
    if (a.ws) {
      if (a.ws_bytes < bytes)
        return fail(SW_ERR_INVALID_ARG, "workspace of %zu bytes, %zu needed", a.ws_bytes, bytes);
      p = (char*)a.ws;
      return SW_OK;
    }
    int st = refuse_capture(s, what);
    if (st != SW_OK) return st;
    void* v = nullptr;
    if ((st = workspace_alloc(&v, bytes, s)) != SW_OK) return st;
    p = (char*)v;
    own = true;
    return SW_OK;
  }
};

}  // namespace
}  // namespace lin

using namespace lin;

int64_t linear_attn_fwd_workspace(const LinAttnArgs& a) {
  int cus;
  if (device_cus(&cus) != SW_OK) return 0;
  return (int64_t)make_layout(a, make_plan(a, false, cus), false).bytes;
}

int64_t linear_attn_bwd_workspace(const LinAttnArgs& a) {
  int cus;
  if (device_cus(&cus) != SW_OK) return 0;
  return (int64_t)make_layout(a, make_plan(a, true, cus), true).bytes;
}

int linear_attn_fwd(const LinAttnArgs& a) {
  int cus, st;
  if ((st = device_cus(&cus)) != SW_OK) return st;
  const Plan p = make_plan(a, false, cus);
  if ((st = check_grid(a, p, false)) != SW_OK) return st;
  const Layout l = make_layout(a, p, false);
  const hipStream_t s = current_stream();
  Workspace ws(s);
  if ((st = ws.get(a, l.bytes, "sw_linear_attn_fwd")) != SW_OK) return st;
  const int r = (int)(a.H / a.Hk);
  WalkArgs w = walk_args(a, p);
  Job j = make_job(a, {a.q, r}, {a.k, r}, {a.v, 1}, false);
  j.rscale = fabsf(a.scale);
  j.init = a.h0;
  j.last = a.h_last;
  set_out(j, a, a.o, a.H, a.V, !a.bf16);
  if (p.cut) {
    j.carry = (float*)(ws.p + l.carry[0]);
    j.decay = (float*)(ws.p + l.decay[0]);
    w.job[0] = j;
    if ((st = launch_walk_any(a, w, CARRY, a.K, a.V, p.nt_v, p.tiles_v, s)) != SW_OK) return st;
    FoldArgs f{};
    f.job[0] = {j.carry, j.decay, a.h0, false};
    if ((st = launch_fold(a, p, f, 1, s)) != SW_OK) return st;
  }
  w.job[0] = j;
  if ((st = launch_walk_any(a, w, OUT, a.K, a.V, p.nt_v, p.tiles_v, s)) != SW_OK) return st;
  if (!a.cu || a.L == 0) return SW_OK;
  ClearArgs c{};
  int n = 0;
  add_clear(c, &n, a.o, a.H * a.V * (a.bf16 ? 2 : 4));
  return launch_clear(a, c, n, s);
}

int linear_attn_bwd(const LinAttnArgs& a) {
  int cus, st;
  if ((st = device_cus(&cus)) != SW_OK) return st;
  ClearArgs c{};
  int n = 0;
  const int64_t es = a.bf16 ? 2 : 4;
  add_clear(c, &n, a.dq, a.Hk * a.K * es);
  add_clear(c, &n, a.dk, a.Hk * a.K * es);
  if (a.H == 0) return launch_clear(a, c, n, current_stream());
  const Plan p = make_plan(a, true, cus);
  if ((st = check_grid(a, p, true)) != SW_OK) return st;
  const Layout l = make_layout(a, p, true);
  const hipStream_t s = current_stream();
  Workspace ws(s);
  if ((st = ws.get(a, l.bytes, "sw_linear_attn_bwd")) != SW_OK) return st;
  const int r = (int)(a.H / a.Hk);
  const Role q{a.q, r}, k{a.k, r}, v{a.v, 1}, dout{a.dout, 1};
  const bool shared = r > 1;
  auto at = [&](size_t off) { return (float*)(ws.p + off); };

  WalkArgs w = walk_args(a, p);
  Job jq = make_job(a, dout, v, k, true);
  jq.rscale = fabsf(a.scale);
  jq.init = a.h0;
  Job jk = make_job(a, v, dout, q, true);
  jk.reverse = true;
  jk.wscale = a.scale;  // the state holds the scale with its sign
  jk.rscale = jk.neg ? -1.0f : 1.0f;
  jk.init = a.dh_last;
  Job jv = make_job(a, k, q, dout, false);
  jv.reverse = true;
  jv.wscale = a.scale;
  jv.rscale = jv.neg ? -1.0f : 1.0f;
  jv.init = a.dh_last;
  jv.last = a.dh0;
  set_out(jv, a, a.dv, a.H, a.V, !a.bf16);
  set_out(jq, a, shared ? at(l.dq) : a.dq, a.H, a.K, shared || !a.bf16);
  set_out(jk, a, shared ? at(l.dk) : a.dk, a.H, a.K, shared || !a.bf16);
  if (p.cut) {
    jq.carry = at(l.carry[0]);
    jq.decay = at(l.decay[0]);
    jk.carry = jv.carry = at(l.carry[1]);
    jk.decay = jv.decay = at(l.decay[1]);
    w.job[0] = jq;
    w.job[1] = jk;
    w.njobs = 2;
    if ((st = launch_walk_any(a, w, CARRY, a.V, a.K, p.nt_k, p.tiles_k, s)) != SW_OK) return st;
    FoldArgs f{};
    f.job[0] = {jq.carry, jq.decay, a.h0, false};
    f.job[1] = {jk.carry, jk.decay, a.dh_last, true};
    if ((st = launch_fold(a, p, f, 2, s)) != SW_OK) return st;
  }
  // dk, then dq, and their parts of dg
  jk.A = a.k;
  jk.adiv = r;
  if (a.L <= 1) jk.A.sl = a.K;
  jk.avec = rows_vec(jk.A, a.K, a.bf16);
  jk.sums = jq.sums = at(l.sums);
  jk.kept = jq.kept = at(l.kept);
  jq.A = a.q;
  jq.adiv = r;
  if (a.L <= 1) jq.A.sl = a.K;
  jq.avec = rows_vec(jq.A, a.K, a.bf16);
  jq.dlast = a.dh_last;
  jq.dvec = (uintptr_t)a.dh_last % 16 == 0;
  if (a.g_head) {
    jq.by_slot = (double*)at(l.by_slot);
  } else if (p.tiles_k == 1) {
    jq.dg = a.dg;
    jq.dg_st = a.H;
    jq.dg_sh = 1;
  } else {
    jq.dg = at(l.share);
    jq.dg_st = 1;
    jq.dg_sh = a.B * a.L;
    jq.dg_sq = a.H * jq.dg_sh;
  }
  w.njobs = 1;
  w.job[0] = jk;
  if ((st = launch_walk_any(a, w, GRAD_K, a.V, a.K, p.nt_k, p.tiles_k, s)) != SW_OK) return st;
  w.job[0] = jq;
  if ((st = launch_walk_any(a, w, GRAD_Q, a.V, a.K, p.nt_k, p.tiles_k, s)) != SW_OK) return st;
  w.job[0] = jv;
  if ((st = launch_walk_any(a, w, OUT, a.K, a.V, p.nt_v, p.tiles_v, s)) != SW_OK) return st;

  const int64_t T = a.B * a.L;
  if (a.g_head) {
    hipLaunchKernelGGL(dg_head_kernel, dim3((unsigned)a.H), dim3(64), 0, s, jq.by_slot, a.dg,
                       p.slots * p.tiles_k, a.H);
    if ((st = check_launch("dg_head_kernel")) != SW_OK) return st;
  } else if (p.tiles_k > 1 && T > 0) {
    const int64_t wgs = (T * a.H + 255) / 256 < 4096 ? (T * a.H + 255) / 256 : 4096;
    hipLaunchKernelGGL(dg_tiles_kernel, dim3((unsigned)wgs), dim3(256), 0, s, jq.dg, a.dg,
                       (int)p.tiles_k, a.H, T);
    if ((st = check_launch("dg_tiles_kernel")) != SW_OK) return st;
  }
  const int64_t groups = T * a.Hk;
  if (shared && groups > 0) {
    ShareArgs h{};
    h.part[0] = at(l.dq);
    h.part[1] = at(l.dk);
    h.out[0] = a.dq;
    h.out[1] = a.dk;
    h.groups = groups;
    h.r = r;
    h.W = (int)a.K;
    const bool four = a.K % 4 == 0 && ((uintptr_t)a.dq | (uintptr_t)a.dk) % 16 == 0;
    const int64_t n = groups * a.K / (four ? 4 : 1);
    const int64_t wgs = (n + 255) / 256 < 16384 ? (n + 255) / 256 : 16384;
    const dim3 grid((unsigned)wgs, 2), block(256);
    if (a.bf16 && four)
      hipLaunchKernelGGL((share_kernel<true, 4>), grid, block, 0, s, h);
    else if (a.bf16)
      hipLaunchKernelGGL((share_kernel<true, 1>), grid, block, 0, s, h);
    else if (four)
      hipLaunchKernelGGL((share_kernel<false, 4>), grid, block, 0, s, h);
    else
      hipLaunchKernelGGL((share_kernel<false, 1>), grid, block, 0, s, h);
    if ((st = check_launch("share_kernel")) != SW_OK) return st;
  }
  if (!a.cu || a.L == 0) return SW_OK;
  add_clear(c, &n, a.dv, a.H * a.V * es);
  if (!a.g_head) add_clear(c, &n, a.dg, a.H * 4);
  return launch_clear(a, c, n, s);
}

// ---------------------------------------------------------------- one step

namespace lin {
namespace {

// S <- e^g S + k v^T, o = scale S^T q for one (sequence, head) and tile of 4 LC
// columns: LC lanes hold four columns each of one row of S, 256 / LC rows at a
// time, so that a row of the tile is one contiguous read and write; the rows'
// parts of o meet in LDS.  Bound by the state's traffic, read and written once.
template <class E, bool VEC>
__global__ __launch_bounds__(256) void step_kernel(LinStepArgs a, int lc, int tiles) {
  __shared__ float sk[LINATTN_MAX_WIDTH], sq[LINATTN_MAX_WIDTH];
  __shared__ __align__(16) float so[1024];
  const int tid = threadIdx.x;
  uint32_t w = blockIdx.x;
  const int tile = w % (uint32_t)tiles;
  w /= (uint32_t)tiles;
  const int h = w % (uint32_t)a.H, K = (int)a.K, V = (int)a.V;
  const int64_t b = w / (uint32_t)a.H;
  const int64_t slot = a.slots ? a.slots[b] : b;
  const int hk = h / (int)(a.H / a.Hk);
  const int v0 = tile * 4 * lc, cols = V - v0 < 4 * lc ? V - v0 : 4 * lc;
  E* o = (E*)a.o + (b * a.H + h) * a.V + v0;
  auto put = [&](int c, float x) {
    if constexpr (sizeof(E) == 2)
      o[c] = (E)bf16_rne(x);
    else
      o[c] = x;
  };
  if (slot < 0 || slot >= a.pool) {
    for (int c = tid; c < cols; c += 256) put(c, 0.0f);
    return;
  }
  const int col = tid % lc * 4, row0 = tid / lc, rows = 256 / lc;
  float* S = a.state + (slot * a.H + h) * a.K * a.V + v0 + col;
  constexpr int U = 8;  // rows of a thread in flight
  f4 s[U];
  auto load = [&](int i0) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u * rows;
      s[u] = f4{0.f, 0.f, 0.f, 0.f};
      if (i < K) {
        if (VEC) {
          if (col < cols) s[u] = *reinterpret_cast<const f4*>(S + (int64_t)i * V);
        } else {
#pragma unroll
          for (int c = 0; c < 4; ++c)
            if (col + c < cols) s[u][c] = S[(int64_t)i * V + c];
        }
      }
    }
  };
  load(row0);
  const E* q = (const E*)a.q + b * a.q_sb + hk * a.q_sh;
  const E* k = (const E*)a.k + b * a.k_sb + hk * a.k_sh;
  const E* v = (const E*)a.v + b * a.v_sb + h * a.v_sh + v0 + col;
  if (tid < K) {
    sk[tid] = widen1(k[tid]);
    sq[tid] = widen1(q[tid]);
  }
  f4 vv;
#pragma unroll
  for (int c = 0; c < 4; ++c) vv[c] = col + c < cols ? widen1(v[c]) : 0.0f;
  const float dec =
      exp2_of((double)clamp_g(a.g[b * a.g_sb + h * a.g_sh]) * 1.4426950408889634);
  __syncthreads();
  f4 acc = {0.f, 0.f, 0.f, 0.f};
  for (int i0 = row0; i0 < K; i0 += U * rows) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u * rows;
      if (i < K) {
        const float kk = sk[i], qq = sq[i];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          s[u][c] = __builtin_fmaf(kk, vv[c], dec * s[u][c]);
          acc[c] = __builtin_fmaf(qq, s[u][c], acc[c]);
        }
        if (VEC) {
          if (col < cols) *reinterpret_cast<f4*>(S + (int64_t)i * V) = s[u];
        } else {
#pragma unroll
          for (int c = 0; c < 4; ++c)
            if (col + c < cols) S[(int64_t)i * V + c] = s[u][c];
        }
      }
    }
    if (i0 + U * rows < K) load(i0 + U * rows);
  }
  *reinterpret_cast<f4*>(so + row0 * 4 * lc + col) = acc;
  __syncthreads();
  if (tid < cols) {
    float x = 0.0f;
    for (int i = 0; i < rows; ++i) x += so[i * 4 * lc + tid];
    put(tid, a.scale * x);
  }
}

}  // namespace
}  // namespace lin

int linear_attn_step(const LinStepArgs& a) {
  if (a.B * a.H == 0) return SW_OK;
  int cus, st;
  if ((st = device_cus(&cus)) != SW_OK) return st;
  const bool vec = a.V % 4 == 0 && (uintptr_t)a.state % 16 == 0;
  // tiles of 128 columns, or of fewer where that leaves compute units without work
  int lc = 32;
  while (lc > 1 && 2 * lc >= a.V) lc /= 2;  // no wider than the state
  while (lc > 8 && a.B * a.H * ((a.V + 4 * lc - 1) / (4 * lc)) < 2 * (int64_t)cus) lc /= 2;
  const int64_t tiles = (a.V + 4 * lc - 1) / (4 * lc);
  const int64_t wgs = a.B * a.H * tiles;
  if (wgs > SW_MAX_WGS)
    return fail(SW_ERR_UNSUPPORTED, "%lld sequences of %lld heads exceed the launch limit",
                (long long)a.B, (long long)a.H);
  const dim3 grid((unsigned)wgs), block(256);
  const hipStream_t s = current_stream();
  if (a.bf16) {
    if (vec)
      hipLaunchKernelGGL((step_kernel<uint16_t, true>), grid, block, 0, s, a, lc, (int)tiles);
    else
      hipLaunchKernelGGL((step_kernel<uint16_t, false>), grid, block, 0, s, a, lc, (int)tiles);
  } else {
    if (vec)
      hipLaunchKernelGGL((step_kernel<float, true>), grid, block, 0, s, a, lc, (int)tiles);
    else
      hipLaunchKernelGGL((step_kernel<float, false>), grid, block, 0, s, a, lc, (int)tiles);
  }
  return check_launch("step_kernel");
}

}  // namespace sw
