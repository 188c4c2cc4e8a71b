// Gated linear recurrence over time that P workers share, its adjoint, and the step of single tokens.
//
//   given gates      h_t = a_t h_{t-1} + x_t
//   sigmoid gates    h_t = a_t h_{t-1} + (1 - a_t) x_t,  a_t = 1 / (1 + exp(-g_t))
//   adjoint          d_t = dh_t + b_{t+1},  b_t = a_t d_t,  b_len = dhT,  dh_0 = b_0;  du_t = d_t,  da_t = d_t h_{t-1}
//
// Each channel is a chain of its own; along time the steps are affine maps, which compose: (A, B) after (A', B') is
// (A A', A B' + B).  So a workgroup of eight waves takes a tile of steps, L to a wave, and 64 V channels: each wave composes its steps,
// the eight maps meet in LDS, and each wave then runs its steps from the state in front of it, all from registers.  Where
// sequences and channels fill the card, a workgroup goes through all of time; where they are few, every tile is a workgroup's (below).
// The workers' boundaries are those of arrays only: a state passes them as it passes tiles.
#include <algorithm>
#include <cstddef>

#include "block8.h"
#include "buffer.h"
#include "common.h"
#include "profile.h"

namespace distdl {

constexpr int kScanInline = 16;  // workers whose pointers travel with the launch; more are in a table
constexpr int kScanWaves = 8;
constexpr int kScanV = 2;        // channels of a lane
constexpr int kScanCols = 64 * kScanV;

struct ScanWorker {
  const void *a, *x, *h, *dh;  // h: input of the adjoint
  void *o0, *o1;               // forward: h; adjoint: da, dx
};

struct ScanArgs {
  ScanWorker w[kScanInline];
  const ScanWorker* more;
  int64_t n_c;
  int32_t T, part, extra;  // worker p has part + (p < extra) steps
  int32_t P, n_b, groups;
  const int32_t* lengths;
  const float *h0, *end;  // end: dhT of the adjoint
  float *hT;              // forward: hT; adjoint: dh0
  // the kernels of few chains:
  uint64_t* words;               // tickets taken; then what the tiles publish
  uint32_t tasks, tiles;         // of all chains; of one
  uint32_t tiles_wide, tiles_rest;  // of a worker with part + 1 steps, with part
};

// Worker p's arrays, from the table or from the launch's own arguments (of which they are the first).  Read as constants, into scalar
// registers: a vector load of them would wait for all data under way, and the compiler would take what it gives for different in each lane.
// The table's address is taken in the kernel itself: the arguments' is not known in a function that the compiler might not inline.
static_assert(offsetof(ScanArgs, w) == 0, "the kernels' first argument starts with the workers");
typedef const __attribute__((address_space(4))) ScanWorker* ScanTable;
#define SCAN_TABLE(s) ((s).more ? (ScanTable)(uint64_t)(s).more : (ScanTable)__builtin_amdgcn_kernarg_segment_ptr())
__device__ __forceinline__ ScanWorker scan_worker(ScanTable table, int p) {
  const ScanTable w = table + p;
  return ScanWorker{w->a, w->x, w->h, w->dh, w->o0, w->o1};
}

struct ScanSpan {  // the worker that holds step t, and its steps
  int p, lo, hi;
};
__device__ __forceinline__ ScanSpan scan_span(const ScanArgs& s, int t) {
  const int wide = s.extra * (s.part + 1);
  ScanSpan r;
  if (t < wide) {
    r.p = (uint32_t)t / (uint32_t)(s.part + 1);
    r.lo = r.p * (s.part + 1);
    r.hi = r.lo + s.part + 1;
  } else {
    r.p = s.extra + (uint32_t)(t - wide) / (uint32_t)s.part;
    r.lo = wide + (r.p - s.extra) * s.part;
    r.hi = r.lo + s.part;
  }
  return r;
}

// The two channels of a lane in one step: neighbours in one access of twice the size (PAIR), where every row starts at a multiple of that, and
// otherwise 64 apart in two, each at its natural alignment.  Measured (us, pairs; one by one): bf16 65536 x 1024
// 102, 154, adjoint of 8 x 4096 x 2048 180, 194, of 16 x 2048 x 2048 168, 197; fp32 16 x 2048 x 2048 160, 159, its adjoint 277, 286.
template <bool PAIR>
__device__ __forceinline__ int scan_channel(int lane, int v) { return PAIR ? lane * 2 + v : lane + 64 * v; }

// Steps of one array as a wave reads and writes them: a buffer from its group's first channel of some step on, whose byte offsets are
// the lane's (the same for all steps; one that fails the check where the channel does not exist) and the step's (uniform).
// So a step costs a scalar addition and no vector ones.
struct ScanLane {
  uint32_t off[2];
  // nowhere, unless `is` (which is uniform)
  __device__ __forceinline__ ScanLane where(bool is) const { return ScanLane{{is ? off[0] : kOob, is ? off[1] : kOob}}; }
};
template <class E, bool PAIR>
__device__ __forceinline__ ScanLane scan_lane(int64_t left) {
  ScanLane l;
#pragma unroll
  for (int v = 0; v < 2; ++v) {
    const int c = scan_channel<PAIR>(threadIdx.x & 63, v);
    l.off[v] = c < left ? c * (uint32_t)sizeof(E) : kOob;
  }
  return l;
}
__device__ __forceinline__ __amdgpu_buffer_rsrc_t scan_rows(const void* p) { return rsrc_of(p, kOob); }

template <class E, bool PAIR>
struct ScanRaw {
  uint32_t v[2];
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t r, const ScanLane& l, uint32_t step) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      if constexpr (sizeof(E) == 4) v[i] = __builtin_amdgcn_raw_buffer_load_b32(r, l.off[i], step, 0);
      else v[i] = (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(r, l.off[i], step, 0);
    }
  }
  __device__ __forceinline__ void values(float* f) const {
#pragma unroll
    for (int i = 0; i < 2; ++i) f[i] = __uint_as_float(sizeof(E) == 4 ? v[i] : v[i] << 16);
  }
};
template <>
struct ScanRaw<float, true> {
  u32x2 v;
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t r, const ScanLane& l, uint32_t step) {
    v = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(r, l.off[0], step, 0));
  }
  __device__ __forceinline__ void values(float* f) const {
    f[0] = __uint_as_float(v[0]);
    f[1] = __uint_as_float(v[1]);
  }
};
template <>
struct ScanRaw<uint16_t, true> {
  uint32_t v;
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t r, const ScanLane& l, uint32_t step) {
    v = __builtin_amdgcn_raw_buffer_load_b32(r, l.off[0], step, 0);
  }
  __device__ __forceinline__ void values(float* f) const {
    f[0] = bf16_lo(v);
    f[1] = bf16_hi(v);
  }
};
template <class E, bool PAIR>
__device__ __forceinline__ void scan_put(__amdgpu_buffer_rsrc_t r, const ScanLane& l, uint32_t step, const float* v) {
  if constexpr (PAIR) {
    if constexpr (sizeof(E) == 4) __builtin_amdgcn_raw_buffer_store_b64(u32x2{__float_as_uint(v[0]), __float_as_uint(v[1])}, r, l.off[0], step, 0);
    else __builtin_amdgcn_raw_buffer_store_b32(to_bf16(v[0], v[1]), r, l.off[0], step, 0);
  } else {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      if constexpr (sizeof(E) == 4) __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(v[i]), r, l.off[i], step, 0);
      else __builtin_amdgcn_raw_buffer_store_b16(to_bf16(v[i]), r, l.off[i], step, 0);
    }
  }
}

// a = 1 / (1 + e) and 1 - a = e / (1 + e) with e = exp(-g), which keeps 1 - a where a is near one.  e is held below 2^126, so that no
// infinity meets a zero; the minimum is the one that keeps NaNs.
template <int GATE>
__device__ __forceinline__ void scan_gate(float g, float& a, float& rest) {
  if constexpr (GATE == DISTDL_GATE_GIVEN) {
    a = g;
    rest = 1.f;
  } else {
    const float e = __builtin_amdgcn_exp2f(__builtin_elementwise_minimum(g * -1.4426950408889634f, 126.f));
    a = __builtin_amdgcn_rcpf(1.f + e);
    rest = e * a;
  }
}

// The factor of a map.  Sigmoid gates are at most one, and a product of them that is lost to zero would have lost any state.  Given gates may grow and
// shrink in turn: their product is a number of 64 bits, of at most 2^1000, and so is a state on its way through maps.  What single steps keep in the
// range of 32 bits is in range there, and a state of zero, which meets no infinity, stays zero.  Measured (us; products held in the range of 32 bits before):
// 65536 x 1024 bf16 107 (102), its adjoint 186 (173), 32768 x 1024 fp32 93 (93), its adjoint 144 (140); with many chains no difference.
template <int GATE>
struct ScanProduct {
  typedef float Factor;
  float m = 1.f;
  __device__ __forceinline__ void more(float a) { m *= a; }
  __device__ __forceinline__ Factor factor() const { return m; }
};
template <>
struct ScanProduct<DISTDL_GATE_GIVEN> {
  typedef double Factor;
  float m = 1.f;  // product of mantissas of 1/2 to 1: of a wave's steps it is no less than 2^-16
  int e = 0;
  __device__ __forceinline__ void more(float a) {
    m *= __builtin_amdgcn_frexp_mantf(a);
    e += __builtin_amdgcn_frexp_expf(a);
  }
  __device__ __forceinline__ Factor factor() const { return __builtin_amdgcn_ldexp((double)m, min(e, 1000)); }
};
template <int GATE>
using ScanFactor = typename ScanProduct<GATE>::Factor;

__device__ __forceinline__ float scan_apply(float A, float state, float B) { return fmaf(A, state, B); }
__device__ __forceinline__ double scan_apply(double A, double state, float B) { return fma(A, state, (double)B); }
__device__ __forceinline__ float scan_then(float first, float then) { return first * then; }
__device__ __forceinline__ double scan_then(double first, double then) { return fmax(fmin(first * then, 0x1p1000), -0x1p1000); }

// The maps of a workgroup's waves
template <int GATE>
struct ScanMaps {
  ScanFactor<GATE> A[kScanWaves][kScanCols];
  float B[kScanWaves][kScanCols];
};

// (the compiler does not know that it is the same in all lanes, and would make every branch on it one of lanes)
__device__ __forceinline__ int scan_wave() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }

struct ScanPlace {
  int group, b, c;  // c: first channel of the group
  int n, len;       // channels of this lane; steps of the sequence
};
template <bool PAIR>
__device__ __forceinline__ ScanPlace scan_place(const ScanArgs& s, uint32_t chain) {
  ScanPlace r;
  r.group = chain % s.groups;
  r.b = chain / s.groups;
  r.c = r.group * kScanCols;
  const int64_t left = s.n_c - r.c;
  const int lane = threadIdx.x & 63;
  r.n = (scan_channel<PAIR>(lane, 0) < left) + (scan_channel<PAIR>(lane, 1) < left);
  r.len = s.lengths ? max(0, min(s.T, ((const __attribute__((address_space(4))) int32_t*)(uint64_t)s.lengths)[r.b])) : s.T;
  return r;
}

// h0, or dhT of the adjoint
template <bool PAIR>
__device__ __forceinline__ void scan_start(const ScanArgs& s, const ScanPlace& at, const float* from, float* state) {
#pragma unroll
  for (int v = 0; v < kScanV; ++v) state[v] = from && v < at.n ? from[at.b * s.n_c + at.c + scan_channel<PAIR>(threadIdx.x & 63, v)] : 0.f;
}

// The maps of all waves, each behind the one before it: `mine` is the state in front of this wave's steps, `state` that behind the tile.
template <int GATE>
__device__ __forceinline__ void scan_meet(ScanMaps<GATE>& lds, const ScanFactor<GATE>* A, const float* B, float* state, float* mine) {
  const int wave = scan_wave(), lane = threadIdx.x & 63;
#pragma unroll
  for (int v = 0; v < kScanV; ++v) {
    lds.A[wave][v * 64 + lane] = A[v];
    lds.B[wave][v * 64 + lane] = B[v];
  }
  __syncthreads();
  ScanFactor<GATE> at[kScanV], here[kScanV];
#pragma unroll
  for (int v = 0; v < kScanV; ++v) at[v] = state[v];
#pragma unroll
  for (int w = 0; w < kScanWaves; ++w) {
#pragma unroll
    for (int v = 0; v < kScanV; ++v) {
      if (w == wave) here[v] = at[v];
      at[v] = scan_apply(lds.A[w][v * 64 + lane], at[v], lds.B[w][v * 64 + lane]);
    }
  }
#pragma unroll
  for (int v = 0; v < kScanV; ++v) {
    mine[v] = here[v];
    state[v] = at[v];
  }
}

// hT, or dh0 of the adjoint
template <bool PAIR>
__device__ __forceinline__ void scan_finish(const ScanArgs& s, const ScanPlace& at, const float* state) {
  if (!s.hT) return;
  float* to = s.hT + at.b * s.n_c + at.c;
#pragma unroll
  for (int v = 0; v < kScanV; ++v)
    if (v < at.n) to[scan_channel<PAIR>(threadIdx.x & 63, v)] = state[v];
}

// A wave's steps of one tile.  Both kernels run through a tile in straight lines: steps that are not there are loads and stores that fail
// their check, so the next tile's loads are under way while this tile's waves meet and write (behind a branch the compiler
// waits for them where the branches join).  Only the arithmetic knows whole tiles from others.
struct ScanTile {
  int64_t row;          // element of its earliest step in the worker's arrays
  int next, from, lo;   // where the tile after it starts; first step; the worker's first step
  int p, cnt, live;     // worker; steps; those inside the sequence
};

template <class E, int GATE, bool PAIR>
__global__ __launch_bounds__(64 * kScanWaves) void scan_fwd_kernel(ScanArgs s) {
  constexpr int L = 8;
  __shared__ ScanMaps<GATE> lds[2];
  const ScanTable table = SCAN_TABLE(s);
  const ScanPlace at = scan_place<PAIR>(s, xcd_order(blockIdx.x, gridDim.x));
  const int wave = scan_wave();
  const ScanLane off = scan_lane<E, PAIR>(s.n_c - at.c);
  const uint32_t hop = (uint32_t)(s.n_c * sizeof(E));
  ScanRaw<E, PAIR> ra[L], rx[L];
  auto tile = [&](int t0, bool is) __attribute__((always_inline)) {
    ScanTile t;
    const ScanSpan sp = scan_span(s, t0);
    t.p = sp.p;
    t.lo = sp.lo;
    t.next = min(sp.hi, t0 + kScanWaves * L);
    t.from = t0 + wave * L;
    t.cnt = is ? max(0, min(L, t.next - t.from)) : 0;
    t.live = max(0, min(t.cnt, at.len - t.from));
    t.row = ((int64_t)at.b * (sp.hi - sp.lo) + (t.from - sp.lo)) * s.n_c + at.c;
    const ScanWorker w = scan_worker(table, t.p);
    const auto pa = scan_rows((const E*)w.a + t.row), px = scan_rows((const E*)w.x + t.row);
#pragma unroll
    for (int i = 0; i < L; ++i) {
      const ScanLane o = off.where(i < t.live);
      ra[i].load(pa, o, i * hop);
      rx[i].load(px, o, i * hop);
    }
    return t;
  };
  ScanTile t = tile(0, true);
  float state[kScanV];
  scan_start<PAIR>(s, at, s.h0, state);
  for (int turn = 0;; turn ^= 1) {
    float a[L][kScanV], u[L][kScanV], B[kScanV], h[kScanV];
    ScanFactor<GATE> A[kScanV];
#pragma unroll
    for (int i = 0; i < L; ++i) {
      float g[kScanV], x[kScanV];
      ra[i].values(g);
      rx[i].values(x);
#pragma unroll
      for (int v = 0; v < kScanV; ++v) {
        float rest;
        scan_gate<GATE>(g[v], a[i][v], rest);
        u[i][v] = rest * x[v];  // (0 where there is no step)
      }
    }
    if (t.live < L) {
#pragma unroll
      for (int i = 0; i < L; ++i)
#pragma unroll
        for (int v = 0; v < kScanV; ++v) a[i][v] = i < t.live ? a[i][v] : 1.f;
    }
#pragma unroll
    for (int v = 0; v < kScanV; ++v) {
      ScanProduct<GATE> all;
      B[v] = 0.f;  // (times the first gate as well, so that one that is not a number stays in the map)
#pragma unroll
      for (int i = 0; i < L; ++i) {
        all.more(a[i][v]);
        B[v] = fmaf(a[i][v], B[v], u[i][v]);
      }
      A[v] = all.factor();
    }
    const ScanTile now = t;
    const bool more = now.next < s.T;
    t = tile(more ? now.next : now.next - 1, more);
    scan_meet<GATE>(lds[turn], A, B, state, h);
#pragma unroll
    for (int i = 0; i < L; ++i)
#pragma unroll
      for (int v = 0; v < kScanV; ++v) u[i][v] = h[v] = fmaf(a[i][v], h[v], u[i][v]);
    if (now.live < L) {
#pragma unroll
      for (int i = 0; i < L; ++i)
#pragma unroll
        for (int v = 0; v < kScanV; ++v) u[i][v] = i < now.live ? u[i][v] : 0.f;
    }
    const auto po = scan_rows((E*)scan_worker(table, now.p).o0 + now.row);
#pragma unroll
    for (int i = 0; i < L; ++i) scan_put<E, PAIR>(po, off.where(i < now.cnt), i * hop, u[i]);
    if (!more) break;
  }
  if (wave == 0) scan_finish<PAIR>(s, at, state);
}

// Backwards in time: wave 0 has a tile's last steps, and step i of a wave is the i-th from its end.
template <class E, int GATE, bool PAIR>
__global__ __launch_bounds__(64 * kScanWaves) void scan_bwd_kernel(ScanArgs s) {
  constexpr int L = sizeof(ScanRaw<E, PAIR>) == 4 ? 8 : 4;  // what the registers hold beside the next tile's loads
  constexpr bool X = GATE != DISTDL_GATE_GIVEN;
  __shared__ ScanMaps<GATE> lds[2];
  const ScanTable table = SCAN_TABLE(s);
  const ScanPlace at = scan_place<PAIR>(s, xcd_order(blockIdx.x, gridDim.x));
  const int wave = scan_wave();
  const ScanLane off = scan_lane<E, PAIR>(s.n_c - at.c);
  const uint32_t hop = (uint32_t)(s.n_c * sizeof(E));
  ScanRaw<E, PAIR> ra[L], rx[L], rd[L], rh[L], edge;  // edge: the state before a worker's first step, the last one of the worker before
  auto tile = [&](int t1, bool is) __attribute__((always_inline)) {
    ScanTile t;
    const ScanSpan sp = scan_span(s, t1 - 1);
    t.p = sp.p;
    t.lo = sp.lo;
    t.next = max(sp.lo, t1 - kScanWaves * L);
    t.from = t1 - 1 - wave * L;  // step i: from - i
    t.cnt = is ? max(0, min(L, t.from + 1 - t.next)) : 0;
    t.live = t.cnt - max(0, min(t.cnt, t.from + 1 - at.len));  // (steps behind the sequence's end come first)
    t.row = ((int64_t)at.b * (sp.hi - sp.lo) + (t.from - t.cnt + 1 - sp.lo)) * s.n_c + at.c;
    const ScanWorker w = scan_worker(table, t.p);
    const auto pa = scan_rows((const E*)w.a + t.row), pd = scan_rows((const E*)w.dh + t.row), ph = scan_rows((const E*)w.h + t.row - s.n_c);
    const auto px = scan_rows((const E*)(X ? w.x : w.a) + t.row);
#pragma unroll
    for (int i = 0; i < L; ++i) {
      const bool in = i >= t.cnt - t.live && i < t.cnt;
      const ScanLane o = off.where(in);
      const uint32_t step = in ? (t.cnt - 1 - i) * hop : 0;
      ra[i].load(pa, o, step);
      rd[i].load(pd, o, step);
      if (X) rx[i].load(px, o, step);
      rh[i].load(ph, off.where(in && t.from - i > t.lo), step);
    }
    const bool first = t.live > 0 && t.from - t.cnt + 1 == t.lo && t.lo > 0;
    const ScanSpan b = scan_span(s, first ? t.lo - 1 : 0);
    edge.load(scan_rows((const E*)scan_worker(table, b.p).h + ((int64_t)at.b * (b.hi - b.lo) + (b.hi - b.lo - 1)) * s.n_c + at.c), off.where(first), 0);
    return t;
  };
  float start[kScanV];  // the state in front of step 0, in 32 bits
  scan_start<PAIR>(s, at, s.h0, start);
  ScanTile t = tile(s.T, true);
  float state[kScanV];
  scan_start<PAIR>(s, at, s.end, state);
  for (int turn = 0;; turn ^= 1) {
    // dx = d rest, da = d slope
    float a[L][kScanV], d[L][kScanV], rest[L][kScanV], slope[L][kScanV], B[kScanV], back[kScanV], last[kScanV];
    ScanFactor<GATE> A[kScanV];
    edge.values(last);
#pragma unroll
    for (int v = 0; v < kScanV; ++v) last[v] = t.lo == 0 ? start[v] : last[v];
#pragma unroll
    for (int i = 0; i < L; ++i) {
      float g[kScanV], x[kScanV] = {}, before[kScanV];
      ra[i].values(g);
      rd[i].values(d[i]);
      if (X) rx[i].values(x);
      rh[i].values(before);
#pragma unroll
      for (int v = 0; v < kScanV; ++v) {
        if (t.from - i == t.lo) before[v] = last[v];
        scan_gate<GATE>(g[v], a[i][v], rest[i][v]);
        slope[i][v] = X ? (before[v] - x[v]) * (a[i][v] * rest[i][v]) : before[v];
      }
    }
    if (t.live < L) {
#pragma unroll
      for (int i = 0; i < L; ++i) {
        const bool in = i >= t.cnt - t.live && i < t.cnt;
#pragma unroll
        for (int v = 0; v < kScanV; ++v) {
          a[i][v] = in ? a[i][v] : 1.f;  // (d is 0 there)
          rest[i][v] = in ? rest[i][v] : 0.f;
          slope[i][v] = in ? slope[i][v] : 0.f;
        }
      }
    }
#pragma unroll
    for (int v = 0; v < kScanV; ++v) {
      ScanProduct<GATE> all;
      all.more(a[0][v]);
      B[v] = a[0][v] * d[0][v];
#pragma unroll
      for (int i = 1; i < L; ++i) {
        all.more(a[i][v]);
        B[v] = a[i][v] * (B[v] + d[i][v]);
      }
      A[v] = all.factor();
    }
    const ScanTile now = t;
    const bool more = now.next > 0;
    t = tile(more ? now.next : now.next + 1, more);
    scan_meet<GATE>(lds[turn], A, B, state, back);
    const ScanWorker w = scan_worker(table, now.p);
    const auto o0 = scan_rows((E*)w.o0 + now.row), o1 = scan_rows((E*)w.o1 + now.row);
#pragma unroll
    for (int i = 0; i < L; ++i) {
      float da[kScanV], dx[kScanV];
#pragma unroll
      for (int v = 0; v < kScanV; ++v) {
        const float all = d[i][v] + back[v];
        back[v] = a[i][v] * all;
        const float live = i < now.cnt - now.live ? 0.f : all;  // (what passes through the steps behind a sequence's end may be infinite)
        da[v] = live * slope[i][v];
        dx[v] = live * rest[i][v];
      }
      const ScanLane o = off.where(i < now.cnt);
      const uint32_t step = i < now.cnt ? (now.cnt - 1 - i) * hop : 0;
      scan_put<E, PAIR>(o0, o, step, da);
      scan_put<E, PAIR>(o1, o, step, dx);
    }
    if (!more) break;
  }
  if (wave == 0) scan_finish<PAIR>(s, at, state);
}

// Few chains: time is split, and each tile of it is one workgroup's, which reads it once.  A workgroup keeps the tile in registers, composes its
// map and publishes that; the state in front of the tile is that in front of its run of kScanSuper tiles through the maps of the tiles before it
// in the run; the run's last tile publishes the state behind it.  So sums have one order whatever the order of the workgroups.
//
// What is published are words of a number and the pass's tag, written and read as one: a word with the tag is there, and nothing else
// has to be ordered.  Which tile a workgroup takes is decided by the ticket that it draws when it starts, tiles in the order of
// time: who waits, waits for tickets drawn before its own, so the lowest ticket not yet done never waits and every wait ends, however
// few workgroups the card holds at a time.  Tickets go on from pass to pass: their quotient by the pass's tiles is the tag.
//
// Measured (us): 65536 x 1024 bf16 on four workers 98 to 102 (4.0 to 4.1 TB/s), adjoint of 7 x 2049 x 1001 fp32 66 to 71 (4.6 to 4.9 TB/s where nothing is cut); with time
// read twice, once for the maps, 145 and 88.  What a tile takes from its workgroup's start to its stores, two at a time on a compute unit, bounds it.
// Gates made twice instead of held (tiles twice as long): 100 and 85.  Workgroups that go from tile to tile and have the next
// one's loads under way, whose loads the waits then stand behind: 133 and 83.  Four waves: 107 and 83, sixteen: 215 and 122.
constexpr int kScanSuper = 2 * kScanWaves;
// Chains at most.  Between 128 and 256 the better kernel depends on the steps as well (us, sigmoid gates, one workgroup through all of time; one for a tile): 136
// chains of 512 bf16 steps 18, 20 (adjoint 29, 30), of 2048 56, 47 (121, 99), of 8192 235, 177 (458, 356); 160 chains 18, 21 (30, 33), 57, 54 (127, 136),
// 243, 206 (483, 412); 192 chains 18, 23 (32, 37), 65, 67 (139, 133), 265, 242 (514, 505).  128 is where the second is the better or equal one for all.
constexpr int kScanFew = 128;
constexpr int kScanShort = 128;  // steps that one workgroup goes through as fast

// Steps of a wave, forwards and backwards: what 64 registers hold of them (16 for two workgroups on a compute unit, 24 for one: the same time).
constexpr int kFewSteps = 16, kFewBack = 8;

__global__ __launch_bounds__(256) void scan_clear_kernel(uint64_t* words, size_t n) {
  for (size_t i = blockIdx.x * (size_t)256 + threadIdx.x; i < n; i += gridDim.x * (size_t)256) words[i] = 0;
}

// A word: a number of 32 bits and the tag; or the upper 35 bits of one of 64, rounded (the range, and the 24 significant bits of the others), and 29 of the tag.
constexpr uint64_t kScanTag29 = (uint64_t(1) << 29) - 1;
__device__ __forceinline__ uint64_t scan_word(float v, uint32_t tag) { return (uint64_t)tag << 32 | __float_as_uint(v); }
__device__ __forceinline__ uint64_t scan_word(double v, uint32_t tag) {
  return (((uint64_t)__double_as_longlong(v) + (kScanTag29 + 1) / 2) & ~kScanTag29) | (tag & kScanTag29);
}
__device__ __forceinline__ bool scan_there(float, uint64_t word, uint32_t tag) { return (int32_t)((uint32_t)(word >> 32) - tag) >= 0; }
__device__ __forceinline__ bool scan_there(double, uint64_t word, uint32_t tag) { return (int32_t)(((uint32_t)word - tag) << 3) >= 0; }
__device__ __forceinline__ void scan_number(uint64_t word, float& v) { v = __uint_as_float((uint32_t)word); }
__device__ __forceinline__ void scan_number(uint64_t word, double& v) { v = __longlong_as_double((long long)(word & ~kScanTag29)); }

template <class F>
__device__ __forceinline__ void scan_publish(uint64_t* to, const F* v, uint32_t tag) {
#pragma unroll
  for (int i = 0; i < kScanV; ++i)
    __hip_atomic_store(to + i * 64 + (threadIdx.x & 63), scan_word(v[i], tag), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// Waits for the words of N places (a place that is null is not waited for): states, or factors (F) and sums of maps in turn.  A later tag also
// ends the wait.
template <class F, int N>
__device__ __forceinline__ void scan_await(const uint64_t* const (&from)[N], uint64_t (&w)[N][kScanV], uint32_t tag) {
  const uint64_t* lead = nullptr;  // the last of them alone first: whoever waits should not fill the memory's queues
#pragma unroll
  for (int k = 0; k < N; ++k) lead = from[k] ? from[k] : lead;
  if (lead)
    while (!__all(scan_there(0.f, __hip_atomic_load(lead + 64 + (threadIdx.x & 63), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT), tag)))
      __builtin_amdgcn_s_sleep(2);
  for (;;) {
    bool there = true;
#pragma unroll
    for (int k = 0; k < N; ++k)
#pragma unroll
      for (int i = 0; i < kScanV; ++i)
        w[k][i] = from[k] ? __hip_atomic_load(from[k] + i * 64 + (threadIdx.x & 63), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT)
                          : N > 1 && k % 2 == 0 ? scan_word(F(0), tag) : scan_word(0.f, tag);
#pragma unroll
    for (int k = 0; k < N; ++k)
#pragma unroll
      for (int i = 0; i < kScanV; ++i) there &= N > 1 && k % 2 == 0 ? scan_there(F(0), w[k][i], tag) : scan_there(0.f, w[k][i], tag);
    if (__all(there)) return;
    __builtin_amdgcn_s_sleep(1);
  }
}

struct ScanTask {
  uint32_t tag, chain, k;  // k: tile of the chain in the order of the pass
};
__device__ __forceinline__ ScanTask scan_task(const ScanArgs& s, uint32_t (&lds)[2]) {
  if (threadIdx.x == 0) {
    const uint64_t ticket = __hip_atomic_fetch_add(s.words, (uint64_t)1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    const uint64_t pass = ticket / s.tasks;
    lds[0] = (uint32_t)pass + 1;
    lds[1] = (uint32_t)(ticket - pass * s.tasks);
  }
  __syncthreads();
  const uint32_t chains = (uint32_t)s.groups * s.n_b, at = __builtin_amdgcn_readfirstlane(lds[1]);
  ScanTask t;
  t.tag = __builtin_amdgcn_readfirstlane(lds[0]);
  t.k = at / chains;
  t.chain = at - t.k * chains;
  return t;
}

// Where tile `tile` lies: its worker, the worker's steps, the tile's first one and the one behind it.
struct ScanSlice {
  int p, lo, hi, from, to;
};
__device__ __forceinline__ ScanSlice scan_slice(const ScanArgs& s, uint32_t tile, int steps) {
  const uint32_t wide = s.extra * s.tiles_wide;
  ScanSlice r;
  if (tile < wide) {
    r.p = tile / s.tiles_wide;
    tile -= r.p * s.tiles_wide;
    r.lo = r.p * (s.part + 1);
    r.hi = r.lo + s.part + 1;
  } else {
    const uint32_t q = (tile - wide) / s.tiles_rest;
    tile -= wide + q * s.tiles_rest;
    r.p = s.extra + q;
    r.lo = s.extra * (s.part + 1) + q * s.part;
    r.hi = r.lo + s.part;
  }
  r.from = r.lo + tile * steps;
  r.to = min(r.hi, r.from + steps);
  return r;
}

// From the map of each wave's steps: publishes the tile's, gives the state in front of this wave's steps and, in the last wave, that behind the tile.
template <int GATE, bool PAIR>
__device__ __forceinline__ void scan_join(const ScanArgs& s, const ScanPlace& at, const ScanTask& task, const float* from, ScanMaps<GATE>& own,
                                          ScanMaps<GATE>& run, float* front, const ScanFactor<GATE>* A, const float* B, float* mine, float* end) {
  typedef ScanFactor<GATE> F;
  const int lane = threadIdx.x & 63, wave = scan_wave();
  const uint32_t super = task.k / kScanSuper, j = task.k % kScanSuper;
  const bool closes = j == kScanSuper - 1, last = task.k == s.tiles - 1;
  uint64_t* const maps = s.words + 16 + ((size_t)task.chain * s.tiles + super * kScanSuper) * 2 * kScanCols;  // those of the run
  uint64_t* const states = s.words + 16 + (size_t)s.groups * s.n_b * s.tiles * 2 * kScanCols +
                           ((size_t)task.chain * ((s.tiles + kScanSuper - 1) / kScanSuper) + super) * kScanCols;  // the one behind the run
#pragma unroll
  for (int v = 0; v < kScanV; ++v) {
    own.A[wave][v * 64 + lane] = A[v];
    own.B[wave][v * 64 + lane] = B[v];
  }
  __syncthreads();
  if (wave == kScanWaves - 1 && !closes && !last) {
    F all[kScanV], sum[kScanV];
#pragma unroll
    for (int v = 0; v < kScanV; ++v) {
      all[v] = 1;
      sum[v] = 0;
#pragma unroll
      for (int w = 0; w < kScanWaves; ++w) {
        all[v] = scan_then(all[v], own.A[w][v * 64 + lane]);
        sum[v] = scan_apply(own.A[w][v * 64 + lane], sum[v], own.B[w][v * 64 + lane]);
      }
    }
    float last_sum[kScanV];
#pragma unroll
    for (int v = 0; v < kScanV; ++v) last_sum[v] = sum[v];
    scan_publish(maps + j * 2 * kScanCols, all, task.tag);
    scan_publish(maps + (j * 2 + 1) * kScanCols, last_sum, task.tag);
  }
  const uint32_t i = 2 * wave;  // the maps of two tiles of the run
  const uint64_t* const m = maps + i * 2 * kScanCols;
  const uint64_t* const words[4] = {i < j ? m : nullptr, i < j ? m + kScanCols : nullptr, i + 1 < j ? m + 2 * kScanCols : nullptr,
                                    i + 1 < j ? m + 3 * kScanCols : nullptr};
  uint64_t got[4][kScanV];
  scan_await<F>(words, got, task.tag);
  if (wave == 0) {
    float start[kScanV];
    const uint64_t* const before[1] = {states - kScanCols};
    uint64_t word[1][kScanV];
    if (super > 0) {
      scan_await<float>(before, word, task.tag);
#pragma unroll
      for (int v = 0; v < kScanV; ++v) scan_number(word[0][v], start[v]);
    } else {
      scan_start<PAIR>(s, at, from, start);
    }
#pragma unroll
    for (int v = 0; v < kScanV; ++v) front[v * 64 + lane] = start[v];
  }
#pragma unroll
  for (int v = 0; v < kScanV; ++v) {
    F a0, a1;
    float b0, b1;
    scan_number(got[0][v], a0);
    scan_number(got[1][v], b0);
    scan_number(got[2][v], a1);
    scan_number(got[3][v], b1);
    a0 = i < j ? a0 : F(1);  // (the others are zeros)
    a1 = i + 1 < j ? a1 : F(1);
    run.A[wave][v * 64 + lane] = scan_then(a0, a1);
    run.B[wave][v * 64 + lane] = (float)scan_apply(a1, F(b0), b1);
  }
  __syncthreads();
  F state[kScanV];
#pragma unroll
  for (int v = 0; v < kScanV; ++v) state[v] = front[v * 64 + lane];
#pragma unroll
  for (int w = 0; w < kScanWaves; ++w)
#pragma unroll
    for (int v = 0; v < kScanV; ++v) state[v] = scan_apply(run.A[w][v * 64 + lane], state[v], run.B[w][v * 64 + lane]);
#pragma unroll
  for (int w = 0; w < kScanWaves; ++w)
#pragma unroll
    for (int v = 0; v < kScanV; ++v) {
      if (w == wave) mine[v] = state[v];
      state[v] = scan_apply(own.A[w][v * 64 + lane], state[v], own.B[w][v * 64 + lane]);
    }
#pragma unroll
  for (int v = 0; v < kScanV; ++v) end[v] = state[v];
  if (wave == kScanWaves - 1) {
    if (last) scan_finish<PAIR>(s, at, end);
    else if (closes) scan_publish(states, end, task.tag);
  }
}

template <class E, int GATE, bool PAIR>
__global__ __launch_bounds__(64 * kScanWaves, 4) void scan_few_fwd_kernel(ScanArgs s) {
  constexpr int L = kFewSteps;
  __shared__ ScanMaps<GATE> own, run;
  __shared__ float front[kScanCols];
  __shared__ uint32_t drawn[2];
  const ScanTable table = SCAN_TABLE(s);
  const ScanTask task = scan_task(s, drawn);
  const ScanPlace at = scan_place<PAIR>(s, task.chain);
  const int wave = scan_wave();
  const ScanLane off = scan_lane<E, PAIR>(s.n_c - at.c);
  const uint32_t hop = (uint32_t)(s.n_c * sizeof(E));
  const ScanSlice t = scan_slice(s, task.k, kScanWaves * L);
  const int first = t.from + wave * L, cnt = max(0, min(L, t.to - first)), live = max(0, min(cnt, at.len - first));
  const int64_t row = ((int64_t)at.b * (t.hi - t.lo) + (first - t.lo)) * s.n_c + at.c;
  const ScanWorker w = scan_worker(table, t.p);
  const auto pa = scan_rows((const E*)w.a + row), px = scan_rows((const E*)w.x + row), po = scan_rows((E*)w.o0 + row);
  ScanRaw<E, PAIR> ra[L], rx[L];
#pragma unroll
  for (int i = 0; i < L; ++i) {
    const ScanLane o = off.where(i < live);
    ra[i].load(pa, o, i * hop);
    rx[i].load(px, o, i * hop);
  }
  float a[L][kScanV], u[L][kScanV], B[kScanV], h[kScanV], end[kScanV];
  ScanFactor<GATE> A[kScanV];
#pragma unroll
  for (int i = 0; i < L; ++i) {
    float g[kScanV], x[kScanV];
    ra[i].values(g);
    rx[i].values(x);
#pragma unroll
    for (int v = 0; v < kScanV; ++v) {
      float rest;
      scan_gate<GATE>(g[v], a[i][v], rest);
      u[i][v] = rest * x[v];  // (0 where there is no step)
    }
  }
  if (live < L) {
#pragma unroll
    for (int i = 0; i < L; ++i)
#pragma unroll
      for (int v = 0; v < kScanV; ++v) a[i][v] = i < live ? a[i][v] : 1.f;
  }
#pragma unroll
  for (int v = 0; v < kScanV; ++v) {
    ScanProduct<GATE> all;
    B[v] = 0.f;
#pragma unroll
    for (int i = 0; i < L; ++i) {
      all.more(a[i][v]);
      B[v] = fmaf(a[i][v], B[v], u[i][v]);
    }
    A[v] = all.factor();
  }
  scan_join<GATE, PAIR>(s, at, task, s.h0, own, run, front, A, B, h, end);
#pragma unroll
  for (int i = 0; i < L; ++i)
#pragma unroll
    for (int v = 0; v < kScanV; ++v) u[i][v] = h[v] = fmaf(a[i][v], h[v], u[i][v]);
  if (live < L) {
#pragma unroll
    for (int i = 0; i < L; ++i)
#pragma unroll
      for (int v = 0; v < kScanV; ++v) u[i][v] = i < live ? u[i][v] : 0.f;
  }
#pragma unroll
  for (int i = 0; i < L; ++i) scan_put<E, PAIR>(po, off.where(i < cnt), i * hop, u[i]);
}

// Backwards in time: tile 0 and wave 0 have the last steps, and step i of a wave is the i-th from its end.
template <class E, int GATE, bool PAIR>
__global__ __launch_bounds__(64 * kScanWaves, 4) void scan_few_bwd_kernel(ScanArgs s) {
  constexpr int L = kFewBack;
  constexpr bool X = GATE != DISTDL_GATE_GIVEN;
  __shared__ ScanMaps<GATE> own, run;
  __shared__ float front[kScanCols];
  __shared__ uint32_t drawn[2];
  const ScanTable table = SCAN_TABLE(s);
  const ScanTask task = scan_task(s, drawn);
  const ScanPlace at = scan_place<PAIR>(s, task.chain);
  const int wave = scan_wave();
  const ScanLane off = scan_lane<E, PAIR>(s.n_c - at.c);
  const uint32_t hop = (uint32_t)(s.n_c * sizeof(E));
  const ScanSlice t = scan_slice(s, s.tiles - 1 - task.k, kScanWaves * L);
  const int from = t.to - 1 - wave * L, cnt = max(0, min(L, from + 1 - t.from));  // step i: from - i
  const int dead = max(0, min(cnt, from + 1 - at.len));                           // steps behind the sequence's end; they come first
  const int64_t row = ((int64_t)at.b * (t.hi - t.lo) + (from - cnt + 1 - t.lo)) * s.n_c + at.c;
  const ScanWorker w = scan_worker(table, t.p);
  const auto pa = scan_rows((const E*)w.a + row), pd = scan_rows((const E*)w.dh + row), ph = scan_rows((const E*)w.h + row - s.n_c);
  const auto px = scan_rows((const E*)(X ? w.x : w.a) + row), o0 = scan_rows((E*)w.o0 + row), o1 = scan_rows((E*)w.o1 + row);
  ScanRaw<E, PAIR> ra[L], rx[L], rd[L], rh[L], edge;  // edge: the state before a worker's first step, the last one of the worker before
#pragma unroll
  for (int i = 0; i < L; ++i) {
    const bool in = i >= dead && i < cnt;
    const ScanLane o = off.where(in);
    const uint32_t step = in ? (cnt - 1 - i) * hop : 0;
    ra[i].load(pa, o, step);
    rd[i].load(pd, o, step);
    if (X) rx[i].load(px, o, step);
    rh[i].load(ph, off.where(in && from - i > t.lo), step);
  }
  const bool edged = cnt > dead && from - cnt + 1 == t.lo && t.lo > 0;
  const ScanSpan b = scan_span(s, edged ? t.lo - 1 : 0);
  edge.load(scan_rows((const E*)scan_worker(table, b.p).h + ((int64_t)at.b * (b.hi - b.lo) + (b.hi - b.lo - 1)) * s.n_c + at.c), off.where(edged), 0);
  float last[kScanV];  // the state in front of a worker's first step, of the first worker in 32 bits
  if (t.lo == 0) scan_start<PAIR>(s, at, s.h0, last);
  // dx = d rest, da = d slope
  float a[L][kScanV], d[L][kScanV], rest[L][kScanV], slope[L][kScanV], B[kScanV], back[kScanV], end[kScanV];
  ScanFactor<GATE> A[kScanV];
  if (t.lo > 0) edge.values(last);
#pragma unroll
  for (int i = 0; i < L; ++i) {
    float g[kScanV], x[kScanV] = {}, before[kScanV];
    ra[i].values(g);
    rd[i].values(d[i]);
    if (X) rx[i].values(x);
    rh[i].values(before);
#pragma unroll
    for (int v = 0; v < kScanV; ++v) {
      if (from - i == t.lo) before[v] = last[v];
      scan_gate<GATE>(g[v], a[i][v], rest[i][v]);
      slope[i][v] = X ? (before[v] - x[v]) * (a[i][v] * rest[i][v]) : before[v];
    }
  }
  if (dead > 0 || cnt < L) {
#pragma unroll
    for (int i = 0; i < L; ++i) {
      const bool in = i >= dead && i < cnt;
#pragma unroll
      for (int v = 0; v < kScanV; ++v) {
        a[i][v] = in ? a[i][v] : 1.f;  // (d is 0 there)
        rest[i][v] = in ? rest[i][v] : 0.f;
        slope[i][v] = in ? slope[i][v] : 0.f;
      }
    }
  }
#pragma unroll
  for (int v = 0; v < kScanV; ++v) {
    ScanProduct<GATE> all;
    B[v] = 0.f;
#pragma unroll
    for (int i = 0; i < L; ++i) {
      all.more(a[i][v]);
      B[v] = a[i][v] * (B[v] + d[i][v]);
    }
    A[v] = all.factor();
  }
  scan_join<GATE, PAIR>(s, at, task, s.end, own, run, front, A, B, back, end);
#pragma unroll
  for (int i = 0; i < L; ++i) {
    float da[kScanV], dx[kScanV];
#pragma unroll
    for (int v = 0; v < kScanV; ++v) {
      const float all = d[i][v] + back[v];
      back[v] = a[i][v] * all;
      const float live = i < dead ? 0.f : all;  // (what passes through the steps behind a sequence's end may be infinite)
      da[v] = live * slope[i][v];
      dx[v] = live * rest[i][v];
    }
    const ScanLane o = off.where(i < cnt);
    const uint32_t step = i < cnt ? (cnt - 1 - i) * hop : 0;
    scan_put<E, PAIR>(o0, o, step, da);
    scan_put<E, PAIR>(o1, o, step, dx);
  }
}

// One token of each row: its state lies at row slots[row] of the pool.  A row without a slot of the pool is idle.
template <class E, int GATE>
__global__ __launch_bounds__(256) void scan_step_kernel(const E* __restrict__ a, const E* __restrict__ x, float* __restrict__ state,
                                                        const int32_t* __restrict__ slots, E* __restrict__ h, int64_t n_slots,
                                                        int64_t n_c) {
  const int64_t row = blockIdx.y, c = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
  if (c >= n_c) return;
  const int n = (int)min((int64_t)8, n_c - c);
  const int64_t slot = slots ? slots[row] : row, o = row * n_c + c;
  float out[8] = {};
  if (slot >= 0 && slot < n_slots) {
    float* const at = state + slot * n_c + c;
    Eight<E> ra, rx;
    Eight<float> rs;
    ra.load(a + o, n);
    rx.load(x + o, n);
    rs.load(at, n);
    float g[8], u[8];
    ra.values(g);
    rx.values(u);
    rs.values(out);
#pragma unroll
    for (int v = 0; v < 8; ++v) {
      float f, rest;
      scan_gate<GATE>(g[v], f, rest);
      out[v] = fmaf(f, out[v], rest * u[v]);
    }
    store8(at, out, n);
  }
  store8(h + o, out, n);
}

}  // namespace distdl

struct distdl_scan_plan {
  int64_t n_b = 0, T = 0, n_c = 0;
  int P = 1, gate = 0;
  distdl_dtype dtype = DISTDL_F32;
  int groups = 1;
  bool few = false;  // chains, so that time has to be split
  distdl::DevArray<distdl::ScanWorker> table;
  distdl::StreamScratch words[2][2];  // by direction and kind of tiles, which have numbers of their own
};

namespace distdl {

static int scan_check(const void* v, size_t size, const char* what, int j) {
  if (!v) return set_error(DISTDL_ERR_NULL, "scan: %s[%d] is null", what, j);
  if ((uintptr_t)v % size) return set_error(DISTDL_ERR_INVALID_ARG, "scan: %s[%d] is not aligned to its elements", what, j);
  return DISTDL_OK;
}

static int scan_args(distdl_scan_plan* p, const std::vector<ScanWorker>& w, hipStream_t st, ScanArgs* s) {
  s->more = nullptr;
  s->T = (int32_t)p->T;
  s->n_c = p->n_c;
  s->part = (int32_t)(p->T / p->P);
  s->extra = (int32_t)(p->T % p->P);
  s->P = p->P;
  s->n_b = (int32_t)p->n_b;
  s->groups = p->groups;
  int rc = DISTDL_OK;
  if (p->P <= kScanInline) {
    std::copy(w.begin(), w.end(), s->w);
  } else {
    if ((rc = p->table.upload(w, st))) return rc;
    s->more = p->table.dev;
  }
  return rc;
}

// What the tiles of `steps` steps publish.  The memory starts as zeros, the tag of no pass; a recorded pass cannot see to that.
static int scan_words(StreamScratch& scratch, int steps, hipStream_t st, ScanArgs* s) {
  s->tiles_wide = (s->part + 1 + steps - 1) / steps;
  s->tiles_rest = (s->part + steps - 1) / steps;
  s->tiles = s->extra * s->tiles_wide + (s->P - s->extra) * s->tiles_rest;
  const int64_t chains = (int64_t)s->groups * s->n_b, supers = (s->tiles + kScanSuper - 1) / kScanSuper;
  s->tasks = (uint32_t)(chains * s->tiles);
  const size_t words = 16 + (size_t)chains * (2 * (int64_t)s->tiles + supers) * kScanCols;
  bool is_new = true;
  for (const StreamScratch::Block& b : scratch.blocks) is_new = is_new && b.stream != st;
  if (is_new) {
    hipStreamCaptureStatus capture = hipStreamCaptureStatusNone;
    DISTDL_HIP_TRY(hipStreamIsCapturing(st, &capture));
    if (capture != hipStreamCaptureStatusNone)
      return set_error(DISTDL_ERR_INVALID_ARG, "scan: the plan's first call on this stream, which is being captured");
  }
  float* at = nullptr;
  const int rc = scratch.get(2 * words, st, &at);
  if (rc) return rc;
  s->words = (uint64_t*)at;
  if (is_new)
    hipLaunchKernelGGL(scan_clear_kernel, dim3((unsigned)std::min<size_t>((words + 255) / 256, 4096)), dim3(256), 0, st, s->words, words);
  DISTDL_HIP_TRY(hipGetLastError());
  return DISTDL_OK;
}

template <class E, int GATE, bool PAIR>
static int launch_scan(distdl_scan_plan* p, ScanArgs& s, bool back, hipStream_t st) {
  const dim3 block(64 * kScanWaves);
  if (p->few) {
    const int rc = scan_words(p->words[back][PAIR], kScanWaves * (back ? kFewBack : kFewSteps), st, &s);
    if (rc) return rc;
    if (back) hipLaunchKernelGGL((scan_few_bwd_kernel<E, GATE, PAIR>), dim3(s.tasks), dim3(64 * kScanWaves), 0, st, s);
    else hipLaunchKernelGGL((scan_few_fwd_kernel<E, GATE, PAIR>), dim3(s.tasks), dim3(64 * kScanWaves), 0, st, s);
  } else {
    const dim3 grid((unsigned)((int64_t)s.groups * s.n_b));
    if (back) hipLaunchKernelGGL((scan_bwd_kernel<E, GATE, PAIR>), grid, block, 0, st, s);
    else hipLaunchKernelGGL((scan_fwd_kernel<E, GATE, PAIR>), grid, block, 0, st, s);
  }
  return DISTDL_OK;
}

// Whether every row of every array starts at a multiple of two elements.
static bool scan_pairs(const distdl_scan_plan* p, const std::vector<ScanWorker>& w) {
  uintptr_t bits = (uintptr_t)(p->n_c * (int64_t)dtype_size(p->dtype));
  for (const ScanWorker& v : w) bits |= (uintptr_t)v.a | (uintptr_t)v.x | (uintptr_t)v.h | (uintptr_t)v.dh | (uintptr_t)v.o0 | (uintptr_t)v.o1;
  return bits % (2 * dtype_size(p->dtype)) == 0;
}

template <class F>
static void scan_kind(distdl_dtype dtype, int gate, F f) {
  typedef std::integral_constant<int, DISTDL_GATE_GIVEN> Given;
  typedef std::integral_constant<int, DISTDL_GATE_SIGMOID> Sigmoid;
  if (dtype == DISTDL_F32) {
    if (gate == DISTDL_GATE_GIVEN) f(float(), Given());
    else f(float(), Sigmoid());
  } else {
    if (gate == DISTDL_GATE_GIVEN) f(uint16_t(), Given());
    else f(uint16_t(), Sigmoid());
  }
}

}  // namespace distdl

using namespace distdl;

extern "C" {

int distdl_scan_plan_create(distdl_scan_plan** out, int64_t n_b, int64_t T, int64_t n_c, int P, distdl_gate gate, distdl_dtype dtype) {
  if (!out) return set_error(DISTDL_ERR_NULL, "scan_plan_create: null argument");
  *out = nullptr;
  if (n_b < 1 || T < 1 || n_c < 1 || P < 1) return set_error(DISTDL_ERR_INVALID_ARG, "scan_plan_create: sizes must be >= 1");
  if (gate != DISTDL_GATE_GIVEN && gate != DISTDL_GATE_SIGMOID) return set_error(DISTDL_ERR_UNSUPPORTED, "unknown gate");
  if (dtype != DISTDL_F32 && dtype != DISTDL_BF16) return set_error(DISTDL_ERR_UNSUPPORTED, "unknown dtype");
  if (T < P) return set_error(DISTDL_ERR_EMPTY_PARTITION, "scan: %lld steps over %d workers", (long long)T, P);
  const int64_t groups = (n_c + kScanCols - 1) / kScanCols;
  if (T >= int64_t(1) << 30 || n_c >= int64_t(1) << 25 ||  // (a tile of one wave is addressed in 31 bits)
       n_b >= int64_t(1) << 22 || groups * n_b >= int64_t(1) << 22)
    return set_error(DISTDL_ERR_UNSUPPORTED, "scan: problem too large");
  return guarded([&]() -> int {
    std::unique_ptr<distdl_scan_plan> p(new distdl_scan_plan());
    p->n_b = n_b;
    p->T = T;
    p->n_c = n_c;
    p->P = P;
    p->gate = gate;
    p->dtype = dtype;
    p->groups = (int)groups;
    // Measured (us, one workgroup through all of time; one for a tile): 67 million bf16 steps in 128 chains 123, 104 (adjoint 223, 187), in
    // 256 chains 84, 95 (167, 174); 32 chains of 128 steps 6.5, 6.8 (9.7, 7.8), of 256 9.9, 7.7 (15.6, 8.9), of 1024 30, 11 (49, 18); 8 chains of
    // 4096 steps on 128 workers 232, 28 (410, 29).  A worker has eight steps at least, so that what tiles publish (2 KiB each) is no more than an array.
    p->few = groups * n_b <= kScanFew && T > kScanShort && T / P >= 8 && groups * n_b * (T / 64 + P) < int64_t(1) << 30;
    *out = p.release();
    return DISTDL_OK;
  });
}

int distdl_scan_plan_destroy(distdl_scan_plan* p) {
  if (!p) return DISTDL_OK;
  p->table.release();
  for (auto& of : p->words)
    for (auto& w : of) w.release();
  delete p;
  return DISTDL_OK;
}

int distdl_scan_fwd(distdl_scan_plan* p, const void* const a_dev[], const void* const x_dev[], const float* h0_dev,
                    const int32_t* lengths_dev, void* const h_dev[], float* hT_dev, void* stream) {
  if (!p || !a_dev || !x_dev || !h_dev) return set_error(DISTDL_ERR_NULL, "scan_fwd: null argument");
  if ((uintptr_t)h0_dev % 4 || (uintptr_t)lengths_dev % 4 || (uintptr_t)hT_dev % 4)
    return set_error(DISTDL_ERR_INVALID_ARG, "scan_fwd: h0, lengths or hT is not aligned to its elements");
  return guarded([&]() -> int {
    const size_t size = dtype_size(p->dtype);
    std::vector<ScanWorker> w((size_t)p->P);
    int rc;
    for (int j = 0; j < p->P; ++j) {
      if ((rc = scan_check(a_dev[j], size, "a", j)) || (rc = scan_check(x_dev[j], size, "x", j)) || (rc = scan_check(h_dev[j], size, "h", j)))
        return rc;
      w[j] = ScanWorker{a_dev[j], x_dev[j], nullptr, nullptr, h_dev[j], nullptr};
    }
    hipStream_t st_ = (hipStream_t)stream;
    ScanArgs s;
    if ((rc = scan_args(p, w, st_, &s))) return rc;
    s.lengths = lengths_dev;
    s.h0 = h0_dev;
    s.end = nullptr;
    s.hT = hT_dev;
    {
      ProfScope prof("scan_fwd", st_);
      scan_kind(p->dtype, p->gate, [&](auto e, auto gate) {
        rc = scan_pairs(p, w) ? launch_scan<decltype(e), decltype(gate)::value, true>(p, s, false, st_)
                              : launch_scan<decltype(e), decltype(gate)::value, false>(p, s, false, st_);
      });
    }
    if (rc) return rc;
    DISTDL_HIP_TRY(hipGetLastError());
    return DISTDL_OK;
  });
}

int distdl_scan_bwd(distdl_scan_plan* p, const void* const a_dev[], const void* const x_dev[], const void* const h_dev[],
                    const float* h0_dev, const int32_t* lengths_dev, const void* const dh_dev[], const float* dhT_dev,
                    void* const da_dev[], void* const dx_dev[], float* dh0_dev, void* stream) {
  if (!p || !a_dev || !h_dev || !dh_dev || !da_dev || !dx_dev) return set_error(DISTDL_ERR_NULL, "scan_bwd: null argument");
  if (!x_dev && p->gate != DISTDL_GATE_GIVEN) return set_error(DISTDL_ERR_NULL, "scan_bwd: sigmoid gates need x");
  if ((uintptr_t)h0_dev % 4 || (uintptr_t)lengths_dev % 4 || (uintptr_t)dhT_dev % 4 || (uintptr_t)dh0_dev % 4)
    return set_error(DISTDL_ERR_INVALID_ARG, "scan_bwd: h0, lengths, dhT or dh0 is not aligned to its elements");
  return guarded([&]() -> int {
    const size_t size = dtype_size(p->dtype);
    std::vector<ScanWorker> w((size_t)p->P);
    int rc;
    for (int j = 0; j < p->P; ++j) {
      if ((rc = scan_check(a_dev[j], size, "a", j)) || (p->gate != DISTDL_GATE_GIVEN && (rc = scan_check(x_dev[j], size, "x", j))) ||
          (rc = scan_check(h_dev[j], size, "h", j)) || (rc = scan_check(dh_dev[j], size, "dh", j)) ||
          (rc = scan_check(da_dev[j], size, "da", j)) || (rc = scan_check(dx_dev[j], size, "dx", j)))
        return rc;
      w[j] = ScanWorker{a_dev[j], x_dev ? x_dev[j] : nullptr, h_dev[j], dh_dev[j], da_dev[j], dx_dev[j]};
    }
    hipStream_t st_ = (hipStream_t)stream;
    ScanArgs s;
    if ((rc = scan_args(p, w, st_, &s))) return rc;
    s.lengths = lengths_dev;
    s.h0 = h0_dev;
    s.end = dhT_dev;
    s.hT = dh0_dev;
    {
      ProfScope prof("scan_bwd", st_);
      scan_kind(p->dtype, p->gate, [&](auto e, auto gate) {
        rc = scan_pairs(p, w) ? launch_scan<decltype(e), decltype(gate)::value, true>(p, s, true, st_)
                              : launch_scan<decltype(e), decltype(gate)::value, false>(p, s, true, st_);
      });
    }
    if (rc) return rc;
    DISTDL_HIP_TRY(hipGetLastError());
    return DISTDL_OK;
  });
}

int distdl_scan_step(const void* a_dev, const void* x_dev, float* state_dev, int64_t n_slots, const int32_t* slots_dev, void* h_dev,
                     int64_t rows, int64_t n_c, distdl_gate gate, distdl_dtype dtype, void* stream) {
  if (rows < 0 || n_c < 1 || n_slots < 0) return set_error(DISTDL_ERR_INVALID_ARG, "scan_step: %lld rows of %lld channels, %lld slots",
                                                           (long long)rows, (long long)n_c, (long long)n_slots);
  if (gate != DISTDL_GATE_GIVEN && gate != DISTDL_GATE_SIGMOID) return set_error(DISTDL_ERR_UNSUPPORTED, "unknown gate");
  if (dtype != DISTDL_F32 && dtype != DISTDL_BF16) return set_error(DISTDL_ERR_UNSUPPORTED, "unknown dtype");
  if (rows == 0) return DISTDL_OK;
  if (!a_dev || !x_dev || !h_dev || (!state_dev && n_slots > 0)) return set_error(DISTDL_ERR_NULL, "scan_step: null argument");
  if (!slots_dev && n_slots < rows) return set_error(DISTDL_ERR_INVALID_ARG, "scan_step: %lld states for %lld rows", (long long)n_slots, (long long)rows);
  if (rows > int64_t(65535) * 65535 || n_c >= int64_t(1) << 30) return set_error(DISTDL_ERR_UNSUPPORTED, "scan_step: problem too large");
  const size_t size = dtype_size(dtype);
  if ((uintptr_t)a_dev % size || (uintptr_t)x_dev % size || (uintptr_t)h_dev % size || (uintptr_t)state_dev % 4 || (uintptr_t)slots_dev % 4)
    return set_error(DISTDL_ERR_INVALID_ARG, "scan_step: an array is not aligned to its elements");
  hipStream_t st_ = (hipStream_t)stream;
  {
    ProfScope prof("scan_step", st_);
    const int64_t wide = (n_c + 2047) / 2048;
    for (int64_t row0 = 0; row0 < rows; row0 += 65535) {  // (one launch for any batch that a decoder has)
      const int64_t n = std::min<int64_t>(65535, rows - row0);
      scan_kind(dtype, gate, [&](auto e, auto g) {
        typedef decltype(e) E;
        hipLaunchKernelGGL((scan_step_kernel<E, decltype(g)::value>), dim3((unsigned)wide, (unsigned)n), dim3(256), 0, st_,
                           (const E*)a_dev + row0 * n_c, (const E*)x_dev + row0 * n_c, state_dev + (slots_dev ? 0 : row0 * n_c),
                           slots_dev ? slots_dev + row0 : nullptr, (E*)h_dev + row0 * n_c, slots_dev ? n_slots : n_slots - row0, n_c);
      });
    }
  }
  DISTDL_HIP_TRY(hipGetLastError());
  return DISTDL_OK;
}

}  // extern "C"
