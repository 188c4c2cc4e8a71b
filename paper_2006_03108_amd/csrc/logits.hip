// Log probabilities, entropy and top alternatives of rows of logits whose vocabulary P workers share, their adjoint, and the
// divergence from a teacher's top logits with its gradient.
//
//   z = x / temperature,  lse = log sum exp z,  log p_i = z_i - lse,  H = lse - sum p_i z_i
//   adjoint of (log p_t, H)   dx_i = (dlogp (1[i = t] - p_i) - dH p_i (log p_i + H)) / temperature
//   divergence                sum_k pi_k (log pi_k - log p_{id_k}),  pi = softmax of the teacher's logits / temperature
//                             dx_i = weight / temperature (p_i - sum_{k: id_k = i} pi_k)
//
// The sums over the vocabulary are the all-reduce of the workers' sums: a workgroup reads a row's parts one behind the other, once,
// with a running maximum.  Everything is in units of log 2: d_i = x_i c - mc, c = log2(e) / temperature, mc = c max x as it was
// rounded, so that exp2(d_i) and what is made of mc belong together whatever mc lost, and the partial sums of lanes, waves and parts meet by
// factors exp2(mc - mc').  Then lse = ln 2 (mc + log2 s) and H = ln 2 (log2 s - w / s), s = sum exp2(d), w = sum exp2(d) d: both
// terms of H are positive.
#include <algorithm>
#include <cfloat>
#include <climits>
#include <cstddef>
#include <type_traits>

#include "block8.h"
#include "buffer.h"
#include "common.h"
#include "profile.h"

namespace distdl {

constexpr int kLogitsInline = 16;   // workers whose pointers travel with the launch; more are in a table
constexpr int kLogitsThreads = 256;
constexpr int kLogitsWaves = kLogitsThreads / 64;
constexpr int kTopMost = 64;        // alternatives: one to a lane
constexpr int kStoredMost = 1024;   // a teacher's logits for one row
constexpr float kLn2 = 0.6931471805599453f;

struct LogitsWorker {
  const void* x;
  void* dx;
};

struct LogitsArgs {
  LogitsWorker w[kLogitsInline];
  const LogitsWorker* more;
  int64_t rows;
  int32_t n_v, P, part, extra;     // worker j has part + (j < extra) entries
  int32_t vec_wide, vec_rest;      // vectors of eight entries of a worker with part + 1, with part
  int32_t splits, per;             // of a row's vectors, and how many each has
  float c, inv_t;
  int32_t n_top;
  const int32_t* targets;
  float *logp, *lse, *entropy;
  int32_t* ids;
  float* top;
  const float *dlogp, *dentropy;   // adjoint; lse and entropy are inputs there
  const int32_t* stored_ids;       // the teacher's
  const float *stored, *weight;
  float* loss;
  float4* parts;                   // (max, mc, s, w) of each split
  uint64_t* part_top;              // kTopMost keys of each split
  float* stored_x;                 // the student's logits at the teacher's places
};

static_assert(offsetof(LogitsArgs, w) == 0, "the kernels' first argument starts with the workers");
typedef const __attribute__((address_space(4))) LogitsWorker* LogitsTable;
// (read as constants, into scalar registers; the address of the arguments is taken in the kernel itself)
#define LOGITS_TABLE(s) ((s).more ? (LogitsTable)(uint64_t)(s).more : (LogitsTable)__builtin_amdgcn_kernarg_segment_ptr())

struct LogitsPart {  // worker j's share of the vocabulary
  int32_t n, first, vec0, vecs;
};
__device__ __forceinline__ LogitsPart logits_part(const LogitsArgs& s, int j) {
  const bool wide = j < s.extra;
  LogitsPart p;
  p.n = s.part + wide;
  p.first = j * s.part + min(j, s.extra);
  p.vecs = wide ? s.vec_wide : s.vec_rest;
  p.vec0 = wide ? j * s.vec_wide : s.extra * s.vec_wide + (j - s.extra) * s.vec_rest;
  return p;
}
// the worker of entry `id`
__device__ __forceinline__ int logits_worker_of(const LogitsArgs& s, int id) {
  const int64_t wide = (int64_t)s.extra * (s.part + 1);
  return id < wide ? id / (s.part + 1) : s.extra + (int)((id - wide) / s.part);
}
template <class E>
__device__ __forceinline__ float logits_at(const LogitsArgs& s, LogitsTable table, int64_t row, int id) {
  const int j = logits_worker_of(s, id);
  const LogitsPart p = logits_part(s, j);
  return ld((const E*)table[j].x, (size_t)(row * p.n + (id - p.first)));
}

// Eight neighbouring entries of a row.  A part's last vector starts so that it ends with the part, and of its entries those from `from`
// on are its own: every load is whole and inside the row.  TINY: parts of fewer than eight entries, read one by one.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t logits_row(const void* x, int64_t row, int n, size_t size) {
  return rsrc_of((const char*)x + row * n * size, (uint32_t)n * (uint32_t)size);
}
template <class E, bool TINY>
struct LogitsVector {
  u32x4 raw[sizeof(E) / 2];
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t row, int n, int v) {
    if constexpr (TINY) {
      uint32_t e[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {  // (what lies behind the row fails the check and is 0)
        if constexpr (sizeof(E) == 4) e[i] = __builtin_amdgcn_raw_buffer_load_b32(row, i * 4, 0, 0);
        else e[i] = (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(row, i * 2, 0, 0);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(E) == 4) raw[0][i] = e[i], raw[1][i] = e[i + 4];
        else raw[0][i] = e[2 * i] | e[2 * i + 1] << 16;
      }
    } else {
      const uint32_t o = (uint32_t)min(8 * v, n - 8) * (uint32_t)sizeof(E);
#pragma unroll
      for (int i = 0; i < (int)sizeof(E) / 2; ++i) raw[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(row, o, i * 16, 0));
    }
  }
  // Values; -inf in the places that are not its own.  edge: there may be vectors behind `end`; ragged: the part's last one may begin before its place
  // (both uniform).
  __device__ __forceinline__ void values(float* f, int n, int v, int end, bool edge, bool ragged) {
    if (edge) {
      asm volatile("");  // (a branch: as selections they would cost every vector an instruction for each entry)
#pragma unroll
      for (int i = 0; i < (int)sizeof(E) / 2; ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k) raw[i][k] = v < end ? raw[i][k] : sizeof(E) == 4 ? 0xff800000u : 0xff80ff80u;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (sizeof(E) == 4) {
        f[i] = __uint_as_float(raw[0][i]);
        f[i + 4] = __uint_as_float(raw[1][i]);
      } else {
        f[2 * i] = bf16_lo(raw[0][i]);
        f[2 * i + 1] = bf16_hi(raw[0][i]);
      }
    }
    if (ragged) {
      asm volatile("");
      const int from = v < end ? first_of(n, v) : 8;
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = i >= from && i < n ? f[i] : -INFINITY;
    }
  }
  static __device__ __forceinline__ int place(int n, int v) { return max(0, min(8 * v, n - 8)); }
  static __device__ __forceinline__ int first_of(int n, int v) { return 8 * v - place(n, v); }
};
template <class E>
constexpr int logits_batch() { return sizeof(E) == 2 ? 4 : 2; }  // vectors of a lane under way: 64 bytes

// f(worker, part, first vector of the workgroup's batch, end) for the batches of a row's vectors lo .. hi - 1
__device__ __forceinline__ int logits_row_vectors(const LogitsArgs& s) { return s.extra * s.vec_wide + (s.P - s.extra) * s.vec_rest; }
template <int B, int THREADS, class F>
__device__ __forceinline__ void logits_between(const LogitsArgs& s, int lo, int hi, F f) {
  for (int j = 0; j < s.P; ++j) {
    const LogitsPart p = logits_part(s, j);
    const int from = max(0, lo - p.vec0), to = min(p.vecs, hi - p.vec0);
    for (int base = from; base < to; base += THREADS * B) f(j, p, base, to);
  }
}
// ... of the split's
template <int B, int THREADS, class F>
__device__ __forceinline__ void logits_each(const LogitsArgs& s, int split, F f) {
  const int lo = split * s.per;
  logits_between<B, THREADS>(s, lo, min(lo + s.per, logits_row_vectors(s)), f);
}

// ---- lanes ----------------------------------------------------------------
// The number of lane l ^ O (a power of two, or 63).  IN_REGISTERS: moved within the vector registers, which takes a tenth of the time of a way through LDS, but the
// vector units': for rows that are cut, whose few waves wait for chains of moves (8 rows of 65536 with 20 alternatives: 17.8 -> 16.6 us).  Where waves are
// many, they have enough to do besides (64 alternatives of 2048 rows of 131072: 223 us in registers, 211 through LDS).
template <int CTRL>
__device__ __forceinline__ uint32_t moved(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, false);
}
template <int O>
__device__ __forceinline__ uint32_t moved_lane(uint32_t v) {
  if constexpr (O == 63) {
    return moved_lane<32>(moved_lane<16>(moved<0x140>(v)));  // (rows of 16 lanes mirrored)
  } else if constexpr (O == 32) {
    const auto w = __builtin_amdgcn_permlane32_swap(v, v, false, false);  // the lower half's twice, the upper half's twice
    return threadIdx.x & 32 ? w[0] : w[1];
  } else if constexpr (O == 16) {
    const auto w = __builtin_amdgcn_permlane16_swap(v, v, false, false);  // the even rows' twice, the odd rows' twice
    return threadIdx.x & 16 ? w[0] : w[1];
  } else {
    static_assert(O == 8 || O == 4 || O == 2 || O == 1, "lanes of a row");
    if constexpr (O == 8) return moved<0x128>(v);                    // rotated by 8
    else if constexpr (O == 4) return moved<0x1b>(moved<0x141>(v));  // eights mirrored, then fours
    else return moved<O == 2 ? 0x4e : 0xb1>(v);                      // within fours
  }
}
template <int O, bool IN_REGISTERS>
__device__ __forceinline__ uint32_t other_lane_bits(uint32_t v) {
  if constexpr (IN_REGISTERS) return moved_lane<O>(v);
  else return (uint32_t)__shfl_xor((int)v, O, 64);
}
template <int O, bool IN_REGISTERS, class T>
__device__ __forceinline__ T other_lane(T v) {
  if constexpr (sizeof(T) == 8) {
    const uint32_t lo = other_lane_bits<O, IN_REGISTERS>((uint32_t)v), hi = other_lane_bits<O, IN_REGISTERS>((uint32_t)(v >> 32));
    return (T)((uint64_t)hi << 32 | lo);
  } else {
    return __builtin_bit_cast(T, other_lane_bits<O, IN_REGISTERS>(__builtin_bit_cast(uint32_t, v)));
  }
}

// ---- sums -----------------------------------------------------------------
// The largest entry's own d is what rounding has left of m c: up to 2^-5 where m c is below 2^20, beyond what exp2 takes from 2^31 on (masks of -1e10, alone in a lane or a row), and m c is no
// number at last.  From 2^20 on d is (x - m) c, of the reference m c itself: an operation more, and exact where entries are near the maximum.
constexpr float kFar = 0x1p20f;

struct LogitsSums {
  float m = -INFINITY, mc = 0.f, s = 0.f, w = 0.f;
  __device__ __forceinline__ bool far() const { return fabsf(mc) >= kFar; }
  // d of an entry
  __device__ __forceinline__ float of(float x, float c) const { return far() ? (x - m) * c : fmaf(x, c, -mc); }
  // log p of an entry, total: log2 s.  In units of log 2 the lowest numbers have none, so where d says -inf it is the difference over the temperature.
  __device__ __forceinline__ float log_p(float x, float c, float inv_t, float total) const {
    const float d = of(x, c);
    return d == -INFINITY ? fmaf(x - m, inv_t, -kLn2 * total) : kLn2 * (d - total);
  }
  __device__ __forceinline__ bool none() const { return m == -INFINITY && s == 0.f; }  // every entry is -inf
  // the reference moves up to the maximum m1
  __device__ __forceinline__ void raise(float m1, float c) {
    const float mc1 = m1 == -INFINITY ? 0.f : m1 * c;
    const bool far0 = far(), far1 = fabsf(mc1) >= kFar;
    const float by = far1 ? far0 ? (m - m1) * c : fmaf(-m1, c, mc) : far0 ? fmaf(m, c, -mc1) : mc - mc1;
    const float shift = m == -INFINITY ? 0.f : fmaxf(by, -200.f);  // (where there is nothing to move, nowhere)
    const float f = __builtin_amdgcn_exp2f(shift);
    w = f * fmaf(s, shift, w);
    s *= f;
    m = m1;
    mc = mc1;
  }
  __device__ __forceinline__ void join(LogitsSums o, float c) {
    const float m1 = fmaxf(m, o.m);
    raise(m1, c);
    o.raise(m1, c);
    s += o.s;
    w += o.w;
  }
  __device__ __forceinline__ void join_lanes(float c) {
    float most = m;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor(most, o, 64));
    raise(most, c);
    s = wave_sum(s);
    w = wave_sum(w);
  }
  // The sums of all waves, for all threads.  `shared`: a place for each wave.
  template <int WAVES>
  __device__ __forceinline__ void join_waves(float4* shared, float c) {
    join_lanes(c);
    if (WAVES == 1) return;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = make_float4(m, mc, s, w);
    __syncthreads();
    LogitsSums all;
    constexpr int kAtOnce = WAVES > 4 ? 2 : WAVES;  // (sixteen places in registers at once would leave a compute unit one workgroup: 537 us for 4096 x 131072 distilled, 490 so)
#pragma unroll kAtOnce
    for (int i = 0; i < WAVES; ++i) {
      const float4 v = shared[i];
      LogitsSums one;
      one.m = v.x, one.mc = v.y, one.s = v.z, one.w = v.w;
      all.join(one, c);
    }
    *this = all;
  }
};

// A batch of a lane's values.  The entropy's w counts what exp2 makes 0 as 0, -inf too.
template <int N, bool ENTROPY>
__device__ __forceinline__ void logits_add(LogitsSums& a, const float (&f)[N], float most, float c) {
  if (__any(most > a.m)) a.raise(fmaxf(a.m, most), c);
  if (__builtin_expect(__any(a.far()), 0)) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float d = a.of(f[i], c), e = __builtin_amdgcn_exp2f(d);
      a.s += e;
      if (ENTROPY) a.w = fmaf(e, fmaxf(d, -200.f), a.w);
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float d = fmaf(f[i], c, -a.mc), e = __builtin_amdgcn_exp2f(d);
    a.s += e;
    if (ENTROPY) a.w = fmaf(e, fmaxf(d, -200.f), a.w);
  }
}
// (fmaxf of loaded numbers costs an instruction more for each, which makes signalling NaNs quiet)
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}
__device__ __forceinline__ float max8(const float* f) { return max3(max3(max3(f[0], f[1], f[2]), f[3], f[4]), max3(f[5], f[6], f[7]), f[7]); }

// ---- top alternatives -----------------------------------------------------
// An entry's key: its value as an integer in the same order, above the complement of its place, so that larger keys come first.  0 is no entry.
__device__ __forceinline__ int32_t order_of(float v) {
  const int32_t b = (int32_t)__float_as_uint(v + 0.f);  // (-0 is 0)
  return v != v ? INT_MIN : b ^ ((b >> 31) & 0x7fffffff);  // (a NaN is no alternative)
}
__device__ __forceinline__ uint64_t key_of(int32_t order, int id) { return (uint64_t)((uint32_t)order ^ 0x80000000u) << 32 | (uint32_t)~id; }
__device__ __forceinline__ float value_of(uint64_t key) {
  const int32_t o = (int32_t)((uint32_t)(key >> 32) ^ 0x80000000u);
  return __uint_as_float((uint32_t)(o ^ ((o >> 31) & 0x7fffffff)));
}

// the last rounds of a bitonic sort: a bitonic sequence of `n` lanes becomes a descending one where `down`, else ascending
template <int N, bool IN_REGISTERS, class T>
__device__ __forceinline__ T bitonic(T v, bool down) {
  if constexpr (N > 1) {
    constexpr int O = N / 2;
    const T u = other_lane<O, IN_REGISTERS>(v);
    const bool large = ((threadIdx.x & O) == 0) == down;
    return bitonic<O, IN_REGISTERS>(large == (u > v) ? u : v, down);
  } else {
    return v;
  }
}
template <bool IN_REGISTERS, class T>
__device__ __forceinline__ T sorted_lanes(T v) {  // descending
  v = bitonic<2, IN_REGISTERS>(v, (threadIdx.x & 2) == 0);
  v = bitonic<4, IN_REGISTERS>(v, (threadIdx.x & 4) == 0);
  v = bitonic<8, IN_REGISTERS>(v, (threadIdx.x & 8) == 0);
  v = bitonic<16, IN_REGISTERS>(v, (threadIdx.x & 16) == 0);
  v = bitonic<32, IN_REGISTERS>(v, (threadIdx.x & 32) == 0);
  return bitonic<64, IN_REGISTERS>(v, true);
}
// the 64 largest keys of two descending lists
template <bool IN_REGISTERS>
__device__ __forceinline__ uint64_t merged_lanes(uint64_t a, uint64_t b) {
  b = other_lane<63, IN_REGISTERS>(b);
  return bitonic<64, IN_REGISTERS>(a > b ? a : b, true);
}

// `best` and `waiting` keys of a buffer in LDS.  (Out of line: it is rarely called, and the registers are the streaming loop's.)
typedef __attribute__((address_space(3))) uint64_t* TopBuffer;
template <bool FEW>
__device__ __attribute__((noinline)) uint64_t top_flushed(uint64_t best, TopBuffer buffer, int waiting) {
  const int lane = threadIdx.x & 63;
  while (waiting > 0) {
    const int n = min(waiting, 64), from = waiting - n;
    best = merged_lanes<FEW>(best, sorted_lanes<FEW>(lane < n ? (uint64_t)buffer[from + lane] : (uint64_t)0));
    waiting = from;
  }
  __builtin_amdgcn_wave_barrier();
  return best;
}
template <bool FEW>
__device__ __attribute__((noinline)) int32_t top_nth(int32_t order, int n) { return __builtin_amdgcn_readlane(sorted_lanes<FEW>(order), n - 1); }

constexpr int kTopRoom = 64 + 512;  // keys that wait: a vector of each lane beside less than 64

// A wave's 64 best entries, descending over the lanes, and a buffer of those that wait.  Values at or below `floor`, the n-th best so far, can
// not be among the n: a wave meets entries in the order of their places, so of equal values the first stay.  (A NaN, at first, lets all pass.)  FEW: rows are cut.
template <bool FEW>
struct TopList {
  uint64_t best = 0;
  float floor = NAN;
  int waiting = 0;
  __device__ __forceinline__ bool passes(float v) const { return !(v <= floor); }
  __device__ __forceinline__ void set_floor(int n_top) {
    const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(best >> 32), n_top - 1);
    const float nth = value_of((uint64_t)hi << 32);
    if (hi != 0 && !(nth <= floor)) floor = nth;
  }
  // From the largest of each lane's first entries: the n-th of them is no better than the n-th of all, and may be it.
  __device__ __forceinline__ void start(float most, int n_top) {
    const int32_t nth = top_nth<FEW>(order_of(most), n_top);
    const int32_t below = nth == 0 ? order_of(-FLT_MIN) : nth - 1;  // (-0, which comes next, is no less than 0)
    if (nth > order_of(-INFINITY)) floor = __uint_as_float((uint32_t)(below ^ ((below >> 31) & 0x7fffffff)));
  }
  __device__ __forceinline__ void flush(uint64_t* buffer, int n_top) {
    best = top_flushed<FEW>(best, (TopBuffer)buffer, waiting);
    waiting = 0;
    set_floor(n_top);
  }
  __device__ __forceinline__ void push(uint64_t* buffer, bool in, float v, int id) {
    const uint64_t all = __ballot(in);
    if (in) buffer[waiting + __popcll(all & ((uint64_t(1) << (threadIdx.x & 63)) - 1))] = key_of(order_of(v), id);
    waiting += __popcll(all);
  }
  // A vector of each lane, some lane's largest value `most` of which passes; mostly it is one value of one lane.
  __device__ __forceinline__ void take(uint64_t* buffer, const float* f, float most, int id, int from, int upto, int n_top) {
    int count = 0, first = 0;
#pragma unroll
    for (int i = 7; i >= 0; --i) {
      const bool in = passes(f[i]) && f[i] == f[i] && i >= from && i < upto;
      count += in;
      first = in ? i : first;
    }
    if (!__any(count > 1)) {
      push(buffer, count > 0, most, id + first);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) push(buffer, passes(f[i]) && f[i] == f[i] && i >= from && i < upto, f[i], id + i);
    }
    __builtin_amdgcn_wave_barrier();
    if (waiting >= 64) flush(buffer, n_top);
  }
};

// The target's logit, for the first thread: it is asked for before the row is read.
template <class E>
__device__ __forceinline__ float logits_target(const LogitsArgs& s, LogitsTable table, int64_t row) {
  if (threadIdx.x != 0 || !s.logp) return 0.f;
  const int t = s.targets[row];
  return t >= 0 && t < s.n_v ? logits_at<E>(s, table, row, t) : 0.f;
}

// What a row's sums and alternatives come to.  Every wave has the sums; wave 0 has the list.
__device__ __forceinline__ void logits_finish(const LogitsArgs& s, int64_t row, const LogitsSums& a, uint64_t best, float x_target) {
  const float total = __builtin_amdgcn_logf(a.s);  // log2
  const bool none = a.none();
  if (threadIdx.x == 0) {
    if (s.lse) s.lse[row] = none ? -INFINITY : a.far() ? fmaf(a.m, s.inv_t, kLn2 * total) : kLn2 * (a.mc + total);
    if (s.entropy) s.entropy[row] = none ? 0.f : kLn2 * (total - a.w / a.s);
    if (s.logp) {
      const int t = s.targets[row];
      float v = 0.f;
      if (t >= 0 && t < s.n_v) v = none ? -INFINITY : a.log_p(x_target, s.c, s.inv_t, total);
      s.logp[row] = v;
    }
  }
  if (s.n_top > 0 && threadIdx.x < s.n_top) {
    const int64_t o = row * s.n_top + threadIdx.x;
    if (s.ids) s.ids[o] = best ? (int32_t)~(uint32_t)best : -1;
    if (s.top) s.top[o] = none || !best ? -INFINITY : a.log_p(value_of(best), s.c, s.inv_t, total);
  }
}

// Sums of a row's vectors lo .. hi - 1.
template <class E, bool ENTROPY, bool TINY, int THREADS>
__device__ __forceinline__ void logits_sum(const LogitsArgs& s, LogitsTable table, int64_t row, int lo, int hi, LogitsSums& a) {
  constexpr int B = logits_batch<E>();
  logits_between<B, THREADS>(s, lo, hi, [&](int j, const LogitsPart& p, int base, int to) {
    const __amdgpu_buffer_rsrc_t x = logits_row(table[j].x, row, p.n, sizeof(E));
    LogitsVector<E, TINY> v[B];
    float f[B * 8], all = -INFINITY;
    const int v0 = base + threadIdx.x, end = base + B * THREADS;
#pragma unroll
    for (int b = 0; b < B; ++b) v[b].load(x, p.n, v0 + b * THREADS);
#pragma unroll
    for (int b = 0; b < B; ++b) {
      v[b].values(f + 8 * b, p.n, v0 + b * THREADS, to, end > to, p.n % 8 != 0 && end >= p.vecs);
      all = fmaxf(all, max8(f + 8 * b));
    }
    logits_add<B * 8, ENTROPY>(a, f, all, s.c);
  });
}

// A row, or one of its splits, to a workgroup.  THREADS: 64 for short rows, whose waves have nothing to join.
template <class E, bool ENTROPY, bool TOP, bool FEW, bool TINY, int THREADS>
__global__ __launch_bounds__(THREADS, 8) void logits_fwd_kernel(LogitsArgs s) {
  constexpr int B = logits_batch<E>() / (TOP ? 2 : 1), kWaves = THREADS / 64;
  __shared__ float4 sums[kWaves];
  __shared__ uint64_t buffers[TOP ? kWaves * kTopRoom : 1];
  const LogitsTable table = LOGITS_TABLE(s);
  const int64_t row = blockIdx.x / (uint32_t)s.splits;
  const int split = blockIdx.x % (uint32_t)s.splits, tid = threadIdx.x, wave = tid >> 6;
  uint64_t* const buffer = buffers + (TOP ? wave * kTopRoom : 0);
  const float x_target = s.splits == 1 ? logits_target<E>(s, table, row) : 0.f;
  LogitsSums a;
  TopList<FEW> list;
  bool first = true;
  typedef LogitsVector<E, TINY> Vector;
  if constexpr (TOP) {
    // The next vectors are under way while these are looked through; one place in the code for both, and for what is rarely done.
    const int lo = split * s.per, hi = min(lo + s.per, logits_row_vectors(s));
    for (int j = 0; j < s.P; ++j) {
      const LogitsPart p = logits_part(s, j);
      const int from = max(0, lo - p.vec0), to = min(p.vecs, hi - p.vec0);
      if (from >= to) continue;
      const __amdgpu_buffer_rsrc_t x = logits_row(table[j].x, row, p.n, sizeof(E));
      Vector next[B];
#pragma unroll
      for (int b = 0; b < B; ++b) next[b].load(x, p.n, from + tid + b * THREADS);
      for (int base = from; base < to; base += B * THREADS) {
        const int v0 = base + tid, end = base + B * THREADS;
        Vector v[B];
#pragma unroll
        for (int b = 0; b < B; ++b) {
          v[b] = next[b];
          next[b].load(x, p.n, v0 + (b + B) * THREADS);
        }
        float f[B * 8], most[B], all = -INFINITY;
#pragma unroll
        for (int b = 0; b < B; ++b) {
          v[b].values(f + 8 * b, p.n, v0 + b * THREADS, to, end > to, p.n % 8 != 0 && end >= p.vecs);
          most[b] = max8(f + 8 * b);
          all = fmaxf(all, most[b]);
        }
        logits_add<B * 8, ENTROPY>(a, f, all, s.c);
        if (__any(a.s != a.s)) {  // (a signalling NaN was the maximum of it and a number: made quiet, it is not)
          asm volatile("");
#pragma unroll
          for (int b = 0; b < B; ++b) {
#pragma unroll
            for (int i = 0; i < 8; ++i) f[8 * b + i] = __builtin_canonicalizef(f[8 * b + i]);
            most[b] = max8(f + 8 * b);
          }
        }
        if (first) list.start(all, s.n_top);
        first = false;
        bool any = false;
#pragma unroll
        for (int b = 0; b < B; ++b) any = any || list.passes(most[b]);
        if (__any(any)) {
#pragma unroll 1
          for (int b = 0; b < B; ++b) {
            float g[8], of = most[0];
#pragma unroll
            for (int i = 0; i < 8; ++i) g[i] = f[i];
#pragma unroll
            for (int c = 1; c < B; ++c) {
#pragma unroll
              for (int i = 0; i < 8; ++i) g[i] = b == c ? f[8 * c + i] : g[i];
              of = b == c ? most[c] : of;
            }
            const int i = v0 + b * THREADS;
            list.take(buffer, g, of, p.first + Vector::place(p.n, i), i < to ? Vector::first_of(p.n, i) : 8, p.n, s.n_top);
          }
        }
      }
    }
  } else {
    logits_sum<E, ENTROPY, TINY, THREADS>(s, table, row, split * s.per, min(split * s.per + s.per, logits_row_vectors(s)), a);
  }
  if constexpr (TOP) {
    list.flush(buffer, s.n_top);
    buffer[tid & 63] = list.best;
  }
  a.template join_waves<kWaves>(sums, s.c);
  if constexpr (TOP) {
    if (wave == 0)
      for (int i = 1; i < kWaves; ++i) list.best = merged_lanes<FEW>(list.best, buffers[i * kTopRoom + tid]);
  }
  if (s.splits == 1) {
    logits_finish(s, row, a, list.best, x_target);
    return;
  }
  if (tid == 0) s.parts[blockIdx.x] = make_float4(a.m, a.mc, a.s, a.w);
  if (TOP && tid < s.n_top) s.part_top[(int64_t)blockIdx.x * s.n_top + tid] = list.best;
}

// The splits of a row meet, in a fixed order.
template <int THREADS>
__device__ __forceinline__ LogitsSums logits_joined(const LogitsArgs& s, int64_t row, float4* shared) {
  LogitsSums a;
  for (int i = threadIdx.x; i < s.splits; i += THREADS) {
    const float4 v = s.parts[row * s.splits + i];
    LogitsSums one;
    one.m = v.x, one.mc = v.y, one.s = v.z, one.w = v.w;
    a.join(one, s.c);
  }
  a.join_waves<THREADS / 64>(shared, s.c);
  return a;
}

template <class E>
__global__ __launch_bounds__(kLogitsThreads) void logits_join_kernel(LogitsArgs s) {
  __shared__ float4 sums[kLogitsWaves];
  __shared__ uint64_t lists[kLogitsWaves * 64];
  const LogitsTable table = LOGITS_TABLE(s);
  const int64_t row = blockIdx.x;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  // The lists of four splits at a time, the first ones asked for before the sums are joined.
  constexpr int N = 4;
  uint64_t more[N];
  auto load = [&](int first) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int split = first + i * kLogitsWaves;
      more[i] = split < s.splits && lane < s.n_top ? s.part_top[(row * s.splits + split) * s.n_top + lane] : 0;
    }
  };
  const float x_target = logits_target<E>(s, table, row);
  load(wave);
  const LogitsSums a = logits_joined<kLogitsThreads>(s, row, sums);
  uint64_t best = 0;
  if (s.n_top > 0) {
    for (int first = wave; first < s.splits; first += N * kLogitsWaves) {
      if (first != wave) load(first);
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (first + i * kLogitsWaves < s.splits) best = merged_lanes<true>(best, more[i]);
    }
    lists[tid] = best;
    __syncthreads();
    if (wave == 0)
      for (int i = 1; i < kLogitsWaves; ++i) best = merged_lanes<true>(best, lists[i * 64 + lane]);
  }
  logits_finish(s, row, a, best, x_target);
}

// ---- adjoint --------------------------------------------------------------
template <class E>
__device__ __forceinline__ void logits_store(E* row, const float* f, int at, int from, int n, bool edge) {
  if (edge && (from > 0 || n < 8)) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i >= from && i < n) st(row, (size_t)(at + i), f[i]);
  } else {
    store8(row + at, f, 8);
  }
}

// An lse has 24 bits: of a shifted or masked row little or nothing of what exp needs.  Up to 256 it leaves p right to 4e-5; beyond, the row is read for its sums again, by its
// first workgroup alone where it is cut (the gradient may lie on it).
constexpr float kLseFar = 256.f, kLseNone = 1e30f;

template <class E, bool ENTROPY, bool TINY, int THREADS>
__global__ __launch_bounds__(THREADS) void logits_bwd_kernel(LogitsArgs s) {
  constexpr int B = logits_batch<E>();
  const LogitsTable table = LOGITS_TABLE(s);
  const int64_t row = blockIdx.x / (uint32_t)s.splits;
  const int split = blockIdx.x % (uint32_t)s.splits, tid = threadIdx.x;
  const int target = s.targets ? s.targets[row] : -1;
  const bool live = target >= 0 && target < s.n_v;
  const float lse = s.lse[row], weight = live ? s.dlogp[row] : 0.f, back = ENTROPY ? s.dentropy[row] : 0.f;
  // dx = p (one + two log2 p) / temperature, and the target's dlogp
  const float one = (-weight - (ENTROPY ? back * s.entropy[row] : 0.f)) * s.inv_t, two = -back * kLn2 * s.inv_t;
  const bool nothing = (weight == 0.f && back == 0.f) || lse < -kLseNone;  // such rows are not read
  const bool far = !nothing && fabsf(lse) >= kLseFar;
  const float lc = lse * (1.f / kLn2), at_target = weight * s.inv_t;
  int lo = split * s.per, hi = min(lo + s.per, logits_row_vectors(s));
  LogitsSums a;
  float stotal = 0.f;
  if (far) {
    if (split > 0) return;
    hi = logits_row_vectors(s);
    __shared__ float4 sums[THREADS / 64];
    logits_sum<E, false, TINY, THREADS>(s, table, row, lo, hi, a);
    a.template join_waves<THREADS / 64>(sums, s.c);
    stotal = __builtin_amdgcn_logf(a.s);
  }
  logits_between<B, THREADS>(s, lo, hi, [&](int j, const LogitsPart& p, int base, int to) {
    const __amdgpu_buffer_rsrc_t x = logits_row(table[j].x, row, p.n, sizeof(E));
    E* const dx = (E*)table[j].dx + row * p.n;
    typedef LogitsVector<E, TINY> Vector;
    Vector v[B];
    const bool edge = base + B * THREADS >= to;  // (a last vector, or none)
    if (!nothing) {
#pragma unroll
      for (int b = 0; b < B; ++b) v[b].load(x, p.n, base + b * THREADS + tid);
    }
#pragma unroll
    for (int b = 0; b < B; ++b) {
      float f[8] = {};
      const int i0 = base + b * THREADS + tid;
      const int at = Vector::place(p.n, i0), from = i0 < to ? Vector::first_of(p.n, i0) : 8;
      if (!nothing) {
        v[b].values(f, p.n, i0, to, false, false);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float d = far ? a.of(f[i], s.c) - stotal : fmaf(f[i], s.c, -lc), e = __builtin_amdgcn_exp2f(d);
          f[i] = ENTROPY ? e * fmaf(two, fmaxf(d, -200.f), one) : e * one;
          if (live && p.first + at + i == target) f[i] += at_target;
        }
      }
      logits_store(dx, f, at, from, p.n, edge);
    }
  });
}

// ---- divergence from a teacher's top logits -------------------------------
constexpr int kStoredFew = 64;    // they are compared with each other
constexpr int kStoredWave = 256;  // of a row that a wave has: 5 KiB of LDS, for 32 of them on a compute unit
template <int N>
struct Stored {  // a row's, N at most
  int32_t id[N];
  float p[N];  // the teacher's probabilities
  float x[N];  // the student's logits
  float red[16];
  int32_t table[2 * N], twice;
};
template <int THREADS>
constexpr int stored_most() { return THREADS == 64 ? kStoredWave : kStoredMost; }
template <int WAVES>
__device__ __forceinline__ float group_max(float v, float* red) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  v = red[0];
#pragma unroll
  for (int i = 1; i < WAVES; ++i) v = fmaxf(v, red[i]);
  return v;
}
template <int WAVES>
__device__ __forceinline__ float group_sum(float v, float* red) {
  v = wave_sum(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  v = red[0];
#pragma unroll
  for (int i = 1; i < WAVES; ++i) v += red[i];
  return v;
}
// The teacher's probabilities of a row: false if it has stored nothing.  total: log2 of their sum relative to the largest, `most`.  (Differences from it first: any finite
// numbers have probabilities, masks of the lowest value too.)
template <int THREADS, int N>
__device__ __forceinline__ bool stored_load(const LogitsArgs& s, int64_t row, Stored<N>& t, float& most, float& total) {
  most = -INFINITY;
  bool odd = false;
  for (int k = threadIdx.x; k < s.n_top; k += THREADS) {
    const int id = s.stored_ids[row * s.n_top + k];
    const bool in = id >= 0 && id < s.n_v;
    const float v = in ? s.stored[row * s.n_top + k] : -INFINITY;
    t.id[k] = in ? id : -1;
    t.p[k] = v;
    most = fmaxf(most, v);
    odd = odd || v != v;
  }
  most = group_max<THREADS / 64>(odd ? INFINITY : most, t.red);  // (a NaN ends as NaN: inf - inf)
  if (most == -INFINITY) return false;
  float sum = 0.f;
  for (int k = threadIdx.x; k < s.n_top; k += THREADS) sum += __builtin_amdgcn_exp2f((t.p[k] - most) * s.c);
  sum = group_sum<THREADS / 64>(sum, t.red);
  total = __builtin_amdgcn_logf(sum);
  return true;
}
// The row's loss, and the teacher's logits in t.p become probabilities.  a, stotal: the student's.
template <int THREADS, int N>
__device__ __forceinline__ float stored_loss(const LogitsArgs& s, Stored<N>& t, float most, float total, const LogitsSums& a, float stotal) {
  float loss = 0.f;
  const float inv = __builtin_amdgcn_exp2f(-total);
  for (int k = threadIdx.x; k < s.n_top; k += THREADS) {
    const float d = (t.p[k] - most) * s.c, p = __builtin_amdgcn_exp2f(d) * inv;
    if (!(p == 0.f)) loss = fmaf(p, kLn2 * (d - total) - a.log_p(t.x[k], s.c, s.inv_t, stotal), loss);
    t.p[k] = p;
  }
  return group_sum<THREADS / 64>(loss, t.red);
}

// Whether a place comes twice: they go into a table of twice their number, by a hash of the place.  (All threads of the workgroup.)
template <int THREADS, int N>
__device__ __forceinline__ bool stored_twice(const LogitsArgs& s, Stored<N>& t) {
  const int bits = 32 - __builtin_clz((uint32_t)(2 * s.n_top - 1));  // (n_top is above 1)
  for (int i = threadIdx.x; i < 1 << bits; i += THREADS) t.table[i] = -1;
  if (threadIdx.x == 0) t.twice = 0;
  __syncthreads();
  for (int k = threadIdx.x; k < s.n_top; k += THREADS) {
    const int id = t.id[k];
    if (id < 0) continue;
    for (uint32_t at = (uint32_t)id * 2654435769u >> (32 - bits);; at = (at + 1) & ((1u << bits) - 1)) {  // (half of the table stays free)
      const int before = atomicCAS(&t.table[at], -1, id);
      if (before == id) t.twice = 1;
      if (before == -1 || before == id) break;
    }
  }
  __syncthreads();
  return t.twice != 0;
}

// The teacher's places among a split's vectors lo .. hi - 1 are written once more.  stotal: log2 of the sum.  Looking through all of a row's places for
// each of them is left for rows where one comes twice: 8192 x 1024 with 256 places, bf16, 167 us else.
template <class E, int THREADS, int N>
__device__ __forceinline__ void stored_places(const LogitsArgs& s, LogitsTable table, int64_t row, Stored<N>& t, const LogitsSums& a, float stotal, float scale,
                                              int lo, int hi) {
  const bool search = s.n_top <= kStoredFew || stored_twice<THREADS>(s, t);
  for (int k = threadIdx.x; k < s.n_top; k += THREADS) {
    const int id = t.id[k];
    if (id < 0) continue;
    const int j = logits_worker_of(s, id);
    const LogitsPart p = logits_part(s, j);
    const int v = p.vec0 + (id - p.first) / 8;
    if (v < lo || v >= hi) continue;
    bool is_first = true;
    float sum = search ? 0.f : t.p[k];
    for (int i = 0; search && i < s.n_top; ++i) {  // (a place that is stored twice has the sum, and its first one writes it)
      const bool same = t.id[i] == id;
      sum += same ? t.p[i] : 0.f;
      if (same && i < k) is_first = false;
    }
    if (is_first) st((E*)table[j].dx, (size_t)(row * p.n + (id - p.first)), scale * (__builtin_amdgcn_exp2f(a.of(t.x[k], s.c) - stotal) - sum));
  }
}

// FIRST: the sums of a split and the student's logits at the teacher's places in it.  Else the loss and the gradient, of rows that
// are one workgroup's (splits == 1, which reads the row for its sums too) or of a split.
template <class E, bool FIRST, bool TINY, int THREADS>
__global__ __launch_bounds__(THREADS) void distill_kernel(LogitsArgs s) {
  constexpr int B = logits_batch<E>();
  __shared__ float4 sums[THREADS / 64];
  __shared__ Stored<stored_most<THREADS>()> t;
  const LogitsTable table = LOGITS_TABLE(s);
  const int64_t row = blockIdx.x / (uint32_t)s.splits;
  const int split = blockIdx.x % (uint32_t)s.splits, tid = threadIdx.x;
  float weight = s.weight ? s.weight[row] : 1.f, most = 0.f, total = 0.f;
  LogitsSums a;
  bool any = false;
  if (FIRST) {
    const int lo = split * s.per, hi = lo + s.per;
    for (int k = tid; k < s.n_top; k += THREADS) {
      const int id = s.stored_ids[row * s.n_top + k];
      if (id < 0 || id >= s.n_v) continue;
      const LogitsPart p = logits_part(s, logits_worker_of(s, id));
      const int v = p.vec0 + (id - p.first) / 8;
      if (v >= lo && v < hi) s.stored_x[row * s.n_top + k] = logits_at<E>(s, table, row, id);
    }
  } else {
    any = stored_load<THREADS>(s, row, t, most, total);
    if (!any) weight = 0.f;
    if (any)
      for (int k = tid; k < s.n_top; k += THREADS)
        t.x[k] = t.id[k] < 0 ? 0.f : s.splits > 1 ? s.stored_x[row * s.n_top + k] : logits_at<E>(s, table, row, t.id[k]);
  }
  const bool sum_here = FIRST || s.splits == 1;
  if (sum_here && (FIRST || any)) {
    logits_sum<E, false, TINY, THREADS>(s, table, row, split * s.per, min(split * s.per + s.per, logits_row_vectors(s)), a);
    a.join_waves<THREADS / 64>(sums, s.c);
  }
  if (FIRST) {
    if (tid == 0) s.parts[blockIdx.x] = make_float4(a.m, a.mc, a.s, 0.f);
    return;
  }
  if (any && !sum_here) a = logits_joined<THREADS>(s, row, sums);
  const float stotal = __builtin_amdgcn_logf(a.s);
  if (any && a.none()) {  // no entry that the student could answer with: an infinite loss, and nothing to follow
    if (tid == 0 && split == 0 && s.loss) s.loss[row] = INFINITY;
    weight = 0.f;
  } else if (any) {
    const float loss = stored_loss<THREADS>(s, t, most, total, a, stotal);
    if (tid == 0 && split == 0 && s.loss) s.loss[row] = loss;
  } else if (tid == 0 && split == 0 && s.loss) {
    s.loss[row] = 0.f;
  }
  if (!table[0].dx) return;
  const float scale = weight * s.inv_t;
  const bool far = a.far();
  const bool nothing = weight == 0.f;  // such rows are not read
  __syncthreads();
  logits_each<B, THREADS>(s, split, [&](int j, const LogitsPart& p, int base, int to) {
    const __amdgpu_buffer_rsrc_t x = logits_row(table[j].x, row, p.n, sizeof(E));
    E* const dx = (E*)table[j].dx + row * p.n;
    typedef LogitsVector<E, TINY> Vector;
    Vector v[B];
    const bool edge = base + B * THREADS >= to;  // (a last vector, or none)
    if (!nothing) {
#pragma unroll
      for (int b = 0; b < B; ++b) v[b].load(x, p.n, base + b * THREADS + tid);
    }
#pragma unroll
    for (int b = 0; b < B; ++b) {
      float f[8] = {};
      const int i0 = base + b * THREADS + tid;
      const int at = Vector::place(p.n, i0), from = i0 < to ? Vector::first_of(p.n, i0) : 8;
      if (!nothing) {
        v[b].values(f, p.n, i0, to, false, false);
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = scale * __builtin_amdgcn_exp2f((far ? (f[i] - a.m) * s.c : fmaf(f[i], s.c, -a.mc)) - stotal);  // (mc + stotal, rounded, would be off by what a row is shifted)
      }
      logits_store(dx, f, at, from, p.n, edge);
    }
  });
  if (nothing) return;
  __syncthreads();  // (behind the stores above)
  stored_places<E, THREADS>(s, table, row, t, a, stotal, scale, split * s.per, split * s.per + s.per);
}

// Rows that fit a workgroup's registers (up to 65536 entries of bf16, 32768 of fp32) are read once.  Slot by slot: a slot has a vector for each thread, of one
// worker.  Longer ones would leave a compute unit one workgroup, which reads, computes and writes in turn: 4096 x 131072, bf16, 648 us that way, 490 us read
// twice.
template <class E>
constexpr int distill_slots() { return sizeof(E) == 2 ? 16 : 8; }
template <class E, int THREADS>
__global__ __launch_bounds__(THREADS) void distill_kept_kernel(LogitsArgs s) {
  constexpr int S = distill_slots<E>();
  typedef LogitsVector<E, false> Vector;
  __shared__ float4 sums[THREADS / 64];
  __shared__ Stored<kStoredMost> t;
  const LogitsTable table = LOGITS_TABLE(s);
  const int64_t row = blockIdx.x;
  const int tid = threadIdx.x;
  // f(slot, worker, part, first vector)
  auto slots = [&](auto f) {
    int j = 0, base = 0;
    LogitsPart p = logits_part(s, 0);
#pragma unroll
    for (int i = 0; i < S; ++i) {
      if (j < s.P) {
        f(i, j, p, base);
        base += THREADS;
        if (base >= p.vecs) {
          ++j;
          base = 0;
          p = logits_part(s, min(j, s.P - 1));
        }
      }
    }
  };
  Vector v[S];
  slots([&](int i, int j, const LogitsPart& p, int base) { v[i].load(logits_row(table[j].x, row, p.n, sizeof(E)), p.n, base + tid); });
  float weight = s.weight ? s.weight[row] : 1.f, most = 0.f, total = 0.f;
  const bool any = stored_load<THREADS>(s, row, t, most, total);
  if (any) {
    for (int k = tid; k < s.n_top; k += THREADS) t.x[k] = t.id[k] < 0 ? 0.f : logits_at<E>(s, table, row, t.id[k]);
  } else {
    weight = 0.f;
  }
  LogitsSums a;
  if (any) {
    slots([&](int i, int j, const LogitsPart& p, int base) {
      float f[8];
      v[i].values(f, p.n, base + tid, p.vecs, base + THREADS > p.vecs, p.n % 8 != 0 && base + THREADS >= p.vecs);
      logits_add<8, false>(a, f, max8(f), s.c);
    });
    a.template join_waves<THREADS / 64>(sums, s.c);
  }
  const float stotal = __builtin_amdgcn_logf(a.s);
  float loss = 0.f;
  if (any && a.none()) {  // no entry that the student could answer with: an infinite loss, and nothing to follow
    loss = INFINITY;
    weight = 0.f;
  } else if (any) {
    loss = stored_loss<THREADS>(s, t, most, total, a, stotal);
  }
  if (tid == 0 && s.loss) s.loss[row] = loss;
  const float scale = weight * s.inv_t;
  const bool nothing = weight == 0.f, far = a.far();
  __syncthreads();  // (places of the row are read above, of dx on x)
  slots([&](int i, int j, const LogitsPart& p, int base) {
    E* const dx = (E*)table[j].dx + row * p.n;
    float f[8] = {};
    if (!nothing) {
      v[i].values(f, p.n, base + tid, p.vecs, false, false);
#pragma unroll
      for (int k = 0; k < 8; ++k) f[k] = scale * __builtin_amdgcn_exp2f((far ? (f[k] - a.m) * s.c : fmaf(f[k], s.c, -a.mc)) - stotal);
    }
    const int at = Vector::place(p.n, base + tid), from = base + tid < p.vecs ? Vector::first_of(p.n, base + tid) : 8;
    logits_store(dx, f, at, from, p.n, base + THREADS >= p.vecs);
  });
  if (nothing) return;
  __syncthreads();  // (behind the stores above)
  stored_places<E, THREADS>(s, table, row, t, a, stotal, scale, 0, INT_MAX);
}

}  // namespace distdl

struct distdl_logits_plan {
  int64_t rows = 0;
  int32_t n_v = 0;
  int P = 1;
  distdl_dtype dtype = DISTDL_F32;
  distdl::DevArray<distdl::LogitsWorker> table;
  distdl::StreamScratch scratch;
};

namespace distdl {

// Workgroups of a row.  A row is one workgroup's where rows fill the card; else it is cut, down to half a batch of a workgroup, or to one worker's part of `parts`, of which a
// workgroup reads one behind the other (16 rows of 32000 bf16 on 8 workers with 20 alternatives 32 -> 16 us; not so the distillation, whose workgroups all look at
// all of a row's places: 200 rows of 20000 on 8 with 32 places 26 -> 32).
static int logits_splits(int64_t rows, int vecs, int batch, int parts) {
  const int64_t wanted = (1024 + rows - 1) / rows, halves = vecs / (batch * kLogitsThreads / 2);
  return rows >= 512 || halves < 2 ? 1 : (int)std::min(wanted, std::max<int64_t>(halves, std::min(parts, vecs)));
}

static int logits_args(distdl_logits_plan* p, const void* const x_dev[], void* const dx_dev[], double temperature, int parts, hipStream_t st, LogitsArgs* s) {
  if (!(temperature >= 1e-6 && temperature <= 1e6)) return set_error(DISTDL_ERR_INVALID_ARG, "logits: temperature %g", temperature);
  const size_t size = dtype_size(p->dtype);
  std::vector<LogitsWorker> w((size_t)p->P);
  for (int j = 0; j < p->P; ++j) {
    if (!x_dev[j] || (dx_dev && !dx_dev[j])) return set_error(DISTDL_ERR_NULL, "logits: %s[%d] is null", x_dev[j] ? "dx" : "x", j);
    if ((uintptr_t)x_dev[j] % size || (dx_dev && (uintptr_t)dx_dev[j] % size))
      return set_error(DISTDL_ERR_INVALID_ARG, "logits: an array of worker %d is not aligned to its elements", j);
    w[j] = LogitsWorker{x_dev[j], dx_dev ? dx_dev[j] : nullptr};
  }
  *s = LogitsArgs{};
  if (p->P <= kLogitsInline) {
    std::copy(w.begin(), w.end(), s->w);
  } else {
    const int rc = p->table.upload(w, st);
    if (rc) return rc;
    s->more = p->table.dev;
  }
  s->rows = p->rows;
  s->n_v = p->n_v;
  s->P = p->P;
  s->part = p->n_v / p->P;
  s->extra = p->n_v % p->P;
  s->vec_rest = (s->part + 7) / 8;
  s->vec_wide = (s->part + 8) / 8;
  s->c = (float)(1.4426950408889634 / temperature);
  s->inv_t = (float)(1.0 / temperature);
  const int vecs = s->extra * s->vec_wide + (s->P - s->extra) * s->vec_rest;
  s->splits = logits_splits(p->rows, vecs, size == 2 ? logits_batch<uint16_t>() : logits_batch<float>(), parts);
  s->per = (vecs + s->splits - 1) / s->splits;
  return DISTDL_OK;
}

// floats of scratch on this stream; a plan's first call there cannot be a recorded one
static int logits_scratch(distdl_logits_plan* p, size_t floats, hipStream_t st, float** out) {
  bool is_new = true;
  for (const StreamScratch::Block& b : p->scratch.blocks) is_new = is_new && (b.stream != st || b.floats < floats);
  if (is_new) {
    hipStreamCaptureStatus capture = hipStreamCaptureStatusNone;
    DISTDL_HIP_TRY(hipStreamIsCapturing(st, &capture));
    if (capture != hipStreamCaptureStatusNone)
      return set_error(DISTDL_ERR_INVALID_ARG, "logits: the plan's first such call on this stream, which is being captured");
  }
  return p->scratch.get(floats, st, out);
}

static int logits_aligned(const char* call, std::initializer_list<const void*> all) {
  for (const void* v : all)
    if ((uintptr_t)v % 4) return set_error(DISTDL_ERR_INVALID_ARG, "%s: an array of the rows is not aligned to its elements", call);
  return DISTDL_OK;
}

// Rounds of `threads` threads with `batch` vectors each over a row.
static int64_t logits_rounds(const LogitsArgs& s, int threads, int batch) {
  const int64_t each = (int64_t)threads * batch, wide = (s.vec_wide + each - 1) / each, rest = (s.vec_rest + each - 1) / each;
  return s.extra * wide + (s.P - s.extra) * rest;
}
// Whether a row is one wave's: nothing to join, and where a worker's part is short, no waves without work.  us for 8192 rows, bf16, workgroup / wave:
//   sums                   8192 entries on 1 worker 31 / 26, 16384 on 1 52 / 54, 16384 on 8 140 / 52
//   with 20 alternatives   512 on 1 48 / 16, 16384 on 1 133 / 94; 4096 rows: 512 27 / 11, 16384 73 / 60; 2048 rows: 2048 19 / 14, 4096 20 / 21, 8192 28 / 32;
//                          1024 rows: 1024 12.6 / 9.4, 2048 13.2 / 13.4, 4096 14 / 20; 600 rows: 1024 11.6 / 9.2, 2048 12.0 / 13.4, 8192 18 / 29
//   adjoint                4096 on 1 32 / 27, 8192 on 1 52 / 57, 2048 on 8 203 / 61
//   distillation           4096 on 1 62 / 48, 8192 on 1 88 / 91, 16384 on 8 143 / 166
static int64_t logits_vectors(const LogitsArgs& s) { return s.extra * s.vec_wide + (int64_t)(s.P - s.extra) * s.vec_rest; }
constexpr int kWaveVectors = 4096;  // at most 512 numbers of a lane one behind the other in a sum, as a workgroup has of 131072
static bool logits_wave_sums(const LogitsArgs& s, int batch) {
  return s.splits == 1 && logits_vectors(s) <= kWaveVectors && logits_rounds(s, 64, batch) <= std::max<int64_t>(4, 2 * logits_rounds(s, kLogitsThreads, batch));
}
static bool logits_wave_top(const LogitsArgs& s) { return s.splits == 1 && logits_vectors(s) <= (s.rows >= 4096 ? kWaveVectors : 256); }
static bool logits_wave_adjoint(const LogitsArgs& s, int batch) {
  return s.splits == 1 && logits_rounds(s, 64, batch) <= 2 * logits_rounds(s, kLogitsThreads, batch);
}
// (256 places: 8192 rows of 1024 on 1 57 / 37, of 4096 on 1 72 / 79, 600 of 1000, fp32, 10 / 14)
static bool logits_wave_distill(const LogitsArgs& s, int batch) {
  const bool many = s.n_top > kStoredFew;
  return s.splits == 1 && s.n_top <= kStoredWave && logits_vectors(s) <= (many ? 64 : 128) * batch && (!many || s.rows >= 4096);
}

template <class E, bool ENTROPY, bool TINY>
static void launch_logits_fwd(const LogitsArgs& s, hipStream_t st) {
  const dim3 grid((unsigned)(s.rows * s.splits)), block(kLogitsThreads);
  if (s.n_top > 0) {
    if (logits_wave_top(s)) hipLaunchKernelGGL((logits_fwd_kernel<E, ENTROPY, true, false, TINY, 64>), grid, dim3(64), 0, st, s);
    else if (s.splits > 1) hipLaunchKernelGGL((logits_fwd_kernel<E, ENTROPY, true, true, TINY, kLogitsThreads>), grid, block, 0, st, s);
    else hipLaunchKernelGGL((logits_fwd_kernel<E, ENTROPY, true, false, TINY, kLogitsThreads>), grid, block, 0, st, s);
  } else {
    if (logits_wave_sums(s, logits_batch<E>())) hipLaunchKernelGGL((logits_fwd_kernel<E, ENTROPY, false, false, TINY, 64>), grid, dim3(64), 0, st, s);
    else hipLaunchKernelGGL((logits_fwd_kernel<E, ENTROPY, false, false, TINY, kLogitsThreads>), grid, block, 0, st, s);
  }
  if (s.splits > 1) hipLaunchKernelGGL((logits_join_kernel<E>), dim3((unsigned)s.rows), block, 0, st, s);
}

template <class E, bool ENTROPY, bool TINY>
static void launch_logits_bwd(const LogitsArgs& s, hipStream_t st) {
  const dim3 grid((unsigned)(s.rows * s.splits));
  if (logits_wave_adjoint(s, logits_batch<E>())) hipLaunchKernelGGL((logits_bwd_kernel<E, ENTROPY, TINY, 64>), grid, dim3(64), 0, st, s);
  else hipLaunchKernelGGL((logits_bwd_kernel<E, ENTROPY, TINY, kLogitsThreads>), grid, dim3(kLogitsThreads), 0, st, s);
}

// Threads of a workgroup that keeps a row in its registers; 0: none does.
static int distill_threads(const LogitsArgs& s, int slots) {
  if (s.part < 8) return 0;
  for (int threads : {256, 512}) {
    const int64_t wide = (s.vec_wide + threads - 1) / threads, rest = (s.vec_rest + threads - 1) / threads;
    if (s.extra * wide + (s.P - s.extra) * rest <= slots) return threads;
  }
  return 0;
}

template <class E, bool TINY>
static void launch_distill(const LogitsArgs& s, bool gradient, hipStream_t st) {
  const dim3 grid((unsigned)(s.rows * s.splits)), block(kLogitsThreads);
  if (logits_wave_distill(s, logits_batch<E>())) {
    hipLaunchKernelGGL((distill_kernel<E, false, TINY, 64>), grid, dim3(64), 0, st, s);
    return;
  }
  const int kept = s.splits == 1 && gradient ? distill_threads(s, distill_slots<E>()) : 0;
  if (kept == 256) hipLaunchKernelGGL((distill_kept_kernel<E, 256>), grid, dim3(256), 0, st, s);
  else if (kept == 512) hipLaunchKernelGGL((distill_kept_kernel<E, 512>), grid, dim3(512), 0, st, s);
  if (kept) return;
  // A row that is read twice should still be in the last cache (256 MB) then: so many threads that the rows under way are half of that.
  const size_t bytes = (size_t)s.n_v * sizeof(E);
  if (s.splits > 1) {
    hipLaunchKernelGGL((distill_kernel<E, true, TINY, kLogitsThreads>), grid, block, 0, st, s);
    hipLaunchKernelGGL((distill_kernel<E, false, TINY, kLogitsThreads>), grid, block, 0, st, s);
  } else if (bytes <= 64 << 10 || TINY) {
    hipLaunchKernelGGL((distill_kernel<E, false, TINY, kLogitsThreads>), grid, block, 0, st, s);
  } else if (bytes <= 128 << 10) {
    hipLaunchKernelGGL((distill_kernel<E, false, false, 512>), grid, dim3(512), 0, st, s);
  } else {
    hipLaunchKernelGGL((distill_kernel<E, false, false, 1024>), grid, dim3(1024), 0, st, s);
  }
}

// f(element, whether there is an option, whether a worker has fewer than eight entries)
template <class F>
static void logits_kind(distdl_dtype dtype, bool option, bool tiny, F f) {
  auto by_tiny = [&](auto e, auto o) { tiny ? f(e, o, std::true_type()) : f(e, o, std::false_type()); };
  auto by_option = [&](auto e) { option ? by_tiny(e, std::true_type()) : by_tiny(e, std::false_type()); };
  dtype == DISTDL_F32 ? by_option(float()) : by_option(uint16_t());
}

}  // namespace distdl

using namespace distdl;

extern "C" {

int distdl_logits_plan_create(distdl_logits_plan** out, int64_t rows, int64_t n_v, int P, distdl_dtype dtype) {
  if (!out) return set_error(DISTDL_ERR_NULL, "logits_plan_create: null argument");
  *out = nullptr;
  if (rows < 0 || n_v < 1 || P < 1) return set_error(DISTDL_ERR_INVALID_ARG, "logits_plan_create: %lld rows of %lld entries on %d workers",
                                                     (long long)rows, (long long)n_v, P);
  if (dtype != DISTDL_F32 && dtype != DISTDL_BF16) return set_error(DISTDL_ERR_UNSUPPORTED, "unknown dtype");
  if (n_v < P) return set_error(DISTDL_ERR_EMPTY_PARTITION, "logits: %lld entries over %d workers", (long long)n_v, P);
  if (n_v > 1 << 28 || rows >= kMaxBlocks256 || P > 1 << 12) return set_error(DISTDL_ERR_UNSUPPORTED, "logits: problem too large");
  return guarded([&]() -> int {
    std::unique_ptr<distdl_logits_plan> p(new distdl_logits_plan());
    p->rows = rows;
    p->n_v = (int32_t)n_v;
    p->P = P;
    p->dtype = dtype;
    *out = p.release();
    return DISTDL_OK;
  });
}

int distdl_logits_plan_destroy(distdl_logits_plan* p) {
  if (!p) return DISTDL_OK;
  p->table.release();
  p->scratch.release();
  delete p;
  return DISTDL_OK;
}

int distdl_logprob_fwd(distdl_logits_plan* p, const void* const x_dev[], const int32_t* targets_dev, float* logp_dev, float* lse_dev,
                       float* entropy_dev, int32_t* top_ids_dev, float* top_logp_dev, int n_top, double temperature, void* stream) {
  if (!p || !x_dev) return set_error(DISTDL_ERR_NULL, "logprob_fwd: null argument");
  if (n_top < 0 || n_top > p->n_v) return set_error(DISTDL_ERR_INVALID_ARG, "logprob_fwd: %d alternatives of %d entries", n_top, p->n_v);
  if (n_top > kTopMost) return set_error(DISTDL_ERR_UNSUPPORTED, "logprob_fwd: more than %d alternatives", kTopMost);
  if (p->rows == 0) return DISTDL_OK;
  if (logp_dev && !targets_dev) return set_error(DISTDL_ERR_NULL, "logprob_fwd: log probabilities without targets");
  if (n_top > 0 && !top_ids_dev && !top_logp_dev) return set_error(DISTDL_ERR_NULL, "logprob_fwd: alternatives without a place for them");
  if (n_top == 0 && (top_ids_dev || top_logp_dev)) return set_error(DISTDL_ERR_INVALID_ARG, "logprob_fwd: a place for no alternatives");
  if (!logp_dev && !lse_dev && !entropy_dev && n_top == 0) return set_error(DISTDL_ERR_NULL, "logprob_fwd: no output");
  return guarded([&]() -> int {
    hipStream_t st_ = (hipStream_t)stream;
    LogitsArgs s;
    int rc;
    if ((rc = logits_aligned("logprob_fwd", {targets_dev, logp_dev, lse_dev, entropy_dev, top_ids_dev, top_logp_dev}))) return rc;
    if ((rc = logits_args(p, x_dev, nullptr, temperature, p->P, st_, &s))) return rc;
    s.targets = targets_dev;
    s.logp = logp_dev;
    s.lse = lse_dev;
    s.entropy = entropy_dev;
    s.n_top = n_top;
    s.ids = top_ids_dev;
    s.top = top_logp_dev;
    if (s.splits > 1) {
      const size_t blocks = (size_t)p->rows * s.splits;
      float* at = nullptr;
      if ((rc = logits_scratch(p, blocks * (4 + 2 * (size_t)n_top), st_, &at))) return rc;
      s.parts = (float4*)at;
      s.part_top = (uint64_t*)(at + blocks * 4);
    }
    {
      ProfScope prof("logprob_fwd", st_);
      logits_kind(p->dtype, entropy_dev != nullptr, s.part < 8,
                  [&](auto e, auto entropy, auto tiny) { launch_logits_fwd<decltype(e), decltype(entropy)::value, decltype(tiny)::value>(s, st_); });
    }
    DISTDL_HIP_TRY(hipGetLastError());
    return DISTDL_OK;
  });
}

int distdl_logprob_bwd(distdl_logits_plan* p, const void* const x_dev[], const int32_t* targets_dev, const float* lse_dev,
                       const float* entropy_dev, const float* dlogp_dev, const float* dentropy_dev, void* const dx_dev[], double temperature,
                       void* stream) {
  if (!p || !x_dev || !dx_dev) return set_error(DISTDL_ERR_NULL, "logprob_bwd: null argument");
  if (p->rows == 0) return DISTDL_OK;
  if (!lse_dev || (!dlogp_dev && !dentropy_dev)) return set_error(DISTDL_ERR_NULL, "logprob_bwd: no lse, or no gradient");
  if (dlogp_dev && !targets_dev) return set_error(DISTDL_ERR_NULL, "logprob_bwd: gradients of log probabilities without targets");
  if (dentropy_dev && !entropy_dev) return set_error(DISTDL_ERR_NULL, "logprob_bwd: the entropy's gradient without the entropy");
  return guarded([&]() -> int {
    hipStream_t st_ = (hipStream_t)stream;
    LogitsArgs s;
    int rc;
    if ((rc = logits_aligned("logprob_bwd", {targets_dev, lse_dev, entropy_dev, dlogp_dev, dentropy_dev}))) return rc;
    if ((rc = logits_args(p, x_dev, dx_dev, temperature, p->P, st_, &s))) return rc;
    s.targets = dlogp_dev ? targets_dev : nullptr;
    s.lse = const_cast<float*>(lse_dev);
    s.entropy = const_cast<float*>(entropy_dev);
    s.dlogp = dlogp_dev;
    s.dentropy = dentropy_dev;
    {
      ProfScope prof("logprob_bwd", st_);
      logits_kind(p->dtype, dentropy_dev != nullptr, s.part < 8,
                  [&](auto e, auto entropy, auto tiny) { launch_logits_bwd<decltype(e), decltype(entropy)::value, decltype(tiny)::value>(s, st_); });
    }
    DISTDL_HIP_TRY(hipGetLastError());
    return DISTDL_OK;
  });
}

int distdl_distill_fwd_bwd(distdl_logits_plan* p, const void* const x_dev[], const int32_t* ids_dev, const float* teacher_dev, int n_top,
                           const float* weight_dev, float* loss_dev, void* const dx_dev[], double temperature, void* stream) {
  if (!p || !x_dev) return set_error(DISTDL_ERR_NULL, "distill: null argument");
  if (n_top < 1) return set_error(DISTDL_ERR_INVALID_ARG, "distill: %d teacher logits a row", n_top);
  if (n_top > kStoredMost) return set_error(DISTDL_ERR_UNSUPPORTED, "distill: more than %d teacher logits a row", kStoredMost);
  if (p->rows == 0) return DISTDL_OK;
  if (!ids_dev || !teacher_dev || (!loss_dev && !dx_dev)) return set_error(DISTDL_ERR_NULL, "distill: no teacher, or no output");
  return guarded([&]() -> int {
    hipStream_t st_ = (hipStream_t)stream;
    LogitsArgs s;
    int rc;
    if ((rc = logits_aligned("distill", {ids_dev, teacher_dev, weight_dev, loss_dev}))) return rc;
    if ((rc = logits_args(p, x_dev, dx_dev, temperature, 1, st_, &s))) return rc;
    s.stored_ids = ids_dev;
    s.stored = teacher_dev;
    s.n_top = n_top;
    s.weight = weight_dev;
    s.loss = loss_dev;
    if (s.splits > 1) {
      const size_t blocks = (size_t)p->rows * s.splits;
      float* at = nullptr;
      if ((rc = logits_scratch(p, blocks * 4 + (size_t)p->rows * n_top, st_, &at))) return rc;
      s.parts = (float4*)at;
      s.stored_x = at + blocks * 4;
    }
    {
      ProfScope prof("distill", st_);
      logits_kind(p->dtype, false, s.part < 8, [&](auto e, auto, auto tiny) { launch_distill<decltype(e), decltype(tiny)::value>(s, dx_dev != nullptr, st_); });
    }
    DISTDL_HIP_TRY(hipGetLastError());
    return DISTDL_OK;
  });
}

}  // extern "C"
