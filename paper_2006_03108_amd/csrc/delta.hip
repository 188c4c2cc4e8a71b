// The gated delta rule over time that P workers share, its adjoint, and the step of single tokens.
//
//   u_t = beta_t (v_t - a_t S_{t-1}^T k_t),  S_t = a_t S_{t-1} + k_t u_t^T,  o_t = scale S_t^T q_t,  a_t = exp(g_t)
//
// A state S [d_k][d_v] is changed by each step in a direction of its own, so steps do not compose as those of an elementwise
// recurrence do.  But what the C steps of a chunk do to each other is triangular.  With G_i the sum of g over the chunk's steps up to i and
// D_ij = exp(G_i - G_j), S the state in front of the chunk:
//   A = strictly lower (beta_i D_ij k_i k_j),  T = (1 + A)^-1,  P = lower (scale D_ij q_i k_j)
//   X = V - exp(G) (K S),  U = T (beta X),  O = scale exp(G) (Q S) + P U,  S' = exp(G_C) S + K^T (exp(G_C - G) U)
// A, T and P need no state: one launch makes them for all chunks (delta_prepare_kernel).  What is left goes through time, and its columns
// (of d_v) are independent: a workgroup has 16 or 32 columns of a head's state in its registers and goes through all chunks, from product
// to product.  Differences of G are exact: sums in 64 bits and in units of log 2, kept as a multiple of 1/64 and the rest.
#include <algorithm>
#include <cmath>

#include "delta.h"
#include "lds_direct.h"
#include "profile.h"

namespace distdl {

// A factor of exp(-200) is 0 in 32 bits, and so is what it stands between.
__device__ __forceinline__ float bounded(float g) { return g < -200.f ? -200.f : g; }

// The adjoint has what beta multiplies as U / beta, where beta is no less than 2^-64: below, it is 0, which adds nothing to a state, and X is kept in U's place.
__device__ __forceinline__ float divisor(float beta) { return fabsf(beta) < 0x1p-64f ? 0.f : beta; }

// Whether K^T is made of K where it is used.
template <class E>
constexpr bool delta_turned() { return sizeof(E) == 2; }

// ---- a chunk's own matrices -----------------------------------------------
// (The waves of these kernels meet over LDS alone, so their barriers leave global loads and stores under way: lds_barrier.)
template <class E, int C, int DK>
struct DeltaPrepareShared {
  static constexpr int kRow = DK + 8, kLine = C + 4;
  union {
    uint16_t rows[2][delta_pieces<E>()][C][kRow];  // K, Q
    struct {
      float a[C][kLine], t[C][kLine], p[C][kLine];
    };
  };
  static constexpr int kHeads = 2;  // (with four, two workgroups share a compute unit instead of three)
  float whole[kHeads][C], rest[kHeads][C], beta[kHeads][C];  // G = whole + rest
};

// (1 + a)^-1 of a strictly lower matrix in `a`, into `t`, zeros above the diagonal.  Blocks of 16 on the diagonal by substitution, a
// column to a lane; block (i, j) is -T_ii sum_k A_ik T_kj, by distance from the diagonal, in fp32 products.
template <int C, int LINE>
__device__ __forceinline__ void delta_inverse(const float (*a)[LINE], float (*t)[LINE]) {
  constexpr int N = C / 16;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, col = lane & 15, g = lane >> 4;
  if (wave < N) {
    const int at = wave * 16;
    f32x4 left[16][4];  // the block's rows, the same for all lanes
#pragma unroll
    for (int i = 1; i < 16; ++i)
#pragma unroll
      for (int j = 0; j < i; j += 4) left[i][j / 4] = *(const f32x4*)&a[at + i][at + j];
    float x[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = i == col ? 1.f : 0.f;
#pragma unroll
    for (int j = 0; j < 15; ++j)
#pragma unroll
      for (int i = j + 1; i < 16; ++i) x[i] = fmaf(-left[i][j / 4][j % 4], x[j], x[i]);
    if (g == 0) {
#pragma unroll
      for (int i = 0; i < 16; ++i) t[at + i][at + col] = x[i];
    }
  }
  for (int d = 1; d < N; ++d) {
    lds_barrier();
    const int i = wave + d, j = wave;
    if (i < N) {
      f32x4 sum = {};
      for (int k = j; k < i; ++k) {
        const f32x4 left = *(const f32x4*)&a[i * 16 + col][k * 16 + 4 * g];
#pragma unroll
        for (int r = 0; r < 4; ++r) sum = __builtin_amdgcn_mfma_f32_16x16x4f32(left[r], t[k * 16 + 4 * g + r][j * 16 + col], sum, 0, 0, 0);
      }
      f32x4 out = {};
      const f32x4 left = *(const f32x4*)&t[i * 16 + col][i * 16 + 4 * g];
#pragma unroll
      for (int r = 0; r < 4; ++r) out = __builtin_amdgcn_mfma_f32_16x16x4f32(left[r], -sum[r], out, 0, 0, 0);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        t[i * 16 + 4 * g + r][j * 16 + col] = out[r];
        t[j * 16 + 4 * g + r][i * 16 + col] = 0.f;
      }
    }
  }
  lds_barrier();
}

// The places along a fragment's sum that a lane has: element e of step ks.
__device__ __forceinline__ int delta_place(int ks, int e) { return 32 * ks + (e >> 2) * 16 + 4 * ((threadIdx.x & 63) >> 4) + (e & 3); }

// Tiles on and below the diagonal, by rows.
struct DeltaLower {
  int mt, nt;
};
__device__ __forceinline__ DeltaLower delta_lower(int tile) {
  const int mt = tile >= 6 ? 3 : tile >= 3 ? 2 : tile >= 1 ? 1 : 0;
  return DeltaLower{mt, tile - mt * (mt + 1) / 2};
}

// A workgroup has a chunk of a key's head and its heads (or a share of them), whose matrices have K K^T and Q K^T in common: these stay in registers.
template <class E, int C, int DK, bool BACK>
__global__ __launch_bounds__(256, 2) void delta_prepare_kernel(DeltaArgs s) {
  typedef DeltaSizes<C, DK> Z;
  typedef DeltaPrepareShared<E, C, DK> Shared;
  constexpr int NI = delta_pieces<E>();
  extern __shared__ char delta_lds[];
  Shared& m = *(Shared*)delta_lds;
  const DeltaTable table = DELTA_TABLE(s);
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, row = lane & 15, g = lane >> 4;
  const int hk = blockIdx.x % (uint32_t)s.n_hk, at_chunk = blockIdx.x / (uint32_t)s.n_hk;
  const int c = at_chunk % s.chunks, b = at_chunk / s.chunks, share = blockIdx.y, shares = gridDim.y;
  const int e_first = share * s.each / shares, e_end = (share + 1) * s.each / shares;
  const DeltaChunk at = delta_chunk(s, b, c);
  if (at.live == 0) return;  // nobody reads what would be here
  const int64_t step0 = (int64_t)b * at.steps + at.first;  // of the worker's arrays
  const DeltaTable w = table + at.p;

  // The sums of g for a head, by a wave.
  auto sum_up = [&](int e) {
    if (wave >= Shared::kHeads || e + wave >= e_end) return;
    const int h = hk * s.each + e + wave;
    const int64_t head = ((int64_t)b * s.chunks + c) * s.n_h + h;
    const bool live = lane < at.live;
    const int64_t o = (step0 + lane) * s.n_h + h;
    const float beta = !live ? 0.f : BACK ? divisor(w->beta[o]) : w->beta[o];
    double sum = live && w->g ? (double)bounded(w->g[o]) * 1.4426950408889634 : 0.0;
#pragma unroll
    for (int d = 1; d < C; d *= 2) {
      const double before = __shfl_up(sum, d, 64);
      if (lane >= d) sum += before;
    }
    const double last = __shfl(sum, C - 1, 64);
    const float whole = (float)(rint(sum * 64.0) * (1.0 / 64.0)), rest = (float)(sum - (double)whole);
    m.whole[wave][lane] = whole;
    m.rest[wave][lane] = rest;
    m.beta[wave][lane] = beta;
    float* const out = s.steps + head * kStepNumbers * C + lane;
    out[kSince * C] = __builtin_amdgcn_exp2f((float)sum);
    out[kUntil * C] = __builtin_amdgcn_exp2f((float)(last - sum));
    out[kBeta * C] = beta;
    out[kWhole * C] = whole;
    out[kRest * C] = rest;
  };

  // rows of K and Q, zeros behind the end of the sequence and of the row
  constexpr int kPieces = 2 * C * (DK / 8) / 256;
  Eight<E> raw[kPieces];
#pragma unroll
  for (int x = 0; x < kPieces; ++x) {
    const int i = tid + 256 * x, what = i / (C * (DK / 8)), t = i / (DK / 8) % C, col = i % (DK / 8) * 8;
    raw[x].load((const E*)(what ? w->q : w->k) + ((step0 + t) * s.n_hk + hk) * s.d_k + col, t < at.live ? min(8, s.d_k - col) : 0);
  }
  sum_up(e_first);
#pragma unroll
  for (int x = 0; x < kPieces; ++x) {
    const int i = tid + 256 * x, what = i / (C * (DK / 8)), t = i / (DK / 8) % C, col = i % (DK / 8) * 8;
    if constexpr (NI == 1) {
      *(u32x4*)&m.rows[what][0][t][col] = raw[x].a;
    } else {
      float v[8];
      raw[x].values(v);
      const Pieces<3> p = split8(v);
#pragma unroll
      for (int k = 0; k < 3; ++k) *(u32x4*)&m.rows[what][k][t][col] = p.p[k];
    }
  }
  lds_barrier();

  // their fragments
  const int64_t key = ((int64_t)b * s.chunks + c) * s.n_hk + hk, key_at = key * Z::kKeyPiece * NI;
  for (int f = wave + 4 * share; f < (BACK ? 1 : 2) * Z::kTiles * Z::kKeySteps; f += 4 * shares) {  // (the adjoint needs no Q and no P as they are)
    const int what = f / (Z::kTiles * Z::kKeySteps), i = f % (Z::kTiles * Z::kKeySteps), mt = i / Z::kKeySteps, ks = i % Z::kKeySteps;
    Pieces<NI> v;
#pragma unroll
    for (int k = 0; k < NI; ++k) {
      const uint16_t* const r = &m.rows[what][k][mt * 16 + row][32 * ks + 4 * g];
      const u32x2 lo = *(const u32x2*)r, hi = *(const u32x2*)(r + 16);
      v.p[k] = u32x4{lo[0], lo[1], hi[0], hi[1]};
    }
    store_fragment((what ? s.qf : s.kf) + key_at + (int64_t)i * NI * kFragment, v);
  }
  for (int f = wave + 4 * share; f < (BACK ? 2 : delta_turned<E>() ? 0 : 1) * Z::kKeyTiles * Z::kSteps; f += 4 * shares) {
    const int what = f / (Z::kKeyTiles * Z::kSteps), i = f % (Z::kKeyTiles * Z::kSteps), mt = i / Z::kSteps, ts = i % Z::kSteps;
    Pieces<NI> v;
#pragma unroll
    for (int k = 0; k < NI; ++k)
#pragma unroll
      for (int e = 0; e < 8; e += 2)
        v.p[k][e / 2] = m.rows[what][k][delta_place(ts, e)][mt * 16 + row] | (uint32_t)m.rows[what][k][delta_place(ts, e + 1)][mt * 16 + row] << 16;
    store_fragment((what ? s.qtf : s.ktf) + key_at + (int64_t)i * NI * kFragment, v);
  }

  // K K^T and Q K^T, tiles on and below the diagonal: a wave has the same tiles of both
  constexpr int kLower = Z::kLower, kJobs = (kLower + 3) / 4;
  f32x4 kk[kJobs] = {}, qk[kJobs] = {};
#pragma unroll
  for (int i = 0; i < kJobs; ++i) {
    if (wave + 4 * i >= kLower) continue;
    const DeltaLower at_tile = delta_lower(wave + 4 * i);
    for (int ks = 0; ks < Z::kKeySteps; ++ks) {
      Pieces<NI> one, two, right;
#pragma unroll
      for (int k = 0; k < NI; ++k) {
        one.p[k] = *(const u32x4*)&m.rows[0][k][at_tile.mt * 16 + row][32 * ks + 8 * g];
        two.p[k] = *(const u32x4*)&m.rows[1][k][at_tile.mt * 16 + row][32 * ks + 8 * g];
        right.p[k] = *(const u32x4*)&m.rows[0][k][at_tile.nt * 16 + row][32 * ks + 8 * g];
      }
      kk[i] = multiply(one, right, kk[i]);
      qk[i] = multiply(two, right, qk[i]);
    }
  }

  for (int e = e_first; e < e_end; ++e) {
    const int h = hk * s.each + e, slot = (e - e_first) % Shared::kHeads;
    const int64_t head = ((int64_t)b * s.chunks + c) * s.n_h + h;
    lds_barrier();
    if (e > e_first && slot == 0) {
      sum_up(e);
      lds_barrier();
    }
    // A and P, zeros above the diagonal
#pragma unroll
    for (int x = 0; x < kJobs; ++x) {
      if (wave + 4 * x >= kLower) continue;
      const DeltaLower at_tile = delta_lower(wave + 4 * x);
      const int j = at_tile.nt * 16 + row;
      const float whole = m.whole[slot][j], rest = m.rest[slot][j];
      f32x4 a, p;  // (a: A / beta)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int i = at_tile.mt * 16 + 4 * g + r;
        const float decay = i >= j ? __builtin_amdgcn_exp2f((m.whole[slot][i] - whole) + (m.rest[slot][i] - rest)) : 0.f;
        a[r] = i > j ? decay * kk[x][r] : 0.f;
        p[r] = i >= j ? s.scale * decay * qk[x][r] : 0.f;
        m.a[i][j] = m.beta[slot][i] * a[r];
        m.p[i][j] = p[r];
        if (at_tile.mt != at_tile.nt) m.p[at_tile.nt * 16 + 4 * g + r][at_tile.mt * 16 + row] = 0.f;
      }
      if constexpr (BACK) {
        f32x4* const to = (f32x4*)s.tiles + (head * 2 * kLower + wave + 4 * x) * 64 + lane;
        to[0] = a;
        to[kLower * 64] = p;
      }
    }
    lds_barrier();
    delta_inverse<C>(m.a, m.t);
    // fragments that are not all zeros
    for (int f = wave; f < Z::kTiles * Z::kSteps; f += 4) {
      const int mt = f / Z::kSteps, ts = f % Z::kSteps, i = mt * 16 + row;
      const int64_t o = head * Z::kStepPiece * kInner + (int64_t)f * kInner * kFragment;
      if (ts * 2 <= mt) {
        auto across = [&](const float (*from)[Shared::kLine]) {
          return split_tiles(*(const f32x4*)&from[i][32 * ts + 4 * g], *(const f32x4*)&from[i][32 * ts + 16 + 4 * g]);
        };
        store_fragment(s.tf + o, across(m.t));
        if constexpr (!BACK) store_fragment(s.pf + o, across(m.p));
      }
      if (BACK && mt / 2 <= ts) {
        auto down = [&](const float (*from)[Shared::kLine]) {
          float v[8];
#pragma unroll
          for (int x = 0; x < 8; ++x) v[x] = from[delta_place(ts, x)][i];
          return split8(v);
        };
        store_fragment(s.ttf + o, down(m.t));
        store_fragment(s.ptf + o, down(m.p));
      }
    }
  }
}

// ---- through time ---------------------------------------------------------
// A head's columns of a chunk's rows.  A wave has the steps 16 w + 4 g + r and the columns lane % 16 + 16 n: offsets that no chunk changes, and
// columns that do not exist fail the check of any buffer.  Steps from `n` on fail that of this chunk's.
template <class E, int NT>
struct DeltaColumns {
  typedef std::conditional_t<sizeof(E) == 4, uint32_t, uint16_t> Raw;  // (as loaded: a conversion would wait for it)
  uint32_t off[NT][4];
  uint32_t hop, row;
  __device__ __forceinline__ DeltaColumns(const DeltaArgs& s, int tile, int col) : hop((uint32_t)(s.n_h * s.d_v) * (uint32_t)sizeof(E)), row((uint32_t)s.d_v * (uint32_t)sizeof(E)) {
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        off[n][r] = col + 16 * n < s.d_v ? (uint32_t)(16 * tile + 4 * ((threadIdx.x & 63) >> 4) + r) * hop + (uint32_t)(col + 16 * n) * (uint32_t)sizeof(E) : kOob;
  }
  __device__ __forceinline__ __amdgpu_buffer_rsrc_t rows(const DeltaArgs& s, const DeltaWalk& at, int b, int h, int n) const {
    n = __builtin_amdgcn_readfirstlane(n);  // (uniform; what the compiler takes for a lane's own it would load in a loop over lanes)
    return rsrc_of((const E*)at.array + (((int64_t)b * at.steps + at.first) * s.n_h + h) * s.d_v, n > 0 ? (uint32_t)(n - 1) * hop + row : 0u);
  }
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t from, Raw (&raw)[NT][4]) const {
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        if constexpr (sizeof(E) == 4) raw[n][r] = __builtin_amdgcn_raw_buffer_load_b32(from, off[n][r], 0, 0);
        else raw[n][r] = __builtin_amdgcn_raw_buffer_load_b16(from, off[n][r], 0, 0);
      }
  }
  static __device__ __forceinline__ f32x4 values(const Raw (&raw)[4]) {
    f32x4 v;
#pragma unroll
    for (int r = 0; r < 4; ++r) v[r] = __uint_as_float(sizeof(E) == 4 ? raw[r] : (uint32_t)raw[r] << 16);
    return v;
  }
  __device__ __forceinline__ void store(__amdgpu_buffer_rsrc_t to, int n, f32x4 v) const {
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      if constexpr (sizeof(E) == 4) __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(v[r]), to, off[n][r], 0, 0);
      else __builtin_amdgcn_raw_buffer_store_b16(to_bf16(v[r]), to, off[n][r], 0, 0);
    }
  }
};

struct DeltaChain {  // a workgroup's sequence, head and first column
  int b, h, col;
};
template <int NT>
__device__ __forceinline__ DeltaChain delta_chain(const DeltaArgs& s) {
  const uint32_t i = xcd_order(blockIdx.x, gridDim.x);  // a head's slices share an L2
  const uint32_t chain = i / (uint32_t)s.slices, slice = i % (uint32_t)s.slices;
  return DeltaChain{(int)(chain / (uint32_t)s.n_h), (int)(chain % (uint32_t)s.n_h), (int)slice * 16 * NT};
}

struct Nothing {
  __device__ __forceinline__ void operator()() const {}
};
// An operand that the four waves of a workgroup make together and all read: [steps of the sum][column tiles][pieces][lanes].
template <int STEPS, int NT, int N>
struct DeltaShared {
  u32x4 v[STEPS][NT][N][64];
  __device__ __forceinline__ Pieces<N> read(int k, int n) const {
    Pieces<N> o;
#pragma unroll
    for (int i = 0; i < N; ++i) o.p[i] = v[k][n][i][threadIdx.x & 63];
    return o;
  }
  // c[n] += left b for the `count` steps from `first` on: all of b is read before the first product, which the compiler would otherwise make wait
  // for one read after the other
  template <int COUNT, int NA, class F = Nothing>
  __device__ __forceinline__ void multiply_into(const Pieces<NA>* left, int first, f32x4 (&c)[NT], F while_reading = F()) const {
    Pieces<N> right[COUNT][NT];
#pragma unroll
    for (int k = 0; k < COUNT; ++k)
#pragma unroll
      for (int n = 0; n < NT; ++n) right[k][n] = read(first + k, n);
    __builtin_amdgcn_sched_barrier(0);
    while_reading();
    __builtin_amdgcn_sched_barrier(0);
    f32x4 odd[NT] = {};
#pragma unroll
    for (int k = 0; k < COUNT; ++k)
#pragma unroll
      for (int n = 0; n < NT; ++n) (k & 1 ? odd : c)[n] = multiply(left[k], right[k][n], (k & 1 ? odd : c)[n]);
    if (COUNT > 1) {
#pragma unroll
      for (int n = 0; n < NT; ++n) c[n] += odd[n];
    }
  }
  // tile `tile` of 16 rows: half of a step
  __device__ __forceinline__ void write(int tile, int n, f32x4 x) {
    const Pieces<3> p = split_tiles(x, f32x4{});
#pragma unroll
    for (int i = 0; i < N; ++i) ((u32x2*)&v[tile >> 1][n][i][threadIdx.x & 63])[tile & 1] = u32x2{p.p[i][0], p.p[i][1]};
  }
};
// Every STRIDE-th piece from piece `from` on begins a fragment.  `at`: the first one's place, `hop`: from chunk to chunk.
template <int COUNT, int N, int STRIDE>
struct DeltaFragments {
  Pieces<N> v[COUNT];
  const char* at;
  int64_t hop;
  __device__ __forceinline__ void start(const uint16_t* base, int64_t chunk0, int heads, int head, int64_t numbers, int c, int from) {
    hop = (int64_t)heads * numbers * 2;
    at = (const char*)base + ((chunk0 + c) * heads + head) * numbers * 2 + (int64_t)from * kFragment * 2;
  }
  // fragments first .. last - 1; the others' loads are of nothing
  __device__ __forceinline__ void load(int first = 0, int last = COUNT) {
#pragma unroll
    for (int i = 0; i < COUNT; ++i) {
      const __amdgpu_buffer_rsrc_t from = rsrc_of(at, i >= first && i < last ? kOob : 0);
#pragma unroll
      for (int k = 0; k < N; ++k) {
        const int o = (i * STRIDE + k) * kFragment * 2;
        v[i].p[k] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(from, (threadIdx.x & 63) * 16 + (o & 4095), o & ~4095, 0));
      }
    }
  }
};
// exp(G), exp(G_C - G), beta of a wave's steps, and exp(G_C)
struct DeltaSteps {
  f32x4 since, until, beta;
  float decay;
  const float* at;
  int64_t hop;
  __device__ __forceinline__ void start(const DeltaArgs& s, int64_t chunk0, int h, int c) {
    hop = (int64_t)s.n_h * kStepNumbers * kChunk;
    at = s.steps + ((chunk0 + c) * s.n_h + h) * kStepNumbers * kChunk;
  }
  __device__ __forceinline__ void load(int tile) {
    const __amdgpu_buffer_rsrc_t from = rsrc_of(at, kStepNumbers * kChunk * 4);
    const uint32_t o = (uint32_t)(16 * tile + 4 * ((threadIdx.x & 63) >> 4)) * 4;
    since = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(from, o, kSince * kChunk * 4, 0));
    until = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(from, o, kUntil * kChunk * 4, 0));
    beta = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(from, o, kBeta * kChunk * 4, 0));
    decay = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(from, 0, (kChunk - 1) * 4, 0));
  }
};
// K^T of a wave's keys from K of the same: a product of tiles of steps with a matrix of zeros and ones has K's numbers where a lane of the left operand K^T
// wants them.  With bf16 keys that is 8 products and 16 other instructions in the time of the partial sums' reads, and 16 KiB less to load for a
// chunk and to make in front (the call 290 us instead of 316 for 8192 steps of 32 heads); with the three pieces of fp32 keys it is three times that, and fragments are loaded.
template <int KT>
struct DeltaTurn {
  u32x4 ones[KT];  // (16 keys of the 32) of a fragment
  __device__ __forceinline__ DeltaTurn(int wave) {
    const int at = (int)(threadIdx.x & 15) - 4 * (int)((threadIdx.x & 63) >> 4);  // a lane's element that is 1, of four
    const uint32_t lo = at == 0 ? 0x3f80u : at == 1 ? 0x3f800000u : 0u, hi = at == 2 ? 0x3f80u : at == 3 ? 0x3f800000u : 0u;
#pragma unroll
    for (int i = 0; i < KT; ++i) {
      const bool second = KT == 2 ? i == 1 : (wave & 1) != 0;
      ones[i] = second ? u32x4{0u, 0u, lo, hi} : u32x4{lo, hi, 0u, 0u};
    }
  }
  __device__ __forceinline__ void operator()(const Pieces<1> (&k)[4], Pieces<1> (&turned)[2 * KT]) const {
#pragma unroll
    for (int i = 0; i < KT; ++i)
#pragma unroll
      for (int mt = 0; mt < 4; ++mt) {
        const f32x4 v = multiply(k[mt], Pieces<1>{ones[i]}, f32x4{});
        turned[i * 2 + mt / 2].p[0][mt % 2 * 2] = to_bf16(v[0], v[1]);  // (exact)
        turned[i * 2 + mt / 2].p[0][mt % 2 * 2 + 1] = to_bf16(v[2], v[3]);
      }
  }
};
// Tiles of results in fp32, as they lie in the lanes.
template <int TILES, int NT>
struct DeltaTiles {
  f32x4 v[TILES][NT][64];
};

// A wave's rows of the state as the operand of a step over keys.  With DK = 64 they are half a step, the other half is zeros.
template <int KT, int NT>
__device__ __forceinline__ void delta_own(const f32x4 (&state)[KT][NT], int wave, Pieces<3> (&own)[NT]) {
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    if constexpr (KT == 2) own[n] = split_tiles(state[0][n], state[1][n]);
    else own[n] = wave & 1 ? split_tiles(f32x4{}, state[0][n]) : split_tiles(state[0][n], f32x4{});
  }
}
// K times a wave's rows of the state: its part of every tile of steps
template <int NT, int NA, class F>
__device__ __forceinline__ void delta_partial(const Pieces<NA>* left, const Pieces<3> (&own)[NT], int wave, DeltaTiles<16, NT>& to, F meanwhile) {
  f32x4 part[4][NT];
#pragma unroll
  for (int mt = 0; mt < 4; ++mt)
#pragma unroll
    for (int n = 0; n < NT; ++n) part[mt][n] = multiply(left[mt], own[n], f32x4{});
  __builtin_amdgcn_sched_barrier(0);
  meanwhile();
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int mt = 0; mt < 4; ++mt)
#pragma unroll
    for (int n = 0; n < NT; ++n) to.v[mt * 4 + wave][n][threadIdx.x & 63] = part[mt][n];
}
template <int NT, class F>
__device__ __forceinline__ void delta_joined(const DeltaTiles<16, NT>& from, int tile, f32x4 (&x)[NT], F while_reading) {
  f32x4 v[NT][4];
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int i = 0; i < 4; ++i) v[n][i] = from.v[tile * 4 + i][n][threadIdx.x & 63];
  __builtin_amdgcn_sched_barrier(0);
  while_reading();
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int n = 0; n < NT; ++n) x[n] = (v[n][0] + v[n][1]) + (v[n][2] + v[n][3]);
}

// A wave's rows of the state += left b
template <int KT, int NT, int NA, class F = Nothing>
__device__ __forceinline__ void delta_state(const DeltaShared<2, NT, 3>& b, const Pieces<NA>* left, f32x4 (&state)[KT][NT], F while_reading = F()) {
  Pieces<3> right[2][NT];
#pragma unroll
  for (int k = 0; k < 2; ++k)
#pragma unroll
    for (int n = 0; n < NT; ++n) right[k][n] = b.read(k, n);
  __builtin_amdgcn_sched_barrier(0);
  while_reading();
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int k = 0; k < 2; ++k)
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < KT; ++i) state[i][n] = multiply(left[i * 2 + k], right[k][n], state[i][n]);
}

// A workgroup takes 16 NT columns of a head's state through all chunks.  Of its first four waves, wave w has a quarter of the state's rows and the tile of steps
// 16 w .. 16 w + 15 of X and U, so the chunk's matrices are read by one wave each, straight into the registers that the last chunk's have left:
// every load has most of a chunk's time.  K S is the sum of what the waves' rows give.  These parts, beta X and U go through LDS, a barrier for each, which
// waits for LDS alone (lds_barrier).  Four more waves make the outputs, which nothing waits for.
template <class E, int DK, int NT, bool STORE>
__global__ __launch_bounds__(STORE ? 256 : 512, 2) void delta_fwd_kernel(DeltaArgs s) {
  typedef DeltaSizes<kChunk, DK> Z;
  typedef DeltaColumns<E, NT> Columns;
  constexpr int NI = delta_pieces<E>(), KT = DK / 64, KS = Z::kKeySteps;
  __shared__ DeltaTiles<16, NT> of_keys;  // K S: tile of steps, wave
  __shared__ DeltaShared<STORE ? 1 : KS, NT, 3> for_queries;
  __shared__ DeltaShared<2, NT, 3> for_inner, for_state;
  __shared__ DeltaShared<2, NT, STORE ? 1 : 3> for_out;
  const DeltaTable table = DELTA_TABLE(s);
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63, g = lane >> 4, tile = wave & 3;
  const DeltaChain chain = delta_chain<NT>(s);
  const int b = chain.b, h = chain.h, hk = h / s.each, col = chain.col + (lane & 15);
  const int len = delta_length(s, b), chunks = delta_live_chunks(s, len);
  const int64_t chunk0 = (int64_t)b * s.chunks;
  const Columns columns(s, tile, col);
  DeltaWalk walk;

  if (!STORE && wave >= 4) {  // O = scale exp(G) (Q S) + P U
    auto outputs = [&](int p) { return table[p].o; };
    DeltaFragments<KS, NI, NI> qf;
    DeltaFragments<2, kInner, kInner> pf;
    const int steps_in = tile < 2 ? 1 : 2;  // of the sums over steps, those that are not all zeros
    DeltaSteps steps;
    qf.start(s.qf, chunk0, s.n_hk, hk, Z::kKeyPiece * NI, 0, tile * KS * NI);
    pf.start(s.pf, chunk0, s.n_h, h, Z::kStepPiece * kInner, 0, tile * 2 * kInner);
    steps.start(s, chunk0, h, 0);
    walk.start(s, 0, outputs);
    if (chunks > 0) {
      qf.load();
      pf.load(0, steps_in);
      steps.load(tile);
    }
    __builtin_amdgcn_s_waitcnt(kWaitVmcnt0);  // (so that the loop's waits count its own loads alone)
    for (int c = 0; c < chunks; ++c) {
      const bool more = c + 1 < chunks;
      lds_barrier();
      f32x4 out[NT] = {};
      for_queries.template multiply_into<KS>(qf.v, 0, out);
#pragma unroll
      for (int n = 0; n < NT; ++n) out[n] *= steps.since * s.scale;
      if (more) qf.at += qf.hop, steps.at += steps.hop;
      qf.load();
      steps.load(tile);
      lds_barrier();
      lds_barrier();
      if (wave >= 6) for_out.template multiply_into<2>(pf.v, 0, out);
      else for_out.template multiply_into<1>(pf.v, 0, out);
      if (more) pf.at += pf.hop;
      pf.load(0, steps_in);
      const int count = walk.count(), live = walk.live(len);
      const __amdgpu_buffer_rsrc_t to = columns.rows(s, walk, b, h, count);
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        if (live < count) {
#pragma unroll
          for (int r = 0; r < 4; ++r) out[n][r] = 16 * tile + 4 * g + r < live ? out[n][r] : 0.f;
        }
        columns.store(to, n, out[n]);
      }
      if (c + 1 < s.chunks) walk.ahead(s, outputs);
    }
    for (int c = chunks; c < s.chunks; ++c) {
      const __amdgpu_buffer_rsrc_t to = columns.rows(s, walk, b, h, walk.count());
#pragma unroll
      for (int n = 0; n < NT; ++n) columns.store(to, n, f32x4{});
      if (c + 1 < s.chunks) walk.ahead(s, outputs);
    }
    return;
  }

  f32x4 state[KT][NT];
  const int64_t state_at = ((int64_t)b * s.n_h + h) * s.d_k * s.d_v;
#pragma unroll
  for (int i = 0; i < KT; ++i)
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int k = 16 * (wave * KT + i) + 4 * g + r, v = col + 16 * n;
        state[i][n][r] = s.h0 && k < s.d_k && v < s.d_v ? s.h0[state_at + (int64_t)k * s.d_v + v] : 0.f;
      }
  auto values = [&](int p) { return table[p].v; };
  DeltaFragments<4, NI, KS * NI> kf;  // of all tiles of steps, for the wave's step over keys
  DeltaFragments<2, kInner, kInner> tf;
  const int steps_in = wave < 2 ? 1 : 2;
  DeltaFragments<2 * KT, NI, NI> ktf;
  constexpr bool kTurned = delta_turned<E>();
  const DeltaTurn<KT> turn(wave);
  DeltaSteps steps;
  kf.start(s.kf, chunk0, s.n_hk, hk, Z::kKeyPiece * NI, 0, wave * KT / 2 * NI);
  if constexpr (!kTurned) ktf.start(s.ktf, chunk0, s.n_hk, hk, Z::kKeyPiece * NI, 0, tile * KT * 2 * NI);
  tf.start(s.tf, chunk0, s.n_h, h, Z::kStepPiece * kInner, 0, tile * 2 * kInner);
  steps.start(s, chunk0, h, 0);
  walk.start(s, 0, values);
  typename Columns::Raw raw[NT][4];
  if (chunks > 0) {
    columns.load(columns.rows(s, walk, b, h, walk.live(len)), raw);
    kf.load();
    tf.load(0, steps_in);
    if constexpr (!kTurned) ktf.load();
    steps.load(tile);
  }
  __builtin_amdgcn_s_waitcnt(kWaitVmcnt0);
  for (int c = 0; c < chunks; ++c) {
    const bool more = c + 1 < chunks;
    const int64_t head = (chunk0 + c) * s.n_h + h;
    // K S
    Pieces<3> own[NT];
    delta_own<KT, NT>(state, wave, own);
    delta_partial<NT>(kf.v, own, wave, of_keys, [&] {
      if constexpr (!kTurned) ktf.load();
    });
    if constexpr (!STORE) {
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int k = 0; k < 3; ++k) {
          if constexpr (KT == 2) {
            for_queries.v[wave][n][k][lane] = own[n].p[k];
          } else {
            const u32x4 v = own[n].p[k];
            ((u32x2*)&for_queries.v[wave >> 1][n][k][lane])[wave & 1] = wave & 1 ? u32x2{v[2], v[3]} : u32x2{v[0], v[1]};
          }
        }
    }
    if (more) kf.at += kf.hop;
    lds_barrier();
    if constexpr (STORE) {
      float* const to = s.states + head * DK * s.dvp;
#pragma unroll
      for (int i = 0; i < KT; ++i)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (col + 16 * n < s.dvp) to[(int64_t)(16 * (wave * KT + i) + 4 * g + r) * s.dvp + col + 16 * n] = state[i][n][r];
    }
    // X = V - exp(G) (K S)
    f32x4 x[NT];
    delta_joined<NT>(of_keys, tile, x, [&] {
      if constexpr (kTurned) turn(kf.v, ktf.v);
      kf.load();
    });
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      x[n] = Columns::values(raw[n]) - steps.since * x[n];
      for_inner.write(wave, n, x[n] * steps.beta);
    }
    if (more) walk.ahead(s, values);
    columns.load(columns.rows(s, walk, b, h, walk.live(len)), raw);
    lds_barrier();
    // U = T (beta X)
    f32x4 u[NT] = {};
    if (wave >= 2) for_inner.template multiply_into<2>(tf.v, 0, u);
    else for_inner.template multiply_into<1>(tf.v, 0, u);
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      for_state.write(wave, n, u[n] * steps.until);
      if (!STORE) for_out.write(wave, n, u[n]);
      if (STORE && col + 16 * n < s.dvp) {
#pragma unroll
        for (int r = 0; r < 4; ++r) s.u[(head * kChunk + 16 * wave + 4 * g + r) * s.dvp + col + 16 * n] = steps.beta[r] == 0.f ? x[n][r] : u[n][r];
      }
    }
#pragma unroll
    for (int i = 0; i < KT; ++i)
#pragma unroll
      for (int n = 0; n < NT; ++n) state[i][n] *= steps.decay;
    if (more) {
      tf.at += tf.hop;
      steps.at += steps.hop;
    }
    lds_barrier();
    // S' = exp(G_C) S + K^T (exp(G_C - G) U)
    delta_state<KT, NT>(for_state, ktf.v, state, [&] {
      tf.load(0, steps_in);
      steps.load(tile);
    });
    if (!kTurned && more) ktf.at += ktf.hop;
  }
  if (s.hT) {
#pragma unroll
    for (int i = 0; i < KT; ++i)
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int k = 16 * (wave * KT + i) + 4 * g + r, v = col + 16 * n;
          if (k < s.d_k && v < s.d_v) s.hT[state_at + (int64_t)k * s.d_v + v] = state[i][n][r];
        }
  }
}

// The gradient of the state, backwards through the chunks, in the same way:
//   dU = P^T dO + exp(G_C - G) (K dS'),  dR = T^T dU,  dS = exp(G_C) dS' + Q^T (scale exp(G) dO) - K^T (exp(G) beta dR)
// with R = beta X.  dS' and dR are kept for the kernel behind it.  The second four waves make the two products of dO, a chunk ahead.
template <class E, int DK, int NT>
__global__ __launch_bounds__(512, 2) void delta_bwd_kernel(DeltaArgs s) {
  typedef DeltaSizes<kChunk, DK> Z;
  typedef DeltaColumns<E, NT> Columns;
  constexpr int NI = delta_pieces<E>(), KT = DK / 64, KS = Z::kKeySteps;
  __shared__ DeltaTiles<16, NT> of_keys;         // K dS': tile of steps, wave
  __shared__ DeltaShared<2, NT, 3> for_inner, for_state;
  __shared__ DeltaShared<2, NT, NI> grads;     // dO
  __shared__ DeltaShared<2, NT, 3> for_queries;  // scale exp(G) dO
  __shared__ DeltaTiles<4, NT> of_inner[2];       // P^T dO, by turns
  __shared__ DeltaTiles<4 * KT, NT> of_queries[2];  // Q^T (scale exp(G) dO)
  const DeltaTable table = DELTA_TABLE(s);
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63, g = lane >> 4, tile = wave & 3;
  const DeltaChain chain = delta_chain<NT>(s);
  const int b = chain.b, h = chain.h, hk = h / s.each, col = chain.col + (lane & 15);
  const int len = delta_length(s, b), chunks = delta_live_chunks(s, len);
  const int64_t chunk0 = (int64_t)b * s.chunks;

  if (wave >= 4) {
    if (chunks == 0) return;
    const Columns columns(s, tile, col);
    auto arrays = [&](int p) { return table[p].d_o; };
    DeltaWalk walk;
    DeltaFragments<2, kInner, kInner> ptf;
    DeltaFragments<2 * KT, NI, NI> qtf;
    DeltaSteps steps;
    int c = chunks - 1;  // the chunk that is made
    ptf.start(s.ptf, chunk0, s.n_h, h, Z::kStepPiece * kInner, c, tile * 2 * kInner);
    qtf.start(s.qtf, chunk0, s.n_hk, hk, Z::kKeyPiece * NI, c, tile * KT * 2 * NI);
    steps.start(s, chunk0, h, c);
    walk.start(s, c, arrays);
    typename Columns::Raw raw[NT][4];
    columns.load(columns.rows(s, walk, b, h, walk.live(len)), raw);
    ptf.load(tile / 2);
    qtf.load();
    steps.load(tile);
    __builtin_amdgcn_s_waitcnt(kWaitVmcnt0);  // (so that the loop's waits count its own loads alone)
    // Three barriers a chunk, one chunk before the other waves.
    for (; c >= 0; --c) {
      const bool more = c > 0;
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const f32x4 v = Columns::values(raw[n]);
        grads.write(tile, n, v);  // (bf16 numbers are their upper halves)
        for_queries.write(tile, n, v * (steps.since * s.scale));
      }
      if (more) {
        walk.back(s, arrays);
        steps.at -= steps.hop;
      }
      columns.load(columns.rows(s, walk, b, h, walk.live(len)), raw);
      steps.load(tile);
      lds_barrier();
      f32x4 u[NT] = {}, sum[KT][NT] = {};
      if (wave < 6) grads.template multiply_into<2>(ptf.v, 0, u);
      else grads.template multiply_into<1>(ptf.v + 1, 1, u);
#pragma unroll
      for (int n = 0; n < NT; ++n) of_inner[c & 1].v[tile][n][lane] = u[n];
      if (more) ptf.at -= ptf.hop;
      ptf.load(tile / 2);
      delta_state<KT, NT>(for_queries, qtf.v, sum);
#pragma unroll
      for (int k = 0; k < KT; ++k)
#pragma unroll
        for (int n = 0; n < NT; ++n) of_queries[c & 1].v[tile * KT + k][n][lane] = sum[k][n];
      if (more) qtf.at -= qtf.hop;
      qtf.load();
      lds_barrier();
      lds_barrier();
    }
    // (the other waves' last chunk: nothing is written while they read what was made for it)
    lds_barrier();
    lds_barrier();
    lds_barrier();
    return;
  }

  f32x4 state[KT][NT];  // dS
  const int64_t state_at = ((int64_t)b * s.n_h + h) * s.d_k * s.d_v;
#pragma unroll
  for (int i = 0; i < KT; ++i)
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int k = 16 * (wave * KT + i) + 4 * g + r, v = col + 16 * n;
        state[i][n][r] = s.dhT && k < s.d_k && v < s.d_v ? s.dhT[state_at + (int64_t)k * s.d_v + v] : 0.f;
      }
  DeltaFragments<4, NI, KS * NI> kf;
  DeltaFragments<2, kInner, kInner> ttf;
  DeltaFragments<2 * KT, NI, NI> ktf;
  DeltaSteps steps;
  const int last = max(chunks - 1, 0);
  kf.start(s.kf, chunk0, s.n_hk, hk, Z::kKeyPiece * NI, last, wave * KT / 2 * NI);
  ktf.start(s.ktf, chunk0, s.n_hk, hk, Z::kKeyPiece * NI, last, tile * KT * 2 * NI);
  ttf.start(s.ttf, chunk0, s.n_h, h, Z::kStepPiece * kInner, last, tile * 2 * kInner);
  steps.start(s, chunk0, h, last);
  if (chunks > 0) {
    kf.load();
    ttf.load(wave / 2);
    ktf.load();
    steps.load(tile);
    __builtin_amdgcn_s_waitcnt(kWaitVmcnt0);
    lds_barrier();
    lds_barrier();
    lds_barrier();
  }
  for (int c = chunks - 1; c >= 0; --c) {
    const bool more = c > 0;
    const int64_t head = (chunk0 + c) * s.n_h + h;
    Pieces<3> own[NT];
    delta_own<KT, NT>(state, wave, own);
    delta_partial<NT>(kf.v, own, wave, of_keys, [&] { ktf.load(); });
    if (more) kf.at -= kf.hop;
    lds_barrier();
    {
      float* const to = s.dstates + head * DK * s.dvp;
#pragma unroll
      for (int i = 0; i < KT; ++i)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (col + 16 * n < s.dvp) to[(int64_t)(16 * (wave * KT + i) + 4 * g + r) * s.dvp + col + 16 * n] = state[i][n][r];
    }
    f32x4 u[NT];
    delta_joined<NT>(of_keys, tile, u, [&] { kf.load(); });
#pragma unroll
    for (int n = 0; n < NT; ++n) for_inner.write(wave, n, of_inner[c & 1].v[wave][n][lane] + u[n] * steps.until);
    lds_barrier();
    f32x4 r_[NT] = {};
    if (wave < 2) for_inner.template multiply_into<2>(ttf.v, 0, r_);
    else for_inner.template multiply_into<1>(ttf.v + 1, 1, r_);
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      for_state.write(wave, n, r_[n] * -(steps.since * steps.beta));
      if (col + 16 * n < s.dvp) {
#pragma unroll
        for (int r = 0; r < 4; ++r) s.dr[(head * kChunk + 16 * wave + 4 * g + r) * s.dvp + col + 16 * n] = r_[n][r];
      }
    }
#pragma unroll
    for (int i = 0; i < KT; ++i)
#pragma unroll
      for (int n = 0; n < NT; ++n) state[i][n] = of_queries[c & 1].v[wave * KT + i][n][lane] + state[i][n] * steps.decay;
    if (more) {
      ttf.at -= ttf.hop;
      steps.at -= steps.hop;
    }
    lds_barrier();
    delta_state<KT, NT>(for_state, ktf.v, state, [&] {
      ttf.load(wave / 2);
      steps.load(tile);
    });
    if (more) ktf.at -= ktf.hop;
  }
  if (s.dh0) {
#pragma unroll
    for (int i = 0; i < KT; ++i)
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int k = 16 * (wave * KT + i) + 4 * g + r, v = col + 16 * n;
          if (k < s.d_k && v < s.d_v) s.dh0[state_at + (int64_t)k * s.d_v + v] = state[i][n][r];
        }
  }
}

// ---- a chunk's gradients --------------------------------------------------
// With the states and their gradients known, chunks are independent.  A workgroup has a chunk of a key's head, whose heads it adds up in order:
//   dA = -strictly lower (dR U^T),  dP = lower (dO U^T),  M = dA beta D,  N = scale D dP,  M and N of k_i k_j and q_i k_j
//   dq = N K + scale exp(G) (dO S^T)
//   dk = N^T Q + (M + M^T) K - exp(G) beta (dR S^T) + Y,  Y = exp(G_C - G) (U dS'^T)
//   dv = beta dR,  dbeta_i = dR_i U_i / beta_i  (u = beta r, and dbeta = du r, of the step itself; with beta of 0, r_i = X_i - sum_j A_ij / beta_i u_j)
//   dG_i = sums of (M k k + N q k) over row i less those over column i, and the rows' products of q, k with what they were multiplied by; what
//   exp(G_C) multiplies goes to the last step;  dg_t = sum of dG from t on
template <class E, int C, int DK>
struct DeltaGradShared {
  static constexpr int kRow = 72, kTiles = C / 16, kKeyTiles = DK / 16;  // 64 columns at a time
  union {
    struct {
      uint16_t dr[3][C][kRow], u[3][C][kRow], d_o[delta_pieces<E>()][C][kRow];
    };
    uint16_t inner[3][3][C][kRow];  // pieces of M + M^T, N, N^T; in a row, a lane's eight numbers of a step of the sum one behind the other
  };
  float row_sum[2][kTiles][C], col_sum[2][2][C];
  float dots[kKeyTiles][C], ends[kKeyTiles][C], us[C], both[kKeyTiles];
  float steps[kStepNumbers][C];
  f32x4 kept[2 * kTiles * kKeyTiles / 8][512];  // a thread's sums over the heads in front
};

__device__ __forceinline__ int place_of(int col) { return (col & 0x23) | (col >> 2 & 3) << 3 | (col >> 4 & 1) << 2; }

// Element e of a lane's eight: a sum of pieces is exact from the smallest on.
template <int N>
__device__ __forceinline__ float from_fragment(const Pieces<N>& p, int e) {
  float v = 0.f;
#pragma unroll
  for (int k = N - 1; k >= 0; --k) v += e & 1 ? bf16_hi(p.p[k][e / 2]) : bf16_lo(p.p[k][e / 2]);
  return v;
}

__device__ __forceinline__ float sum16(float v) {  // over a row of 16 lanes
  v += row_rotated<8>(v);
  v += row_rotated<4>(v);
  v += row_rotated<2>(v);
  return v + row_rotated<1>(v);
}

// Rows of the keys' gradients: a lane's key in step 16 mt0 + 4 g of the chunk, and steps behind it; what does not exist fails the checks.  `first`: the chunk's
// first number in the arrays.
template <class E, int N>
__device__ __forceinline__ void delta_store_keys(const DeltaArgs& s, int64_t first, E* dq, E* dk, const DeltaChunk& at, int mt0, int key, const f32x4 (&sum_q)[N],
                                                 const f32x4 (&sum_k)[N]) {
  const int g = (threadIdx.x & 63) >> 4;
  const uint32_t hop = (uint32_t)(s.n_hk * s.d_k) * (uint32_t)sizeof(E);
  const uint32_t key_off = key < s.d_k ? (uint32_t)(mt0 * 16 + 4 * g) * hop + (uint32_t)key * (uint32_t)sizeof(E) : kOob;
  auto key_rows = [&](E* array, int n) {
    n = __builtin_amdgcn_readfirstlane(n);
    return rsrc_of(array + first, (uint32_t)(n - 1) * hop + (uint32_t)s.d_k * (uint32_t)sizeof(E));
  };
  const __amdgpu_buffer_rsrc_t to_q = key_rows(dq, at.n), to_k = key_rows(dk, at.n);
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const bool in = (mt0 + i) * 16 + 4 * g + r < at.live;
      const uint32_t step_off = (uint32_t)(i * 16 + r) * hop;
      const float q = in ? sum_q[i][r] : 0.f, k = in ? sum_k[i][r] : 0.f;
      if constexpr (sizeof(E) == 4) {
        __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(q), to_q, key_off, step_off, 0);
        __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(k), to_k, key_off, step_off, 0);
      } else {
        __builtin_amdgcn_raw_buffer_store_b16(to_bf16(q), to_q, key_off, step_off, 0);
        __builtin_amdgcn_raw_buffer_store_b16(to_bf16(k), to_k, key_off, step_off, 0);
      }
    }
}

// Bound by the time and the bytes of its loads (a compute unit holds one workgroup): a thread's part of the next 64 columns, of this head or of the next
// one, is loaded into the registers that this one's have left.
// SPLIT: few chunks, whose heads are workgroups of their own; delta_keys_kernel adds up what they leave.
template <class E, int C, int DK, bool SPLIT>
__global__ __launch_bounds__(512, 2) void delta_grad_kernel(DeltaArgs s) {
  static_assert(C == 64, "two steps of a sum over steps");
  typedef DeltaSizes<C, DK> Z;
  typedef DeltaGradShared<E, C, DK> Shared;
  constexpr int NI = delta_pieces<E>(), W = 8;
  constexpr int kMine = Z::kTiles * Z::kKeyTiles / W;  // tiles of a wave: one column of keys, some rows of steps
  constexpr bool kBoth = kMine == 2;  // with 64 keys a wave has tiles of M and of N, with 128 of one of them
  extern __shared__ char delta_lds[];
  Shared& m = *(Shared*)delta_lds;
  const DeltaTable table = DELTA_TABLE(s);
  int tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), kt = kBoth ? wave & 3 : wave, mt0 = wave / Z::kKeyTiles * kMine;
  // Of M and N a wave has the tiles (mt, nt) of its rows mt, which it reads anyway, and one column nt <= mt (the two waves of a SIMD have about as many).
  const int wave_what = wave >> 2, nt = kBoth || wave_what == 0 ? wave & 3 : 3 - (wave & 3);
  struct Item {  // a chunk of a key's head, and which of its heads
    DeltaChunk at;
    int hk, first, end;
    int64_t step0, key0, head0;
    const E* d_o;
  };
  auto item_of = [&](int i) {
    Item x;
    x.first = SPLIT ? i % (uint32_t)s.each : 0;
    x.end = SPLIT ? x.first + 1 : s.each;
    if (SPLIT) i /= (uint32_t)s.each;
    x.hk = i % (uint32_t)s.n_hk;
    const int at_chunk = i / (uint32_t)s.n_hk, c = at_chunk % s.chunks, b = at_chunk / s.chunks;
    x.at = delta_chunk(s, b, c);
    x.at.live = __builtin_amdgcn_readfirstlane(x.at.live);
    x.step0 = (int64_t)b * x.at.steps + x.at.first;
    x.key0 = ((int64_t)b * s.chunks + c) * s.n_hk + x.hk;
    x.head0 = x.key0 * s.each;
    x.d_o = (const E*)table[x.at.p].d_o + (x.step0 * s.n_h + x.hk * s.each) * s.d_v;
    return x;
  };
  // A thread's eight columns of dR, U and dO in a step, and a lane's of the state and its gradient in a key's row.  Offsets inside a head's
  // arrays; columns that do not exist, and steps behind the end, fail the checks.
  const uint32_t stage_off = (uint32_t)((tid >> 3) * s.dvp + (tid & 7) * 8) * 4, state_off = (uint32_t)((kt * 16 + (tid & 15)) * s.dvp + 8 * ((tid & 63) >> 4)) * 4;
  u32x4 r8[2], u8[2], s8[2], d8[2];
  u32x4 o8[sizeof(E) / 2];
  const bool whole_eights = s.d_v % 8 == 0;
  auto load_stage = [&](const Item& x, int e, int v0, uint32_t size) {
    const int64_t rows = (x.head0 + e) * C * s.dvp;
    const int v = v0 + (tid & 7) * 8;
    const uint32_t o = v < s.dvp ? stage_off : kOob;
    const __amdgpu_buffer_rsrc_t from_r = rsrc_of(s.dr + rows + v0, size), from_u = rsrc_of(s.u + rows + v0, size);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      r8[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(from_r, o, 16 * i, 0));
      u8[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(from_u, o, 16 * i, 0));
    }
    const int t = tid >> 3;
    const E* const from = x.d_o + e * s.d_v;
    if (whole_eights) {
      const __amdgpu_buffer_rsrc_t from_o = rsrc_of(from + v0, size);
      const uint32_t o = t < x.at.live && v < s.d_v ? (uint32_t)(t * s.n_h * s.d_v + (tid & 7) * 8) * (uint32_t)sizeof(E) : kOob;
#pragma unroll
      for (int i = 0; i < (int)sizeof(E) / 2; ++i) o8[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(from_o, o, 16 * i, 0));
    } else {
      Eight<E> raw;
      raw.load(from + (int64_t)t * s.n_h * s.d_v + v, t < x.at.live && size ? max(0, min(8, s.d_v - v)) : 0);
      o8[0] = raw.a;
      if constexpr (sizeof(E) == 4) o8[1] = raw.b;
    }
  };
  auto load_eight = [&](const float* states, const Item& x, int e, int v0, uint32_t size, u32x4 (&to)[2]) {
    const __amdgpu_buffer_rsrc_t from = rsrc_of(states + (x.head0 + e) * DK * s.dvp + v0, size);
    const uint32_t o = v0 + 8 * ((tid & 63) >> 4) < s.dvp ? state_off : kOob;
#pragma unroll
    for (int i = 0; i < 2; ++i) to[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(from, o, 16 * i, 0));
  };
  auto load_states = [&](const Item& x, int e, uint32_t size) {
    load_eight(s.states, x, e, 0, size, s8);
    load_eight(s.dstates, x, e, 0, size, d8);
  };
  auto numbers = [](const u32x4 (&raw)[2], float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(raw[i / 4][i % 4]);
  };
  auto load_pieces = [&](const uint16_t* fragments, int at_byte) {
    const __amdgpu_buffer_rsrc_t from = rsrc_of(fragments, kOob);
    Pieces<NI> o;
#pragma unroll
    for (int k = 0; k < NI; ++k) o.p[k] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(from, (tid & 63) * 16, at_byte + k * kFragment * 2, 0));
    return o;
  };
  float step;
  auto load_first = [&](const Item& x, int e, bool there) {
    const uint32_t size = there && x.at.live > 0 ? kOob : 0;
    const __amdgpu_buffer_rsrc_t from = rsrc_of(s.steps + (x.head0 + e) * kStepNumbers * C, size ? kStepNumbers * C * 4 : 0);
    step = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(from, tid * 4, 0, 0));
    load_stage(x, e, 0, size);
    return size;
  };

  const int items = s.n_b * s.chunks * s.n_hk * (SPLIT ? s.each : 1);
  Item it = item_of(blockIdx.x);
  {
    const uint32_t size = load_first(it, it.first, true);
    load_states(it, it.first, size);
  }
  for (int i = blockIdx.x; i < items; i += gridDim.x) {
  const bool another = i + (int)gridDim.x < items;
  const Item next = item_of(another ? i + (int)gridDim.x : i);
  const DeltaChunk at = it.at;
  const int hk = it.hk;
  const int64_t step0 = it.step0, head0 = it.head0;
  const DeltaTable w = table + at.p;
  E* const dq = (E*)w->dq, * const dk = (E*)w->dk, * const dv = (E*)w->dv;
  if (at.live == 0) {
    const int heads = it.end - it.first, columns = heads * s.d_v;
    for (int i = tid; i < (it.first == 0 ? at.n * s.d_k : 0); i += 64 * W) {
      const int64_t o = ((step0 + i / s.d_k) * s.n_hk + hk) * s.d_k + i % s.d_k;
      st(dq, (size_t)o, 0.f);
      st(dk, (size_t)o, 0.f);
    }
    for (int64_t i = tid; i < (int64_t)at.n * columns; i += 64 * W)
      st(dv, (size_t)(((step0 + i / columns) * s.n_h + hk * s.each + it.first) * s.d_v + i % columns), 0.f);
    for (int i = tid; i < at.n * heads; i += 64 * W) {
      const int64_t o = (step0 + i / heads) * s.n_h + hk * s.each + it.first + i % heads;
      if (w->dg) w->dg[o] = 0.f;
      w->dbeta[o] = 0.f;
    }
    const uint32_t size = load_first(next, next.first, another);
    load_states(next, next.first, size);
    it = next;
    continue;
  }
  const int64_t key_at = it.key0 * Z::kKeyPiece * NI;
  const uint16_t *const ktf = s.ktf + key_at, *const qtf = s.qtf + key_at;
  for (int e = it.first; e < it.end; ++e) {
    // (What is made of the thread's number is made again for each head: kept, it would not fit the registers.)
    asm volatile("" : "+v"(tid));
    const int lane = tid & 63, row = lane & 15, g = lane >> 4, key = kt * 16 + row;
    const int h = hk * s.each + e;
    lds_barrier();
    if (tid < kStepNumbers * C) m.steps[tid / C][tid % C] = step;
    f32x4 os[kMine] = {}, rs[kMine] = {}, us[kMine] = {}, acc[4] = {};
    float udot = 0.f, both = 0.f;
    const __amdgpu_buffer_rsrc_t tiles = rsrc_of(s.tiles + (head0 + e) * Z::kLower * 2 * 256, kOob);
    f32x4 made[4];
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const int mt = max(mt0 + x % kMine, nt);
      made[x] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(tiles, lane * 16, ((kBoth ? x / 2 : wave_what) * Z::kLower + mt * (mt + 1) / 2 + nt) * 1024, 0));
    }
    const int t8 = tid >> 3, col8 = (tid & 7) * 8;
    for (int v0 = 0; v0 < s.d_v; v0 += 64) {
      const uint32_t more = v0 + 64 < s.d_v ? kOob : 0;  // (the loads behind the last ones are of nothing)
      lds_barrier();
      {
        float r[8], u[8], out[8];
        numbers(r8, r);
        numbers(u8, u);
        const float beta = m.steps[kBeta][t8], inverse = beta == 0.f ? 1.f : 1.f / beta;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          udot = fmaf(r[i], u[i] * inverse, udot);
          u[i] = beta == 0.f ? 0.f : u[i];
        }
        const Pieces<3> rp = split8(r), up = split8(u);
#pragma unroll
        for (int k = 0; k < 3; ++k) {
          *(u32x4*)&m.dr[k][t8][col8] = rp.p[k];
          *(u32x4*)&m.u[k][t8][col8] = up.p[k];
        }
        if constexpr (NI == 1) {
          *(u32x4*)&m.d_o[0][t8][col8] = o8[0];
        } else {
          float o[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) o[i] = __uint_as_float(o8[i / 4 * (sizeof(E) / 4)][i % 4]);
          const Pieces<3> op = split8(o);
#pragma unroll
          for (int k = 0; k < 3; ++k) *(u32x4*)&m.d_o[k][t8][col8] = op.p[k];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) out[i] = t8 < at.live ? beta * r[i] : 0.f;
        const int v = v0 + col8;
        if (t8 < at.n && v < s.d_v) store8(dv + ((step0 + t8) * s.n_h + h) * s.d_v + v, out, min(8, s.d_v - v));
      }
      load_stage(it, e, v0 + 64, more);
      lds_barrier();
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
        if (v0 + 32 * ks < s.dvp) {
          const int at8 = 32 * ks + 8 * g;
          float sv[8], dv_[8];
          numbers(s8, sv);
          numbers(d8, dv_);
          if (mt0 == 0) {
#pragma unroll
            for (int i = 0; i < 8; ++i) both = fmaf(sv[i], dv_[i], both);
          }
          const int next_v = v0 + 32 * ks + 32;
          const uint32_t more_v = next_v < s.dvp ? kOob : 0;
          auto rows3 = [&](const uint16_t (*from)[C][Shared::kRow], int mt) {
            Pieces<3> o;
#pragma unroll
            for (int k = 0; k < 3; ++k) o.p[k] = *(const u32x4*)&from[k][mt * 16 + row][at8];
            return o;
          };
          auto products = [&](auto what) {
            const Pieces<3> right = rows3(m.u, nt), sp = split8(sv);
            load_eight(s.states, it, e, next_v, more_v, s8);
#pragma unroll
            for (int i = 0; i < kMine; ++i) {
              Pieces<NI> o;
#pragma unroll
              for (int k = 0; k < NI; ++k) o.p[k] = *(const u32x4*)&m.d_o[k][(mt0 + i) * 16 + row][at8];
              const Pieces<3> r = rows3(m.dr, mt0 + i);
              os[i] = multiply(o, sp, os[i]);
              rs[i] = multiply(r, sp, rs[i]);
              if (mt0 + i >= nt) {
                if constexpr (what != 1) acc[i] = multiply(r, right, acc[i]);
                if constexpr (what == 1) acc[i] = multiply(o, right, acc[i]);
                if constexpr (what == 2) acc[2 + i % 2] = multiply(o, right, acc[2 + i % 2]);
              }
            }
          };
          if constexpr (kBoth) products(std::integral_constant<int, 2>());
          else if (wave_what) products(std::integral_constant<int, 1>());
          else products(std::integral_constant<int, 0>());
          numbers(d8, dv_);
          const Pieces<3> dp = split8(dv_);
          load_eight(s.dstates, it, e, next_v, more_v, d8);
#pragma unroll
          for (int i = 0; i < kMine; ++i) us[i] = multiply(rows3(m.u, mt0 + i), dp, us[i]);
        }
      }
    }
    lds_barrier();
    asm volatile("" : "+v"(tid));
    Pieces<NI> kk[Z::kSteps], qq[Z::kSteps];
#pragma unroll
    for (int k = 0; k < Z::kSteps; ++k) {
      kk[k] = load_pieces(ktf, (kt * Z::kSteps + k) * NI * kFragment * 2);
      qq[k] = load_pieces(qtf, (kt * Z::kSteps + k) * NI * kFragment * 2);
    }
    // M and N, in pieces; what A and P were made of is in them still: M k k = -dA A, of which beta is left out along the rows, and N q k = dP P
    const int j = nt * 16 + row;
    const float whole = m.steps[kWhole][j], rest = m.steps[kRest][j];
    float down[2] = {};
    auto tile_of = [&](auto what, auto diagonal, int x, int mt) {
      f32x4 mine, across;
      const int i0 = mt * 16 + 4 * g;
      const f32x4 whole_i = *(const f32x4*)&m.steps[kWhole][i0], rest_i = *(const f32x4*)&m.steps[kRest][i0], beta_i = *(const f32x4*)&m.steps[kBeta][i0];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const bool below = !diagonal || 4 * g + r > row, in = below || (what && 4 * g + r == row);
        float decay = __builtin_amdgcn_exp2f(in ? (whole_i[r] - whole) + (rest_i[r] - rest) : 0.f);
        if constexpr (diagonal) asm volatile("" : "+v"(decay));  // (no branch around it)
        const float all = decay * acc[x][r] * (what ? s.scale : -beta_i[r]), part = what ? acc[x][r] * made[x][r] : -acc[x][r] * made[x][r];
        mine[r] = in ? all : 0.f;
        const float mine_part = below ? part : 0.f;
        down[kBoth ? x / 2 : 0] += what ? mine_part : mine_part * beta_i[r];
        across[r] = sum16(mine_part);
      }
      const float across_of = row < 2 ? row ? across[1] : across[0] : row == 2 ? across[2] : across[3];
      if (row < 4) m.row_sum[what][nt][i0 + row] = across_of;
      const Pieces<3> p = split_tiles(mine, f32x4{});
#pragma unroll
      for (int k = 0; k < 3; ++k) {
        const u32x2 v = {p.p[k][0], p.p[k][1]};
        if constexpr (what) {
          *(u32x2*)&m.inner[2][k][j][place_of(i0)] = v;
#pragma unroll
          for (int r = 0; r < 4; ++r) m.inner[1][k][i0 + r][place_of(j)] = (uint16_t)(v[r / 2] >> (16 * (r & 1)));
          if (!diagonal && (mt ^ nt) == 1) {  // above the diagonal, in a step of the sum that is not all zeros
            *(u32x2*)&m.inner[1][k][j][place_of(i0)] = u32x2{0, 0};
            *(u32x2*)&m.inner[2][k][mt * 16 + row][place_of(nt * 16 + 4 * g)] = u32x2{0, 0};
          }
        } else if constexpr (!diagonal) {
          *(u32x2*)&m.inner[0][k][j][place_of(i0)] = v;
#pragma unroll
          for (int r = 0; r < 4; ++r) m.inner[0][k][i0 + r][place_of(j)] = (uint16_t)(v[r / 2] >> (16 * (r & 1)));
        } else {
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const uint16_t one = (uint16_t)(v[r / 2] >> (16 * (r & 1)));
            if (4 * g + r >= row) m.inner[0][k][i0 + r][place_of(j)] = one;
            if (4 * g + r > row) m.inner[0][k][j][place_of(i0) + r] = one;
          }
        }
      }
    };
    auto tiles_of = [&](auto what, int first, int count) {
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const int mt = mt0 + x % kMine;
        if (x < first || x >= first + count || mt < nt) continue;
        if (mt == nt) tile_of(what, std::true_type(), x, mt);
        else tile_of(what, std::false_type(), x, mt);
      }
    };
    if (kBoth) {
      tiles_of(std::integral_constant<int, 0>(), 0, 2);
      tiles_of(std::integral_constant<int, 1>(), 2, 2);
    } else if (wave_what) {
      tiles_of(std::integral_constant<int, 1>(), 0, 4);
    } else {
      tiles_of(std::integral_constant<int, 0>(), 0, 4);
    }
    // the next columns: of the next head, or of another chunk
    const bool last = e + 1 == it.end;
    const Item& then = last ? next : it;
    const int then_e = last ? next.first : e + 1;
    const uint32_t then_size = load_first(then, then_e, !last || another);
#pragma unroll
    for (int x = 0; x < (kBoth ? 2 : 1); ++x) {
      down[x] += __shfl_xor(down[x], 16, 64);
      down[x] += __shfl_xor(down[x], 32, 64);
      if (g == 0) m.col_sum[kBoth ? x : wave_what][mt0 / 2][j] = down[x];
    }
    // what the states' products come to (a lane's numbers of the fragments of Q^T and K^T are its numbers of a tile of results)
    f32x4 sum_q[kMine], sum_k[kMine];
    {
#pragma unroll
      for (int i = 0; i < kMine; ++i) {
        const int t0 = (mt0 + i) * 16 + 4 * g;
        f32x4 all, end;
        const f32x4 since = *(const f32x4*)&m.steps[kSince][t0], until = *(const f32x4*)&m.steps[kUntil][t0], beta = *(const f32x4*)&m.steps[kBeta][t0];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int at8 = i % 2 * 4 + r;  // (a wave's first tile is an even one)
          const float qv = from_fragment(mt0 + i < 2 ? qq[0] : qq[1], at8), kv = from_fragment(mt0 + i < 2 ? kk[0] : kk[1], at8);
          const float one = s.scale * since[r] * os[i][r], two = since[r] * beta[r] * rs[i][r], three = until[r] * us[i][r];
          all[r] = sum16(fmaf(qv, one, -kv * (two + three)));
          end[r] = sum16(kv * three);
          sum_q[i][r] = one;
          sum_k[i][r] = three - two;
        }
        const float one_all = row < 2 ? row ? all[1] : all[0] : row == 2 ? all[2] : all[3];
        const float one_end = row < 2 ? row ? end[1] : end[0] : row == 2 ? end[2] : end[3];
        if (row < 4) {
          m.dots[kt][t0 + row] = one_all;
          m.ends[kt][t0 + row] = one_end;
        }
      }
    }
    both = wave_sum(both);
    if (lane == 0 && mt0 == 0) m.both[kt] = both;
    udot += __shfl_xor(udot, 1, 64);
    udot += __shfl_xor(udot, 2, 64);
    udot += __shfl_xor(udot, 4, 64);
    if ((tid & 7) == 0) m.us[tid >> 3] = udot;
    lds_barrier();
    load_states(then, then_e, then_size);
#pragma unroll
    for (int k = 0; k < Z::kSteps; ++k) {
#pragma unroll
      for (int i = 0; i < kMine; ++i) {
        const int mt = mt0 + i;
        auto across = [&](int what) {
          Pieces<3> o;
#pragma unroll
          for (int x = 0; x < 3; ++x) {
            o.p[x] = *(const u32x4*)&m.inner[what][x][mt * 16 + row][32 * k + 8 * g];
          }
          return o;
        };
        sum_k[i] = multiply(across(0), kk[k], sum_k[i]);
        if (2 * k <= mt) sum_q[i] = multiply(across(1), kk[k], sum_q[i]);
        if (mt / 2 <= k) sum_k[i] = multiply(across(2), qq[k], sum_k[i]);
      }
    }
    if (wave == 0) {
      const int tile = lane >> 4;
      float d = 0.f, end = 0.f, all = 0.f, rows[2] = {};
      const float beta = m.steps[kBeta][lane];
#pragma unroll
      for (int what = 0; what < 2; ++what) {
#pragma unroll
        for (int i = 0; i < Z::kTiles; ++i) {
          const float v = m.row_sum[what][i][lane];  // (what no wave wrote is not used)
          rows[what] += i <= tile ? v : 0.f;
        }
        d += what ? rows[what] : beta * rows[what];
#pragma unroll
        for (int i = 0; i < Z::kTiles / kMine; ++i) d -= m.col_sum[what][i][lane];
      }
#pragma unroll
      for (int i = 0; i < Z::kKeyTiles; ++i) {
        d += m.dots[i][lane];
        end += m.ends[i][lane];
        all += m.both[i];
      }
      end = wave_sum(end);
      if (lane == C - 1) d += end + m.steps[kSince][C - 1] * all;
#pragma unroll
      for (int o = 1; o < C; o *= 2) {
        const float later = __shfl_down(d, o, 64);
        if (lane + o < C) d += later;
      }
      if (lane < at.n) {
        const int64_t o = (step0 + lane) * s.n_h + h;
        if (w->dg) w->dg[o] = lane < at.live ? d : 0.f;
        w->dbeta[o] = lane < at.live ? m.us[lane] + (beta == 0.f ? rows[0] : 0.f) : 0.f;
      }
    }
    if constexpr (SPLIT) {
      f32x4* const to = (f32x4*)s.keys + (head0 + e) * 2 * kMine * 512 + tid;
#pragma unroll
      for (int i = 0; i < kMine; ++i) {
        to[i * 512] = sum_q[i];
        to[(kMine + i) * 512] = sum_k[i];
      }
      continue;
    }
    if (e > 0) {
#pragma unroll
      for (int i = 0; i < kMine; ++i) {
        sum_q[i] += m.kept[i][tid];
        sum_k[i] += m.kept[kMine + i][tid];
      }
    }
    if (e + 1 < s.each) {
#pragma unroll
      for (int i = 0; i < kMine; ++i) {
        m.kept[i][tid] = sum_q[i];
        m.kept[kMine + i][tid] = sum_k[i];
      }
      continue;
    }
    delta_store_keys<E>(s, (step0 * s.n_hk + hk) * s.d_k, dq, dk, at, mt0, key, sum_q, sum_k);
  }
  it = next;
  }
}

// dq and dk of a chunk of a key's head, whose heads' parts lie as the threads of delta_grad_kernel had them: added up in order.
template <class E, int C, int DK>
__global__ __launch_bounds__(512) void delta_keys_kernel(DeltaArgs s) {
  constexpr int kKeyTiles = DK / 16, kMine = C / 16 * kKeyTiles / 8;
  const DeltaTable table = DELTA_TABLE(s);
  const int hk = blockIdx.x % (uint32_t)s.n_hk, at_chunk = blockIdx.x / (uint32_t)s.n_hk, c = at_chunk % s.chunks, b = at_chunk / s.chunks;
  const DeltaChunk at = delta_chunk(s, b, c);
  if (at.live == 0) return;  // (zeros are there)
  const int tid = threadIdx.x, wave = tid >> 6, kt = kMine == 2 ? wave & 3 : wave, mt0 = wave / kKeyTiles * kMine;
  const f32x4* from = (const f32x4*)s.keys + (int64_t)blockIdx.x * s.each * 2 * kMine * 512 + tid;
  f32x4 sum_q[kMine] = {}, sum_k[kMine] = {};
  for (int e = 0; e < s.each; ++e, from += 2 * kMine * 512) {
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
      sum_q[i] += from[i * 512];
      sum_k[i] += from[(kMine + i) * 512];
    }
  }
  const int64_t step0 = (int64_t)b * at.steps + at.first;
  delta_store_keys<E>(s, (step0 * s.n_hk + hk) * s.d_k, (E*)table[at.p].dq, (E*)table[at.p].dk, at, mt0, kt * 16 + (tid & 15), sum_q, sum_k);
}

// ---- single tokens --------------------------------------------------------
// One step of each row: a workgroup has Q V columns of a head's state in its registers, thread (i, j) columns V j and rows i, i + 256 / Q, ...  Read
// once: o = scale (a S^T q + (q k) u) needs no second pass over the new state.  Bound by reading and writing the states.
template <class E, int V, int Q>
__global__ __launch_bounds__(256) void delta_step_kernel(const E* __restrict__ q, const E* __restrict__ k, const E* __restrict__ v,
                                                         const float* __restrict__ g, const float* __restrict__ beta, float* __restrict__ state,
                                                         const int32_t* __restrict__ slots, E* __restrict__ o, int64_t n_slots, int n_h, int each,
                                                         int d_k, int d_v, int groups, float scale) {
  constexpr int kGroups = 256 / Q, R = 128 / kGroups;
  __shared__ float keys[128], queries[128];
  __shared__ float sums[4][Q][2 * V + 1];
  const int tid = threadIdx.x, j = tid % Q, i = tid / Q;
  const uint32_t group = blockIdx.x % (uint32_t)groups, at = blockIdx.x / (uint32_t)groups;
  const int64_t row = at / (uint32_t)n_h;
  const int h = at % (uint32_t)n_h, col = ((int)group * Q + j) * V;
  const int64_t slot = slots ? slots[row] : row;
  const bool in = col < d_v;
  E* const out = o + ((int64_t)row * n_h + h) * d_v + col;
  if (slot < 0 || slot >= n_slots) {
    if (i == 0 && in) {
#pragma unroll
      for (int x = 0; x < V; ++x) st(out, (size_t)x, 0.f);
    }
    return;
  }
  const int64_t key = ((int64_t)row * (n_h / each) + h / each) * d_k, head = (int64_t)row * n_h + h;
  float* const mine = state + ((slot * n_h + h) * d_k + i) * (int64_t)d_v + col;
  float part[R][V];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const bool is = in && i + r * kGroups < d_k;
    float* const from = mine + (int64_t)r * kGroups * d_v;
    if constexpr (V == 4) {
      const f32x4 x = is ? *(const f32x4*)from : f32x4{};
#pragma unroll
      for (int y = 0; y < 4; ++y) part[r][y] = x[y];
    } else {
      part[r][0] = is ? *from : 0.f;
    }
  }
  if (tid < 128) {
    keys[tid] = tid < d_k ? ld(k, (size_t)(key + tid)) : 0.f;
    queries[tid] = tid < d_k ? ld(q, (size_t)(key + tid)) : 0.f;
  }
  const float a = g ? expf(g[head]) : 1.f, b = beta[head];
  float value[V];
#pragma unroll
  for (int x = 0; x < V; ++x) value[x] = in ? ld(v, (size_t)(head * d_v + col + x)) : 0.f;
  __syncthreads();
  float sum[2 * V + 1] = {}, kr[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const float kk = keys[i + r * kGroups], qq = queries[i + r * kGroups];
    kr[r] = kk;
#pragma unroll
    for (int x = 0; x < V; ++x) {
      sum[x] = fmaf(part[r][x], kk, sum[x]);
      sum[V + x] = fmaf(part[r][x], qq, sum[V + x]);
    }
    sum[2 * V] = fmaf(kk, qq, sum[2 * V]);
  }
  // over the rows: the lanes of a wave that have these columns, then the waves
#pragma unroll
  for (int x = 0; x < 2 * V + 1; ++x)
#pragma unroll
    for (int d = Q; d < 64; d *= 2) sum[x] += __shfl_xor(sum[x], d, 64);
  if ((tid & 63) < Q) {
#pragma unroll
    for (int x = 0; x < 2 * V + 1; ++x) sums[tid >> 6][j][x] = sum[x];
  }
  __syncthreads();
#pragma unroll
  for (int x = 0; x < 2 * V + 1; ++x) sum[x] = (sums[0][j][x] + sums[1][j][x]) + (sums[2][j][x] + sums[3][j][x]);
  float u[V];
#pragma unroll
  for (int x = 0; x < V; ++x) u[x] = b * fmaf(-a, sum[x], value[x]);
#pragma unroll
  for (int r = 0; r < R; ++r) {
    if (!in || i + r * kGroups >= d_k) continue;
    float* const to = mine + (int64_t)r * kGroups * d_v;
    if constexpr (V == 4) {
      f32x4 x;
#pragma unroll
      for (int y = 0; y < 4; ++y) x[y] = fmaf(kr[r], u[y], a * part[r][y]);
      *(f32x4*)to = x;
    } else {
      *to = fmaf(kr[r], u[0], a * part[r][0]);
    }
  }
  if (i == 0 && in) {
#pragma unroll
    for (int x = 0; x < V; ++x) st(out, (size_t)x, scale * fmaf(sum[2 * V], u[x], a * sum[V + x]));
  }
}

}  // namespace distdl

struct distdl_delta_plan {
  int32_t n_b = 0, T = 0, n_h = 0, n_hk = 0, d_k = 0, d_v = 0, P = 1;
  float scale = 1;
  distdl_dtype dtype = DISTDL_F32;
  distdl::DevArray<distdl::DeltaWorker> table;
  distdl::StreamScratch scratch;
};

namespace distdl {

constexpr int kDeltaKeys = 128;  // d_k: the state's rows are registers

static int delta_check(const void* v, size_t size, const char* what, int j) {
  if (!v) return set_error(DISTDL_ERR_NULL, "delta: %s[%d] is null", what, j);
  if ((uintptr_t)v % size) return set_error(DISTDL_ERR_INVALID_ARG, "delta: %s[%d] is not aligned to its elements", what, j);
  return DISTDL_OK;
}

static int delta_args(distdl_delta_plan* p, const std::vector<DeltaWorker>& w, hipStream_t st, DeltaArgs* s) {
  *s = DeltaArgs{};
  if (p->P <= kDeltaInline) {
    std::copy(w.begin(), w.end(), s->w);
  } else {
    const int rc = p->table.upload(w, st);
    if (rc) return rc;
    s->more = p->table.dev;
  }
  constexpr int C = kChunk;
  s->P = p->P;
  s->T = p->T;
  s->part = p->T / p->P;
  s->extra = p->T % p->P;
  s->chunks_wide = (s->part + C) / C;
  s->chunks_rest = (s->part + C - 1) / C;
  s->chunks = s->extra * s->chunks_wide + (s->P - s->extra) * s->chunks_rest;
  s->n_b = p->n_b;
  s->n_h = p->n_h;
  s->n_hk = p->n_hk;
  s->each = p->n_h / p->n_hk;
  s->d_k = p->d_k;
  s->d_v = p->d_v;
  s->dvp = (p->d_v + 15) / 16 * 16;
  s->scale = p->scale;
  return DISTDL_OK;
}

// Whether the heads of a chunk's keys are workgroups of their own for its gradients: where the chunks leave half of the compute units without work.  54 chunks of
// keys with three heads, fp32: 45 us one head behind the other, 19 and 4 for their sum; a round of workgroups more than that would cost what it gives.
static bool delta_heads_apart(size_t chunks, int each) { return each > 1 && chunks <= 128; }

// The scratch of a call, one array behind the other at multiples of 256 bytes.
template <class E, int DK>
static int delta_scratch(distdl_delta_plan* p, bool back, hipStream_t st, DeltaArgs* s) {
  constexpr int C = kChunk;
  typedef DeltaSizes<C, DK> Z;
  const size_t keys = (size_t)s->n_b * s->chunks * s->n_hk, heads = (size_t)s->n_b * s->chunks * s->n_h;
  const size_t key = keys * Z::kKeyPiece * delta_pieces<E>() * 2, step = heads * Z::kStepPiece * kInner * 2, state = heads * DK * s->dvp * 4,
               rows = heads * C * s->dvp * 4;
  struct Part {
    void** at;
    size_t bytes;
  } parts[] = {{(void**)&s->kf, key}, {(void**)&s->ktf, back || !delta_turned<E>() ? key : 0}, {(void**)&s->qf, back ? 0 : key}, {(void**)&s->qtf, back ? key : 0},
               {(void**)&s->tf, step}, {(void**)&s->pf, back ? 0 : step}, {(void**)&s->ttf, back ? step : 0}, {(void**)&s->ptf, back ? step : 0},
               {(void**)&s->tiles, back ? heads * 2 * Z::kLower * 1024 : 0}, {(void**)&s->steps, heads * kStepNumbers * C * 4}, {(void**)&s->states, back ? state : 0}, {(void**)&s->dstates, back ? state : 0},
               {(void**)&s->u, back ? rows : 0}, {(void**)&s->dr, back ? rows : 0},
               {(void**)&s->keys, back && delta_heads_apart(keys, s->each) ? heads * 2 * C * DK * 4 : 0}};
  size_t all = 0;
  for (const Part& v : parts) all += (v.bytes + 255) / 256 * 256;
  bool is_new = true;
  for (const StreamScratch::Block& v : p->scratch.blocks) is_new = is_new && (v.stream != st || v.floats < all / 4);
  if (is_new) {
    hipStreamCaptureStatus capture = hipStreamCaptureStatusNone;
    DISTDL_HIP_TRY(hipStreamIsCapturing(st, &capture));
    if (capture != hipStreamCaptureStatusNone)
      return set_error(DISTDL_ERR_INVALID_ARG, "delta: the plan's first such call on this stream, which is being captured");
  }
  float* base = nullptr;
  const int rc = p->scratch.get(all / 4, st, &base);
  if (rc) return rc;
  char* at = (char*)base;
  for (const Part& v : parts) {
    *v.at = v.bytes ? at : nullptr;
    at += (v.bytes + 255) / 256 * 256;
  }
  return DISTDL_OK;
}

template <class E, int DK, bool BACK>
static int launch_delta(distdl_delta_plan* p, DeltaArgs& s, hipStream_t st) {
  constexpr int C = kChunk;
  int rc = delta_scratch<E, DK>(p, BACK, st, &s);
  if (rc) return rc;
  constexpr auto prepare = delta_prepare_kernel<E, C, DK, BACK>;
  if ((rc = allow_large_lds<prepare>())) return rc;
  const dim3 chunks((unsigned)((int64_t)s.n_b * s.chunks * s.n_hk));
  // A key's heads are shared out among workgroups that still fit one to a compute unit (54 chunks of keys with three heads, fp32, adjoint: 24 -> 14 us; more
  // than that make K K^T again for nothing, 135 chunks with two heads, fp32: 23 -> 28).
  const unsigned shares = std::min((unsigned)s.each, std::max(1u, 256u / chunks.x));
  hipLaunchKernelGGL(prepare, dim3(chunks.x, shares), dim3(256), sizeof(DeltaPrepareShared<E, C, DK>), st, s);
  // A workgroup, of which a compute unit holds one, takes 32 columns where those of 16 would be more than a round.
  const int64_t chains = (int64_t)s.n_b * s.n_h;
  const bool two = s.d_v > 16 && chains * ((s.d_v + 15) / 16) > 256;
  s.slices = two ? (s.d_v + 31) / 32 : (s.d_v + 15) / 16;
  const dim3 groups((unsigned)(chains * s.slices));
  if (two) hipLaunchKernelGGL((delta_fwd_kernel<E, DK, 2, BACK>), groups, dim3(BACK ? 256 : 512), 0, st, s);
  else hipLaunchKernelGGL((delta_fwd_kernel<E, DK, 1, BACK>), groups, dim3(BACK ? 256 : 512), 0, st, s);
  if constexpr (BACK) {
    if (two) hipLaunchKernelGGL((delta_bwd_kernel<E, DK, 2>), groups, dim3(512), 0, st, s);
    else hipLaunchKernelGGL((delta_bwd_kernel<E, DK, 1>), groups, dim3(512), 0, st, s);
    if (s.keys) {
      constexpr auto grad = delta_grad_kernel<E, C, DK, true>;
      if ((rc = allow_large_lds<grad>())) return rc;
      hipLaunchKernelGGL(grad, dim3(std::min(chunks.x * s.each, 256u)), dim3(512), sizeof(DeltaGradShared<E, C, DK>), st, s);
      hipLaunchKernelGGL((delta_keys_kernel<E, C, DK>), chunks, dim3(512), 0, st, s);
    } else {
      constexpr auto grad = delta_grad_kernel<E, C, DK, false>;
      if ((rc = allow_large_lds<grad>())) return rc;
      hipLaunchKernelGGL(grad, dim3(std::min(chunks.x, 256u)), dim3(512), sizeof(DeltaGradShared<E, C, DK>), st, s);
    }
  }
  return DISTDL_OK;
}

template <bool BACK>
static int launch_delta(distdl_delta_plan* p, DeltaArgs& s, hipStream_t st) {
  const bool wide = p->d_k > 64;
  if (p->dtype == DISTDL_F32) return wide ? launch_delta<float, 128, BACK>(p, s, st) : launch_delta<float, 64, BACK>(p, s, st);
  return wide ? launch_delta<uint16_t, 128, BACK>(p, s, st) : launch_delta<uint16_t, 64, BACK>(p, s, st);
}

template <class E, int V, int Q>
static void launch_delta_step(const void* q, const void* k, const void* v, const float* g, const float* beta, float* state, const int32_t* slots,
                              void* o, int64_t n_slots, int64_t rows, int n_h, int each, int d_k, int d_v, float scale, hipStream_t st) {
  const int groups = (d_v + V * Q - 1) / (V * Q);
  hipLaunchKernelGGL((delta_step_kernel<E, V, Q>), dim3((unsigned)(rows * n_h * groups)), dim3(256), 0, st, (const E*)q, (const E*)k, (const E*)v, g,
                     beta, state, slots, (E*)o, n_slots, n_h, each, d_k, d_v, groups, scale);
}

template <class E>
static void delta_step_kind(const void* q, const void* k, const void* v, const float* g, const float* beta, float* state, const int32_t* slots, void* o,
                            int64_t n_slots, int64_t rows, int n_h, int each, int d_k, int d_v, float scale, hipStream_t st) {
  if (d_v % 4 || (uintptr_t)state % 16)
    launch_delta_step<E, 1, 32>(q, k, v, g, beta, state, slots, o, n_slots, rows, n_h, each, d_k, d_v, scale, st);
  else if (d_v <= 32 || rows * n_h < 512)
    launch_delta_step<E, 4, 8>(q, k, v, g, beta, state, slots, o, n_slots, rows, n_h, each, d_k, d_v, scale, st);
  else
    launch_delta_step<E, 4, 32>(q, k, v, g, beta, state, slots, o, n_slots, rows, n_h, each, d_k, d_v, scale, st);
}

// What every call asks of the sizes.
static int delta_sizes(const char* call, int64_t n_h, int64_t n_hk, int64_t d_k, int64_t d_v, double scale, distdl_dtype dtype) {
  if (n_h < 1 || n_hk < 1 || d_k < 1 || d_v < 1) return set_error(DISTDL_ERR_INVALID_ARG, "%s: sizes must be >= 1", call);
  if (n_h % n_hk) return set_error(DISTDL_ERR_INVALID_ARG, "%s: %lld heads on %lld heads of keys", call, (long long)n_h, (long long)n_hk);
  if (!std::isfinite(scale)) return set_error(DISTDL_ERR_INVALID_ARG, "%s: scale %g", call, scale);
  if (dtype != DISTDL_F32 && dtype != DISTDL_BF16) return set_error(DISTDL_ERR_UNSUPPORTED, "unknown dtype");
  if (d_k > kDeltaKeys) return set_error(DISTDL_ERR_UNSUPPORTED, "%s: d_k of more than %d", call, kDeltaKeys);
  // (a chunk of an array of keys or values stays below 2^31 bytes: the kernels' offsets inside it have 32 bits)
  if (n_h > 1 << 20 || d_v > 1 << 20 || n_h * d_v > 1 << 22 || n_hk * d_k > 1 << 22) return set_error(DISTDL_ERR_UNSUPPORTED, "%s: problem too large", call);
  return DISTDL_OK;
}

}  // namespace distdl

using namespace distdl;

extern "C" {

int distdl_delta_plan_create(distdl_delta_plan** out, int64_t n_b, int64_t T, int64_t n_h, int64_t n_hk, int64_t d_k, int64_t d_v, int P, double scale,
                             distdl_dtype dtype) {
  if (!out) return set_error(DISTDL_ERR_NULL, "delta_plan_create: null argument");
  *out = nullptr;
  if (n_b < 1 || T < 1 || P < 1) return set_error(DISTDL_ERR_INVALID_ARG, "delta_plan_create: sizes must be >= 1");
  const int rc = delta_sizes("delta_plan_create", n_h, n_hk, d_k, d_v, scale, dtype);
  if (rc) return rc;
  if (T < P) return set_error(DISTDL_ERR_EMPTY_PARTITION, "delta: %lld steps over %d workers", (long long)T, P);
  if (T >= int64_t(1) << 30 || n_b >= 1 << 20 || n_b * (T / kChunk + P) >= kMaxBlocks256 / n_hk / 2 || n_b * n_h * ((d_v + 15) / 16) >= kMaxBlocks256 / 2)
    return set_error(DISTDL_ERR_UNSUPPORTED, "delta: problem too large");
  return guarded([&]() -> int {
    std::unique_ptr<distdl_delta_plan> p(new distdl_delta_plan());
    p->n_b = (int32_t)n_b;
    p->T = (int32_t)T;
    p->n_h = (int32_t)n_h;
    p->n_hk = (int32_t)n_hk;
    p->d_k = (int32_t)d_k;
    p->d_v = (int32_t)d_v;
    p->P = P;
    p->scale = (float)scale;
    p->dtype = dtype;
    *out = p.release();
    return DISTDL_OK;
  });
}

int distdl_delta_plan_destroy(distdl_delta_plan* p) {
  if (!p) return DISTDL_OK;
  p->table.release();
  p->scratch.release();
  delete p;
  return DISTDL_OK;
}

int distdl_delta_fwd(distdl_delta_plan* p, const void* const q_dev[], const void* const k_dev[], const void* const v_dev[], const float* const g_dev[],
                     const float* const beta_dev[], const float* h0_dev, const int32_t* lengths_dev, void* const o_dev[], float* hT_dev, void* stream) {
  if (!p || !q_dev || !k_dev || !v_dev || !beta_dev || !o_dev) return set_error(DISTDL_ERR_NULL, "delta_fwd: null argument");
  if ((uintptr_t)h0_dev % 4 || (uintptr_t)lengths_dev % 4 || (uintptr_t)hT_dev % 4)
    return set_error(DISTDL_ERR_INVALID_ARG, "delta_fwd: h0, lengths or hT is not aligned to its elements");
  return guarded([&]() -> int {
    const size_t size = dtype_size(p->dtype);
    std::vector<DeltaWorker> w((size_t)p->P);
    int rc;
    for (int j = 0; j < p->P; ++j) {
      if ((rc = delta_check(q_dev[j], size, "q", j)) || (rc = delta_check(k_dev[j], size, "k", j)) || (rc = delta_check(v_dev[j], size, "v", j)) ||
          (g_dev && (rc = delta_check(g_dev[j], 4, "g", j))) || (rc = delta_check(beta_dev[j], 4, "beta", j)) ||
          (rc = delta_check(o_dev[j], size, "o", j)))
        return rc;
      w[j] = DeltaWorker{q_dev[j], k_dev[j], v_dev[j], g_dev ? g_dev[j] : nullptr, beta_dev[j], o_dev[j]};
    }
    hipStream_t st_ = (hipStream_t)stream;
    DeltaArgs s;
    if ((rc = delta_args(p, w, st_, &s))) return rc;
    s.h0 = h0_dev;
    s.lengths = lengths_dev;
    s.hT = hT_dev;
    {
      ProfScope prof("delta_fwd", st_);
      rc = launch_delta<false>(p, s, st_);
    }
    if (rc) return rc;
    DISTDL_HIP_TRY(hipGetLastError());
    return DISTDL_OK;
  });
}

int distdl_delta_bwd(distdl_delta_plan* p, const void* const q_dev[], const void* const k_dev[], const void* const v_dev[], const float* const g_dev[],
                     const float* const beta_dev[], const float* h0_dev, const int32_t* lengths_dev, const void* const do_dev[], const float* dhT_dev,
                     void* const dq_dev[], void* const dk_dev[], void* const dv_dev[], float* const dg_dev[], float* const dbeta_dev[], float* dh0_dev,
                     void* stream) {
  if (!p || !q_dev || !k_dev || !v_dev || !beta_dev || !do_dev || !dq_dev || !dk_dev || !dv_dev || !dbeta_dev)
    return set_error(DISTDL_ERR_NULL, "delta_bwd: null argument");
  if (dg_dev && !g_dev) return set_error(DISTDL_ERR_NULL, "delta_bwd: gradients of g without g");
  if ((uintptr_t)h0_dev % 4 || (uintptr_t)lengths_dev % 4 || (uintptr_t)dhT_dev % 4 || (uintptr_t)dh0_dev % 4)
    return set_error(DISTDL_ERR_INVALID_ARG, "delta_bwd: h0, lengths, dhT or dh0 is not aligned to its elements");
  return guarded([&]() -> int {
    const size_t size = dtype_size(p->dtype);
    std::vector<DeltaWorker> w((size_t)p->P);
    int rc;
    for (int j = 0; j < p->P; ++j) {
      if ((rc = delta_check(q_dev[j], size, "q", j)) || (rc = delta_check(k_dev[j], size, "k", j)) || (rc = delta_check(v_dev[j], size, "v", j)) ||
          (g_dev && (rc = delta_check(g_dev[j], 4, "g", j))) || (rc = delta_check(beta_dev[j], 4, "beta", j)) ||
          (rc = delta_check(do_dev[j], size, "do", j)) || (rc = delta_check(dq_dev[j], size, "dq", j)) || (rc = delta_check(dk_dev[j], size, "dk", j)) ||
          (rc = delta_check(dv_dev[j], size, "dv", j)) || (dg_dev && (rc = delta_check(dg_dev[j], 4, "dg", j))) ||
          (rc = delta_check(dbeta_dev[j], 4, "dbeta", j)))
        return rc;
      w[j] = DeltaWorker{q_dev[j],  k_dev[j],  v_dev[j],  g_dev ? g_dev[j] : nullptr,   beta_dev[j],  nullptr,
                         do_dev[j], dq_dev[j], dk_dev[j], dv_dev[j], dg_dev ? dg_dev[j] : nullptr, dbeta_dev[j]};
    }
    hipStream_t st_ = (hipStream_t)stream;
    DeltaArgs s;
    if ((rc = delta_args(p, w, st_, &s))) return rc;
    s.h0 = h0_dev;
    s.lengths = lengths_dev;
    s.dhT = dhT_dev;
    s.dh0 = dh0_dev;
    {
      ProfScope prof("delta_bwd", st_);
      rc = launch_delta<true>(p, s, st_);
    }
    if (rc) return rc;
    DISTDL_HIP_TRY(hipGetLastError());
    return DISTDL_OK;
  });
}

int distdl_delta_step(const void* q_dev, const void* k_dev, const void* v_dev, const float* g_dev, const float* beta_dev, float* state_dev,
                      int64_t n_slots, const int32_t* slots_dev, void* o_dev, int64_t rows, int64_t n_h, int64_t n_hk, int64_t d_k, int64_t d_v,
                      double scale, distdl_dtype dtype, void* stream) {
  if (rows < 0 || n_slots < 0) return set_error(DISTDL_ERR_INVALID_ARG, "delta_step: %lld rows, %lld slots", (long long)rows, (long long)n_slots);
  const int rc = delta_sizes("delta_step", n_h, n_hk, d_k, d_v, scale, dtype);
  if (rc) return rc;
  if (rows == 0) return DISTDL_OK;
  if (!q_dev || !k_dev || !v_dev || !beta_dev || !o_dev || (!state_dev && n_slots > 0)) return set_error(DISTDL_ERR_NULL, "delta_step: null argument");
  if (!slots_dev && n_slots < rows) return set_error(DISTDL_ERR_INVALID_ARG, "delta_step: %lld states for %lld rows", (long long)n_slots, (long long)rows);
  if (rows >= kMaxBlocks256 / (n_h * ((d_v + 31) / 32))) return set_error(DISTDL_ERR_UNSUPPORTED, "delta_step: problem too large");
  const size_t size = dtype_size(dtype);
  if ((uintptr_t)q_dev % size || (uintptr_t)k_dev % size || (uintptr_t)v_dev % size || (uintptr_t)o_dev % size || (uintptr_t)g_dev % 4 ||
      (uintptr_t)beta_dev % 4 || (uintptr_t)state_dev % 4 || (uintptr_t)slots_dev % 4)
    return set_error(DISTDL_ERR_INVALID_ARG, "delta_step: an array is not aligned to its elements");
  hipStream_t st_ = (hipStream_t)stream;
  {
    ProfScope prof("delta_step", st_);
    auto* launch = dtype == DISTDL_F32 ? delta_step_kind<float> : delta_step_kind<uint16_t>;
    launch(q_dev, k_dev, v_dev, g_dev, beta_dev, state_dev, slots_dev, o_dev, n_slots, rows, (int)n_h, (int)(n_h / n_hk), (int)d_k, (int)d_v,
           (float)scale, st_);
  }
  DISTDL_HIP_TRY(hipGetLastError());
  return DISTDL_OK;
}

}  // extern "C"
