// Root-mean-square norm over features that P workers share, with the residual's addition in front, and its adjoint.
//
//   forward   s = x + r;  rstd = 1 / sqrt(mean(s^2) + eps);  y = s rstd g        y in the tensor's type or in 8-bit blocks
//   adjoint   n = s rstd;  e = dy g;  ds = dsum + rstd (e - n mean(e n));  dg = sum over rows of dy n
//
// The sum over features is the all-reduce of the workers' partial sums; here it is one sum over all arrays of a row.  Both directions read
// and write every element once and are bound by memory, so a row is held in registers between its sum and its use, and a workgroup that
// goes from row to row has the next row's loads under way meanwhile.  A wave takes pieces of 512 features of one worker, each through a
// buffer that ends with the worker's row, so that features that are not there need no test.  A row belongs to 1, 4, 8 or 16 waves, by
// what keeps at most two pieces in a wave (adjoint: one); rows wider than that, over 16384 features (adjoint: 8192), are read twice, the second
// time from the caches, and dg is made by a launch of its own in front.
// ROWS16: every row starts at a multiple of 16 bytes, a lane's eight features are neighbours (two accesses of fp32, one of bf16).  Otherwise
// they are 64 apart, each access at its natural alignment: wide accesses that straddle cost more than narrow ones.
//
// Measured: forward 8192 x 4096 bf16 on two workers, residual in, sum and 8-bit codes out, 50 us (4.8 TB/s), on one with a bf16 answer in their place 51 (5.2 TB/s), its
// adjoint 52 (5.2 TB/s) and 5 for the sum of dg's parts; adjoint 5003 x 2000 fp32 on three workers, of whose pieces of 512 places half are empty,
// 34 us (4.7 TB/s) and 5 for the sum of dg's parts; forward 4 x 4096 3.7 us, a launch and a trip to memory.
#include <algorithm>
#include <cfloat>
#include <cstddef>

#include "block8.h"
#include "buffer.h"
#include "common.h"
#include "profile.h"

namespace distdl {

constexpr int kNormInline = 8;  // workers whose pointers travel with the launch; more are in a table
constexpr int kPiece = 512;     // features of a wave at a time

struct NormWorker {
  const void* x;       // forward: x; adjoint: s
  const void* r;       // forward: r or null; adjoint: dsum or null
  const float* g;
  const void* dy;      // adjoint
  void* s;             // forward: s or null; adjoint: ds
  void* y;             // forward: y or null; adjoint: dg
  uint8_t* q;          // forward: codes or null
  uint8_t* qs;         // their scales, [blocks][rows]
  int32_t piece0;      // first piece
  int32_t n;           // features
};

struct NormArgs {
  NormWorker w[kNormInline];
  const NormWorker* more;  // all of them, where they are more than kNormInline
  int32_t P, pieces;       // workers; pieces of a row
  int64_t rows;
  float inv_n, eps;
  float* rstd;             // forward: written if not null; adjoint: read
  float* partial;          // adjoint: [parts][512 pieces] sums of dy n
};

// The table's address is taken in the kernel itself, and its records are read as constants, into scalar registers.
static_assert(offsetof(NormArgs, w) == 0, "the kernels' first argument starts with the workers");
typedef const __attribute__((address_space(4))) NormWorker* NormTable;
#define NORM_TABLE(a) ((a).more ? (NormTable)(uint64_t)(a).more : (NormTable)__builtin_amdgcn_kernarg_segment_ptr())

struct NormPiece {
  NormWorker w;
  int col;  // first feature in the worker; behind all of them for a piece that is not there
};
__device__ __forceinline__ NormPiece norm_piece(NormTable table, int P, int pieces, int piece) {
  int j = 0;
  while (j + 1 < P && piece >= table[j + 1].piece0) ++j;
  const NormTable t = table + j;
  NormPiece p;
  p.w = NormWorker{t->x, t->r, t->g, t->dy, t->s, t->y, t->q, t->qs, t->piece0, t->n};
  p.col = piece < pieces ? (piece - t->piece0) * kPiece : t->n;
  return p;
}

// Row `row` of a worker's array: a buffer that ends with it.
template <class E>
__device__ __forceinline__ __amdgpu_buffer_rsrc_t norm_row(const void* p, int64_t row, int n) {
  return rsrc_of((const E*)p + row * n, (uint32_t)n * sizeof(E));
}

// A lane's eight features of a piece, as they lie in memory
template <class E, bool ROWS16>
struct NormRaw {
  uint32_t v[8];
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t r, int col, int lane) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t at = (uint32_t)(col + lane + 64 * i) * sizeof(E);
      if constexpr (sizeof(E) == 4) v[i] = __builtin_amdgcn_raw_buffer_load_b32(r, at, 0, 0);
      else v[i] = (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(r, at, 0, 0);
    }
  }
  __device__ __forceinline__ void values(float* f) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(sizeof(E) == 4 ? v[i] : v[i] << 16);
  }
};
template <>
struct NormRaw<float, true> {
  u32x4 a, b;
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t r, int col, int lane) {
    const uint32_t at = (uint32_t)(col + lane * 8) * 4;
    a = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, at, 0, 0));
    b = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, at + 16, 0, 0));
  }
  __device__ __forceinline__ void values(float* f) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[i] = __uint_as_float(a[i]);
      f[i + 4] = __uint_as_float(b[i]);
    }
  }
};
template <>
struct NormRaw<uint16_t, true> {
  u32x4 a;
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t r, int col, int lane) {
    a = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, (uint32_t)(col + lane * 8) * 2, 0, 0));
  }
  __device__ __forceinline__ void values(float* f) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = bf16_lo(a[i]);
      f[2 * i + 1] = bf16_hi(a[i]);
    }
  }
};

template <class E, bool ROWS16>
__device__ __forceinline__ void norm_put(__amdgpu_buffer_rsrc_t r, int col, int lane, const float* f) {
  if constexpr (!ROWS16) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t at = (uint32_t)(col + lane + 64 * i) * sizeof(E);
      if constexpr (sizeof(E) == 4) __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(f[i]), r, at, 0, 0);
      else __builtin_amdgcn_raw_buffer_store_b16(to_bf16(f[i]), r, at, 0, 0);
    }
  } else if constexpr (sizeof(E) == 4) {
    const uint32_t at = (uint32_t)(col + lane * 8) * 4;
    __builtin_amdgcn_raw_buffer_store_b128(u32x4{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])}, r, at, 0, 0);
    __builtin_amdgcn_raw_buffer_store_b128(u32x4{__float_as_uint(f[4]), __float_as_uint(f[5]), __float_as_uint(f[6]), __float_as_uint(f[7])}, r, at + 16, 0, 0);
  } else {
    __builtin_amdgcn_raw_buffer_store_b128(u32x4{to_bf16(f[0], f[1]), to_bf16(f[2], f[3]), to_bf16(f[4], f[5]), to_bf16(f[6], f[7])}, r,
                                           (uint32_t)(col + lane * 8) * 2, 0, 0);
  }
}

// The piece in 8 bits: a block of 128 lies in 16 lanes (a DPP row), or in all lanes, two features each.
template <bool ROWS16>
__device__ __forceinline__ void norm_put_codes(const NormPiece& p, int64_t row, int64_t rows, int lane, const float* f) {
  const auto q = norm_row<uint8_t>(p.w.q, row, p.w.n);
  if constexpr (ROWS16) {
    float mx = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) mx = fmaxf(mx, fabsf(f[i]));
    const int byte = scale_byte(row16_max(mx));
    const float inv = scale_inverse(byte);
    const uint32_t at = (uint32_t)(p.col + lane * 8);
    __builtin_amdgcn_raw_buffer_store_b32(pack_e4m3(f[0] * inv, f[1] * inv, f[2] * inv, f[3] * inv), q, at, 0, 0);
    __builtin_amdgcn_raw_buffer_store_b32(pack_e4m3(f[4] * inv, f[5] * inv, f[6] * inv, f[7] * inv), q, at + 4, 0, 0);
    if ((lane & 15) == 0 && (int)at < p.w.n) p.w.qs[(int64_t)(at >> 7) * rows + row] = (uint8_t)byte;
  } else {
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      float mx = row16_max(fmaxf(fabsf(f[2 * b]), fabsf(f[2 * b + 1])));
      mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
      mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
      const int byte = scale_byte(mx);
      const float inv = scale_inverse(byte);
      const uint32_t c = pack_e4m3(f[2 * b] * inv, f[2 * b + 1] * inv, 0.f, 0.f);
      const uint32_t at = (uint32_t)(p.col + lane + 128 * b);
      __builtin_amdgcn_raw_buffer_store_b8((uint8_t)c, q, at, 0, 0);
      __builtin_amdgcn_raw_buffer_store_b8((uint8_t)(c >> 8), q, at + 64, 0, 0);
      const int first = p.col + 128 * b;
      if (lane == 0 && first < p.w.n) p.w.qs[(int64_t)(first >> 7) * rows + row] = (uint8_t)byte;
    }
  }
}

// Sum over the waves of a row
template <int W>
__device__ __forceinline__ float row_sum(float v, float (*lds)[16], int& turn) {
  v = wave_sum(v);
  if constexpr (W > 1) {
    // two sets in turn: a wave may write the next row's sum while another still reads this one's
    float* const at = lds[turn ^= 1];
    if ((threadIdx.x & 63) == 0) at[threadIdx.x >> 6] = v;
    __syncthreads();
    v = at[0];
#pragma unroll
    for (int w = 1; w < W; ++w) v += at[w];
  }
  return v;
}

constexpr int norm_threads(int W) { return W == 1 ? 256 : 64 * W; }  // a workgroup is one row, or four of one wave each

template <class E, int W, int R, bool ROWS16, bool WIDE>
__global__ __launch_bounds__(norm_threads(W)) void norm_fwd_kernel(NormArgs a) {
  constexpr int kRows = norm_threads(W) / (64 * W);
  __shared__ float lds[2][16];
  const NormTable table = NORM_TABLE(a);
  int turn = 0;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), w = wave % W;
  const int sets = WIDE ? (a.pieces + W * R - 1) / (W * R) : 1;
  NormPiece at[R];
  NormRaw<E, ROWS16> x[R], r[R];
  float g[R][8];
  auto place = [&](int set) __attribute__((always_inline)) {
#pragma unroll
    for (int k = 0; k < R; ++k) {
      at[k] = norm_piece(table, a.P, a.pieces, (set * R + k) * W + w);
      NormRaw<float, ROWS16> raw;
      raw.load(rsrc_of(at[k].w.g, (uint32_t)at[k].w.n * 4), at[k].col, lane);
      raw.values(g[k]);
    }
  };
  auto load = [&](int64_t row) __attribute__((always_inline)) {
#pragma unroll
    for (int k = 0; k < R; ++k) {
      x[k].load(norm_row<E>(at[k].w.x, row, at[k].w.n), at[k].col, lane);
      if (at[k].w.r) r[k].load(norm_row<E>(at[k].w.r, row, at[k].w.n), at[k].col, lane);
    }
  };
  float v[R][8];
  auto add = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int k = 0; k < R; ++k) {
      x[k].values(v[k]);
      if (at[k].w.r) {
        float u[8];
        r[k].values(u);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[k][i] += u[i];
      }
    }
  };
  const int64_t step = (int64_t)gridDim.x * kRows;
  int64_t row = (int64_t)blockIdx.x * kRows + wave / W;
  if (!WIDE) {
    place(0);
    if (row < a.rows) load(row);
  }
  for (; row < a.rows; row += step) {  // (rows of a workgroup of several waves are the same for all of them)
    float sum = 0.f;
    for (int set = 0; set < sets; ++set) {
      if (WIDE) {
        place(set);
        load(row);
      }
      add();
#pragma unroll
      for (int k = 0; k < R; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i) sum = fmaf(v[k][i], v[k][i], sum);
    }
    if (!WIDE) load(min(row + step, a.rows - 1));
    const float rstd = 1.f / sqrtf(fmaf(row_sum<W>(sum, lds, turn), a.inv_n, a.eps));
    if (a.rstd && lane == 0 && w == 0) a.rstd[row] = rstd;
    for (int set = 0; set < sets; ++set) {
      if (WIDE) {
        place(set);
        load(row);
        add();
      }
#pragma unroll
      for (int k = 0; k < R; ++k) {
        const NormWorker& p = at[k].w;
        if (p.s) norm_put<E, ROWS16>(norm_row<E>(p.s, row, p.n), at[k].col, lane, v[k]);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[k][i] = v[k][i] * rstd * g[k][i];  // (n = s rstd first, as the adjoint has it)
        if (p.y) norm_put<E, ROWS16>(norm_row<E>(p.y, row, p.n), at[k].col, lane, v[k]);
        if (p.q) norm_put_codes<ROWS16>(at[k], row, a.rows, lane, v[k]);
      }
    }
  }
}

// A workgroup takes every gridDim'th group of rows and keeps its part of dg in registers; norm_dg_kernel sums the parts in a fixed
// order.  Rows wider than the registers (WIDE) leave the parts to norm_dg_wide_kernel.
template <class E, int W, int R, bool ROWS16, bool WIDE>
__global__ __launch_bounds__(norm_threads(W)) void norm_bwd_kernel(NormArgs a) {
  constexpr int kRows = norm_threads(W) / (64 * W);
  __shared__ float lds[2][16];
  const NormTable table = NORM_TABLE(a);
  int turn = 0;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), w = wave % W;
  const int sets = WIDE ? (a.pieces + W * R - 1) / (W * R) : 1;
  NormPiece at[R];
  NormRaw<E, ROWS16> x[R], dy[R], r[R];
  float g[R][8], dg[R][8] = {};
  float rstd = 0.f;
  auto place = [&](int set) __attribute__((always_inline)) {
#pragma unroll
    for (int k = 0; k < R; ++k) {
      at[k] = norm_piece(table, a.P, a.pieces, (set * R + k) * W + w);
      NormRaw<float, ROWS16> raw;
      raw.load(rsrc_of(at[k].w.g, (uint32_t)at[k].w.n * 4), at[k].col, lane);
      raw.values(g[k]);
    }
  };
  auto load = [&](int64_t row) __attribute__((always_inline)) {
    rstd = a.rstd[row];
#pragma unroll
    for (int k = 0; k < R; ++k) {
      x[k].load(norm_row<E>(at[k].w.x, row, at[k].w.n), at[k].col, lane);
      dy[k].load(norm_row<E>(at[k].w.dy, row, at[k].w.n), at[k].col, lane);
      if (at[k].w.r) r[k].load(norm_row<E>(at[k].w.r, row, at[k].w.n), at[k].col, lane);
    }
  };
  const int64_t step = (int64_t)gridDim.x * kRows;
  int64_t row = (int64_t)blockIdx.x * kRows + wave / W;
  if (!WIDE) {
    place(0);
    if (row < a.rows) load(row);
  }
  for (; row < a.rows; row += step) {
    float n[R][8], e[R][8], u[R][8] = {}, dot = 0.f, scale = rstd;
    auto spread = [&](bool first) __attribute__((always_inline)) {
      scale = rstd;
#pragma unroll
      for (int k = 0; k < R; ++k) {
        x[k].values(n[k]);
        dy[k].values(e[k]);
        if (at[k].w.r) r[k].values(u[k]);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          n[k][i] *= scale;
          if (!WIDE) dg[k][i] = fmaf(e[k][i], n[k][i], dg[k][i]);
          e[k][i] *= g[k][i];
          if (first) dot = fmaf(e[k][i], n[k][i], dot);
        }
      }
    };
    for (int set = 0; set < sets; ++set) {
      if (WIDE) {
        place(set);
        load(row);
      }
      spread(true);
    }
    if (!WIDE) load(min(row + step, a.rows - 1));
    const float mean = row_sum<W>(dot, lds, turn) * a.inv_n;
    for (int set = 0; set < sets; ++set) {
      if (WIDE) {
        place(set);
        load(row);
        spread(false);
      }
#pragma unroll
      for (int k = 0; k < R; ++k) {
#pragma unroll
        for (int i = 0; i < 8; ++i) e[k][i] = fmaf(scale, fmaf(-n[k][i], mean, e[k][i]), at[k].w.r ? u[k][i] : 0.f);
        norm_put<E, ROWS16>(norm_row<E>(at[k].w.s, row, at[k].w.n), at[k].col, lane, e[k]);
      }
    }
  }
  if constexpr (!WIDE) {
    float* const to = a.partial + (int64_t)blockIdx.x * a.pieces * kPiece;
    if constexpr (kRows == 1) {
#pragma unroll
      for (int k = 0; k < R; ++k)
        if (k * W + w < a.pieces) {
#pragma unroll
          for (int i = 0; i < 8; ++i) to[(k * W + w) * kPiece + (ROWS16 ? lane * 8 + i : lane + 64 * i)] = dg[k][i];
        }
    } else {  // four rows at a time: their parts meet in LDS
      __shared__ float part[kRows][R * kPiece];
#pragma unroll
      for (int k = 0; k < R; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i) part[wave][k * kPiece + i * 64 + lane] = dg[k][i];
      __syncthreads();
      for (int c = threadIdx.x; c < a.pieces * kPiece; c += 256) {
        const int in = c % kPiece, u = c - in + (ROWS16 ? (in & 7) * 64 + (in >> 3) : in);
        to[c] = (part[0][u] + part[1][u]) + (part[2][u] + part[3][u]);
      }
    }
  }
}

// The parts of dg for wide rows: a wave takes a piece and every (4 gridDim.y)'th row.
template <class E, bool ROWS16>
__global__ __launch_bounds__(256) void norm_dg_wide_kernel(NormArgs a) {
  __shared__ float part[4][8][64];
  const NormTable table = NORM_TABLE(a);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const NormPiece at = norm_piece(table, a.P, a.pieces, blockIdx.x);
  float dg[8] = {};
  for (int64_t row = blockIdx.y * 4 + wave; row < a.rows; row += (int64_t)gridDim.y * 4) {
    NormRaw<E, ROWS16> x, dy;
    float n[8], e[8];
    x.load(norm_row<E>(at.w.x, row, at.w.n), at.col, lane);
    dy.load(norm_row<E>(at.w.dy, row, at.w.n), at.col, lane);
    x.values(n);
    dy.values(e);
    const float rstd = a.rstd[row];
#pragma unroll
    for (int i = 0; i < 8; ++i) dg[i] = fmaf(e[i], n[i] * rstd, dg[i]);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) part[wave][i][lane] = dg[i];
  __syncthreads();
  if (wave == 0) {
    float* const to = a.partial + ((int64_t)blockIdx.y * a.pieces + blockIdx.x) * kPiece;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      to[ROWS16 ? lane * 8 + i : lane + 64 * i] = (part[0][i][lane] + part[1][i][lane]) + (part[2][i][lane] + part[3][i][lane]);
  }
}

// dg from its parts: a workgroup takes 16 columns, a row of 16 threads every 64th part.
__global__ __launch_bounds__(1024) void norm_dg_kernel(NormArgs a, int parts) {
  __shared__ float lds[64][17];
  const NormTable table = NORM_TABLE(a);
  const int x = threadIdx.x & 15, y = threadIdx.x >> 4, c = blockIdx.x * 16 + x, columns = a.pieces * kPiece;
  float sum = 0.f;
  for (int p = y; p < parts; p += 64) sum += a.partial[(int64_t)p * columns + c];
  lds[y][x] = sum;
  __syncthreads();
  for (int half = 32; half > 0; half >>= 1) {
    if (y < half) lds[y][x] += lds[y + half][x];
    __syncthreads();
  }
  const NormPiece at = norm_piece(table, a.P, a.pieces, blockIdx.x / (kPiece / 16));
  const int col = at.col + c % kPiece;
  if (y == 0 && col < at.w.n) ((float*)at.w.y)[col] = lds[0][x];
}

}  // namespace distdl

struct distdl_rmsnorm_plan {
  int64_t rows = 0, n_f = 0;
  int P = 1;
  double eps = 0;
  distdl_dtype dtype = DISTDL_F32;
  std::vector<int32_t> piece0, size;
  int32_t pieces = 0;
  distdl::DevArray<distdl::NormWorker> table;
  distdl::StreamScratch partial;
};

namespace distdl {

// The launch for rows of so many pieces: waves of a row, pieces of a wave, wide or not.  The adjoint holds three arrays, gains and sums:
// a wave has one piece there (two take 165 registers for fp32, three waves to a SIMD).
template <bool BACK, class F>
static void norm_shape(int pieces, F f) {
  typedef std::integral_constant<int, 1> One;
  typedef std::integral_constant<int, 2> Two;
  typedef std::integral_constant<int, 4> Four;
  typedef std::integral_constant<int, 8> Eight;
  typedef std::integral_constant<int, 16> Sixteen;
  if constexpr (BACK) {
    if (pieces <= 1) f(One(), One(), std::false_type());
    else if (pieces <= 2) f(Two(), One(), std::false_type());
    else if (pieces <= 4) f(Four(), One(), std::false_type());
    else if (pieces <= 8) f(Eight(), One(), std::false_type());
    else if (pieces <= 16) f(Sixteen(), One(), std::false_type());
    else f(Sixteen(), One(), std::true_type());
  } else {
    if (pieces <= 1) f(One(), One(), std::false_type());
    else if (pieces <= 2) f(One(), Two(), std::false_type());
    else if (pieces <= 4) f(Four(), One(), std::false_type());
    else if (pieces <= 8) f(Four(), Two(), std::false_type());
    else if (pieces <= 16) f(Eight(), Two(), std::false_type());
    else if (pieces <= 32) f(Sixteen(), Two(), std::false_type());
    else f(Sixteen(), Two(), std::true_type());
  }
}

// Whether every row of every array starts at a multiple of 16 bytes (gains and codes at multiples of 16 and 4).
static bool norm_rows16(const std::vector<NormWorker>& w, size_t size) {
  uintptr_t bits = 0;
  for (const NormWorker& v : w)
    bits |= (uintptr_t)(v.n * size) | (uintptr_t)v.x | (uintptr_t)v.r | (uintptr_t)v.g | (uintptr_t)v.dy | (uintptr_t)v.s |
            (v.dy ? 0 : (uintptr_t)v.y) | (uintptr_t)v.q * 4;
  return bits % 16 == 0;
}

static int norm_args(distdl_rmsnorm_plan* p, const std::vector<NormWorker>& w, hipStream_t st, NormArgs* a) {
  a->more = nullptr;
  a->P = p->P;
  a->pieces = p->pieces;
  a->rows = p->rows;
  a->inv_n = (float)(1.0 / (double)p->n_f);
  a->eps = p->eps > 0 ? std::max((float)p->eps, FLT_MIN) : 0.f;  // (rows of zeros stay zeros under any eps that is not zero)
  a->partial = nullptr;
  if (p->P <= kNormInline) {
    std::copy(w.begin(), w.end(), a->w);
    return DISTDL_OK;
  }
  const int rc = p->table.upload(w, st);
  a->more = p->table.dev;
  return rc;
}

static int norm_check(const void* v, size_t size, const char* what, int j) {
  if (!v) return set_error(DISTDL_ERR_NULL, "rmsnorm: %s[%d] is null", what, j);
  if ((uintptr_t)v % size) return set_error(DISTDL_ERR_INVALID_ARG, "rmsnorm: %s[%d] is not aligned to its elements", what, j);
  return DISTDL_OK;
}

template <class E, bool ROWS16>
static void launch_norm_fwd(const NormArgs& a, hipStream_t st) {
  norm_shape<false>(a.pieces, [&](auto W, auto R, auto wide) {
    const int rows = norm_threads(W) / (64 * W);
    const int64_t groups = (a.rows + rows - 1) / rows;
    hipLaunchKernelGGL((norm_fwd_kernel<E, W, R, ROWS16, wide>), dim3((unsigned)std::min<int64_t>(groups, 4096 / W)), dim3(norm_threads(W)), 0, st, a);
  });
}

template <class E, bool ROWS16>
static int launch_norm_bwd(distdl_rmsnorm_plan* p, NormArgs& a, hipStream_t st) {
  int rc = DISTDL_OK, parts = 0;
  norm_shape<true>(a.pieces, [&](auto W, auto R, auto wide) {
    const int rows = norm_threads(W) / (64 * W);
    const int64_t groups = (a.rows + rows - 1) / rows;
    const int grid = (int)std::min<int64_t>(groups, W == 1 ? 1024 : 4096 / W);
    parts = wide ? (int)std::min<int64_t>((a.rows + 3) / 4, 64) : grid;
    rc = p->partial.get((size_t)parts * a.pieces * kPiece, st, &a.partial);
    if (rc) return;
    // Before norm_bwd_kernel, whose dx may lie on s or dy.
    if (wide) hipLaunchKernelGGL((norm_dg_wide_kernel<E, ROWS16>), dim3(a.pieces, parts), dim3(256), 0, st, a);
    hipLaunchKernelGGL((norm_bwd_kernel<E, W, R, ROWS16, wide>), dim3((unsigned)grid), dim3(norm_threads(W)), 0, st, a);
  });
  if (rc) return rc;
  hipLaunchKernelGGL(norm_dg_kernel, dim3(a.pieces * (kPiece / 16)), dim3(1024), 0, st, a, parts);
  return DISTDL_OK;
}

}  // namespace distdl

using namespace distdl;

extern "C" {

int distdl_rmsnorm_plan_create(distdl_rmsnorm_plan** out, int64_t rows, int64_t n_f, int P, double eps, distdl_dtype dtype) {
  if (!out) return set_error(DISTDL_ERR_NULL, "rmsnorm_plan_create: null argument");
  *out = nullptr;
  if (rows < 0 || n_f < 1 || P < 1) return set_error(DISTDL_ERR_INVALID_ARG, "rmsnorm_plan_create: %lld rows of %lld features on %d workers",
                                                     (long long)rows, (long long)n_f, P);
  if (!(eps >= 0) || !std::isfinite(eps)) return set_error(DISTDL_ERR_INVALID_ARG, "rmsnorm_plan_create: eps %g", eps);
  if (dtype != DISTDL_F32 && dtype != DISTDL_BF16) return set_error(DISTDL_ERR_UNSUPPORTED, "unknown dtype");
  if (n_f < P) return set_error(DISTDL_ERR_EMPTY_PARTITION, "rmsnorm: %lld features over %d workers", (long long)n_f, P);
  if (n_f > 1 << 24 || rows >= kMaxBlocks256 || P > 1 << 12) return set_error(DISTDL_ERR_UNSUPPORTED, "rmsnorm: problem too large");
  return guarded([&]() -> int {
    std::unique_ptr<distdl_rmsnorm_plan> p(new distdl_rmsnorm_plan());
    p->rows = rows;
    p->n_f = n_f;
    p->P = P;
    p->eps = eps;
    p->dtype = dtype;
    for (int j = 0; j < P; ++j) {
      p->size.push_back((int32_t)(n_f / P + (j < n_f % P ? 1 : 0)));
      p->piece0.push_back(p->pieces);
      p->pieces += (p->size.back() + kPiece - 1) / kPiece;
    }
    *out = p.release();
    return DISTDL_OK;
  });
}

int distdl_rmsnorm_plan_destroy(distdl_rmsnorm_plan* p) {
  if (!p) return DISTDL_OK;
  p->table.release();
  p->partial.release();
  delete p;
  return DISTDL_OK;
}

int distdl_rmsnorm_fwd(distdl_rmsnorm_plan* p, const void* const x_dev[], const void* const r_dev[], const float* const g_dev[],
                       void* const s_dev[], void* const y_dev[], void* const q_dev[], void* const qs_dev[], float* rstd_dev,
                       void* stream) {
  if (!p || !x_dev || !g_dev) return set_error(DISTDL_ERR_NULL, "rmsnorm_fwd: null argument");
  if ((q_dev == nullptr) != (qs_dev == nullptr)) return set_error(DISTDL_ERR_NULL, "rmsnorm_fwd: codes without scales, or scales without codes");
  if (!s_dev && !y_dev && !q_dev && !rstd_dev) return set_error(DISTDL_ERR_NULL, "rmsnorm_fwd: no output");
  if (p->rows == 0) return DISTDL_OK;
  return guarded([&]() -> int {
    const size_t size = dtype_size(p->dtype);
    std::vector<NormWorker> w((size_t)p->P);
    int rc;
    for (int j = 0; j < p->P; ++j) {
      if ((rc = norm_check(x_dev[j], size, "x", j)) || (rc = norm_check(g_dev[j], 4, "g", j)) || (r_dev && (rc = norm_check(r_dev[j], size, "r", j))) ||
          (s_dev && (rc = norm_check(s_dev[j], size, "s", j))) || (y_dev && (rc = norm_check(y_dev[j], size, "y", j))) ||
          (q_dev && ((rc = norm_check(q_dev[j], 1, "q", j)) || (rc = norm_check(qs_dev[j], 1, "qs", j)))))
        return rc;
      w[j] = NormWorker{x_dev[j], r_dev ? r_dev[j] : nullptr, g_dev[j], nullptr, s_dev ? s_dev[j] : nullptr, y_dev ? y_dev[j] : nullptr,
                        q_dev ? (uint8_t*)q_dev[j] : nullptr, q_dev ? (uint8_t*)qs_dev[j] : nullptr, p->piece0[j], p->size[j]};
    }
    if ((uintptr_t)rstd_dev % 4) return set_error(DISTDL_ERR_INVALID_ARG, "rmsnorm_fwd: rstd is not aligned to its elements");
    hipStream_t st_ = (hipStream_t)stream;
    NormArgs a;
    if ((rc = norm_args(p, w, st_, &a))) return rc;
    a.rstd = rstd_dev;
    {
      ProfScope prof("rmsnorm_fwd", st_);
      if (p->dtype == DISTDL_F32) norm_rows16(w, 4) ? launch_norm_fwd<float, true>(a, st_) : launch_norm_fwd<float, false>(a, st_);
      else norm_rows16(w, 2) ? launch_norm_fwd<uint16_t, true>(a, st_) : launch_norm_fwd<uint16_t, false>(a, st_);
    }
    DISTDL_HIP_TRY(hipGetLastError());
    return DISTDL_OK;
  });
}

int distdl_rmsnorm_bwd(distdl_rmsnorm_plan* p, const void* const s_dev[], const float* const g_dev[], const float* rstd_dev,
                       const void* const dy_dev[], const void* const dsum_dev[], void* const dx_dev[], float* const dg_dev[],
                       void* stream) {
  if (!p || !s_dev || !g_dev || (!rstd_dev && p->rows > 0) || !dy_dev || !dx_dev || !dg_dev) return set_error(DISTDL_ERR_NULL, "rmsnorm_bwd: null argument");
  return guarded([&]() -> int {
    const size_t size = dtype_size(p->dtype);
    std::vector<NormWorker> w((size_t)p->P);
    int rc;
    for (int j = 0; j < p->P; ++j) {
      if ((rc = norm_check(dg_dev[j], 4, "dg", j))) return rc;
      if (p->rows > 0 && ((rc = norm_check(s_dev[j], size, "s", j)) || (rc = norm_check(g_dev[j], 4, "g", j)) ||
                          (rc = norm_check(dy_dev[j], size, "dy", j)) || (dsum_dev && (rc = norm_check(dsum_dev[j], size, "dsum", j))) ||
                          (rc = norm_check(dx_dev[j], size, "dx", j))))
        return rc;
      w[j] = NormWorker{s_dev[j], dsum_dev ? dsum_dev[j] : nullptr, g_dev[j], dy_dev[j], dx_dev[j], dg_dev[j], nullptr, nullptr,
                        p->piece0[j], p->size[j]};
    }
    if ((uintptr_t)rstd_dev % 4) return set_error(DISTDL_ERR_INVALID_ARG, "rmsnorm_bwd: rstd is not aligned to its elements");
    hipStream_t st_ = (hipStream_t)stream;
    NormArgs a;
    if ((rc = norm_args(p, w, st_, &a))) return rc;
    a.rstd = const_cast<float*>(rstd_dev);
    {
      ProfScope prof("rmsnorm_bwd", st_);
      if (p->rows == 0) hipLaunchKernelGGL(norm_dg_kernel, dim3(a.pieces * (kPiece / 16)), dim3(1024), 0, st_, a, 0);  // (sums of nothing)
      else if (p->dtype == DISTDL_F32) rc = norm_rows16(w, 4) ? launch_norm_bwd<float, true>(p, a, st_) : launch_norm_bwd<float, false>(p, a, st_);
      else rc = norm_rows16(w, 2) ? launch_norm_bwd<uint16_t, true>(p, a, st_) : launch_norm_bwd<uint16_t, false>(p, a, st_);
      if (rc) return rc;
    }
    DISTDL_HIP_TRY(hipGetLastError());
    return DISTDL_OK;
  });
}

}  // extern "C"
