// Root-mean-square norm over features that P workers share, with the residual's addition in front, and its adjoint.
//
//   forward   s = x + r;  rstd = 1 / sqrt(mean(s^2) + eps);  y = s rstd g        y in the tensor's type or in 8-bit blocks
//   adjoint   n = s rstd;  e = dy g;  ds = dsum + rstd (e - n mean(e n));  dg = sum over rows of dy n
//
// The sum over features is the all-reduce of the workers' partial sums; here it is one sum over all arrays of a row.  Both directions read
// and write every element once and are bound by memory, so a row is held in registers between its sum and its use.  A thread takes
// units of eight features: 16 lanes (a DPP row) hold a block of 128, whose largest magnitude needs no LDS; a
// worker's units are padded to blocks, so that no block crosses arrays.  A row belongs to one wave (up to 512 features a register set) or to
// a workgroup of four, by what keeps at most four units in a thread; wider rows are read twice, the second time from the caches.
#include <algorithm>

#include "block8.h"
#include "common.h"
#include "profile.h"

namespace distdl {

constexpr int kNormInline = 8;  // workers whose pointers travel with the launch; more are in a table

struct NormWorker {
  const void* x;       // forward: x; adjoint: s
  const void* r;       // forward: r or null; adjoint: dsum or null
  const float* g;
  const void* dy;      // adjoint
  void* s;             // forward: s or null; adjoint: ds
  void* y;             // forward: y or null; adjoint: dg
  uint8_t* q;          // forward: codes or null
  uint8_t* qs;         // their scales, [blocks][rows]
  int32_t unit0;       // first unit
  int32_t n;           // features
};

struct NormArgs {
  NormWorker w[kNormInline];
  const NormWorker* more;  // all of them, where they are more than kNormInline
  int32_t P, units;        // workers; units of a row, those that pad blocks among them
  int64_t rows;
  float inv_n, eps;
  float* rstd;             // forward: written if not null; adjoint: read
  float* partial;          // adjoint: [parts][8 units] sums of dy n
};

__device__ __forceinline__ const NormWorker& norm_worker(const NormArgs& a, int j) { return a.more ? a.more[j] : a.w[j]; }

// Where a unit lies: its worker and its first feature there.  P is small and the loop uniform: its loads are scalar.
struct NormPlace {
  const void *x, *r, *dy;
  const float* g;
  void *s, *y;
  uint8_t *q, *qs;
  int32_t n, col, left;  // the worker's features; first feature; features of the unit
};
__device__ __forceinline__ NormPlace norm_place(const NormArgs& a, int unit) {
  NormPlace p{};
  for (int j = 0; j < a.P; ++j) {
    const NormWorker& w = norm_worker(a, j);
    if (unit >= w.unit0) {
      p = NormPlace{w.x, w.r, w.dy, w.g, w.s, w.y, w.q, w.qs, w.n, (unit - w.unit0) * 8, 0};
    }
  }
  p.left = unit < a.units ? max(0, min(8, p.n - p.col)) : 0;
  return p;
}

// Sum over the threads of a row: one wave, or the four waves of a workgroup.
template <int T>
__device__ __forceinline__ float row_sum(float v, float* lds, int& turn) {
  v = wave_sum(v);
  if constexpr (T == 256) {
    // two sets in turn: a wave may write the next row's sum while another still reads this one's
    float* const at = lds + (turn ^= 4);
    if ((threadIdx.x & 63) == 0) at[threadIdx.x >> 6] = v;
    __syncthreads();
    v = (at[0] + at[1]) + (at[2] + at[3]);
  }
  return v;
}

template <class E, int T, int R, bool WIDE>
__global__ __launch_bounds__(256) void norm_fwd_kernel(NormArgs a) {
  __shared__ float lds[8];
  int turn = 0;
  const int t = threadIdx.x % T;
  const int64_t row = (int64_t)blockIdx.x * (256 / T) + threadIdx.x / T;
  if (T < 256 && row >= a.rows) return;  // (whole waves)
  NormPlace at[R];
  Eight<E> x[R], r[R];
  float v[R][8];
  float sum = 0.f;
  const int sets = WIDE ? (a.units + T * R - 1) / (T * R) : 1;
  for (int set = 0; set < sets; ++set) {
#pragma unroll
    for (int k = 0; k < R; ++k) {
      at[k] = norm_place(a, (set * R + k) * T + t);
      x[k].load((const E*)at[k].x + row * at[k].n + at[k].col, at[k].left);
      if (at[k].r) r[k].load((const E*)at[k].r + row * at[k].n + at[k].col, at[k].left);
    }
#pragma unroll
    for (int k = 0; k < R; ++k) {
      x[k].values(v[k]);
      if (at[k].r) {
        float u[8];
        r[k].values(u);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[k][i] += u[i];
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) sum = fmaf(v[k][i], v[k][i], sum);
    }
  }
  const float rstd = 1.f / sqrtf(fmaf(row_sum<T>(sum, lds, turn), a.inv_n, a.eps));
  if (a.rstd && t == 0) a.rstd[row] = rstd;
  for (int set = 0; set < sets; ++set) {
#pragma unroll
    for (int k = 0; k < R; ++k) {
      if (WIDE) {
        at[k] = norm_place(a, (set * R + k) * T + t);
        x[k].load((const E*)at[k].x + row * at[k].n + at[k].col, at[k].left);
        x[k].values(v[k]);
        if (at[k].r) {
          float u[8];
          r[k].load((const E*)at[k].r + row * at[k].n + at[k].col, at[k].left);
          r[k].values(u);
#pragma unroll
          for (int i = 0; i < 8; ++i) v[k][i] += u[i];
        }
      }
      const int left = at[k].left;
      const int64_t to = row * at[k].n + at[k].col;
      if (at[k].s && left > 0) store8((E*)at[k].s + to, v[k], left);
      Eight<float> gain;
      float g[8], mx = 0.f;
      gain.load(at[k].g + at[k].col, left);
      gain.values(g);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        v[k][i] = i < left ? v[k][i] * rstd * g[i] : 0.f;
        mx = fmaxf(mx, fabsf(v[k][i]));
      }
      if (at[k].y && left > 0) store8((E*)at[k].y + to, v[k], left);
      mx = row16_max(mx);
      if (at[k].q && left > 0) {
        const int byte = scale_byte(mx);
        const float inv = scale_inverse(byte);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[k][i] *= inv;
        store8_codes(at[k].q + to, u32x2{pack_e4m3(v[k][0], v[k][1], v[k][2], v[k][3]), pack_e4m3(v[k][4], v[k][5], v[k][6], v[k][7])}, left);
        if ((t & 15) == 0) at[k].qs[(int64_t)(at[k].col >> 7) * a.rows + row] = (uint8_t)byte;
      }
    }
  }
}

// A workgroup takes every gridDim'th group of rows and keeps its part of dg in registers; norm_dg_kernel sums the parts in a fixed
// order.  Rows wider than the registers (WIDE) leave the parts to norm_dg_wide_kernel.
template <class E, int T, int R, bool WIDE>
__global__ __launch_bounds__(256) void norm_bwd_kernel(NormArgs a) {
  __shared__ float lds[8];
  int turn = 0;
  const int t = threadIdx.x % T, lane_row = threadIdx.x / T;
  NormPlace at[R];
  float g[R][8], dg[R][8];
  auto gains = [&](int k) {
    Eight<float> gain;
    gain.load(at[k].g + at[k].col, at[k].left);
    gain.values(g[k]);
  };
#pragma unroll
  for (int k = 0; k < R; ++k) {
    if (!WIDE) {
      at[k] = norm_place(a, k * T + t);
      gains(k);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) dg[k][i] = 0.f;
  }
  const int sets = WIDE ? (a.units + T * R - 1) / (T * R) : 1;
  for (int64_t row0 = (int64_t)blockIdx.x * (256 / T); row0 < a.rows; row0 += (int64_t)gridDim.x * (256 / T)) {
    const int64_t row = row0 + lane_row;
    if (T < 256 && row >= a.rows) break;  // (whole waves, in the last turn)
    const float rstd = a.rstd[row];
    Eight<E> x[R], dy[R], r[R];
    float n[R][8], e[R][8], dot = 0.f;
    auto load = [&](int set, bool with_r) {
#pragma unroll
      for (int k = 0; k < R; ++k) {
        if (WIDE) at[k] = norm_place(a, (set * R + k) * T + t);
        const int64_t from = row * at[k].n + at[k].col;
        x[k].load((const E*)at[k].x + from, at[k].left);
        dy[k].load((const E*)at[k].dy + from, at[k].left);
        if (with_r && at[k].r) r[k].load((const E*)at[k].r + from, at[k].left);
        if (WIDE) gains(k);
      }
    };
    auto spread = [&](bool first) {
#pragma unroll
      for (int k = 0; k < R; ++k) {
        x[k].values(n[k]);
        dy[k].values(e[k]);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          n[k][i] *= rstd;
          if (!WIDE) dg[k][i] = fmaf(e[k][i], n[k][i], dg[k][i]);
          e[k][i] *= g[k][i];
          if (first) dot = fmaf(e[k][i], n[k][i], dot);
        }
      }
    };
    for (int set = 0; set < sets; ++set) {
      load(set, !WIDE);
      spread(true);
    }
    const float mean = row_sum<T>(dot, lds, turn) * a.inv_n;
    for (int set = 0; set < sets; ++set) {
      if (WIDE) {
        load(set, true);
        spread(false);
      }
#pragma unroll
      for (int k = 0; k < R; ++k) {
        if (at[k].left <= 0) continue;
        float u[8];
        if (at[k].r) r[k].values(u);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float d = rstd * fmaf(-n[k][i], mean, e[k][i]);
          e[k][i] = at[k].r ? u[i] + d : d;
        }
        store8((E*)at[k].s + row * at[k].n + at[k].col, e[k], at[k].left);
      }
    }
  }
  if constexpr (!WIDE) {
    float* const to = a.partial + (int64_t)blockIdx.x * a.units * 8;
    if constexpr (T == 256) {
#pragma unroll
      for (int k = 0; k < R; ++k)
        if (k * T + t < a.units) store8(to + (k * T + t) * 8, dg[k], 8);
    } else {
      __shared__ float part[4][R * T * 8];
#pragma unroll
      for (int k = 0; k < R; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i) part[lane_row][i * R * T + k * T + t] = dg[k][i];
      __syncthreads();
      for (int c = threadIdx.x; c < a.units * 8; c += 256) {
        const int u = (c & 7) * R * T + (c >> 3);
        to[c] = (part[0][u] + part[1][u]) + (part[2][u] + part[3][u]);
      }
    }
  }
}

// The parts of dg for wide rows: a wave takes 64 units and every (4 gridDim.y)'th row.
template <class E>
__global__ __launch_bounds__(256) void norm_dg_wide_kernel(NormArgs a) {
  __shared__ float part[4][8][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, unit = blockIdx.x * 64 + lane;
  const NormPlace at = norm_place(a, unit);
  float dg[8] = {};
  for (int64_t row = blockIdx.y * 4 + wave; row < a.rows; row += (int64_t)gridDim.y * 4) {
    Eight<E> x, dy;
    float n[8], e[8];
    x.load((const E*)at.x + row * at.n + at.col, at.left);
    dy.load((const E*)at.dy + row * at.n + at.col, at.left);
    x.values(n);
    dy.values(e);
    const float rstd = a.rstd[row];
#pragma unroll
    for (int i = 0; i < 8; ++i) dg[i] = fmaf(e[i], n[i] * rstd, dg[i]);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) part[wave][i][lane] = dg[i];
  __syncthreads();
  if (wave == 0 && unit < a.units) {
#pragma unroll
    for (int i = 0; i < 8; ++i) dg[i] = (part[0][i][lane] + part[1][i][lane]) + (part[2][i][lane] + part[3][i][lane]);
    store8(a.partial + ((int64_t)blockIdx.y * a.units + unit) * 8, dg, 8);
  }
}

// dg from its parts: a workgroup takes 16 columns, a row of 16 threads every 64th part.
__global__ __launch_bounds__(1024) void norm_dg_kernel(NormArgs a, int parts) {
  __shared__ float lds[64][17];
  const int x = threadIdx.x & 15, y = threadIdx.x >> 4, c = blockIdx.x * 16 + x, columns = a.units * 8;
  float sum = 0.f;
  if (c < columns)
    for (int p = y; p < parts; p += 64) sum += a.partial[(int64_t)p * columns + c];
  lds[y][x] = sum;
  __syncthreads();
  for (int half = 32; half > 0; half >>= 1) {
    if (y < half) lds[y][x] += lds[y + half][x];
    __syncthreads();
  }
  if (y == 0 && c < columns) {
    for (int j = 0; j < a.P; ++j) {
      const NormWorker& w = norm_worker(a, j);
      const int col = c - w.unit0 * 8;
      if (col >= 0 && col < w.n) ((float*)w.y)[col] = lds[0][x];
    }
  }
}

}  // namespace distdl

struct distdl_rmsnorm_plan {
  int64_t rows = 0, n_f = 0;
  int P = 1;
  double eps = 0;
  distdl_dtype dtype = DISTDL_F32;
  std::vector<int32_t> unit0, size;
  int32_t units = 0;
  distdl::DevArray<distdl::NormWorker> table;
  distdl::StreamScratch partial;
};

namespace distdl {

// The launch of rows of `units`: threads of a row, units of a thread, wide or not.  A wave for each row needs no barrier; beyond two units a
// thread a row goes to four waves, which keeps more of them loading at once.
template <class F>
static void norm_shape(int units, F f) {
  if (units <= 64) f(std::integral_constant<int, 64>(), std::integral_constant<int, 1>(), std::false_type());
  else if (units <= 128) f(std::integral_constant<int, 64>(), std::integral_constant<int, 2>(), std::false_type());
  else if (units <= 256) f(std::integral_constant<int, 256>(), std::integral_constant<int, 1>(), std::false_type());
  else if (units <= 512) f(std::integral_constant<int, 256>(), std::integral_constant<int, 2>(), std::false_type());
  else if (units <= 1024) f(std::integral_constant<int, 256>(), std::integral_constant<int, 4>(), std::false_type());
  else f(std::integral_constant<int, 256>(), std::integral_constant<int, 4>(), std::true_type());
}

static int norm_args(distdl_rmsnorm_plan* p, const std::vector<NormWorker>& w, hipStream_t st, NormArgs* a) {
  a->more = nullptr;
  a->P = p->P;
  a->units = p->units;
  a->rows = p->rows;
  a->inv_n = (float)(1.0 / (double)p->n_f);
  a->eps = (float)p->eps;
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

template <class E>
static void launch_norm_fwd(const NormArgs& a, hipStream_t st) {
  norm_shape(a.units, [&](auto T, auto R, auto wide) {
    const int64_t groups = (a.rows + 256 / T - 1) / (256 / T);
    hipLaunchKernelGGL((norm_fwd_kernel<E, T, R, wide>), dim3((unsigned)groups), dim3(256), 0, st, a);
  });
}

template <class E>
static int launch_norm_bwd(distdl_rmsnorm_plan* p, NormArgs& a, hipStream_t st) {
  int rc = DISTDL_OK, parts = 0;
  norm_shape(a.units, [&](auto T, auto R, auto wide) {
    const int64_t groups = (a.rows + 256 / T - 1) / (256 / T);
    const int grid = (int)std::min<int64_t>(groups, 1024);
    parts = wide ? (int)std::min<int64_t>((a.rows + 3) / 4, 64) : grid;
    rc = p->partial.get((size_t)parts * a.units * 8, st, &a.partial);
    if (rc) return;
    hipLaunchKernelGGL((norm_bwd_kernel<E, T, R, wide>), dim3(wide ? (unsigned)std::min<int64_t>(groups, 4096) : (unsigned)grid),
                       dim3(256), 0, st, a);
    if (wide) hipLaunchKernelGGL((norm_dg_wide_kernel<E>), dim3((a.units + 63) / 64, parts), dim3(256), 0, st, a);
  });
  if (rc) return rc;
  hipLaunchKernelGGL(norm_dg_kernel, dim3((a.units * 8 + 15) / 16), dim3(1024), 0, st, a, parts);
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
      p->unit0.push_back(p->units);
      p->units += (p->size.back() + kBlock8 - 1) / kBlock8 * (kBlock8 / 8);
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
                        q_dev ? (uint8_t*)q_dev[j] : nullptr, q_dev ? (uint8_t*)qs_dev[j] : nullptr, p->unit0[j], p->size[j]};
    }
    if ((uintptr_t)rstd_dev % 4) return set_error(DISTDL_ERR_INVALID_ARG, "rmsnorm_fwd: rstd is not aligned to its elements");
    hipStream_t st_ = (hipStream_t)stream;
    NormArgs a;
    if ((rc = norm_args(p, w, st_, &a))) return rc;
    a.rstd = rstd_dev;
    {
      ProfScope prof("rmsnorm_fwd", st_);
      if (p->dtype == DISTDL_F32) launch_norm_fwd<float>(a, st_);
      else launch_norm_fwd<uint16_t>(a, st_);
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
                        p->unit0[j], p->size[j]};
    }
    if ((uintptr_t)rstd_dev % 4) return set_error(DISTDL_ERR_INVALID_ARG, "rmsnorm_bwd: rstd is not aligned to its elements");
    hipStream_t st_ = (hipStream_t)stream;
    NormArgs a;
    if ((rc = norm_args(p, w, st_, &a))) return rc;
    a.rstd = const_cast<float*>(rstd_dev);
    {
      ProfScope prof("rmsnorm_bwd", st_);
      if (p->rows == 0) hipLaunchKernelGGL(norm_dg_kernel, dim3((a.units * 8 + 15) / 16), dim3(1024), 0, st_, a, 0);  // (sums of nothing)
      else if ((rc = p->dtype == DISTDL_F32 ? launch_norm_bwd<float>(p, a, st_) : launch_norm_bwd<uint16_t>(p, a, st_))) return rc;
    }
    DISTDL_HIP_TRY(hipGetLastError());
    return DISTDL_OK;
  });
}

}  // extern "C"
