// Matrices to 8-bit blocks: rows, columns (transposed), or tiles of 128 x 128 in both orders.
//
// One pass, bound by memory: every element is read once, and one or two bytes are written for it.  A workgroup takes a tile of 128 x 128; a
// thread holds 8 x 8 of it, so that a row's block lies in 16 lanes (a DPP row) and a column's in all sixteen rows of
// threads, whose magnitudes meet in LDS.  A thread's 8 x 8 codes are turned in registers and go through LDS, so that both orders
// are written in runs of a whole block.
//
// Measured: 8192 x 4096 bf16 to codes in both orders 31 us (4.3 TB/s), to the transposed ones alone 33 (3.0 TB/s), of an array that other work has put out of the
// caches; the same array again and again 27, 21 (rows alone 21).  4096 x 4096 fp32 in tiles, both orders, again and again 17.  145 registers for blocks of rows leave three
// waves to a SIMD, and a call for one order holds both orders' maxima.  A thread with half the elements, 512 to a
// workgroup: 48 us.  Neighbouring tiles on one XCD: 36 us for 33.
#include <algorithm>
#include <cstddef>

#include "block8.h"
#include "common.h"
#include "profile.h"

namespace distdl {

struct QuantArray {
  const void* x;
  uint8_t *q, *s, *qt, *st;  // codes and scales, and those of the transpose; either pair may be null
  int64_t rows, cols;
  uint32_t tile0, tiles_c;   // first workgroup; tiles side by side
};

// The arrays travel with the launch; more of them take several launches.  A table on the device would have to belong to someone: this call has
// no plan, and may be made by several threads, recorded, and made again with other arrays, without end.  Up to 16 arrays take 1 KiB of arguments,
// more of them launches with 3 KiB (us, 1 array 8.5 and 8.7; 40 arrays 57 and 52.5, as with a table).
template <int N>
struct QuantArgs {
  QuantArray a[N];
  int32_t n;
};
// The arguments' address is taken in the kernel itself, and the records are read as constants, into scalar registers.
static_assert(offsetof(QuantArgs<16>, a) == 0, "the kernel's first argument starts with the arrays");
typedef const __attribute__((address_space(4))) QuantArray* QuantTable;

// TILES: one scale for the tile.  Otherwise each order has blocks of its own.
template <class E, bool TILES, int N>
__global__ __launch_bounds__(256) void quant8_kernel(QuantArgs<N> args) {
  __shared__ float meet[4][kBlock8];
  // column c's 16-byte piece p lies at p ^ ((c >> 3) & 7): the lanes of a wave write eight columns apart
  __shared__ alignas(16) uint8_t turned[kBlock8][kBlock8];
  const QuantTable table = (QuantTable)__builtin_amdgcn_kernarg_segment_ptr();
  int i = 0;
  while (i + 1 < args.n && blockIdx.x >= table[i + 1].tile0) ++i;
  const QuantTable t = table + i;
  const QuantArray m{t->x, t->q, t->s, t->qt, t->st, t->rows, t->cols, t->tile0, t->tiles_c};
  const uint32_t tile = blockIdx.x - m.tile0;
  const int64_t r0 = (int64_t)(tile / m.tiles_c) * kBlock8, c0 = (int64_t)(tile % m.tiles_c) * kBlock8;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t row = r0 + ty * 8, col = c0 + tx * 8;
  const int n = (int)max((int64_t)0, min((int64_t)8, m.cols - col));
  float v[8][8];
  {
    Eight<E> x[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k].load((const E*)m.x + (row + k) * m.cols + col, row + k < m.rows ? n : 0);
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k].values(v[k]);
  }
  float rmax[8], cmax[8] = {};
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    float mx = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      mx = fmaxf(mx, fabsf(v[k][j]));
      cmax[j] = fmaxf(cmax[j], fabsf(v[k][j]));
    }
    rmax[k] = row16_max(mx);
  }
  // columns: over the four rows of lanes of a wave, then over the waves
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    cmax[j] = fmaxf(cmax[j], __shfl_xor(cmax[j], 16, 64));
    cmax[j] = fmaxf(cmax[j], __shfl_xor(cmax[j], 32, 64));
    if (lane < 16) meet[wave][tx * 8 + j] = cmax[j];
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < 8; ++j)
    cmax[j] = fmaxf(fmaxf(meet[0][tx * 8 + j], meet[1][tx * 8 + j]), fmaxf(meet[2][tx * 8 + j], meet[3][tx * 8 + j]));
  if (TILES) {
    float all = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) all = fmaxf(all, cmax[j]);
    all = row16_max(all);
#pragma unroll
    for (int k = 0; k < 8; ++k) rmax[k] = cmax[k] = all;
  }
  if (m.q) {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int byte = scale_byte(rmax[k]);
      const float inv = scale_inverse(byte);
      if (row + k < m.rows && n > 0) {
        store8_codes(m.q + (row + k) * m.cols + col,
                     u32x2{pack_e4m3(v[k][0] * inv, v[k][1] * inv, v[k][2] * inv, v[k][3] * inv),
                           pack_e4m3(v[k][4] * inv, v[k][5] * inv, v[k][6] * inv, v[k][7] * inv)}, n);
        if (!TILES && tx == 0) m.s[(c0 >> 7) * m.rows + row + k] = (uint8_t)byte;
      }
      if (TILES && threadIdx.x == 0 && k == 0) m.s[tile] = (uint8_t)byte;
    }
  }
  if (m.qt) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int byte = scale_byte(cmax[j]);
      const float inv = scale_inverse(byte);
      *(u32x2*)&turned[tx * 8 + j][((ty >> 1) ^ (tx & 7)) * 16 + (ty & 1) * 8] = u32x2{pack_e4m3(v[0][j] * inv, v[1][j] * inv, v[2][j] * inv, v[3][j] * inv),
                                                   pack_e4m3(v[4][j] * inv, v[5][j] * inv, v[6][j] * inv, v[7][j] * inv)};
      if (!TILES && ty == 0 && j < n) m.st[(r0 >> 7) * m.cols + col + j] = (uint8_t)byte;
      if (TILES && threadIdx.x == 0 && j == 0) m.st[(c0 >> 7) * ((m.rows + kBlock8 - 1) >> 7) + (r0 >> 7)] = (uint8_t)byte;
    }
    __syncthreads();
    // eight lanes write a column's 128 codes
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int c = (threadIdx.x >> 3) + 32 * k, piece = (threadIdx.x & 7) * 16;
      const uint8_t* const from = &turned[c][piece ^ ((c >> 3) & 7) * 16];
      if (c0 + c >= m.cols) continue;
      const int left = (int)max((int64_t)0, min((int64_t)16, m.rows - r0 - piece));
      uint8_t* to = m.qt + (c0 + c) * m.rows + r0 + piece;
      if (left == 16) {
        *(u32x4_any*)to = *(const u32x4*)from;
      } else {
        for (int b = 0; b < left; ++b) to[b] = from[b];
      }
    }
  }
}

template <int N>
static int launch_quant(const std::vector<QuantArray>& a, int64_t all_tiles, bool tiles, distdl_dtype dtype, hipStream_t st) {
  for (size_t first = 0; first < a.size(); first += N) {
    QuantArgs<N> args;
    args.n = (int32_t)std::min(a.size() - first, (size_t)N);
    const uint32_t tile0 = a[first].tile0;
    const int64_t end = first + args.n < a.size() ? a[first + args.n].tile0 : all_tiles;
    for (int i = 0; i < args.n; ++i) {
      args.a[i] = a[first + i];
      args.a[i].tile0 -= tile0;
    }
    const dim3 grid((unsigned)(end - tile0)), block(256);
    if (dtype == DISTDL_F32) {
      if (tiles) hipLaunchKernelGGL((quant8_kernel<float, true, N>), grid, block, 0, st, args);
      else hipLaunchKernelGGL((quant8_kernel<float, false, N>), grid, block, 0, st, args);
    } else {
      if (tiles) hipLaunchKernelGGL((quant8_kernel<uint16_t, true, N>), grid, block, 0, st, args);
      else hipLaunchKernelGGL((quant8_kernel<uint16_t, false, N>), grid, block, 0, st, args);
    }
    DISTDL_HIP_TRY(hipGetLastError());
  }
  return DISTDL_OK;
}

}  // namespace distdl

using namespace distdl;

extern "C" int distdl_quant8(const void* const x_dev[], const int64_t rows[], const int64_t cols[], int n_arrays, int tiles,
                             void* const q_dev[], void* const s_dev[], void* const qt_dev[], void* const st_dev[], distdl_dtype dtype,
                             void* stream) {
  if (!x_dev || !rows || !cols) return set_error(DISTDL_ERR_NULL, "quant8: null argument");
  if ((q_dev == nullptr) != (s_dev == nullptr) || (qt_dev == nullptr) != (st_dev == nullptr))
    return set_error(DISTDL_ERR_NULL, "quant8: codes without scales, or scales without codes");
  if (!q_dev && !qt_dev) return set_error(DISTDL_ERR_NULL, "quant8: no output");
  if (n_arrays < 1) return set_error(DISTDL_ERR_INVALID_ARG, "quant8: %d arrays", n_arrays);
  if (dtype != DISTDL_F32 && dtype != DISTDL_BF16) return set_error(DISTDL_ERR_UNSUPPORTED, "unknown dtype");
  return guarded([&]() -> int {
    std::vector<QuantArray> a;
    int64_t at = 0;
    for (int i = 0; i < n_arrays; ++i) {
      if (rows[i] < 0 || cols[i] < 0) return set_error(DISTDL_ERR_INVALID_ARG, "quant8: array %d is %lld x %lld", i, (long long)rows[i], (long long)cols[i]);
      if (rows[i] == 0 || cols[i] == 0) continue;
      if (rows[i] > int64_t(1) << 32 || cols[i] > int64_t(1) << 32) return set_error(DISTDL_ERR_UNSUPPORTED, "quant8: array %d is too large", i);
      if (!x_dev[i] || (q_dev && (!q_dev[i] || !s_dev[i])) || (qt_dev && (!qt_dev[i] || !st_dev[i])))
        return set_error(DISTDL_ERR_NULL, "quant8: array %d is null", i);
      if ((uintptr_t)x_dev[i] % dtype_size(dtype)) return set_error(DISTDL_ERR_INVALID_ARG, "quant8: array %d is not aligned to its elements", i);
      const int64_t tr = (rows[i] + kBlock8 - 1) / kBlock8, tc = (cols[i] + kBlock8 - 1) / kBlock8;
      a.push_back(QuantArray{x_dev[i], q_dev ? (uint8_t*)q_dev[i] : nullptr, q_dev ? (uint8_t*)s_dev[i] : nullptr,
                             qt_dev ? (uint8_t*)qt_dev[i] : nullptr, qt_dev ? (uint8_t*)st_dev[i] : nullptr, rows[i], cols[i], (uint32_t)at, (uint32_t)tc});
      if (tr >= kMaxBlocks256 || tc >= kMaxBlocks256 || (at += tr * tc) >= kMaxBlocks256)
        return set_error(DISTDL_ERR_UNSUPPORTED, "quant8: too many elements");
    }
    if (a.empty()) return DISTDL_OK;
    hipStream_t st_ = (hipStream_t)stream;
    ProfScope prof("quant8", st_);
    return a.size() <= 16 ? launch_quant<16>(a, at, tiles != 0, dtype, st_) : launch_quant<48>(a, at, tiles != 0, dtype, st_);
  });
}
