// Products of 8-bit operands with a scale for each block of 128 along the sum, over a P_fo x P_fi partition of the weights.
//
//   forward           y_i  = sum_j x_j W_ij^T          x in blocks of rows, W in tiles of 128 x 128
//   data gradient     dx_j = sum_i dy_i W_ij           dy in blocks of rows, the transposed W in tiles
//   weight gradient   dW_ij = dy_i^T x_j               the transposes of both in blocks of rows (along the batch)
//
// All three are C[m][n] = sum over segments and k of A[m][k] B[n][k] with k contiguous in both; a worker of the sum is a segment, whose
// blocks start anew.  Accumulators are fp32, fed by one of two matrix instructions:
//
//   v_mfma_scale_f32_16x16x128_f8f6f4 takes codes and scales as they are, at 5 PFLOP/s, but adds eight neighbouring products at a time in a
//   window: beside a product of 2^8 and 2^8, what lies below 2^3 is cut off (measured, each of the 127 other places; the
//   groups' sums and the accumulator keep all 24 bits).  A result is off by at most 2^-10 of the sum of the groups' largest products,
//   1.3e-5 of its size for N(0, 1) operands: 1/300 of a bf16 result's last place.  That is fewer bits than an fp32 sum has, and a choice:
//   each operand's rounding to codes puts a product off by up to 2^-4 of itself already.  Bf16 results whose cheapest tiles are the largest take it: 1.2 % of
//   those of 4096^3 differ from the rounded fp32 sum's (3.2 % where the numbers of a row differ by factors of exp(2 N(0, 1))), by one place, and both are equally far
//   (1.66e-3 of their size) from the unrounded sum.  A plan for fp32 results never takes it.
//
//   v_mfma_f32_16x16x32_bf16 takes codes times scales, which are exact in bf16 (an instruction converts two), at 2.5 PFLOP/s: sums of 128 to 8192
//   N(0, 1) products are 1e-8 to 3e-7 off.  Fp32 results take it (weight gradients among them), and products whose time
//   is not that of the matrix instructions.
//
// Measured (us a launch by the profiler, which counts its start and end, 2.5 for a launch of one workgroup): 8 x 4096 x 4096 7.2 (2.3 TB/s of weights; a launch
// and a trip to memory are most of it), 256 x 4096 x 4096 on 2 x 2 workers 18 (a pass among others 15), 8192 x 4096 x 4096 142 to 154 (1.8 to 1.9 PFLOP/s, 73 % of
// the library's 8192^3), the same in fp32 265 to 290 (0.95 to 1.02 PFLOP/s: conversions, of which a wave makes one for 2.7 products).
#include <algorithm>
#include <cstddef>
#include <map>
#include <tuple>

#include "block8.h"
#include "buffer.h"
#include "common.h"
#include "lds_direct.h"
#include "profile.h"

namespace distdl {

struct ProdSeg {  // one worker's part of a sum
  const uint8_t *a, *as, *b, *bs;
  int64_t k;
};
struct ProdOut {
  void* c;
  int32_t m, n;
  uint32_t tile0;       // its first workgroup
  uint32_t tiles_m;     // workgroups along m
  int32_t seg0, segs;
};
static_assert(sizeof(ProdOut) == 32 && sizeof(ProdSeg) == 40, "read from the launch's arguments as they lie there");
constexpr int kProdInline = 16;  // results and segments that travel with the launch; more are in a table
struct ProdArgs {
  ProdOut out[kProdInline];
  ProdSeg seg[4 * kProdInline];
  const ProdOut* more_out;
  const ProdSeg* more_seg;
  int32_t n_out;
};

typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));

// Eight codes times their scale, exactly: bf16's numbers go down to 2^-133, and what lies below in an operand is all that is rounded.  The instruction
// reads the exponent of `scale` alone.
__device__ __forceinline__ float scale_exponent(int byte) { return __uint_as_float((uint32_t)byte << 23); }
__device__ __forceinline__ v8bf codes_to_bf16(uint32_t lo, uint32_t hi, float scale) {
  union {
    v2bf p[4];
    v8bf v;
  } u;
  u.p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false);
  u.p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
  u.p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false);
  u.p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
  return u.v;
}

// Results and workers' parts of a sum, from the tables or from the launch's own arguments, read into scalar registers.  The addresses are taken
// in the kernel itself: the arguments' is not known in a function that the compiler might not inline.
struct ProdTables {
  const __attribute__((address_space(4))) ProdOut* outs;
  const __attribute__((address_space(4))) ProdSeg* segs;
  int n_out;
  __device__ __forceinline__ ProdOut out(int i) const {
    const auto p = outs + i;
    return ProdOut{p->c, p->m, p->n, p->tile0, p->tiles_m, p->seg0, p->segs};
  }
  __device__ __forceinline__ ProdSeg seg(int i) const {
    const auto p = segs + i;
    return ProdSeg{p->a, p->as, p->b, p->bs, p->k};
  }
  __device__ __forceinline__ ProdOut of(uint32_t block) const {  // the result that workgroup `block` belongs to
    int o = 0;
    while (o + 1 < n_out && block >= outs[o + 1].tile0) ++o;
    return out(o);
  }
};
static_assert(offsetof(ProdArgs, out) == 0, "the kernels' first argument starts with the results");
#define PROD_TABLES(args)                                                                                                  \
  ProdTables {                                                                                                             \
    (args).more_out ? (const __attribute__((address_space(4))) ProdOut*)(uint64_t)(args).more_out                          \
                    : (const __attribute__((address_space(4))) ProdOut*)__builtin_amdgcn_kernarg_segment_ptr(),            \
        (args).more_seg ? (const __attribute__((address_space(4))) ProdSeg*)(uint64_t)(args).more_seg                      \
                        : (const __attribute__((address_space(4))) ProdSeg*)((const __attribute__((address_space(4))) char*) \
                              __builtin_amdgcn_kernarg_segment_ptr() + offsetof(ProdArgs, seg)),                           \
        (args).n_out                                                                                                       \
  }

// 16 codes from k on of a row of n < 16, zeros behind its end
__device__ __forceinline__ u32x4 short_row(const uint8_t* row, int k, int n) {
  uint64_t lo = 0, hi = 0;
#pragma unroll 1
  for (int i = k; i < n; ++i) {
    const uint64_t c = row[i];
    if (i - k < 8) lo |= c << (8 * (i - k));
    else hi |= c << (8 * (i - k - 8));
  }
  return u32x4{(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)};
}
// 16 codes from k on of a row of n, zeros behind its end: one load, of the row's last 16 where it would pass the end, and a shift.
__device__ __forceinline__ u32x4 load16_codes(const uint8_t* row, int k, int n) {
  if (n < 16) return short_row(row, k, n);
  const int from = min(k, n - 16), skip = min(k - from, 16) * 8;  // bits that are another piece's
  const u32x4 c = *(const u32x4_any*)(row + from);
  uint64_t lo = (uint64_t)c[1] << 32 | c[0], hi = (uint64_t)c[3] << 32 | c[2];
  if (skip >= 64) {
    lo = skip < 128 ? hi >> (skip - 64) : 0;
    hi = 0;
  } else if (skip > 0) {
    lo = lo >> skip | hi << (64 - skip);
    hi >>= skip;
  }
  return u32x4{(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)};
}

// Four consecutive results of a row
__device__ __forceinline__ void prod_store(float* c, int m, int n, int cols, v4f v) {
  float* const to = c + (int64_t)m * cols + n;
  typedef v4f v4f_any __attribute__((aligned(4)));
  if (n + 3 < cols) {
    *(v4f_any*)to = v;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (n + e < cols) to[e] = v[e];
  }
}
__device__ __forceinline__ void prod_store(uint16_t* c, int m, int n, int cols, v4f v) {
  uint16_t* const to = c + (int64_t)m * cols + n;
  typedef u32x2 u32x2_two __attribute__((aligned(2)));
  if (n + 3 < cols) {
    *(u32x2_two*)to = u32x2{to_bf16(v[0], v[1]), to_bf16(v[2], v[3])};
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (n + e < cols) to[e] = to_bf16(v[e]);
  }
}

// Rows of any length and alignment to rows of whole 16-byte pieces, zeros behind their end: what tiles read where an operand's rows are
// neither.  One pass over the operands; the products of more than 64 rows that follow take several times as long.
struct ProdCopy {
  const uint8_t* from;
  u32x4* to;
  uint32_t n, pieces, total, block0;  // codes of a row; pieces of a row, of all rows; first workgroup
};
constexpr int kCopyInline = 32;
struct ProdCopies {
  ProdCopy c[kCopyInline];
  const ProdCopy* more;
  int32_t n;
};
__global__ __launch_bounds__(256) void prod8_pieces_kernel(ProdCopies args) {
  static_assert(offsetof(ProdCopies, c) == 0, "the kernel's first argument starts with the copies");
  typedef const __attribute__((address_space(4))) ProdCopy* Table;
  const Table table = args.more ? (Table)(uint64_t)args.more : (Table)__builtin_amdgcn_kernarg_segment_ptr();
  int i = 0;
  while (i + 1 < args.n && blockIdx.x >= table[i + 1].block0) ++i;
  const Table c = table + i;
  const uint32_t first = (blockIdx.x - c->block0) * 1024 + threadIdx.x;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const uint32_t at = first + 256 * k;
    if (at >= c->total) break;
    const uint32_t row = at / c->pieces, p = at - row * c->pieces;
    c->to[at] = load16_codes(c->from + (int64_t)row * c->n, (int)p * 16, (int)c->n);
  }
}

// Few rows of x (16 MI of them at most): reading the weights is all there is to do, once and as fast as memory gives them.  A workgroup takes 16
// rows of the weights, its eight waves every eighth block of k; operands go from memory to registers, U blocks of them under way
// at a time, and the waves' sums meet in LDS.  Rows of any length and alignment.
template <class C, bool B_TILES, int MI, int U>
__global__ __launch_bounds__(512) void prod8_rows_kernel(ProdArgs args) {
  __shared__ v4f meet[8][MI][64];
  const ProdTables tables = PROD_TABLES(args);
  const ProdOut out = tables.of(blockIdx.x);
  const int n0 = (int)(blockIdx.x - out.tile0) * 16;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r16 = lane & 15, g = lane >> 4;
  // (rows that are not there are others' once more: what comes of them is not stored)
  const int n = min(n0 + r16, out.n - 1);
  int m[MI];
#pragma unroll
  for (int i = 0; i < MI; ++i) m[i] = min(i * 16 + r16, out.m - 1);
  v4f acc[MI] = {};
  int total = 0, sg = 0, base = 0;  // blocks of all segments; the segment at hand and its first block
  for (int i = 0; i < out.segs; ++i) total += ((int)tables.seg(out.seg0 + i).k + 127) / 128;
  ProdSeg seg = tables.seg(out.seg0);
  int k = (int)seg.k, blocks = (k + 127) / 128;
  for (int t0 = wave; t0 < total; t0 += 8 * U) {
    u32x4 fb[U][2], fa[U][MI][2], mask[U][2];
    int sb[U], sa[U][MI];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (t0 + 8 * u >= total) break;
      while (t0 + 8 * u - base >= blocks) {
        base += blocks;
        seg = tables.seg(out.seg0 + ++sg);
        k = (int)seg.k;
        blocks = (k + 127) / 128;
      }
      const int kb = t0 + 8 * u - base;
      const uint8_t* const b = seg.b + (int64_t)n * k;
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        // A piece that passes the row's end is the row's last 16 codes, without those that are another piece's: in which place of
        // a product a k stands is the same for both operands, and no matter.
        const int at = kb * 128 + p * 64 + g * 16, from = min(at, k - 16), skip = (at - from) * 8;
#pragma unroll
        for (int d = 0; d < 4; ++d) mask[u][p][d] = skip >= 32 * d + 32 ? 0u : 0xFFFFFFFFu << max(0, skip - 32 * d);
        if (k >= 16) {
          fb[u][p] = *(const u32x4_any*)(b + from);
#pragma unroll
          for (int i = 0; i < MI; ++i) fa[u][i][p] = *(const u32x4_any*)(seg.a + (int64_t)m[i] * k + from);
        } else {
          mask[u][p] = u32x4{~0u, ~0u, ~0u, ~0u};
          fb[u][p] = short_row(b, at, k);
#pragma unroll
          for (int i = 0; i < MI; ++i) fa[u][i][p] = short_row(seg.a + (int64_t)m[i] * k, at, k);
        }
      }
      sb[u] = B_TILES ? seg.bs[(int64_t)(n >> 7) * blocks + kb] : seg.bs[(int64_t)kb * out.n + n];
#pragma unroll
      for (int i = 0; i < MI; ++i) sa[u][i] = seg.as[(int64_t)kb * out.m + m[i]];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (t0 + 8 * u >= total) break;
      const float f = scale_exponent(sb[u]);
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        const u32x4 b = fb[u][p] & mask[u][p];
        const v8bf b0 = codes_to_bf16(b[0], b[1], f), b1 = codes_to_bf16(b[2], b[3], f);
#pragma unroll
        for (int i = 0; i < MI; ++i) {
          const float e = scale_exponent(sa[u][i]);
          const u32x4 a = fa[u][i][p] & mask[u][p];
          acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b0, codes_to_bf16(a[0], a[1], e), acc[i], 0, 0, 0);
          acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b1, codes_to_bf16(a[2], a[3], e), acc[i], 0, 0, 0);
        }
      }
    }
  }
#pragma unroll
  for (int i = 0; i < MI; ++i) meet[wave][i][lane] = acc[i];
  __syncthreads();
  if (wave < MI) {
    v4f sum = meet[0][wave][lane];
#pragma unroll
    for (int w = 1; w < 8; ++w) sum += meet[w][wave][lane];
    if (wave * 16 + r16 < out.m) prod_store((C*)out.c, wave * 16 + r16, n0 + g * 4, out.n, sum);
  }
}

// Rows of whole 16-byte pieces.  TM x TN results a workgroup of WM x WN waves, 128 k a stage, ST stages in LDS.  Stages are filled by loads that go straight to LDS (no
// registers, no instructions to store them) while earlier ones are multiplied; a stage costs one barrier.  A wave's load brings eight
// rows of 128 bytes: lane L asks for piece (L & 7) ^ (L >> 3) of row L >> 3, so that row r's piece p lies at p ^ (r & 7) and the lanes
// that read together find different banks.  Rows and pieces that are not there fail the check of their buffer and arrive as zeros.
// The scales of the stage's rows come the same way, a byte to a word of LDS.
// FP8: the codes' own matrix instruction, else bf16 ones on codes that are converted as they leave LDS.  WK > 1: a stage is WK blocks
// of 128 k, each for a WK'th of the waves, which add up at the end.  What a wave does between two barriers is a
// chain (LDS, conversion, products), of which small tiles would have a short one on each SIMD otherwise.
template <class C, bool B_TILES, bool FP8, int TM, int TN, int WM, int WN, int WK, int ST>
__global__ __launch_bounds__(64 * WM * WN * WK) void prod8_tile_kernel(ProdArgs args) {
  constexpr int NW = WM * WN * WK, MI = TM / WM / 16, NI = TN / WN / 16;
  constexpr int kData = (TM + TN) * 128, kBlock = kData + (TM + TN) * 4, kStage = WK * kBlock;
  constexpr int kLoads = (TM + TN) / 8 / NW;                                            // a wave's loads of codes for a stage
  constexpr int kScales = ((TM + TN) / 64 + NW - 1) / NW;                               // and of scales (some twice, where waves are many)
  static_assert((TM + TN) / 8 % NW == 0 && TM % 64 == 0 && TN % 64 == 0, "whole loads");
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  const uint32_t block = xcd_order(blockIdx.x, gridDim.x);
  const ProdTables tables = PROD_TABLES(args);
  const ProdOut out = tables.of(block);
  const uint32_t tile = block - out.tile0, tiles_n = ((uint32_t)out.n + TN - 1) / TN;
  // eight rows of tiles are walked column by column: what an XCD works on at a time shares its operands in that XCD's L2
  const uint32_t band = tile / (8 * tiles_n), in_band = tile - band * 8 * tiles_n, high = min(8u, out.tiles_m - band * 8);
  const int m0 = (int)((band * 8 + in_band % high) * TM), n0 = (int)(in_band / high * TN);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave % WM * (TM / WM), wn = wave / WM % WN * (TN / WN), wk = wave / (WM * WN), r16 = lane & 15, g = lane >> 4;
  const uint32_t lds0 = lds_address(lds);

  // Loads.  A wave brings groups of eight rows wave, wave + NW, ... of A, then of B, and one or more runs of 64 scales.
  constexpr int kLoadsA = TM / 8 / NW;
  static_assert(TM / 8 % NW == 0 && TN / 8 % NW == 0, "the same loads for all waves");
  const int piece = ((lane & 7) ^ (lane >> 3)) * 16;
  int seg_i = -1, left = 0, rest = 0;  // the segment that is loaded; blocks of it that are not yet; k of its last block
  uint32_t at_k = 0, into = 0;         // first k of the next block; where it goes in LDS
  lds_u32x4 ra, rb, rs[kScales];
  uint32_t voff[kLoads], soff[kScales], at_s[kScales], hop[kScales];
  auto open = [&]() __attribute__((always_inline)) {                  // the buffers and offsets of the next segment
    const ProdSeg seg = tables.seg(out.seg0 + ++seg_i);
    const uint32_t k = (uint32_t)seg.k;
    left = (int)((k + 127) / 128);
    rest = (int)(k - (left - 1) * 128);
    at_k = 0;
    ra = lds_direct_rsrc(seg.a + (int64_t)m0 * k, (uint32_t)min((int64_t)0x7fffffe0, (int64_t)(out.m - m0) * k));
    rb = lds_direct_rsrc(seg.b + (int64_t)n0 * k, (uint32_t)min((int64_t)0x7fffffe0, (int64_t)(out.n - n0) * k));
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const bool is_a = i < kLoadsA;
      const int r = ((is_a ? i : i - kLoadsA) * NW + wave) * 8 + (lane >> 3);
      voff[i] = r < (is_a ? out.m - m0 : out.n - n0) ? (uint32_t)r * k + piece : kOob;
    }
#pragma unroll
    for (int i = 0; i < kScales; ++i) {
      const int l = (wave * kScales + i) % ((TM + TN) / 64);
      const bool is_a = l * 64 < TM;
      const int r = is_a ? m0 + l * 64 + lane : n0 + l * 64 - TM + lane;
      const uint32_t width = is_a ? out.m : B_TILES ? (out.n + 127) >> 7 : out.n;
      rs[i] = lds_direct_rsrc(is_a ? seg.as : seg.bs, left * width);
      if (is_a) soff[i] = r < out.m ? r : kOob;
      else soff[i] = r < out.n ? (B_TILES ? (uint32_t)(r >> 7) * left : r) : kOob;
      hop[i] = is_a ? out.m : B_TILES ? 1 : out.n;
      at_s[i] = 0;
    }
  };
  auto load = [&]() __attribute__((always_inline)) {                  // the next block to the next place; zeros behind the last one
    if (left == 0 && seg_i + 1 < out.segs) open();
    const bool gone = left <= 0 || (left == 1 && piece >= rest);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int l = i < kLoadsA ? i * NW + wave : TM / 8 + (i - kLoadsA) * NW + wave;
      load_to_lds(i < kLoadsA ? ra : rb, lds0 + into + l * 1024, gone ? kOob : voff[i], at_k);
    }
#pragma unroll
    for (int i = 0; i < kScales; ++i) {
      const int l = (wave * kScales + i) % ((TM + TN) / 64);
      load_byte_to_lds(rs[i], lds0 + into + kData + l * 256, left > 0 ? soff[i] : kOob, left > 0 ? at_s[i] : 0);
      at_s[i] += hop[i];
    }
    at_k = left > 1 ? at_k + 128 : 0;
    --left;
    into = into == ST * kStage - kBlock ? 0 : into + kBlock;
  };
  auto load_stage = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < WK; ++i) load();
  };
  int total = 0;
  for (int i = 0; i < out.segs; ++i) total += (int)((tables.seg(out.seg0 + i).k + 127) / 128);
  total = (total + WK - 1) / WK;

  v4f acc[NI][MI] = {};  // B's rows are the matrix instruction's rows, so that a lane holds four consecutive n of one m
#pragma unroll
  for (int i = 0; i < ST - 1; ++i)
    if (i < total) load_stage();
  uint32_t from = 0;
  const uint32_t at_a = (wm + r16) * 128, at_b = (TM + wn + r16) * 128, at_sa = kData + (wm + r16) * 4, at_sb = kData + (TM + wn + r16) * 4;
  const uint32_t p0 = (g ^ (r16 & 7)) * 16, p1 = ((g + 4) ^ (r16 & 7)) * 16;
  for (int s = 0; s < total; ++s) {
    if (total - 1 - s >= ST - 2) asm volatile("s_waitcnt vmcnt(%0)" ::"n"((ST - 2) * WK * (kLoads + kScales)) : "memory");
    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    lds_barrier();  // this stage is there for all waves, and all have read the one before it
    const char* const at = lds + from + wk * kBlock;
    from = from == (ST - 1) * kStage ? 0 : from + kStage;
    // The operands' reads first, then the next loads: the scalar work of those runs while LDS answers.
    int sa[MI], sb[NI];
#pragma unroll
    for (int i = 0; i < MI; ++i) sa[i] = *(const uint8_t*)(at + at_sa + i * 64);
#pragma unroll
    for (int j = 0; j < NI; ++j) sb[j] = *(const uint8_t*)(at + at_sb + j * 64);
    if constexpr (FP8) {
      auto both = [&](const char* p) __attribute__((always_inline)) {
        const u32x4 lo = *(const u32x4*)(p + p0), hi = *(const u32x4*)(p + p1);
        v8i f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          f[i] = (int)lo[i];
          f[i + 4] = (int)hi[i];
        }
        return f;
      };
      if (s + ST - 1 < total) load_stage();
      v8i fa[MI];
#pragma unroll
      for (int i = 0; i < MI; ++i) fa[i] = both(at + at_a + i * 2048);
#pragma unroll
      for (int j = 0; j < NI; ++j) {
        const v8i fb = both(at + at_b + j * 2048);
#pragma unroll
        for (int i = 0; i < MI; ++i)
          acc[j][i] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fb, fa[i], acc[j][i], 0, 0, 0, sb[j], 0, sa[i]);
      }
    } else {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t p = h ? p1 : p0;
        u32x4 ca[MI], cb[NI];
#pragma unroll
        for (int i = 0; i < MI; ++i) ca[i] = *(const u32x4*)(at + at_a + i * 2048 + p);
#pragma unroll
        for (int j = 0; j < NI; ++j) cb[j] = *(const u32x4*)(at + at_b + j * 2048 + p);
        if (h == 0 && s + ST - 1 < total) load_stage();
        v8bf fa[MI][2];
#pragma unroll
        for (int i = 0; i < MI; ++i) {
          const float f = scale_exponent(sa[i]);
          fa[i][0] = codes_to_bf16(ca[i][0], ca[i][1], f);
          fa[i][1] = codes_to_bf16(ca[i][2], ca[i][3], f);
        }
#pragma unroll
        for (int j = 0; j < NI; ++j) {
          const float f = scale_exponent(sb[j]);
          const v8bf b0 = codes_to_bf16(cb[j][0], cb[j][1], f), b1 = codes_to_bf16(cb[j][2], cb[j][3], f);
#pragma unroll
          for (int i = 0; i < MI; ++i) {
            acc[j][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b0, fa[i][0], acc[j][i], 0, 0, 0);
            acc[j][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b1, fa[i][1], acc[j][i], 0, 0, 0);
          }
        }
      }
    }
  }
  if constexpr (WK > 1) {
    static_assert((WK - 1) * TM * TN * 4 <= ST * kStage, "the other waves' sums fit where the stages were");
    v4f* const sums = (v4f*)lds + (wave % (WM * WN)) * (NI * MI * 64) + lane;
    lds_barrier();  // (no load is under way: the last stage was waited for)
    if (wk > 0) {
#pragma unroll
      for (int j = 0; j < NI; ++j)
#pragma unroll
        for (int i = 0; i < MI; ++i) sums[((wk - 1) * WM * WN * NI * MI + j * MI + i) * 64] = acc[j][i];
    }
    lds_barrier();
    if (wk > 0) return;
#pragma unroll
    for (int w = 0; w < WK - 1; ++w)
#pragma unroll
      for (int j = 0; j < NI; ++j)
#pragma unroll
        for (int i = 0; i < MI; ++i) acc[j][i] += sums[(w * WM * WN * NI * MI + j * MI + i) * 64];
  }
#pragma unroll
  for (int i = 0; i < MI; ++i) {
    const int m = m0 + wm + i * 16 + r16;
    if (m >= out.m) continue;
#pragma unroll
    for (int j = 0; j < NI; ++j) prod_store((C*)out.c, m, n0 + wn + j * 16 + g * 4, out.n, acc[j][i]);
  }
}

}  // namespace distdl

struct distdl_linear8_plan {
  int64_t n_b = 0, n_fi = 0, n_fo = 0;
  int P_fo = 1, P_fi = 1;
  distdl_dtype dtype = DISTDL_F32;
  std::vector<int64_t> fo, fi;  // features of each worker
  distdl::DevArray<distdl::ProdOut> outs;
  distdl::DevArray<distdl::ProdSeg> segs;
  distdl::DevArray<distdl::ProdCopy> copies;
  distdl::StreamScratch pieces;
};

namespace distdl {

static int prod_check(const void* v, size_t size, const char* what, int j) {
  if (!v) return set_error(DISTDL_ERR_NULL, "linear8: %s[%d] is null", what, j);
  if ((uintptr_t)v % size) return set_error(DISTDL_ERR_INVALID_ARG, "linear8: %s[%d] is not aligned to its elements", what, j);
  return DISTDL_OK;
}

// Tiles of TM x TN over all results: their first workgroups.  Returns the number of workgroups.
static int64_t prod_tiles(std::vector<ProdOut>& outs, int TM, int TN) {
  int64_t tiles = 0;
  for (ProdOut& o : outs) {
    o.tile0 = (uint32_t)std::min<int64_t>(tiles, UINT32_MAX);
    o.tiles_m = (uint32_t)((o.m + TM - 1) / TM);
    tiles += (int64_t)o.tiles_m * ((o.n + TN - 1) / TN);
  }
  return tiles;
}

// Makes the rows of all operands whole 16-byte pieces: those that are not are copied to the plan's scratch.
static int prod_pieces(distdl_linear8_plan* p, const std::vector<ProdOut>& outs, std::vector<ProdSeg>& segs, hipStream_t st) {
  // An operand of several results is copied once: its place in `copies`.  Operands may start at one address and differ in rows or their length
  // (a matrix and its first rows), so these belong to what is remembered.
  std::map<std::tuple<const void*, int64_t, int64_t>, size_t> seen;
  std::vector<ProdCopy> copies;
  std::vector<std::pair<const uint8_t**, size_t>> users;
  int64_t pieces = 0, blocks = 0;
  for (const ProdOut& o : outs)
    for (int i = o.seg0; i < o.seg0 + o.segs; ++i) {
      ProdSeg& g = segs[i];
      const int64_t wide = (g.k + 15) / 16;
      const struct {
        const uint8_t** p;
        int64_t rows;
      } sides[2] = {{&g.a, o.m}, {&g.b, o.n}};
      for (const auto& side : sides) {
        if (g.k % 16 == 0 && (uintptr_t)*side.p % 16 == 0) continue;
        const auto it = seen.emplace(std::make_tuple((const void*)*side.p, side.rows, g.k), copies.size());
        if (it.second) {
          const int64_t total = side.rows * wide;
          if (total >= int64_t(1) << 31 || (blocks += (total + 1023) / 1024) >= kMaxBlocks256) return set_error(DISTDL_ERR_UNSUPPORTED, "linear8: problem too large");
          copies.push_back(ProdCopy{*side.p, (u32x4*)(pieces * 16), (uint32_t)g.k, (uint32_t)wide, (uint32_t)total, (uint32_t)(blocks - (total + 1023) / 1024)});
          pieces += total;
        }
        users.emplace_back(side.p, it.first->second);
      }
    }
  for (ProdSeg& g : segs) g.k = (g.k + 15) / 16 * 16;
  if (copies.empty()) return DISTDL_OK;
  float* scratch = nullptr;
  int rc = p->pieces.get((size_t)pieces * 4, st, &scratch);
  if (rc) return rc;
  for (ProdCopy& c : copies) c.to = (u32x4*)((char*)scratch + (uintptr_t)c.to);
  for (const auto& u : users) *u.first = (const uint8_t*)copies[u.second].to;
  ProdCopies args;
  args.n = (int32_t)copies.size();
  args.more = nullptr;
  if (copies.size() <= (size_t)kCopyInline) {
    std::copy(copies.begin(), copies.end(), args.c);
  } else {
    if ((rc = p->copies.upload(copies, st))) return rc;
    args.more = p->copies.dev;
  }
  hipLaunchKernelGGL(prod8_pieces_kernel, dim3((unsigned)blocks), dim3(256), 0, st, args);
  return DISTDL_OK;
}

template <class C, bool B_TILES, bool FP8, int TM, int TN, int WM, int WN, int WK, int ST>
static int launch_prod_tile(const ProdArgs& args, int64_t tiles, hipStream_t st) {
  constexpr int bytes = ST * WK * (TM + TN) * 132;
  static_assert(bytes <= 160 * 1024, "LDS of a compute unit");
  const int rc = allow_large_lds<prod8_tile_kernel<C, B_TILES, FP8, TM, TN, WM, WN, WK, ST>>();
  if (rc) return rc;
  hipLaunchKernelGGL((prod8_tile_kernel<C, B_TILES, FP8, TM, TN, WM, WN, WK, ST>), dim3((unsigned)tiles), dim3(64 * WM * WN * WK), bytes, st, args);
  return DISTDL_OK;
}

template <class C, bool B_TILES>
static int launch_prod_as(ProdArgs& args, std::vector<ProdOut>& outs, std::vector<ProdSeg>& segs, distdl_linear8_plan* p, hipStream_t st) {
  enum { kRows, kSmall, kMiddle, kLarge } kind;
  int64_t tiles = 0, rows = 0, longest = 0;
  for (const ProdOut& o : outs) rows = std::max<int64_t>(rows, o.m);
  for (const ProdSeg& g : segs) longest = std::max<int64_t>(longest, g.k);
  if (rows <= 64) {
    kind = kRows;
    tiles = prod_tiles(outs, 64, 16);
  } else {
    // Offsets within a tile have 31 bits.
    if (longest > 1 << 24) return set_error(DISTDL_ERR_UNSUPPORTED, "linear8: a sum of %lld products for more than 64 rows", (long long)longest);
    const int rc = prod_pieces(p, outs, segs, st);
    if (rc) return rc;
    // What a round of 256 tiles takes for a block of k, in units of 0.05 us: measured at K = 2048 and 4096, 0.59 to 0.67 us for 64 x 64, 1.2 to 1.5
    // for 128 x 128, 1.9 for 256 x 256 on 8-bit instructions, 2.2 for 256 x 128 on bf16 ones.  (2048 x 4096 x 4096, 128 large
    // tiles: 61 us for 74 with 512 of 128 x 128; in fp32, 2048^3, 128 large tiles: 35 us for 24 with 256.)
    const int64_t small = prod_tiles(outs, 64, 64), middle = prod_tiles(outs, 128, 128), large = prod_tiles(outs, 256, sizeof(C) == 2 ? 256 : 128);
    const auto rounds = [](int64_t n) { return (n + 255) / 256; };
    const int64_t cost[3] = {rounds(small) * 13, rounds(middle) * 26, rounds(large) * (sizeof(C) == 2 ? 38 : 44)};
    kind = kLarge;
    if (cost[1] < cost[2]) kind = kMiddle;
    if (cost[0] < std::min(cost[1], cost[2]) || longest > 1 << 22) kind = kSmall;
    tiles = kind == kLarge ? large : kind == kMiddle ? prod_tiles(outs, 128, 128) : prod_tiles(outs, 64, 64);
  }
  if (tiles >= kMaxBlocks256 / 2) return set_error(DISTDL_ERR_UNSUPPORTED, "linear8: problem too large");
  args.n_out = (int32_t)outs.size();
  args.more_out = nullptr;
  args.more_seg = nullptr;
  if (outs.size() <= (size_t)kProdInline && segs.size() <= (size_t)(4 * kProdInline)) {
    std::copy(outs.begin(), outs.end(), args.out);
    std::copy(segs.begin(), segs.end(), args.seg);
  } else {
    int rc;
    if ((rc = p->outs.upload(outs, st)) || (rc = p->segs.upload(segs, st))) return rc;
    args.more_out = p->outs.dev;
    args.more_seg = p->segs.dev;
  }
  if (kind == kLarge) {
    if constexpr (sizeof(C) == 2) return launch_prod_tile<C, B_TILES, true, 256, 256, 2, 4, 1, 2>(args, tiles, st);
    else return launch_prod_tile<C, B_TILES, false, 256, 128, 4, 2, 1, 3>(args, tiles, st);
  }
  if (kind == kMiddle) return launch_prod_tile<C, B_TILES, false, 128, 128, 2, 2, 2, 2>(args, tiles, st);
  if (kind == kSmall) return launch_prod_tile<C, B_TILES, false, 64, 64, 1, 2, 4, 2>(args, tiles, st);
  const dim3 grid((unsigned)tiles);
  if (rows <= 16) hipLaunchKernelGGL((prod8_rows_kernel<C, B_TILES, 1, 4>), grid, dim3(512), 0, st, args);
  else if (rows <= 32) hipLaunchKernelGGL((prod8_rows_kernel<C, B_TILES, 2, 2>), grid, dim3(512), 0, st, args);
  else if (rows <= 48) hipLaunchKernelGGL((prod8_rows_kernel<C, B_TILES, 3, 2>), grid, dim3(512), 0, st, args);
  else hipLaunchKernelGGL((prod8_rows_kernel<C, B_TILES, 4, 2>), grid, dim3(512), 0, st, args);
  return DISTDL_OK;
}

static int launch_prod(distdl_linear8_plan* p, std::vector<ProdOut>& outs, std::vector<ProdSeg>& segs, bool f32, bool b_tiles,
                       const char* name, hipStream_t st) {
  ProdArgs args;
  int rc;
  {
    ProfScope prof(name, st);
    if (f32) rc = b_tiles ? launch_prod_as<float, true>(args, outs, segs, p, st) : launch_prod_as<float, false>(args, outs, segs, p, st);
    else rc = launch_prod_as<uint16_t, true>(args, outs, segs, p, st);
  }
  if (rc) return rc;
  DISTDL_HIP_TRY(hipGetLastError());
  return DISTDL_OK;
}

}  // namespace distdl

using namespace distdl;

extern "C" {

int distdl_linear8_plan_create(distdl_linear8_plan** out, int64_t n_b, int64_t n_fi, int64_t n_fo, int P_fo, int P_fi, distdl_dtype dtype) {
  if (!out) return set_error(DISTDL_ERR_NULL, "linear8_plan_create: null argument");
  *out = nullptr;
  if (n_b < 1 || n_fi < 1 || n_fo < 1 || P_fo < 1 || P_fi < 1)
    return set_error(DISTDL_ERR_INVALID_ARG, "linear8_plan_create: sizes must be >= 1");
  if (dtype != DISTDL_F32 && dtype != DISTDL_BF16) return set_error(DISTDL_ERR_UNSUPPORTED, "unknown dtype");
  if (n_fo < P_fo || n_fi < P_fi)
    return set_error(DISTDL_ERR_EMPTY_PARTITION, "linear8: %lld x %lld features over %d x %d workers", (long long)n_fo, (long long)n_fi, P_fo, P_fi);
  if (n_b >= int64_t(1) << 30 || n_fi >= int64_t(1) << 30 || n_fo >= int64_t(1) << 30 || (int64_t)P_fo * P_fi > 1 << 16)
    return set_error(DISTDL_ERR_UNSUPPORTED, "linear8: problem too large");
  return guarded([&]() -> int {
    std::unique_ptr<distdl_linear8_plan> p(new distdl_linear8_plan());
    p->n_b = n_b;
    p->n_fi = n_fi;
    p->n_fo = n_fo;
    p->P_fo = P_fo;
    p->P_fi = P_fi;
    p->dtype = dtype;
    for (int i = 0; i < P_fo; ++i) p->fo.push_back(n_fo / P_fo + (i < n_fo % P_fo ? 1 : 0));
    for (int j = 0; j < P_fi; ++j) p->fi.push_back(n_fi / P_fi + (j < n_fi % P_fi ? 1 : 0));
    *out = p.release();
    return DISTDL_OK;
  });
}

int distdl_linear8_plan_destroy(distdl_linear8_plan* p) {
  if (!p) return DISTDL_OK;
  p->outs.release();
  p->segs.release();
  p->copies.release();
  p->pieces.release();
  delete p;
  return DISTDL_OK;
}

int distdl_linear8_fwd(distdl_linear8_plan* p, const void* const xq_dev[], const void* const xs_dev[], const void* const wq_dev[],
                       const void* const ws_dev[], void* const y_dev[], void* stream) {
  if (!p || !xq_dev || !xs_dev || !wq_dev || !ws_dev || !y_dev) return set_error(DISTDL_ERR_NULL, "linear8_fwd: null argument");
  return guarded([&]() -> int {
    int rc;
    std::vector<ProdOut> outs;
    std::vector<ProdSeg> segs;
    for (int j = 0; j < p->P_fi; ++j)
      if ((rc = prod_check(xq_dev[j], 1, "xq", j)) || (rc = prod_check(xs_dev[j], 1, "xs", j))) return rc;
    for (int i = 0; i < p->P_fo; ++i) {
      if ((rc = prod_check(y_dev[i], dtype_size(p->dtype), "y", i))) return rc;
      outs.push_back(ProdOut{y_dev[i], (int32_t)p->n_b, (int32_t)p->fo[i], 0, 0, (int32_t)segs.size(), p->P_fi});
      for (int j = 0; j < p->P_fi; ++j) {
        const int w = i * p->P_fi + j;
        if ((rc = prod_check(wq_dev[w], 1, "wq", w)) || (rc = prod_check(ws_dev[w], 1, "ws", w))) return rc;
        segs.push_back(ProdSeg{(const uint8_t*)xq_dev[j], (const uint8_t*)xs_dev[j], (const uint8_t*)wq_dev[w], (const uint8_t*)ws_dev[w], p->fi[j]});
      }
    }
    return launch_prod(p, outs, segs, p->dtype == DISTDL_F32, true, "linear8_fwd", (hipStream_t)stream);
  });
}

int distdl_linear8_bwd_x(distdl_linear8_plan* p, const void* const dyq_dev[], const void* const dys_dev[], const void* const wtq_dev[],
                         const void* const wts_dev[], void* const dx_dev[], void* stream) {
  if (!p || !dyq_dev || !dys_dev || !wtq_dev || !wts_dev || !dx_dev) return set_error(DISTDL_ERR_NULL, "linear8_bwd_x: null argument");
  return guarded([&]() -> int {
    int rc;
    std::vector<ProdOut> outs;
    std::vector<ProdSeg> segs;
    for (int i = 0; i < p->P_fo; ++i)
      if ((rc = prod_check(dyq_dev[i], 1, "dyq", i)) || (rc = prod_check(dys_dev[i], 1, "dys", i))) return rc;
    for (int j = 0; j < p->P_fi; ++j) {
      if ((rc = prod_check(dx_dev[j], dtype_size(p->dtype), "dx", j))) return rc;
      outs.push_back(ProdOut{dx_dev[j], (int32_t)p->n_b, (int32_t)p->fi[j], 0, 0, (int32_t)segs.size(), p->P_fo});
      for (int i = 0; i < p->P_fo; ++i) {
        const int w = i * p->P_fi + j;
        if ((rc = prod_check(wtq_dev[w], 1, "wtq", w)) || (rc = prod_check(wts_dev[w], 1, "wts", w))) return rc;
        segs.push_back(ProdSeg{(const uint8_t*)dyq_dev[i], (const uint8_t*)dys_dev[i], (const uint8_t*)wtq_dev[w], (const uint8_t*)wts_dev[w], p->fo[i]});
      }
    }
    return launch_prod(p, outs, segs, p->dtype == DISTDL_F32, true, "linear8_bwd_x", (hipStream_t)stream);
  });
}

int distdl_linear8_bwd_w(distdl_linear8_plan* p, const void* const dytq_dev[], const void* const dyts_dev[], const void* const xtq_dev[],
                         const void* const xts_dev[], float* const dw_dev[], void* stream) {
  if (!p || !dytq_dev || !dyts_dev || !xtq_dev || !xts_dev || !dw_dev) return set_error(DISTDL_ERR_NULL, "linear8_bwd_w: null argument");
  return guarded([&]() -> int {
    int rc;
    std::vector<ProdOut> outs;
    std::vector<ProdSeg> segs;
    for (int j = 0; j < p->P_fi; ++j)
      if ((rc = prod_check(xtq_dev[j], 1, "xtq", j)) || (rc = prod_check(xts_dev[j], 1, "xts", j))) return rc;
    for (int i = 0; i < p->P_fo; ++i) {
      if ((rc = prod_check(dytq_dev[i], 1, "dytq", i)) || (rc = prod_check(dyts_dev[i], 1, "dyts", i))) return rc;
      for (int j = 0; j < p->P_fi; ++j) {
        const int w = i * p->P_fi + j;
        if ((rc = prod_check(dw_dev[w], 4, "dw", w))) return rc;
        outs.push_back(ProdOut{dw_dev[w], (int32_t)p->fo[i], (int32_t)p->fi[j], 0, 0, (int32_t)segs.size(), 1});
        segs.push_back(ProdSeg{(const uint8_t*)dytq_dev[i], (const uint8_t*)dyts_dev[i], (const uint8_t*)xtq_dev[j], (const uint8_t*)xts_dev[j], p->n_b});
      }
    }
    return launch_prod(p, outs, segs, true, false, "linear8_bwd_w", (hipStream_t)stream);
  });
}

}  // extern "C"
