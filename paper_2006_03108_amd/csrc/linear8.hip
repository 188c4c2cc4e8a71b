// Products of 8-bit operands with a scale for each block of 128 along the sum, over a P_fo x P_fi partition of the weights.
//
//   forward           y_i  = sum_j x_j W_ij^T          x in blocks of rows, W in tiles of 128 x 128
//   data gradient     dx_j = sum_i dy_i W_ij           dy in blocks of rows, the transposed W in tiles
//   weight gradient   dW_ij = dy_i^T x_j               the transposes of both in blocks of rows (along the batch)
//
// All three are C[m][n] = sum over segments and k of A[m][k] B[n][k] with k contiguous in both; a worker of the sum is a segment, whose
// blocks start anew.  Codes times scales are exact in bf16 (one instruction for two), so bf16 matrix instructions
// add exact products in fp32; measured, sums of 128 to 8192 products of N(0, 1) operands are 1e-8 to 3e-7 of their size off.
#include <algorithm>

#include "block8.h"
#include "common.h"
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
constexpr int kProdInline = 16;  // results and segments that travel with the launch; more are in a table
struct ProdArgs {
  ProdOut out[kProdInline];
  ProdSeg seg[4 * kProdInline];
  const ProdOut* more_out;
  const ProdSeg* more_seg;
  int32_t n_out;
};

typedef float v4f __attribute__((ext_vector_type(4)));
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));

// Eight codes times their scale, exactly (numbers below 2^-126 aside)
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

// 16 codes, those from n on zero
__device__ __forceinline__ u32x4 load16_codes(const uint8_t* p, int64_t n) {
  if (n >= 16) return *(const u32x4_any*)p;
  u32x4 c = {0u, 0u, 0u, 0u};
#pragma unroll
  for (int i = 0; i < 16; ++i)
    if (i < n) c[i >> 2] |= (uint32_t)p[i] << (8 * (i & 3));
  return c;
}

// Any sizes, strides of rows and alignment: 128 x 128 results a workgroup, 64 x 64 a wave, 128 k at a time through LDS.  The 16-byte
// piece p of row r lies at piece p ^ (r & 7), so that the eight rows that lanes read together lie in different banks.
template <class C, bool B_TILES>
__global__ __launch_bounds__(256) void prod8_any_kernel(ProdArgs args) {
  __shared__ u32x4 lds[2][kBlock8][8];
  int o = 0;
  while (o + 1 < args.n_out && blockIdx.x >= (args.more_out ? args.more_out[o + 1].tile0 : args.out[o + 1].tile0)) ++o;
  const ProdOut out = args.more_out ? args.more_out[o] : args.out[o];
  const uint32_t tile = blockIdx.x - out.tile0;
  const int m0 = (int)(tile % out.tiles_m) * 128, n0 = (int)(tile / out.tiles_m) * 128;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int wm = (wave & 1) * 64, wn = (wave >> 1) * 64, r16 = lane & 15, g = lane >> 4;
  v4f acc[4][4] = {};  // [n][m]: B's rows are the matrix instruction's rows, so that a lane holds four consecutive n of one m
  for (int sg = 0; sg < out.segs; ++sg) {
    const ProdSeg seg = args.more_seg ? args.more_seg[out.seg0 + sg] : args.seg[out.seg0 + sg];
    const int64_t blocks = (seg.k + kBlock8 - 1) / kBlock8;
    for (int64_t kb = 0; kb < blocks; ++kb) {
      u32x4 ra[4], rb[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = i * 32 + (threadIdx.x >> 3), p = threadIdx.x & 7;
        const int64_t k = kb * kBlock8 + p * 16;
        ra[i] = load16_codes(seg.a + (m0 + r) * seg.k + k, m0 + r < out.m ? seg.k - k : 0);
        rb[i] = load16_codes(seg.b + (n0 + r) * seg.k + k, n0 + r < out.n ? seg.k - k : 0);
      }
      int sa[4], sb[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int64_t m = min(m0 + wm + i * 16 + r16, out.m - 1), n = min(n0 + wn + i * 16 + r16, out.n - 1);
        sa[i] = seg.as[kb * out.m + m];
        sb[i] = B_TILES ? seg.bs[(n >> 7) * blocks + kb] : seg.bs[kb * out.n + n];
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = i * 32 + (threadIdx.x >> 3), p = threadIdx.x & 7;
        lds[0][r][p ^ (r & 7)] = ra[i];
        lds[1][r][p ^ (r & 7)] = rb[i];
      }
      __syncthreads();
      auto piece = [&](int side, int row, int p) { return lds[side][row][(g + 4 * p) ^ (row & 7)]; };
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        v8bf fa[4][2];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const u32x4 c = piece(0, wm + i * 16 + r16, p);
          const float s = scale_value(sa[i]);
          fa[i][0] = codes_to_bf16(c[0], c[1], s);
          fa[i][1] = codes_to_bf16(c[2], c[3], s);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const u32x4 c = piece(1, wn + j * 16 + r16, p);
          const float s = scale_value(sb[j]);
          const v8bf b0 = codes_to_bf16(c[0], c[1], s), b1 = codes_to_bf16(c[2], c[3], s);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            acc[j][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b0, fa[i][0], acc[j][i], 0, 0, 0);
            acc[j][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b1, fa[i][1], acc[j][i], 0, 0, 0);
          }
        }
      }
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int m = m0 + wm + i * 16 + r16;
    if (m >= out.m) continue;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int n = n0 + wn + j * 16 + g * 4;
      C* const to = (C*)out.c + (int64_t)m * out.n + n;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (n + e < out.n) st(to, e, acc[j][i][e]);
    }
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
};

namespace distdl {

static int prod_check(const void* v, size_t size, const char* what, int j) {
  if (!v) return set_error(DISTDL_ERR_NULL, "linear8: %s[%d] is null", what, j);
  if ((uintptr_t)v % size) return set_error(DISTDL_ERR_INVALID_ARG, "linear8: %s[%d] is not aligned to its elements", what, j);
  return DISTDL_OK;
}

static int launch_prod(distdl_linear8_plan* p, std::vector<ProdOut>& outs, const std::vector<ProdSeg>& segs, bool f32, bool b_tiles,
                       const char* name, hipStream_t st) {
  int64_t tiles = 0;
  for (ProdOut& o : outs) {
    o.tile0 = (uint32_t)tiles;
    o.tiles_m = (uint32_t)((o.m + 127) / 128);
    tiles += (int64_t)o.tiles_m * ((o.n + 127) / 128);
  }
  if (tiles >= kMaxBlocks256) return set_error(DISTDL_ERR_UNSUPPORTED, "linear8: problem too large");
  ProdArgs args;
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
  {
    ProfScope prof(name, st);
    const dim3 grid((unsigned)tiles), block(256);
    if (f32) {
      if (b_tiles) hipLaunchKernelGGL((prod8_any_kernel<float, true>), grid, block, 0, st, args);
      else hipLaunchKernelGGL((prod8_any_kernel<float, false>), grid, block, 0, st, args);
    } else {
      if (b_tiles) hipLaunchKernelGGL((prod8_any_kernel<uint16_t, true>), grid, block, 0, st, args);
      else hipLaunchKernelGGL((prod8_any_kernel<uint16_t, false>), grid, block, 0, st, args);
    }
  }
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
