// The update of many arrays at once: AdamW (decoupled weight decay) with moments in 32 bits or in 8.
//
//   g' = g * gscale;  m = b1 m + (1 - b1) g';  v = b2 v + (1 - b2) g'^2
//   p  = p (1 - lr wd) - lr / (1 - b1^t) * m / (sqrt(v) / sqrt(1 - b2^t) + eps)
//
// One pass: every number is read and written once, 16 bytes an element with 8-bit moments and a 32-bit gradient, 28 with 32-bit ones, so
// memory bounds it.  A workgroup takes consecutive elements of one array, from a table that a stream's first call makes; a thread takes
// eight at a time, so that 16 lanes (one DPP row) hold a block of 128 and its scales need no LDS.  Measured: 168 million weights, bf16
// gradients, 8-bit moments and bf16 copies 509 to 565 us (4.8 to 5.3 TB/s); 67 million with fp32 moments and copies 348 us (5.4 TB/s).  A thread
// has eight elements of fp32 moments (twice as many: 361 us) and sixteen of 8-bit ones (half as many: 550 us, twice: 603).
//
// 8-bit moments: m and r = sqrt(v) as e4m3 codes (r, since v has twice the range), rounded up or down at random with the
// remainder's probability.  Rounded to nearest a moving average with b2 = 0.999 would never move: a step changes r by 0.05 %, half
// a unit of e4m3 is 3 to 6 %.  r > 0 is never rounded to zero, which would divide m by eps.  The
// random bits are a hash of the seed, the step and the element's place, so a call repeats to the bit.
//
// Products and sums are not contracted into fused ones: the update is the same, to the bit, as that of the formula's operations one by one.
#include <algorithm>
#include <cfloat>
#include <cmath>

#include "block8.h"
#include "common.h"
#include "profile.h"

#pragma clang fp contract(off)

namespace distdl {

constexpr int adam_chunk(bool s8) { return s8 ? 4096 : 2048; }  // elements of a workgroup of 256 threads

struct AdamChunk {
  uint32_t array, chunk;
};

struct AdamArray {  // what a launch needs of one array
  float* p;
  const void* g;
  void *m, *v;
  uint8_t *ms, *vs;
  uint16_t* copy;
  int64_t count;
  uint32_t place;  // of its first element in the hash: the arrays lie one behind the other, each at a multiple of 128
  uint32_t chunk0;  // its first workgroup
};

struct AdamArgs {
  float beta1, keep1, beta2, keep2;  // keep: 1 - beta
  float decay, rate, grow, eps;      // 1 - lr wd; lr / (1 - b1^t); 1 / sqrt(1 - b2^t)
  uint32_t key;
  double lr, b1, b2;                 // for a step that is read on the device
  uint32_t seed;
  const int64_t* step;
  const float* gscale;
};

// What each workgroup takes: the last array whose first workgroup is not behind it (those of no elements come before the array that is at their place).
__global__ __launch_bounds__(256) void adamw_chunks_kernel(AdamChunk* __restrict__ chunks, uint32_t n_chunks, const AdamArray* __restrict__ arrays,
                                                           uint32_t n_arrays) {
  const uint32_t c = blockIdx.x * 256 + threadIdx.x;
  if (c >= n_chunks) return;
  uint32_t lo = 0, hi = n_arrays;  // arrays[lo].chunk0 <= c < arrays[hi].chunk0
  while (hi - lo > 1) {
    const uint32_t mid = (lo + hi) / 2;
    if (arrays[mid].chunk0 <= c) lo = mid;
    else hi = mid;
  }
  chunks[c] = AdamChunk{lo, c - arrays[lo].chunk0};
}

// (the multipliers are 2^32 over the golden ratio and the fractions of sqrt(2) and sqrt(3))
__device__ __forceinline__ uint32_t adam_noise(uint32_t place, uint32_t key) {
  uint32_t x = place * 0x9E3779B1u + key;
  x = (x ^ (x >> 15)) * 0x6A09E667u;
  x = (x ^ (x >> 13)) * 0xBB67AE85u;
  return x ^ (x >> 16);
}

// y (a code's worth of at most 448) to a number that e4m3 holds: up with the probability of the remainder, of which the
// upper 16 of 20 bits count.  Below 2^-6 codes are as far apart as just above it, so that is where the rounding is done.
__device__ __forceinline__ float rounded_at_random(float y, uint32_t noise16) {
  const float size = fabsf(y);
  const bool small = size < kCodeNormal;
  float t = small ? size + kCodeNormal : size;
  t = __uint_as_float((__float_as_uint(t) + (noise16 << 4)) & ~0xFFFFFu);
  return copysignf(small ? t - kCodeNormal : t, y);
}

template <bool G16, bool S8>
__global__ __launch_bounds__(256) void adamw_kernel(const AdamChunk* __restrict__ chunks, const AdamArray* __restrict__ arrays,
                                                    AdamArgs s) {
  const AdamChunk ch = chunks[blockIdx.x];
  const AdamArray a = arrays[ch.array];
  const float gscale = s.gscale ? *s.gscale : 1.f;
  if (s.step) {  // the step's number on the device: its factors once a workgroup
    __shared__ float factor[2];
    __shared__ uint32_t key;
    if (threadIdx.x == 0) {
      const int64_t t = *s.step;
      factor[0] = (float)(s.lr / (1.0 - pow(s.b1, (double)t)));
      factor[1] = (float)(1.0 / sqrt(1.0 - pow(s.b2, (double)t)));
      key = s.seed * 0x6A09E667u + (uint32_t)t * 0xBB67AE85u;
    }
    __syncthreads();
    s.rate = factor[0];
    s.grow = factor[1];
    s.key = key;
  }
  constexpr int kChunk = adam_chunk(S8), kTimes = kChunk / 2048;
  typedef typename std::conditional<G16, uint16_t, float>::type G;
  Eight<float> p[kTimes], m[kTimes], v[kTimes];
  Eight<G> g[kTimes];
  u32x2 m8[kTimes], v8[kTimes];
  int mb[kTimes], vb[kTimes];
  const int64_t first = (int64_t)ch.chunk * kChunk + threadIdx.x * 8;
#pragma unroll
  for (int k = 0; k < kTimes; ++k) {  // all loads before the first use
    const int64_t at = first + k * 2048;
    const int n = (int)max((int64_t)0, min((int64_t)8, a.count - at));
    g[k].load((const G*)a.g + at, n);
    p[k].load(a.p + at, n);
    if constexpr (S8) {
      m8[k] = load8_codes((const uint8_t*)a.m + at, n);
      v8[k] = load8_codes((const uint8_t*)a.v + at, n);
      mb[k] = n > 0 ? a.ms[at >> 7] : 1;
      vb[k] = n > 0 ? a.vs[at >> 7] : 1;
    } else {
      m[k].load((const float*)a.m + at, n);
      v[k].load((const float*)a.v + at, n);
    }
  }
#pragma unroll
  for (int k = 0; k < kTimes; ++k) {
    const int64_t at = first + k * 2048;
    const int n = (int)max((int64_t)0, min((int64_t)8, a.count - at));
    float pv[8], gv[8], mv[8], vv[8];
    p[k].values(pv);
    g[k].values(gv);
    if constexpr (S8) {
      unpack_e4m3(m8[k][0], mv);
      unpack_e4m3(m8[k][1], mv + 4);
      unpack_e4m3(v8[k][0], vv);
      unpack_e4m3(v8[k][1], vv + 4);
      const float ms = scale_value(mb[k]), vs = scale_value(vb[k]);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        mv[i] *= ms;
        const float r = vv[i] * vs;
        vv[i] = r * r;
      }
    } else {
      m[k].values(mv);
      v[k].values(vv);
    }
    float mmax = 0.f, rmax = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float gi = gv[i] * gscale;
      mv[i] = mv[i] * s.beta1 + gi * s.keep1;
      vv[i] = vv[i] * s.beta2 + gi * gi * s.keep2;
      const float root = sqrtf(vv[i]);
      pv[i] = pv[i] * s.decay - mv[i] / (root * s.grow + s.eps) * s.rate;
      if constexpr (S8) {
        vv[i] = root;
        mmax = fmaxf(mmax, fabsf(mv[i]));
        rmax = fmaxf(rmax, root);
      }
    }
    if (n > 0) {
      store8(a.p + at, pv, n);
      if (a.copy) store8(a.copy + at, pv, n);
      if constexpr (!S8) {
        store8((float*)a.m + at, mv, n);
        store8((float*)a.v + at, vv, n);
      }
    }
    if constexpr (S8) {
      const int mb1 = scale_byte(row16_max(mmax)), vb1 = scale_byte(row16_max(rmax));
      const float mi = scale_inverse(mb1), vi = scale_inverse(vb1);
      const uint32_t place = a.place + (uint32_t)at;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint32_t r = adam_noise(place + i, s.key);
        mv[i] = rounded_at_random(mv[i] * mi, r >> 16);
        const float q = vv[i] * vi;
        vv[i] = rounded_at_random(q, r & 0xFFFFu);
        if (q > 0.f) vv[i] = fmaxf(vv[i], kCodeMin);
      }
      if (n > 0) {
        store8_codes((uint8_t*)a.m + at, u32x2{pack_e4m3(mv[0], mv[1], mv[2], mv[3]), pack_e4m3(mv[4], mv[5], mv[6], mv[7])}, n);
        store8_codes((uint8_t*)a.v + at, u32x2{pack_e4m3(vv[0], vv[1], vv[2], vv[3]), pack_e4m3(vv[4], vv[5], vv[6], vv[7])}, n);
        if ((threadIdx.x & 15) == 0) {
          a.ms[at >> 7] = (uint8_t)mb1;
          a.vs[at >> 7] = (uint8_t)vb1;
        }
      }
    }
  }
}

}  // namespace distdl

struct distdl_adamw_plan {
  std::vector<int64_t> count;
  std::vector<uint32_t> place, chunk0;
  bool g16 = false, s8 = false;
  int64_t n_chunks = 0;
  distdl::StreamScratch chunks;
  distdl::DevArray<distdl::AdamArray> arrays;
};

using namespace distdl;

extern "C" {

int distdl_adamw_plan_create(distdl_adamw_plan** out, const int64_t count[], int n_arrays, distdl_dtype g_dtype, int states8) {
  if (!out) return set_error(DISTDL_ERR_NULL, "adamw_plan_create: null argument");
  *out = nullptr;
  if (!count) return set_error(DISTDL_ERR_NULL, "adamw_plan_create: null argument");
  if (n_arrays < 1) return set_error(DISTDL_ERR_INVALID_ARG, "adamw_plan_create: %d arrays", n_arrays);
  if (g_dtype != DISTDL_F32 && g_dtype != DISTDL_BF16) return set_error(DISTDL_ERR_UNSUPPORTED, "unknown dtype");
  const int size = adam_chunk(states8 != 0);
  int64_t chunks = 0;
  for (int i = 0; i < n_arrays; ++i) {
    if (count[i] < 0) return set_error(DISTDL_ERR_INVALID_ARG, "adamw_plan_create: array %d has %lld elements", i, (long long)count[i]);
    if (count[i] > int64_t(1) << 40) return set_error(DISTDL_ERR_UNSUPPORTED, "adamw_plan_create: array %d is too large", i);
    chunks += (count[i] + size - 1) / size;
    if (chunks >= kMaxBlocks256) return set_error(DISTDL_ERR_UNSUPPORTED, "adamw_plan_create: too many elements");
  }
  return guarded([&]() -> int {
    std::unique_ptr<distdl_adamw_plan> p(new distdl_adamw_plan());
    p->g16 = g_dtype == DISTDL_BF16;
    p->s8 = states8 != 0;
    p->n_chunks = chunks;
    int64_t place = 0, at = 0;
    for (int i = 0; i < n_arrays; ++i) {
      p->count.push_back(count[i]);
      p->place.push_back((uint32_t)place);
      place += (count[i] + kBlock8 - 1) / kBlock8 * kBlock8;
      p->chunk0.push_back((uint32_t)at);
      at += (count[i] + size - 1) / size;
    }
    *out = p.release();
    return DISTDL_OK;
  });
}

int distdl_adamw_plan_destroy(distdl_adamw_plan* p) {
  if (!p) return DISTDL_OK;
  p->chunks.release();
  p->arrays.release();
  delete p;
  return DISTDL_OK;
}

int distdl_adamw_step(distdl_adamw_plan* p, void* const p_dev[], const void* const g_dev[], void* const m_dev[],
                      void* const v_dev[], void* const ms_dev[], void* const vs_dev[], void* const copy_dev[],
                      const distdl_adamw_args* h, void* stream) {
  if (!p || !p_dev || !g_dev || !m_dev || !v_dev || !h) return set_error(DISTDL_ERR_NULL, "adamw_step: null argument");
  if (p->s8 && (!ms_dev || !vs_dev)) return set_error(DISTDL_ERR_NULL, "adamw_step: 8-bit moments need their scales");
  if (!(h->lr >= 0) || !std::isfinite(h->lr) || !(h->beta1 >= 0 && h->beta1 < 1) || !(h->beta2 >= 0 && h->beta2 < 1) ||
      !(h->eps > 0) || !std::isfinite(h->eps) || !std::isfinite(h->weight_decay) || h->weight_decay < 0)
    return set_error(DISTDL_ERR_INVALID_ARG, "adamw_step: lr %g, beta %g and %g, eps %g, weight decay %g", h->lr, h->beta1, h->beta2,
                     h->eps, h->weight_decay);
  if (!h->step_dev && h->step < 1) return set_error(DISTDL_ERR_INVALID_ARG, "adamw_step: step %lld", (long long)h->step);
  if ((uintptr_t)h->step_dev % 8 || (uintptr_t)h->gscale_dev % 4)
    return set_error(DISTDL_ERR_INVALID_ARG, "adamw_step: the step's number or the gradient's factor is not aligned to its size");
  const size_t n = p->count.size();
  return guarded([&]() -> int {
    std::vector<AdamArray> arrays(n);
    for (size_t i = 0; i < n; ++i) {
      AdamArray& a = arrays[i];
      a = AdamArray{(float*)p_dev[i], g_dev[i], m_dev[i], v_dev[i], p->s8 ? (uint8_t*)ms_dev[i] : nullptr,
                    p->s8 ? (uint8_t*)vs_dev[i] : nullptr, copy_dev ? (uint16_t*)copy_dev[i] : nullptr, p->count[i], p->place[i], p->chunk0[i]};
      if (p->count[i] == 0) continue;
      if (!a.p || !a.g || !a.m || !a.v || (p->s8 && (!a.ms || !a.vs)))
        return set_error(DISTDL_ERR_NULL, "adamw_step: array %zu is null", i);
      if ((uintptr_t)a.p % 4 || (uintptr_t)a.g % (p->g16 ? 2 : 4) || (!p->s8 && ((uintptr_t)a.m % 4 || (uintptr_t)a.v % 4)) ||
          (uintptr_t)a.copy % 2)
        return set_error(DISTDL_ERR_INVALID_ARG, "adamw_step: array %zu is not aligned to its elements", i);
    }
    if (p->n_chunks == 0) return DISTDL_OK;
    hipStream_t st_ = (hipStream_t)stream;
    bool is_new = true;  // to this stream, whose first call makes the table of workgroups
    for (const StreamScratch::Block& b : p->chunks.blocks) is_new = is_new && b.stream != st_;
    if (is_new) {
      hipStreamCaptureStatus cap = hipStreamCaptureStatusNone;
      DISTDL_HIP_TRY(hipStreamIsCapturing(st_, &cap));
      if (cap != hipStreamCaptureStatusNone)
        return set_error(DISTDL_ERR_INVALID_ARG, "adamw_step: the plan's first call on this stream, which is being captured");
    }
    int rc = p->arrays.upload(arrays, st_);
    if (rc) return rc;
    float* table = nullptr;
    static_assert(sizeof(AdamChunk) == 2 * sizeof(float), "two words a workgroup");
    if ((rc = p->chunks.get(2 * (size_t)p->n_chunks, st_, &table))) return rc;
    AdamChunk* const chunks = (AdamChunk*)table;
    if (is_new) {
      hipLaunchKernelGGL(adamw_chunks_kernel, dim3((unsigned)((p->n_chunks + 255) / 256)), dim3(256), 0, st_, chunks, (uint32_t)p->n_chunks, p->arrays.dev, (uint32_t)n);
      DISTDL_HIP_TRY(hipGetLastError());
    }
    const double t = h->step_dev ? 1.0 : (double)h->step;
    AdamArgs s;
    s.beta1 = (float)h->beta1;
    s.keep1 = (float)(1 - h->beta1);
    s.beta2 = (float)h->beta2;
    s.keep2 = (float)(1 - h->beta2);
    s.decay = (float)(1 - h->lr * h->weight_decay);
    s.rate = (float)(h->lr / (1 - std::pow(h->beta1, t)));
    s.grow = (float)(1 / std::sqrt(1 - std::pow(h->beta2, t)));
    s.eps = std::max((float)h->eps, FLT_MIN);  // (never the zero that a smaller one would be in 32 bits: weights without gradients would divide by it)
    s.key = h->seed * 0x6A09E667u + (uint32_t)h->step * 0xBB67AE85u;
    s.lr = h->lr;
    s.b1 = h->beta1;
    s.b2 = h->beta2;
    s.seed = h->seed;
    s.step = h->step_dev;
    s.gscale = h->gscale_dev;
    {
      ProfScope prof("adamw", st_);
      const dim3 grid((unsigned)p->n_chunks);
      if (p->s8) {
        if (p->g16) hipLaunchKernelGGL((adamw_kernel<true, true>), grid, dim3(256), 0, st_, chunks, p->arrays.dev, s);
        else hipLaunchKernelGGL((adamw_kernel<false, true>), grid, dim3(256), 0, st_, chunks, p->arrays.dev, s);
      } else {
        if (p->g16) hipLaunchKernelGGL((adamw_kernel<true, false>), grid, dim3(256), 0, st_, chunks, p->arrays.dev, s);
        else hipLaunchKernelGGL((adamw_kernel<false, false>), grid, dim3(256), 0, st_, chunks, p->arrays.dev, s);
      }
    }
    DISTDL_HIP_TRY(hipGetLastError());
    return DISTDL_OK;
  });
}

}  // extern "C"
