// What the kernels of the gated delta rule share: arguments, chunks, operand pieces (gfx950).
//
// A matrix operand of v_mfma_f32_16x16x32_bf16 is, for each lane, eight numbers of a row (or column) lane % 16: a fragment of 16 x 32
// numbers, 1 KiB.  The sums' order is free, so the 32 numbers that a fragment is summed over are taken as lane group g = lane / 16
// gets them from two 16 x 16 tiles of results: 4 g + 0 .. 3 of the first, 4 g + 0 .. 3 of the second.  So one product's results are the next one's
// right operand as they lie in the lanes.
//
// Numbers that are not bf16 already are sums of three bf16 parts, which hold all 24 bits (hi, and what is left, twice); products keep
// the parts whose sum of ranks is below three: six products of two such operands, three of one with a bf16 operand.
#pragma once
#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>
#include <type_traits>

#include "block8.h"
#include "buffer.h"
#include "common.h"

namespace distdl {

constexpr int kChunk = 64;        // steps
constexpr int kDeltaInline = 16;  // workers whose pointers travel with the launch; more are in a table

struct DeltaWorker {
  const void *q, *k, *v;
  const float *g, *beta;
  void* o;
  const void* d_o;  // adjoint
  void *dq, *dk, *dv;
  float *dg, *dbeta;
};

struct DeltaArgs {
  DeltaWorker w[kDeltaInline];
  const DeltaWorker* more;
  int32_t P, T, part, extra;          // worker p has part + (p < extra) steps
  int32_t chunks_wide, chunks_rest;   // chunks of a worker with part + 1 steps, with part
  int32_t chunks, n_b, n_h, n_hk, each;  // each: heads of a key's head
  int32_t d_k, d_v, dvp;              // dvp: d_v up to a multiple of 16
  int32_t slices;                     // of the columns of a head
  float scale;
  const int32_t* lengths;
  const float *h0, *dhT;
  float *hT, *dh0;
  // made by the kernel in front, for each sequence, chunk and key's head ...
  uint16_t *kf, *ktf, *qf, *qtf;      // fragments of K, K^T, Q, Q^T
  // ... and for each sequence, chunk and head
  uint16_t *tf, *pf, *ttf, *ptf;      // fragments of T and P, and of their transposes
  float* tiles;                       // A / beta and P, tiles on and below the diagonal as they lie in the lanes
  float* steps;                       // of each step: kStepNumbers of them, [C] each
  float *states, *dstates;            // [DK][dvp] at a chunk's start; the gradient at its end
  float *u, *dr;                      // [C][dvp]; in u X where beta is 0
  float* keys;                        // parts of dq and dk, where a chunk's heads are workgroups of their own
};

static_assert(offsetof(DeltaArgs, w) == 0, "the kernels' first argument starts with the workers");
typedef const __attribute__((address_space(4))) DeltaWorker* DeltaTable;
// (read as constants, into scalar registers; the address of the arguments is taken in the kernel itself)
#define DELTA_TABLE(s) ((s).more ? (DeltaTable)(uint64_t)(s).more : (DeltaTable)__builtin_amdgcn_kernarg_segment_ptr())

// A chunk: steps first .. first + n - 1 of worker p, which has `steps` of them; `live` of them lie inside the sequence.
struct DeltaChunk {
  int32_t p, first, n, steps, live;
};
__device__ __forceinline__ DeltaChunk delta_chunk(const DeltaArgs& s, int b, int c) {
  DeltaChunk r;
  const int wide = s.extra * s.chunks_wide;
  if (c < wide) {
    r.p = c / s.chunks_wide;
    r.first = (c - r.p * s.chunks_wide) * kChunk;
    r.steps = s.part + 1;
  } else {
    const int i = (c - wide) / s.chunks_rest;
    r.p = s.extra + i;
    r.first = (c - wide - i * s.chunks_rest) * kChunk;
    r.steps = s.part;
  }
  r.n = min(kChunk, r.steps - r.first);
  const int64_t at = (int64_t)r.p * s.part + min(r.p, s.extra) + r.first;  // of the whole
  const int64_t len = s.lengths ? s.lengths[b] : s.T;
  r.live = (int)max((int64_t)0, min((int64_t)r.n, len - at));
  return r;
}

__device__ __forceinline__ int delta_length(const DeltaArgs& s, int b) {
  return __builtin_amdgcn_readfirstlane(s.lengths ? max(0, min(s.lengths[b], s.T)) : s.T);
}
// How many chunks have some of a sequence's steps; they come first.
__device__ __forceinline__ int delta_live_chunks(const DeltaArgs& s, int len) {
  if (len == 0) return 0;
  const int last = len - 1, wide = s.extra * (s.part + 1);
  if (last < wide) return last / (s.part + 1) * s.chunks_wide + last % (s.part + 1) / kChunk + 1;
  return s.extra * s.chunks_wide + (last - wide) / s.part * s.chunks_rest + (last - wide) % s.part / kChunk + 1;
}

// A walk along the chunks that reads nothing but a worker's pointer, where it comes to another worker: one of its arrays.
struct DeltaWalk {
  int32_t p, first, steps, before;  // before: the worker's first step
  const char* array;
  template <class F>
  __device__ __forceinline__ void enter(const DeltaArgs& s, int worker, F pointer) {
    p = worker;
    steps = s.part + (p < s.extra);
    before = p * s.part + min(p, s.extra);
    array = (const char*)pointer(p);
  }
  template <class F>
  __device__ __forceinline__ void start(const DeltaArgs& s, int c, F pointer) {
    const int wide = s.extra * s.chunks_wide;
    enter(s, c < wide ? c / s.chunks_wide : s.extra + (c - wide) / s.chunks_rest, pointer);
    first = (c < wide ? c % s.chunks_wide : (c - wide) % s.chunks_rest) * kChunk;
  }
  template <class F>
  __device__ __forceinline__ void ahead(const DeltaArgs& s, F pointer) {
    first += kChunk;
    if (first >= steps) {
      enter(s, p + 1, pointer);
      first = 0;
    }
  }
  template <class F>
  __device__ __forceinline__ void back(const DeltaArgs& s, F pointer) {
    first -= kChunk;
    if (first < 0) {
      enter(s, p - 1, pointer);
      first = (steps - 1) / kChunk * kChunk;
    }
  }
  __device__ __forceinline__ int count() const { return min(kChunk, steps - first); }
  __device__ __forceinline__ int live(int len) const { return max(0, min(count(), len - before - first)); }
};

// ---- operand pieces -------------------------------------------------------
typedef __bf16 delta_bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

template <int N>
struct Pieces {
  u32x4 p[N];
};

// Eight numbers, exactly: the upper halves of the numbers, of what is left, and of what is left then.
__device__ __forceinline__ Pieces<3> split8(const float* v) {
  Pieces<3> o;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float a = v[2 * i], b = v[2 * i + 1];
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      o.p[k][i] = __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
      if (k < 2) {
        a -= __uint_as_float(__float_as_uint(a) & 0xffff0000u);
        b -= __uint_as_float(__float_as_uint(b) & 0xffff0000u);
      }
    }
  }
  return o;
}
// two tiles of results as the next product's operand
__device__ __forceinline__ Pieces<3> split_tiles(f32x4 a, f32x4 b) {
  const float v[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
  return split8(v);
}
// Eight numbers of the tensors' type: one piece of bf16, three of fp32.
template <class E>
constexpr int delta_pieces() { return sizeof(E) == 2 ? 1 : 3; }

// c += a b, the smallest products first
template <int NA, int NB>
__device__ __forceinline__ f32x4 multiply(const Pieces<NA>& a, const Pieces<NB>& b, f32x4 c) {
  constexpr int kMost = (NA > NB ? NA : NB) - 1;
#pragma unroll
  for (int r = kMost; r >= 0; --r)
#pragma unroll
    for (int i = 0; i < NA; ++i) {
      const int j = r - i;
      if (j >= 0 && j < NB)
        c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(delta_bf16x8, a.p[i]), __builtin_bit_cast(delta_bf16x8, b.p[j]), c, 0, 0, 0);
    }
  return c;
}

constexpr int kFragment = 512;  // numbers
template <int N>
__device__ __forceinline__ Pieces<N> load_fragment(const uint16_t* at) {
  Pieces<N> o;
#pragma unroll
  for (int i = 0; i < N; ++i) o.p[i] = *(const u32x4*)(at + i * kFragment + (threadIdx.x & 63) * 8);
  return o;
}
template <int N>
__device__ __forceinline__ void store_fragment(uint16_t* at, const Pieces<N>& v) {
#pragma unroll
  for (int i = 0; i < N; ++i) *(u32x4*)(at + i * kFragment + (threadIdx.x & 63) * 8) = v.p[i];
}

template <int C, int DK>
struct DeltaSizes {
  static constexpr int kTiles = C / 16, kLower = kTiles * (kTiles + 1) / 2, kSteps = C / 32;       // of a chunk's steps as rows, and as what is summed over
  static constexpr int kKeyTiles = DK / 16, kKeySteps = DK / 32;
  // numbers of one piece of all fragments
  static constexpr int64_t kKeyPiece = (int64_t)C * DK, kStepPiece = (int64_t)C * C;
};
constexpr int kInner = 3;  // pieces of T and P
// exp(G), exp(G_C - G), beta, and the two parts of G / log 2
constexpr int kSince = 0, kUntil = 1, kBeta = 2, kWhole = 3, kRest = 4, kStepNumbers = 5;

}  // namespace distdl
