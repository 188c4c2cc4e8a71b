// 8-bit numbers in blocks of 128, and the pieces that kernels over rows share (gfx950).
//
// A number is an e4m3 code times 2^(byte - 127), one byte (e8m0) for each block.  The byte is the smallest power of two for which
// no magnitude of the block exceeds 448 codes.  A power of two costs nothing: e4m3 keeps three bits of mantissa at any
// scale, so a finer one would only move the range (2^-9 .. 448 codes) by less than a factor of two, multiplying by it is
// exact in both directions, and the matrix instructions take it as an operand.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>
#include <cstring>

namespace distdl {

constexpr int kBlock8 = 128;
constexpr float kCodeMin = 0.001953125f;    // 2^-9, the smallest e4m3 number
constexpr float kCodeNormal = 0.015625f;    // 2^-6, the smallest normal one

// Biased exponent of the block's scale.  448 = 1.75 * 2^8: a mantissa above 1.75 (0x600000) carries.  At least 1 (2^-126): a
// subnormal scale would have no exact inverse.  255 (NaN) for a block that holds an infinity; NaNs are not in `amax`
// and become NaN codes where they are.
__device__ __forceinline__ int scale_byte(float amax) {
  const uint32_t bits = __float_as_uint(amax);
  const int byte = (int)((bits + 0x1FFFFFu) >> 23) - 8;
  return bits >= 0x7F800000u ? 255 : max(byte, 1);
}
__device__ __forceinline__ float scale_value(int byte) {
  return __uint_as_float(byte == 255 ? 0x7FC00000u : byte == 0 ? 0x00400000u : (uint32_t)byte << 23);
}
// 2^(127 - byte), and 0 for 255: the codes of such a block are NaN or 0, and it stands for NaN throughout
__device__ __forceinline__ float scale_inverse(int byte) { return byte == 255 ? 0.f : __uint_as_float((uint32_t)(254 - byte) << 23); }

// Four fp32 numbers (magnitudes up to 448, or NaN) to e4m3, nearest even, and back.
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d) {
  int v = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, v, true);
}
__device__ __forceinline__ void unpack_e4m3(uint32_t v, float* out) {
  const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)v, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)v, true);
  out[0] = lo[0];
  out[1] = lo[1];
  out[2] = hi[0];
  out[3] = hi[1];
}

// ---- eight elements of a row at a time ------------------------------------
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
// (rows of an odd number of elements start anywhere: the accesses are as wide as for aligned ones, the address is not)
typedef u32x4 u32x4_any __attribute__((aligned(1)));
typedef u32x2 u32x2_any __attribute__((aligned(1)));

__device__ __forceinline__ float bf16_lo(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t v) { return __uint_as_float(v & 0xffff0000u); }
// Nearest even, NaNs stay NaN: one instruction for two
__device__ __forceinline__ uint32_t to_bf16(float lo, float hi) {
  typedef __bf16 pair_bf16 __attribute__((ext_vector_type(2)));
  typedef float pair_f32 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(pair_f32{lo, hi}, pair_bf16));
}
__device__ __forceinline__ uint16_t to_bf16(float v) { return __builtin_bit_cast(uint16_t, (__bf16)v); }

// The raw bits of eight elements: those below `n` of them, zeros for the rest.
template <class T>
struct Eight;
template <>
struct Eight<float> {
  u32x4 a, b;
  __device__ __forceinline__ void load(const float* p, int n) {
    if (n >= 8) {
      a = *(const u32x4_any*)p;
      b = *(const u32x4_any*)(p + 4);
    } else {
      const uint32_t* q = (const uint32_t*)p;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        a[i] = i < n ? q[i] : 0u;
        b[i] = i + 4 < n ? q[i + 4] : 0u;
      }
    }
  }
  __device__ __forceinline__ void values(float* v) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[i] = __uint_as_float(a[i]);
      v[i + 4] = __uint_as_float(b[i]);
    }
  }
};
template <>
struct Eight<uint16_t> {
  u32x4 a;
  __device__ __forceinline__ void load(const uint16_t* p, int n) {
    if (n >= 8) {
      a = *(const u32x4_any*)p;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) a[i] = (2 * i < n ? p[2 * i] : 0u) | (2 * i + 1 < n ? (uint32_t)p[2 * i + 1] << 16 : 0u);
    }
  }
  __device__ __forceinline__ void values(float* v) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = bf16_lo(a[i]);
      v[2 * i + 1] = bf16_hi(a[i]);
    }
  }
};

__device__ __forceinline__ void store8(float* p, const float* v, int n) {
  if (n >= 8) {
    u32x4 a, b;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      a[i] = __float_as_uint(v[i]);
      b[i] = __float_as_uint(v[i + 4]);
    }
    *(u32x4_any*)p = a;
    *(u32x4_any*)(p + 4) = b;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) p[i] = v[i];
  }
}
__device__ __forceinline__ void store8(uint16_t* p, const float* v, int n) {
  if (n >= 8) {
    u32x4 a;
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] = to_bf16(v[2 * i], v[2 * i + 1]);
    *(u32x4_any*)p = a;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) p[i] = to_bf16(v[i]);
  }
}
// Eight codes
__device__ __forceinline__ void store8_codes(uint8_t* p, u32x2 c, int n) {
  if (n >= 8) {
    *(u32x2_any*)p = c;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) p[i] = (uint8_t)(c[i >> 2] >> (8 * (i & 3)));
  }
}
__device__ __forceinline__ u32x2 load8_codes(const uint8_t* p, int n) {
  u32x2 c = {0u, 0u};
  if (n >= 8) return *(const u32x2_any*)p;
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (i < n) c[i >> 2] |= (uint32_t)p[i] << (8 * (i & 3));
  return c;
}

// Workgroups go to the eight XCDs in turn; this numbers them so that neighbours meet in one XCD, and so in one L2: the lines that two of
// them share (rows that are no multiple of 128 bytes) are put together there instead of being written in parts.
__device__ __forceinline__ uint32_t xcd_order(uint32_t block, uint32_t blocks) {
  const uint32_t x = block & 7, each = blocks >> 3, left = blocks & 7;
  return x * each + min(x, left) + (block >> 3);
}

// ---- reductions over lanes ------------------------------------------------
template <int ror>
__device__ __forceinline__ float row_rotated(float v) {  // lanes of a row of 16, rotated (DPP row_ror)
  return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), 0x120 + ror, 0xf, 0xf, false));
}
__device__ __forceinline__ float row16_max(float v) {
  v = fmaxf(v, row_rotated<8>(v));
  v = fmaxf(v, row_rotated<4>(v));
  v = fmaxf(v, row_rotated<2>(v));
  return fmaxf(v, row_rotated<1>(v));
}
// (lanes exchange their sums in pairs, so that all end with the same bits)
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

}  // namespace distdl
