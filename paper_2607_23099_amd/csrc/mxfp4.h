// MXFP4 elements: the operand layout of the dense product and the quantisation of eight values a lane.
#pragma once

#include "common.h"
#include "device.h"

namespace damoe {

// DAMOE_LAYOUT_TILE32: tiles of 32 rows x 256 columns, each the operands of four 32x32x64 scaled MFMAs in lane
// order.  Lane 32 h + r of step j holds the 32 codes of row r, columns 64 j + 32 h .. + 31 (16 bytes at
// 1024 j + 16 lane), one scale block; its four blocks' scale bytes are the dword at 4096 + 4 lane, so an
// operand's scales come in one load and step j takes byte j of it.
constexpr int kTileRows = 32, kTileCols = 256;
constexpr uint32_t kTileCodes = 4096, kTileBytes = kTileCodes + 256;
// Code 0 with scale 1: the padding of a tile.
constexpr uint32_t kScaleOne = 127;

__host__ __device__ inline int64_t tiles_of(int64_t n, int per) { return (n + per - 1) / per; }

// Scale byte of a block from the largest magnitude's bits (of an fp32 value, sign cleared): exponent minus 2
// (the e2m1 maximum is 1.5 x 2^2), at least 2^-127; 1 for a block of zeros, 255 with an infinity or NaN.
__device__ __forceinline__ uint32_t fp4_scale_byte(uint32_t amax_bits) {
  const uint32_t e = amax_bits >> 23;
  return amax_bits == 0 ? kScaleOne : e == 255u ? 255u : e > 2u ? e - 2u : 0u;
}

// 2^(s - 127), a number for s = 255 too (the codes of such a block are set to 0 by the caller).
__device__ __forceinline__ float fp4_scale(uint32_t s) { return __uint_as_float(s == 0u ? 0x00400000u : s << 23); }

template <int CTRL>
__device__ __forceinline__ uint32_t dpp_u32(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xF, 0xF, false);
}

// Maximum over the four lanes of a quad.
__device__ __forceinline__ uint32_t quad_max(uint32_t x) {
  x = max(x, dpp_u32<0xB1>(x));
  return max(x, dpp_u32<0x4E>(x));
}

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef uint16_t u16x2_t __attribute__((ext_vector_type(2)));

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

template <bool NT>
__device__ __forceinline__ uint4 load16(const void* p) {
  const u32x4_t* q = static_cast<const u32x4_t*>(p);
  return __builtin_bit_cast(uint4, NT ? __builtin_nontemporal_load(q) : *q);
}

template <bool NT>
__device__ __forceinline__ void store16(void* p, uint4 v) {
  u32x4_t* q = static_cast<u32x4_t*>(p);
  if constexpr (NT) __builtin_nontemporal_store(__builtin_bit_cast(u32x4_t, v), q);
  else *q = __builtin_bit_cast(u32x4_t, v);
}

// Eight values of a lane, as loaded.
template <bool BF>
struct Eight {
  uint32_t q[BF ? 4 : 8];

  // V: 16-byte loads (the address is 16-byte aligned); NT: with the nontemporal hint.
  template <bool V, bool NT = false>
  __device__ __forceinline__ void load(const void* base, int64_t i) {
    if constexpr (BF) {
      const uint16_t* p = static_cast<const uint16_t*>(base) + i;
      if constexpr (V) {
        const uint4 a = load16<NT>(p);
        q[0] = a.x, q[1] = a.y, q[2] = a.z, q[3] = a.w;
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) q[j] = (uint32_t)p[2 * j] | (uint32_t)p[2 * j + 1] << 16;
      }
    } else {
      const uint32_t* p = static_cast<const uint32_t*>(base) + i;
      if constexpr (V) {
        const uint4 a = load16<NT>(p), b = load16<NT>(p + 4);
        q[0] = a.x, q[1] = a.y, q[2] = a.z, q[3] = a.w;
        q[4] = b.x, q[5] = b.y, q[6] = b.z, q[7] = b.w;
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) q[j] = p[j];
      }
    }
  }

  __device__ __forceinline__ void zero() {
#pragma unroll
    for (uint32_t& v : q) v = 0;
  }

  // Largest magnitude of the eight, as the bits of an fp32 value: magnitudes compare as integers.
  __device__ __forceinline__ uint32_t amax() const {
    if constexpr (BF) {
      u16x2_t m = __builtin_bit_cast(u16x2_t, q[0] & 0x7FFF7FFFu);
#pragma unroll
      for (int j = 1; j < 4; ++j)
        m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2_t, q[j] & 0x7FFF7FFFu));
      return max((uint32_t)m[0], (uint32_t)m[1]) << 16;
    } else {
      uint32_t m = q[0] & 0x7FFFFFFFu;
#pragma unroll
      for (int j = 1; j < 8; ++j) m = max(m, q[j] & 0x7FFFFFFFu);
      return m;
    }
  }

  // Scale byte of the block of a quad's 32 values.
  __device__ __forceinline__ uint32_t scale_byte() const { return fp4_scale_byte(quad_max(amax())); }

  // The eight codes, the first in the low nibble.  The conversion divides by the scale exactly and rounds to
  // nearest even with saturation, subnormal inputs and scales included (checked on the device against the
  // definition over every exponent).
  __device__ __forceinline__ uint32_t codes(uint32_t s) const {
    if (s == 255u) return 0;
    const float f = fp4_scale(s);
    uint32_t r = 0;
    if constexpr (BF) {
      r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2_t, q[0]), f, 0);
      r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2_t, q[1]), f, 1);
      r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2_t, q[2]), f, 2);
      r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2_t, q[3]), f, 3);
    } else {
      r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, __uint_as_float(q[0]), __uint_as_float(q[1]), f, 0);
      r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, __uint_as_float(q[2]), __uint_as_float(q[3]), f, 1);
      r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, __uint_as_float(q[4]), __uint_as_float(q[5]), f, 2);
      r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, __uint_as_float(q[6]), __uint_as_float(q[7]), f, 3);
    }
    return r;
  }
};

// Rows of x into DAMOE_LAYOUT_TILE32 (quantise.hip), for the product's activations.
hipError_t launch_quantise_tiles(const void* x, bool bf, int64_t rows, int32_t cols, int64_t ldx, uint8_t* tiles,
                                 hipStream_t stream);

}  // namespace damoe
