// Sixteen bytes of a matrix row a lane, of any alignment that its elements have, and the types of its elements.
#pragma once

#include "common.h"
#include "device.h"

namespace damoe {

// Global loads and stores of 16 bytes need no more than the element's alignment on this card (the compiler emits them for
// packed types), so odd row lengths and strides cost the lines that they straddle and not a load an element.
template <int ALIGN>
struct __attribute__((packed, aligned(ALIGN))) Packed16 {
  typedef uint32_t V __attribute__((ext_vector_type(4)));
  V v;
};

template <int ALIGN, bool NT = false>
__device__ __forceinline__ uint4 load16_at(const void* p) {
  typedef typename Packed16<ALIGN>::V V;
  if constexpr (NT) {  // the builtin takes the type's own alignment from the pointer
    typedef V U __attribute__((aligned(ALIGN)));
    return __builtin_bit_cast(uint4, __builtin_nontemporal_load(static_cast<const U*>(p)));
  } else {
    return __builtin_bit_cast(uint4, static_cast<const Packed16<ALIGN>*>(p)->v);
  }
}

template <int ALIGN, bool NT = false>
__device__ __forceinline__ void store16_at(void* p, uint4 q) {
  typedef typename Packed16<ALIGN>::V V;
  if constexpr (NT) {
    typedef V U __attribute__((aligned(ALIGN)));
    __builtin_nontemporal_store(__builtin_bit_cast(V, q), static_cast<U*>(p));
  } else {
    static_cast<Packed16<ALIGN>*>(p)->v = __builtin_bit_cast(V, q);
  }
}

// Element type of a matrix: bf16 (BF) or fp32.
template <bool BF>
struct Elem;
template <>
struct Elem<true> {
  typedef uint16_t T;
  static constexpr int kBytes = 2, kPer16 = 8;
};
template <>
struct Elem<false> {
  typedef float T;
  static constexpr int kBytes = 4, kPer16 = 4;
};

// The 16 bytes of a row from `p` on of which n elements (at least one) are the row's; the others are 0.
template <bool BF, bool NT = false>
__device__ __forceinline__ uint4 load_some(const typename Elem<BF>::T* p, int n) {
  typedef Elem<BF> E;
  if (n >= E::kPer16) return load16_at<E::kBytes, NT>(p);
  uint32_t q[4] = {0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < E::kPer16; ++i) {
    if (i >= n) continue;
    if constexpr (BF) q[i / 2] |= (uint32_t)p[i] << (16 * (i & 1));
    else q[i] = __float_as_uint(p[i]);
  }
  return uint4{q[0], q[1], q[2], q[3]};
}

template <bool BF, bool NT = false>
__device__ __forceinline__ void store_some(typename Elem<BF>::T* p, int n, uint4 v) {
  typedef Elem<BF> E;
  if (n >= E::kPer16) return store16_at<E::kBytes, NT>(p, v);
  const uint32_t q[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < E::kPer16; ++i) {
    if (i >= n) continue;
    if constexpr (BF) p[i] = (uint16_t)(q[i / 2] >> (16 * (i & 1)));
    else p[i] = __uint_as_float(q[i]);
  }
}

// The values of 16 bytes as fp32, and back (bf16: round to nearest even, NaN kept).
template <bool BF>
__device__ __forceinline__ void unpack16(uint4 v, float (&f)[Elem<BF>::kPer16]) {
  const uint32_t q[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (BF) {
      f[2 * i] = __uint_as_float(q[i] << 16);
      f[2 * i + 1] = __uint_as_float(q[i] & 0xFFFF0000u);
    } else {
      f[i] = __uint_as_float(q[i]);
    }
  }
}

template <bool BF>
__device__ __forceinline__ uint4 pack16(const float (&f)[Elem<BF>::kPer16]) {
  uint32_t q[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (BF) q[i] = pack_bf16x2(f[2 * i], f[2 * i + 1]);
    else q[i] = __float_as_uint(f[i]);
  }
  return uint4{q[0], q[1], q[2], q[3]};
}

}  // namespace damoe
