// MXFP4 quantisation into the library's layouts, and back.
//
// A lane takes eight consecutive values (one 16-byte load of bf16) and a quad of lanes a 32-value block, so
// loads are contiguous, the block's maximum is two lane exchanges, and a lane's result is one dword of codes.
// Each pass is memory bound: 2 or 4 bytes in and 17/32 out per value, or the reverse.
//
// The lanes' order follows the layout: row-major, a wave has 512 consecutive values; FRAG16, a wave has a quad
// fragment (16 rows x 128 columns, four rows at a time); TILE32, a wave has 8 rows of a 32 x 256 tile, 64
// columns at a time.  So a wave reads whole 128-byte lines of x and its stores fill runs of at least 64 bytes.
#include "mxfp4.h"

namespace damoe {
namespace {

constexpr int kThreads = 256;
constexpr int kUnroll = 4;  // eights a lane handles, loaded together

struct QuantArgs {
  void* x;
  int64_t rows, ld;
  int32_t cols;
  uint8_t* codes;
  uint8_t* scales;
};

// ---------------------------------------------------------------- quantise

// Row-major, eights in order.  Where an eight of the matrix lies in x: rows without a gap (GAP false) are one long row;
// else a block row of the grid has `chunk` rows' eights, few enough that 32 bits number them.
template <bool GAP>
struct Eights {
  int64_t first, n;  // the block row's eights: codes from number `first` on, n of them
  int64_t row0, ld;
  uint32_t n8;

  __device__ __forceinline__ Eights(const QuantArgs& a, int64_t n_all, int64_t chunk) : ld(a.ld), n8((uint32_t)(a.cols / 8)) {
    row0 = GAP ? (int64_t)blockIdx.y * chunk : 0;
    first = GAP ? row0 * n8 : 0;
    n = GAP ? min(chunk, a.rows - row0) * n8 : n_all;
  }
  __device__ __forceinline__ int64_t at(int64_t i) const {
    if constexpr (!GAP) return i * 8;
    const uint32_t r = (uint32_t)i / n8;
    return (row0 + r) * ld + (int64_t)((uint32_t)i - r * n8) * 8;
  }
};

template <bool BF, bool V, bool NT, bool GAP>
__global__ void __launch_bounds__(kThreads) k_quantise_rows(QuantArgs a, int64_t n_all, int64_t chunk) {
  const Eights<GAP> w(a, n_all, chunk);
  const int64_t i0 = (int64_t)blockIdx.x * (kThreads * kUnroll) + threadIdx.x;
  Eight<BF> e[kUnroll];
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    const int64_t i = i0 + u * kThreads;
    if (i < w.n) e[u].template load<V, NT>(a.x, w.at(i));
    else e[u].zero();
  }
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    const int64_t i = i0 + u * kThreads;
    const uint32_t s = e[u].scale_byte();
    if (i >= w.n) continue;
    reinterpret_cast<uint32_t*>(a.codes)[w.first + i] = e[u].codes(s);
    if ((i & 3) == 0) a.scales[(w.first + i) >> 2] = (uint8_t)s;
  }
}

// FRAG16: a wave a quad fragment.  Lane 16 r4 + 4 b + g has row 4 u + r4, columns 32 b + 8 g .. + 7, whose codes
// are bytes 4 b .. + 3 of the fragment's lane 16 g + row.
template <bool BF, bool V, bool NT>
__global__ void __launch_bounds__(kThreads) k_quantise_frag(QuantArgs a, int64_t quads, int32_t per_row) {
  const int lane = threadIdx.x & 63;
  const int64_t q = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (q >= quads) return;
  const int64_t rb = q / per_row;
  const int32_t kq = (int32_t)(q - rb * per_row);
  const int r4 = lane >> 4, b = (lane >> 2) & 3, g = lane & 3;
  uint8_t* out = a.codes + q * kFp4QuadBytes;
  Eight<BF> e[4];
#pragma unroll
  for (int u = 0; u < 4; ++u)
    e[u].template load<V, NT>(a.x, (rb * 16 + 4 * u + r4) * a.ld + (int64_t)kq * 128 + 32 * b + 8 * g);
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const int row = 4 * u + r4;
    const uint32_t s = e[u].scale_byte();
    *reinterpret_cast<uint32_t*>(out + (row + 16 * g) * 16 + 4 * b) = e[u].codes(s);
    if (g == 0) out[1024 + 4 * row + b] = (uint8_t)s;
  }
}

// TILE32: a block a tile, a wave 8 of its rows.  Lane 8 r + 4 h + q has row 8 w + r, columns
// 64 j + 32 h + 8 q .. + 7.
template <bool BF, bool V, bool NT>
__global__ void __launch_bounds__(kThreads) k_quantise_tile(QuantArgs a, int64_t tiles, int32_t per_row) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int r = 8 * w + (lane >> 3), h = (lane >> 2) & 1, q = lane & 3;
  for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
    const int64_t rb = tile / per_row;
    const int64_t row = rb * kTileRows + r;
    const int32_t c0 = (int32_t)(tile - rb * per_row) * kTileCols + 32 * h + 8 * q;
    Eight<BF> e[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (row < a.rows && c0 + 64 * j < a.cols) e[j].template load<V, NT>(a.x, row * a.ld + c0 + 64 * j);
      else e[j].zero();
    }
    uint8_t* out = a.codes + tile * kTileBytes;
    uint32_t sc = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t s = e[j].scale_byte();
      *reinterpret_cast<uint32_t*>(out + 1024 * j + 16 * (32 * h + r) + 4 * q) = e[j].codes(s);
      sc |= s << (8 * j);
    }
    if (q == 0) *reinterpret_cast<uint32_t*>(out + kTileCodes + 4 * (32 * h + r)) = sc;
  }
}

// ---------------------------------------------------------------- dequantise

// Eight values of the codes c and the scale byte s.  The conversions multiply by the scale exactly, results below the
// normal range included, and give infinity past the type's range and NaN for a NaN scale (checked on the device for
// every code under every scale).
template <bool BF, bool V, bool NT>
__device__ __forceinline__ void store8(void* base, int64_t i, uint32_t c, uint32_t s) {
  const float f = e8m0_to_f32(s);
  if constexpr (BF) {
    uint16_t* p = static_cast<uint16_t*>(base) + i;
    const uint4 q = fp4x8_to_bf16x8(c, f);
    if constexpr (V) {
      store16<NT>(p, q);
    } else {
      const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
      for (int j = 0; j < 8; ++j) p[j] = (uint16_t)(w[j / 2] >> (16 * (j & 1)));
    }
  } else {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    const f32x2 v[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, f, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, f, 1),
                        __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, f, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, f, 3)};
    float* p = static_cast<float*>(base) + i;
    if constexpr (V) {
      store16<NT>(p, __builtin_bit_cast(uint4, make_float4(v[0][0], v[0][1], v[1][0], v[1][1])));
      store16<NT>(p + 4, __builtin_bit_cast(uint4, make_float4(v[2][0], v[2][1], v[3][0], v[3][1])));
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) p[j] = v[j / 2][j & 1];
    }
  }
}

template <bool BF, bool V, bool NT, bool GAP>
__global__ void __launch_bounds__(kThreads) k_dequantise_rows(QuantArgs a, int64_t n_all, int64_t chunk) {
  const Eights<GAP> w(a, n_all, chunk);
  const int64_t i0 = (int64_t)blockIdx.x * (kThreads * kUnroll) + threadIdx.x;
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    const int64_t i = i0 + u * kThreads;
    if (i >= w.n) continue;
    store8<BF, V, NT>(a.x, w.at(i), reinterpret_cast<const uint32_t*>(a.codes)[w.first + i], a.scales[(w.first + i) >> 2]);
  }
}

template <bool BF, bool V, bool NT>
__global__ void __launch_bounds__(kThreads) k_dequantise_frag(QuantArgs a, int64_t quads, int32_t per_row) {
  const int lane = threadIdx.x & 63;
  const int64_t q = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (q >= quads) return;
  const int64_t rb = q / per_row;
  const int32_t kq = (int32_t)(q - rb * per_row);
  const int r4 = lane >> 4, b = (lane >> 2) & 3, g = lane & 3;
  const uint8_t* in = a.codes + q * kFp4QuadBytes;
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const int row = 4 * u + r4;
    store8<BF, V, NT>(a.x, (rb * 16 + row) * a.ld + (int64_t)kq * 128 + 32 * b + 8 * g,
                  *reinterpret_cast<const uint32_t*>(in + (row + 16 * g) * 16 + 4 * b), in[1024 + 4 * row + b]);
  }
}

template <bool BF, bool V, bool NT>
__global__ void __launch_bounds__(kThreads) k_dequantise_tile(QuantArgs a, int64_t tiles, int32_t per_row) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int r = 8 * w + (lane >> 3), h = (lane >> 2) & 1, q = lane & 3;
  for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
    const int64_t rb = tile / per_row;
    const int64_t row = rb * kTileRows + r;
    const int32_t c0 = (int32_t)(tile - rb * per_row) * kTileCols + 32 * h + 8 * q;
    const uint8_t* in = a.codes + tile * kTileBytes;
    if (row >= a.rows) continue;
    const uint32_t sc = *reinterpret_cast<const uint32_t*>(in + kTileCodes + 4 * (32 * h + r));
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (c0 + 64 * j < a.cols)
        store8<BF, V, NT>(a.x, row * a.ld + c0 + 64 * j,
                      *reinterpret_cast<const uint32_t*>(in + 1024 * j + 16 * (32 * h + r) + 4 * q),
                      (sc >> (8 * j)) & 255u);
  }
}

// ---------------------------------------------------------------- pack

// Row-major codes and scales into tiles: a block a tile, thread t the 16-byte blocks t of its 256.
__global__ void __launch_bounds__(kThreads) k_pack_tile(const uint8_t* __restrict__ codes,
                                                        const uint8_t* __restrict__ scales, int64_t rows, int32_t cols,
                                                        uint8_t* __restrict__ tiles_out, int64_t tiles,
                                                        int32_t per_row) {
  const int t = threadIdx.x, r = t >> 3, blk = t & 7;  // block blk of row r: step blk / 2, half blk % 2
  for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
    const int64_t rb = tile / per_row;
    const int64_t row = rb * kTileRows + r;
    const int32_t kb = (int32_t)(tile - rb * per_row) * 8 + blk, nkb = cols / 32;
    uint8_t* out = tiles_out + tile * kTileBytes;
    const int lane = 32 * (blk & 1) + r, j = blk >> 1;
    uint4 c = make_uint4(0, 0, 0, 0);
    uint8_t s = (uint8_t)kScaleOne;
    if (row < rows && kb < nkb) {
      c = reinterpret_cast<const uint4*>(codes)[row * nkb + kb];
      s = scales[row * nkb + kb];
    }
    *reinterpret_cast<uint4*>(out + 1024 * j + 16 * lane) = c;
    out[kTileCodes + 4 * lane + j] = s;
  }
}

// ---------------------------------------------------------------- launches

constexpr int64_t kMaxGrid = 1 << 20;
// Eights of a block row of the row-major kernels with gaps.
constexpr int64_t kChunkEights = (int64_t)1 << 30;

// Bytes of x from which its accesses carry the nontemporal hint: what no longer fits the 256 MB cache in front of HBM is
// not worth keeping there.  bf16, quantise / dequantise over and over: 470 MiB 95 / 91 us with the hint, 111 / 126
// without; 256 MiB 54 / 52 and 60 / 72; 128 MiB 28 / 28 and 25 / 29, there the next reader finds the values cached.
constexpr int64_t kNontemporal = (int64_t)256 << 20;

template <class F>
hipError_t by_type(bool bf, bool vec, bool nt, F f) {
  using std::false_type;
  using std::true_type;
  const auto typed = [&](auto b) {
    if (!vec) return f(b, false_type{}, false_type{});
    return nt ? f(b, true_type{}, true_type{}) : f(b, true_type{}, false_type{});
  };
  return bf ? typed(true_type{}) : typed(false_type{});
}

// 16-byte accesses of eights: rows start 16-byte aligned.
bool vec_ok(const void* x, int64_t ld, bool bf) {
  return reinterpret_cast<uintptr_t>(x) % 16 == 0 && ld % (bf ? 8 : 4) == 0;
}

template <bool QUANT>
hipError_t launch(QuantArgs a, bool bf, int32_t layout, hipStream_t stream) {
  if (a.rows == 0) return hipSuccess;
  const bool vec = vec_ok(a.x, a.ld, bf);
  const bool nt = a.rows * a.cols * (bf ? 2 : 4) >= kNontemporal;
  return by_type(bf, vec, nt, [&](auto b, auto v, auto n) {
    constexpr bool B = decltype(b)::value, V = decltype(v)::value, NT = decltype(n)::value;
    if (layout == DAMOE_LAYOUT_ROWMAJOR) {
      const int64_t n8 = a.cols / 8, n_all = a.rows * n8;
      const auto go = [&](auto gap) {
        constexpr bool GAP = decltype(gap)::value;
        const int64_t chunk = GAP ? std::min(a.rows, kChunkEights / n8) : a.rows;
        const dim3 grid((unsigned)tiles_of(chunk * n8, kThreads * kUnroll), (unsigned)((a.rows + chunk - 1) / chunk));
        if constexpr (QUANT) hipLaunchKernelGGL((k_quantise_rows<B, V, NT, GAP>), grid, dim3(kThreads), 0, stream, a, n_all, chunk);
        else hipLaunchKernelGGL((k_dequantise_rows<B, V, NT, GAP>), grid, dim3(kThreads), 0, stream, a, n_all, chunk);
      };
      if (a.ld == a.cols) go(std::false_type{});
      else go(std::true_type{});
    } else if (layout == DAMOE_LAYOUT_FRAG16) {
      const int32_t per_row = a.cols / 128;
      const int64_t quads = a.rows / 16 * per_row;
      const dim3 grid((unsigned)((quads + 3) / 4));
      if constexpr (QUANT) hipLaunchKernelGGL((k_quantise_frag<B, V, NT>), grid, dim3(kThreads), 0, stream, a, quads, per_row);
      else hipLaunchKernelGGL((k_dequantise_frag<B, V, NT>), grid, dim3(kThreads), 0, stream, a, quads, per_row);
    } else {
      const int32_t per_row = (int32_t)tiles_of(a.cols, kTileCols);
      const int64_t tiles = tiles_of(a.rows, kTileRows) * per_row;
      const dim3 grid((unsigned)std::min(tiles, kMaxGrid));
      if constexpr (QUANT) hipLaunchKernelGGL((k_quantise_tile<B, V, NT>), grid, dim3(kThreads), 0, stream, a, tiles, per_row);
      else hipLaunchKernelGGL((k_dequantise_tile<B, V, NT>), grid, dim3(kThreads), 0, stream, a, tiles, per_row);
    }
    return hipGetLastError();
  });
}

// Bounds that keep every grid below 2^32 threads (32 values a thread): 2^36 values, rows of at most 2^20.
constexpr int32_t kMaxCols = 1 << 20;
constexpr int64_t kMaxValues = (int64_t)1 << 36;

damoe_status check(const void* x, int32_t dtype, int64_t rows, int32_t cols, int64_t ldx, int32_t layout,
                   const uint8_t* codes, const uint8_t* scales) {
  if (rows < 0 || cols <= 0 || ldx < cols) return DAMOE_ERR_INVALID_ARG;
  if (dtype != DAMOE_BF16 && dtype != DAMOE_F32) return DAMOE_ERR_UNSUPPORTED;
  if (damoe_mxfp4_bytes(std::max<int64_t>(rows, 16), cols, layout) == 0 || (rows > 0 && damoe_mxfp4_bytes(rows, cols, layout) == 0))
    return DAMOE_ERR_UNSUPPORTED;
  if (rows == 0) return DAMOE_OK;
  if (!x || !codes || (layout == DAMOE_LAYOUT_ROWMAJOR && !scales)) return DAMOE_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(codes) % 16 || reinterpret_cast<uintptr_t>(x) % (dtype == DAMOE_BF16 ? 2 : 4))
    return DAMOE_ERR_INVALID_ARG;
  return DAMOE_OK;
}

}  // namespace

hipError_t launch_quantise_tiles(const void* x, bool bf, int64_t rows, int32_t cols, int64_t ldx, uint8_t* tiles,
                                 hipStream_t stream) {
  return launch<true>(QuantArgs{const_cast<void*>(x), rows, ldx, cols, tiles, nullptr}, bf, DAMOE_LAYOUT_TILE32, stream);
}

}  // namespace damoe

using namespace damoe;

extern "C" {

size_t damoe_mxfp4_bytes(int64_t rows, int32_t cols, int32_t layout) {
  if (rows <= 0 || cols <= 0 || cols % 32 || cols > kMaxCols || rows > kMaxValues / cols) return 0;
  if (layout == DAMOE_LAYOUT_ROWMAJOR) return (size_t)rows * cols / 2;
  if (layout == DAMOE_LAYOUT_FRAG16) return rows % 16 || cols % 128 ? 0 : (size_t)rows * cols / 32 * 17;
  if (layout == DAMOE_LAYOUT_TILE32) return (size_t)tiles_of(rows, kTileRows) * tiles_of(cols, kTileCols) * kTileBytes;
  return 0;
}

damoe_status damoe_mxfp4_quantise(const void* x, int32_t dtype, int64_t rows, int32_t cols, int64_t ldx, int32_t layout,
                                  uint8_t* codes, uint8_t* scales, hipStream_t stream) {
  const damoe_status st = check(x, dtype, rows, cols, ldx, layout, codes, scales);
  if (st != DAMOE_OK) return st;
  const QuantArgs a{const_cast<void*>(x), rows, ldx, cols, codes, scales};
  return launch<true>(a, dtype == DAMOE_BF16, layout, stream) == hipSuccess ? DAMOE_OK : DAMOE_ERR_HIP;
}

damoe_status damoe_mxfp4_dequantise(const uint8_t* codes, const uint8_t* scales, int64_t rows, int32_t cols,
                                    int32_t layout, void* x, int32_t dtype, int64_t ldx, hipStream_t stream) {
  const damoe_status st = check(x, dtype, rows, cols, ldx, layout, codes, scales);
  if (st != DAMOE_OK) return st;
  const QuantArgs a{x, rows, ldx, cols, const_cast<uint8_t*>(codes), const_cast<uint8_t*>(scales)};
  return launch<false>(a, dtype == DAMOE_BF16, layout, stream) == hipSuccess ? DAMOE_OK : DAMOE_ERR_HIP;
}

damoe_status damoe_mxfp4_pack(const uint8_t* codes, const uint8_t* scales, int64_t rows, int32_t cols, uint8_t* tiles,
                              hipStream_t stream) {
  if (rows < 0 || cols <= 0) return DAMOE_ERR_INVALID_ARG;
  if (cols % 32 || (rows > 0 && damoe_mxfp4_bytes(rows, cols, DAMOE_LAYOUT_TILE32) == 0)) return DAMOE_ERR_UNSUPPORTED;
  if (rows == 0) return DAMOE_OK;
  if (!codes || !scales || !tiles) return DAMOE_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(codes) % 16 || reinterpret_cast<uintptr_t>(tiles) % 16) return DAMOE_ERR_INVALID_ARG;
  const int32_t per_row = (int32_t)tiles_of(cols, kTileCols);
  const int64_t n = tiles_of(rows, kTileRows) * per_row;
  hipLaunchKernelGGL(k_pack_tile, dim3((unsigned)std::min(n, kMaxGrid)), dim3(kThreads), 0, stream, codes, scales, rows,
                     cols, tiles, n, per_row);
  return hipGetLastError() == hipSuccess ? DAMOE_OK : DAMOE_ERR_HIP;
}

}  // extern "C"
