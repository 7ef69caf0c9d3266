// The dense MXFP4 product y = add + Q(x) W^T on the scaled fp4 matrix instructions.
//
// Both operands are in DAMOE_LAYOUT_TILE32: W as the caller holds it, Q(x) quantised into the workspace by
// the call.  v_mfma_scale_f32_32x32x64_f8f6f4 multiplies a step of 64 columns: lane 32 h + r holds row r,
// columns 32 h .. + 31, one scale block, and takes its scale from a byte of a register.  Products and scales
// are exact (a product is a multiple of 2^-2 times the scales, at most 36), the sums are fp32.
#include "common.h"
#include "device.h"
#include "mxfp4.h"

namespace damoe {
namespace {

typedef int v8i __attribute__((ext_vector_type(8)));

struct LinearArgs {
  const uint8_t* w;   // tiles of N x K
  const uint8_t* x;   // tiles of T x K
  const void* add;
  void* y;
  int64_t ld_add, ldy;
  int32_t T, N, nk;   // nk: tiles along K
  int32_t y_bf;
};

// Both operands' fp4 codes fill the lower half of the instruction's 8-register operands.
template <int J>
__device__ __forceinline__ floatx16 mfma_fp4(const uint4& a, uint32_t sa, const uint4& b, uint32_t sb, const floatx16& c) {
  const v8i av = {(int)a.x, (int)a.y, (int)a.z, (int)a.w, 0, 0, 0, 0};
  const v8i bv = {(int)b.x, (int)b.y, (int)b.z, (int)b.w, 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(av, bv, c, 4, 4, J, (int)sa, J, (int)sb);
}

// A tile's operand registers of one lane: four steps and their scales.
struct Frag {
  uint4 q[4];
  uint32_t s;

  __device__ __forceinline__ void load(const uint8_t* tile, int lane) {
#pragma unroll
    for (int j = 0; j < 4; ++j) q[j] = *reinterpret_cast<const uint4*>(tile + 1024 * j + 16 * lane);
    s = *reinterpret_cast<const uint32_t*>(tile + kTileCodes + 4 * lane);
  }
};

__device__ __forceinline__ void mfma_tile(const Frag& a, const Frag& b, floatx16& c) {
  c = mfma_fp4<0>(a.q[0], a.s, b.q[0], b.s, c);
  c = mfma_fp4<1>(a.q[1], a.s, b.q[1], b.s, c);
  c = mfma_fp4<2>(a.q[2], a.s, b.q[2], b.s, c);
  c = mfma_fp4<3>(a.q[3], a.s, b.q[3], b.s, c);
}

__device__ __forceinline__ float load_elem(const void* p, int64_t i, bool bf) {
  return bf ? bf16_to_f32(static_cast<const uint16_t*>(p)[i]) : static_cast<const float*>(p)[i];
}

// Rows of W of a block of results: register 4 q + i of lane (r, g) is W row 8 q + 4 g + i, token r.
__device__ __forceinline__ void store_block(const LinearArgs& a, const floatx16& c, int64_t t, int n0, int g) {
  if (t >= a.T) return;
#pragma unroll
  for (int q = 0; q < 4; ++q)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int n = n0 + 8 * q + 4 * g + i;
      if (n >= a.N) continue;
      float v = c[4 * q + i];
      if (a.add) v += load_elem(a.add, t * a.ld_add + n, a.y_bf);
      if (a.y_bf) static_cast<uint16_t*>(a.y)[t * a.ldy + n] = __builtin_bit_cast(uint16_t, (__bf16)v);
      else static_cast<float*>(a.y)[t * a.ldy + n] = v;
    }
}

// A wave: 32 rows of W x 32 NT tokens.
template <int NT>
__global__ void __launch_bounds__(256) k_mxfp4_linear(LinearArgs a) {
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int rb = blockIdx.x * 4 + w, tb0 = blockIdx.y * NT;
  const int nrb = (a.N + 31) / 32, ntb = (a.T + 31) / 32;
  if (rb >= nrb) return;
  floatx16 c[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int i = 0; i < 16; ++i) c[n][i] = 0.f;
  for (int k = 0; k < a.nk; ++k) {
    Frag wf, xf[NT];
    wf.load(a.w + ((int64_t)rb * a.nk + k) * kTileBytes, lane);
#pragma unroll
    for (int n = 0; n < NT; ++n)  // blocks past the last repeat it; their results are not stored
      xf[n].load(a.x + ((int64_t)min(tb0 + n, ntb - 1) * a.nk + k) * kTileBytes, lane);
#pragma unroll
    for (int n = 0; n < NT; ++n) mfma_tile(wf, xf[n], c[n]);
  }
#pragma unroll
  for (int n = 0; n < NT; ++n) store_block(a, c[n], (int64_t)(tb0 + n) * 32 + (lane & 31), rb * 32, lane >> 5);
}

constexpr int32_t kMaxDim = 1 << 20;

bool linear_shape_ok(int32_t T, int32_t N, int32_t K) { return T >= 0 && N > 0 && K > 0; }

bool linear_range_ok(int32_t T, int32_t N, int32_t K) {
  return T <= DAMOE_MAX_T && N <= kMaxDim && K <= kMaxDim && K % 32 == 0 &&
         tiles_of(T, 32) * tiles_of(K, kTileCols) * kTileBytes < (int64_t)1 << 31 &&
         tiles_of(N, 32) * tiles_of(K, kTileCols) * kTileBytes < (int64_t)1 << 31;
}

size_t x_tiles_bytes(int32_t T, int32_t K) {
  return (size_t)tiles_of(T, kTileRows) * tiles_of(K, kTileCols) * kTileBytes;
}

}  // namespace
}  // namespace damoe

using namespace damoe;

extern "C" {

size_t damoe_mxfp4_linear_workspace_size(int32_t T_max, int32_t N, int32_t K) {
  if (!linear_shape_ok(T_max, N, K) || !linear_range_ok(T_max, N, K)) return 0;
  return std::max<size_t>(256, (x_tiles_bytes(T_max, K) + 255) / 256 * 256);
}

damoe_status damoe_mxfp4_linear(const void* x, int32_t xdtype, int64_t ldx, int32_t T, int32_t K, const uint8_t* w,
                                int32_t N, const void* add, int64_t ld_add, void* y, int32_t ydtype, int64_t ldy,
                                void* ws, size_t ws_bytes, hipStream_t stream) {
  if (!linear_shape_ok(T, N, K)) return DAMOE_ERR_INVALID_ARG;
  if (!linear_range_ok(T, N, K)) return DAMOE_ERR_UNSUPPORTED;
  if ((xdtype != DAMOE_BF16 && xdtype != DAMOE_F32) || (ydtype != DAMOE_BF16 && ydtype != DAMOE_F32))
    return DAMOE_ERR_UNSUPPORTED;
  if (ldx < K || ldy < N || (add && ld_add < N)) return DAMOE_ERR_INVALID_ARG;
  if (T == 0) return DAMOE_OK;
  if (!x || !w || !y || !ws) return DAMOE_ERR_INVALID_ARG;
  const uintptr_t xs = xdtype == DAMOE_BF16 ? 2 : 4, ys = ydtype == DAMOE_BF16 ? 2 : 4;
  if (reinterpret_cast<uintptr_t>(x) % xs || reinterpret_cast<uintptr_t>(y) % ys || reinterpret_cast<uintptr_t>(add) % ys ||
      reinterpret_cast<uintptr_t>(w) % 16 || reinterpret_cast<uintptr_t>(ws) % 16)
    return DAMOE_ERR_INVALID_ARG;
  if (ws_bytes < x_tiles_bytes(T, K)) return DAMOE_ERR_WORKSPACE;
  uint8_t* xt = static_cast<uint8_t*>(ws);
  if (launch_quantise_tiles(x, xdtype == DAMOE_BF16, T, K, ldx, xt, stream) != hipSuccess) return DAMOE_ERR_HIP;
  const LinearArgs a{w, xt, add, y, ld_add, ldy, T, N, (int32_t)tiles_of(K, kTileCols), ydtype == DAMOE_BF16};
  const int nt = T <= 32 ? 1 : 4;
  const dim3 grid((unsigned)tiles_of(N, 128), (unsigned)tiles_of(T, 32 * nt));
  if (nt == 1) hipLaunchKernelGGL(k_mxfp4_linear<1>, grid, dim3(256), 0, stream, a);
  else hipLaunchKernelGGL(k_mxfp4_linear<4>, grid, dim3(256), 0, stream, a);
  return hipGetLastError() == hipSuccess ? DAMOE_OK : DAMOE_ERR_HIP;
}

}  // extern "C"
