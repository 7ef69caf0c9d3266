// Rows sorted by expert and back: damoe_sort_rows, damoe_combine_rows and the gradient of the latter.
//
// With q(t, j) = inv_perm[t k + j] the place of slot j of token t:
//   sort     rows[q(t, j)] = w_tj x_t          combine     y_t = add_t + sum_j w_tj rows[q(t, j)]
//   combine's gradient: drows[q(t, j)] = w_tj dy_t, dw_tj = <dy_t, rows[q(t, j)]>
// Each is memory bound: a few operations for 16 bytes.  All of them go by tokens, so that the token's side (x, y, dy) is
// read or written once and only the sorted side k times, and so that no two waves touch one element.
#include "vec.h"

namespace damoe {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;

struct RowArgs {
  const void* x;  // the token's side: x, add or dy
  int64_t ldx;
  const float* w;
  const int32_t* inv_perm;
  void* rows;     // the sorted side
  int64_t ldr;
  void* out;      // y or drows
  int64_t ldo;
  float* dw;
  int32_t T, k, H, R;
  int32_t chunks;  // pieces of 64 x 16 bytes of a row
};

// The token's slots, one a lane: place (-1 where there is none) and factor.  at() and weight() take them from their lanes, which
// all have to be there: what is in the registers of a lane that has left is not laid down.
struct Slots {
  int place = -1;
  float factor = 1.f;

  __device__ __forceinline__ Slots(const RowArgs& a, int64_t t, int lane) {
    if (lane < a.k) {
      place = a.inv_perm[t * a.k + lane];
      if (a.w) factor = a.w[t * a.k + lane];
      if ((uint32_t)place >= (uint32_t)a.R) place = -1;
    }
  }
  __device__ __forceinline__ int at(int j) const { return __builtin_amdgcn_readlane(place, j); }
  __device__ __forceinline__ float weight(int j) const {
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, factor), j));
  }
};

// A wave's piece of work: 64 x 16 bytes of a token's row.
template <class F>
__device__ __forceinline__ void by_pieces(const RowArgs& a, F f) {
  const int64_t n = (int64_t)a.T * a.chunks, stride = (int64_t)gridDim.x * kWaves;
  int64_t i = (int64_t)blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  for (; i < n; i += stride) {
    const int64_t t = i / a.chunks;
    f(t, (int)(i - t * a.chunks));
  }
}

// First column of the lane's 16 bytes.  Lanes past the row's end, of which none may leave (Slots), have its last piece too and
// load and store the same there as the lane whose it is.
template <bool BF>
__device__ __forceinline__ int column(const RowArgs& a, int chunk, int lane) {
  constexpr int P = Elem<BF>::kPer16;
  return min((chunk * kWave + lane) * P, (a.H - 1) / P * P);
}

template <bool BF>
__device__ __forceinline__ uint4 scaled(uint4 v, float w) {
  float f[Elem<BF>::kPer16];
  unpack16<BF>(v, f);
#pragma unroll
  for (float& e : f) e *= w;
  return pack16<BF>(f);
}

// 8192 tokens to 8 x 7168 bf16: 198 us, 5.3 TB/s, a copy's rate (204 with stores past the caches).
template <bool BF>
__global__ void __launch_bounds__(kThreads) k_sort_rows(RowArgs a) {
  typedef typename Elem<BF>::T T;
  const int lane = threadIdx.x & 63;
  by_pieces(a, [&](int64_t t, int chunk) {
    const Slots s(a, t, lane);
    const int c = column<BF>(a, chunk, lane), n = a.H - c;
    const uint4 v = load_some<BF>(static_cast<const T*>(a.x) + t * a.ldx + c, n);
    for (int j = 0; j < a.k; ++j) {
      const int q = s.at(j);
      if (q < 0) continue;
      store_some<BF>(static_cast<T*>(a.rows) + (int64_t)q * a.ldr + c, n, a.w ? scaled<BF>(v, s.weight(j)) : v);
    }
  });
}

// Slots in order, in fp32; one rounding at the end.  Past the caches: 8192 tokens of 8 x 7168 bf16 199 us so (5.9 TB/s), 225
// with plain loads and stores.
template <bool BF>
__global__ void __launch_bounds__(kThreads) k_combine_rows(RowArgs a) {
  typedef typename Elem<BF>::T T;
  constexpr int P = Elem<BF>::kPer16;
  const int lane = threadIdx.x & 63;
  by_pieces(a, [&](int64_t t, int chunk) {
    const Slots s(a, t, lane);
    const int c = column<BF>(a, chunk, lane), n = a.H - c;
    uint4 v[DAMOE_MAX_K];
#pragma unroll
    for (int j = 0; j < DAMOE_MAX_K; ++j) {
      if (j < a.k && s.at(j) >= 0) v[j] = load_some<BF, true>(static_cast<const T*>(a.rows) + (int64_t)s.at(j) * a.ldr + c, n);
    }
    float sum[P] = {};
    if (a.x) unpack16<BF>(load_some<BF>(static_cast<const T*>(a.x) + t * a.ldx + c, n), sum);
#pragma unroll
    for (int j = 0; j < DAMOE_MAX_K; ++j) {
      if (j >= a.k || s.at(j) < 0) continue;
      float f[P];
      unpack16<BF>(v[j], f);
      const float w = s.weight(j);
#pragma unroll
      for (int i = 0; i < P; ++i) sum[i] = fmaf(w, f[i], sum[i]);
    }
    store_some<BF, true>(static_cast<T*>(a.out) + t * a.ldo + c, n, pack16<BF>(sum));
  });
}

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
  return v;
}

// A block takes a token over its whole row: each lane's products in fp32, then the wave's lanes by exchanges, then the waves
// in order.  8192 tokens of 8 x 7168 bf16: 394 us, 5.1 TB/s, half of it written.  At most 128 registers (four waves a SIMD): with 130
// 8192 tokens of 8 x 520 took 68 us for 55.
template <bool BF>
__global__ void __launch_bounds__(kThreads, 4) k_combine_rows_grad(RowArgs a) {
  typedef typename Elem<BF>::T T;
  constexpr int P = Elem<BF>::kPer16;
  __shared__ float part[kWaves][DAMOE_MAX_K];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  for (int64_t t = blockIdx.x; t < a.T; t += gridDim.x) {
    const Slots s(a, t, lane);
    float acc[DAMOE_MAX_K] = {};
    for (int chunk = wave; chunk < a.chunks; chunk += kWaves) {
      const int c = column<BF>(a, chunk, lane), n = a.H - c;
      const bool mine = c == (chunk * kWave + lane) * P;
      const uint4 d = load_some<BF>(static_cast<const T*>(a.x) + t * a.ldx + c, n);
      uint4 v[DAMOE_MAX_K];
      if (a.dw) {
#pragma unroll
        for (int j = 0; j < DAMOE_MAX_K; ++j) {
          if (j < a.k && s.at(j) >= 0) v[j] = load_some<BF, true>(static_cast<const T*>(a.rows) + (int64_t)s.at(j) * a.ldr + c, n);
        }
      }
      float f[P];
      unpack16<BF>(d, f);
#pragma unroll
      for (int j = 0; j < DAMOE_MAX_K; ++j) {
        if (j >= a.k || s.at(j) < 0) continue;
        if (a.dw) {
          float g[P], sum = acc[j];
          unpack16<BF>(v[j], g);
#pragma unroll
          for (int i = 0; i < P; ++i) sum = fmaf(f[i], g[i], sum);
          acc[j] = mine ? sum : acc[j];
        }
        if (a.out) store_some<BF, true>(static_cast<T*>(a.out) + (int64_t)s.at(j) * a.ldo + c, n, a.w ? scaled<BF>(d, s.weight(j)) : d);
      }
    }
    if (!a.dw) continue;
#pragma unroll
    for (int j = 0; j < DAMOE_MAX_K; ++j) {
      if (j >= a.k) continue;
      const float v = wave_sum(acc[j]);
      if (lane == 0) part[wave][j] = v;
    }
    __syncthreads();
    if ((int)threadIdx.x < a.k) {
      float v = 0.f;
#pragma unroll
      for (int i = 0; i < kWaves; ++i) v += part[i][threadIdx.x];
      a.dw[t * a.k + threadIdx.x] = v;
    }
    __syncthreads();
  }
}

// The same for few rows, where blocks of tokens would not fill the card: a wave takes a slot, eight pieces of its row at once.  509
// tokens of 8 x 2048 fp32: 14.1 us, 5.0 TB/s (24.0 by blocks of four waves a slot).
template <bool BF>
__global__ void __launch_bounds__(kThreads) k_combine_rows_grad_slots(RowArgs a) {
  typedef typename Elem<BF>::T T;
  constexpr int P = Elem<BF>::kPer16, N = 8;
  const int lane = threadIdx.x & 63;
  const int64_t slot = (int64_t)blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (slot >= (int64_t)a.T * a.k) return;
  const int64_t t = slot / a.k;
  const int place = a.inv_perm[slot];
  const float w = a.w ? a.w[slot] : 1.f;
  if ((uint32_t)place >= (uint32_t)a.R) {
    if (a.dw && lane == 0) a.dw[slot] = 0.f;
    return;
  }
  const T* x = static_cast<const T*>(a.x) + t * a.ldx;
  const T* row = static_cast<const T*>(a.rows) + place * a.ldr;
  T* out = static_cast<T*>(a.out) + place * a.ldo;
  float acc = 0.f;
  for (int chunk = 0; chunk < a.chunks; chunk += N) {
    uint4 d[N], v[N];
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int c = ((chunk + j) * kWave + lane) * P, n = a.H - c;
      d[j] = v[j] = uint4{0, 0, 0, 0};
      if (n <= 0) continue;
      d[j] = load_some<BF>(x + c, n);
      if (a.dw) v[j] = load_some<BF>(row + c, n);
    }
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int c = ((chunk + j) * kWave + lane) * P, n = a.H - c;
      if (n <= 0) continue;
      if (a.dw) {
        float f[P], g[P];
        unpack16<BF>(d[j], f);
        unpack16<BF>(v[j], g);
#pragma unroll
        for (int i = 0; i < P; ++i) acc = fmaf(f[i], g[i], acc);
      }
      if (a.out) store_some<BF>(out + c, n, a.w ? scaled<BF>(d[j], w) : d[j]);
    }
  }
  if (!a.dw) return;
  acc = wave_sum(acc);
  if (lane == 0) a.dw[slot] = acc;
}

// ---------------------------------------------------------------- launches

// Blocks of a launch at most; beyond them they go on in strides.
constexpr int64_t kMaxBlocks = 1 << 22;

// Bytes of rows below which combine's gradient goes by slots.  By tokens / by slots, us, k = 8: 509 x 2048 fp32 (33 MB) 17.0 /
// 14.5, 1500 x 1024 bf16 (25 MB) 15.7 / 13.0; 700 x 2048 fp32 (46 MB) 22.4 / 31.5, 509 x 7168 bf16 (58 MB) 27.5 / 29.1.  Next to the
// border: 340 x 7168 bf16 (39 MB) 23.2 / 20.9, 640 x 2048 fp32 (42 MB) 22.0 / 23.7, 400 x 7168 bf16 (46 MB) 24.3 / 26.9; with
// shorter rows or fewer slots the slots stay faster (6000 x 512 bf16, 49 MB, 39.4 / 32.0).  Masked slots count as rows.
constexpr int64_t kFewBytes = 40 << 20;

bool shape_ok(int32_t T, int32_t k, int32_t H, int32_t R) {
  return T >= 0 && T <= DAMOE_MAX_T && k >= 1 && k <= DAMOE_MAX_K && H >= 1 && R >= 0;
}

damoe_status check(int32_t T, int32_t k, int32_t H, int32_t R, int32_t dtype) {
  if (!shape_ok(T, k, H, R)) return DAMOE_ERR_INVALID_ARG;
  if (dtype != DAMOE_BF16 && dtype != DAMOE_F32) return DAMOE_ERR_UNSUPPORTED;
  return H > DAMOE_MAX_COLS ? DAMOE_ERR_UNSUPPORTED : DAMOE_OK;
}

// A matrix whose rows are at least as long as the call's, at its element's alignment.
bool matrix_ok(const void* p, int64_t ld, int32_t H, int32_t dtype) {
  return p && ld >= H && reinterpret_cast<uintptr_t>(p) % (dtype == DAMOE_BF16 ? 2 : 4) == 0;
}

bool words_ok(const void* p) { return reinterpret_cast<uintptr_t>(p) % 4 == 0; }

int32_t chunks_of(int32_t H, int32_t dtype) {
  const int32_t n = kWave * (dtype == DAMOE_BF16 ? 8 : 4);
  return (H + n - 1) / n;
}

unsigned blocks_for(int64_t n) { return (unsigned)std::max<int64_t>(1, std::min(kMaxBlocks, n)); }

damoe_status last() { return hipGetLastError() == hipSuccess ? DAMOE_OK : DAMOE_ERR_HIP; }

}  // namespace
}  // namespace damoe

using namespace damoe;

extern "C" {

damoe_status damoe_sort_rows(const void* x, int32_t dtype, int64_t ldx, const float* w, const int32_t* inv_perm, int32_t T,
                             int32_t k, int32_t H, int32_t R, void* rows, int64_t ld_rows, hipStream_t stream) {
  if (const damoe_status s = check(T, k, H, R, dtype)) return s;
  if (T == 0 || R == 0) return DAMOE_OK;
  if (!matrix_ok(x, ldx, H, dtype) || !matrix_ok(rows, ld_rows, H, dtype) || !inv_perm || !words_ok(inv_perm) || !words_ok(w))
    return DAMOE_ERR_INVALID_ARG;
  RowArgs a{x, ldx, w, inv_perm, rows, ld_rows, nullptr, 0, nullptr, T, k, H, R, chunks_of(H, dtype)};
  const dim3 grid(blocks_for(((int64_t)T * a.chunks + kWaves - 1) / kWaves));
  if (dtype == DAMOE_BF16) hipLaunchKernelGGL(k_sort_rows<true>, grid, dim3(kThreads), 0, stream, a);
  else hipLaunchKernelGGL(k_sort_rows<false>, grid, dim3(kThreads), 0, stream, a);
  return last();
}

damoe_status damoe_combine_rows(const void* rows, int32_t dtype, int64_t ld_rows, const float* w, const int32_t* inv_perm,
                                int32_t T, int32_t k, int32_t H, int32_t R, const void* add, int64_t ld_add, void* y, int64_t ldy,
                                hipStream_t stream) {
  if (const damoe_status s = check(T, k, H, R, dtype)) return s;
  if (T == 0) return DAMOE_OK;
  if ((R > 0 && !matrix_ok(rows, ld_rows, H, dtype)) || !matrix_ok(y, ldy, H, dtype) || (add && !matrix_ok(add, ld_add, H, dtype)) ||
      (add == y && ld_add != ldy) || !inv_perm || !words_ok(inv_perm) || !words_ok(w))
    return DAMOE_ERR_INVALID_ARG;
  RowArgs a{add, ld_add, w, inv_perm, const_cast<void*>(rows), ld_rows, y, ldy, nullptr, T, k, H, R, chunks_of(H, dtype)};
  const dim3 grid(blocks_for(((int64_t)T * a.chunks + kWaves - 1) / kWaves));
  if (dtype == DAMOE_BF16) hipLaunchKernelGGL(k_combine_rows<true>, grid, dim3(kThreads), 0, stream, a);
  else hipLaunchKernelGGL(k_combine_rows<false>, grid, dim3(kThreads), 0, stream, a);
  return last();
}

damoe_status damoe_combine_rows_grad(const void* dy, int32_t dtype, int64_t ldy, const void* rows, int64_t ld_rows, const float* w,
                                     const int32_t* inv_perm, int32_t T, int32_t k, int32_t H, int32_t R, void* drows,
                                     int64_t ld_drows, float* dw, hipStream_t stream) {
  if (const damoe_status s = check(T, k, H, R, dtype)) return s;
  if (T == 0 || (!drows && !dw)) return DAMOE_OK;
  if (!matrix_ok(dy, ldy, H, dtype) || (dw && R > 0 && !matrix_ok(rows, ld_rows, H, dtype)) ||
      (drows && R > 0 && !matrix_ok(drows, ld_drows, H, dtype)) || (drows && drows == rows && dw && ld_drows != ld_rows) || !inv_perm ||
      !words_ok(inv_perm) || !words_ok(w) || !words_ok(dw))
    return DAMOE_ERR_INVALID_ARG;
  RowArgs a{dy, ldy, w, inv_perm, const_cast<void*>(rows), ld_rows, drows, ld_drows, dw, T, k, H, R, chunks_of(H, dtype)};
  const bool slots = (int64_t)T * k * H * (dtype == DAMOE_BF16 ? 2 : 4) < kFewBytes;
  const dim3 grid(slots ? (unsigned)(((int64_t)T * k + kWaves - 1) / kWaves) : blocks_for(T));
  const auto kernel = dtype == DAMOE_BF16 ? (slots ? k_combine_rows_grad_slots<true> : k_combine_rows_grad<true>)
                                          : (slots ? k_combine_rows_grad_slots<false> : k_combine_rows_grad<false>);
  hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, stream, a);
  return last();
}

}  // extern "C"
