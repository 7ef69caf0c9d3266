// damoe_adapters: y = add + s B (A x) with a pair (A, B) for each segment of rows.
#include "adapters.h"

namespace damoe {
namespace {

// Few places: `down` and `up` in one launch.  A block takes a tile of at most 16 places and W x Up::kCols columns of y, and
// has the tile's u for itself, by W waves over K; blocks of other columns make it again.
template <bool XB, bool YB, bool WB, int RB, int W>
__global__ void __launch_bounds__(W* kWave) k_adapter_both(DownArgs a, UpArgs b) {
  constexpr int kSets = RB ? RB : 1, kRanks = 16 * kSets;
  typedef Down<XB, WB, kRows, kSets, 1, W> D;
  typedef Up<YB, WB, RB> U;
  typedef Ready<WB> R;
  __shared__ floatx4 red[D::kLds];
  __shared__ __align__(16) char lds[16 * kRanks * R::kBytes];
  __shared__ __align__(16) char runs[W * U::Weights::kLds];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int i = lane & 15, g = lane >> 4;
  Tile tile;
  if (!find_tile<false>(a.off, a.L, a.T, a.places, blockIdx.x, tile)) return;
  const int c0 = (blockIdx.y * W + wave) * U::kCols;
  const float s = b.scale ? b.scale[tile.l] : 1.f;
  D d;
  d.run(a, tile, 0, a.units, 0);
  d.put(red);
  const Places places(a.perm, a.off);
  const int p = min(tile.lo + i, tile.hi - 1), row = places.row(places.load(p), p);
  U v;
  typename U::Weights w;
  if (c0 < b.C) {
    w.template load<false>(b, tile.l, c0, runs + wave * U::Weights::kLds);
    v.rows(tile.lo + i < tile.hi && (uint32_t)row < (uint32_t)a.T ? row : -1);
    v.template load_add<false>(b, nullptr, c0);
  }
  __syncthreads();
  for (int e = threadIdx.x; e < 16 * 4 * kSets; e += W * kWave) {
    const int q = e % (4 * kSets), at = e / (4 * kSets), rho = 4 * q;
    floatx4 f = D::value(red, at, q);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (rho + k >= a.r) f[k] = 0.f;
      else if (a.u && blockIdx.y == 0 && tile.lo + at < tile.hi) a.u[(int64_t)(tile.lo + at) * a.r + rho + k] = f[k];
    }
    R::put(lds, 16, at, rho, kRanks, f);
  }
  __syncthreads();
  if (c0 >= b.C) return;
  v.u.load(lds, 16, i, kRanks, g);
  v.template work<false>(b, w, c0, s);
}

// Whether the u that blocks make again costs less than a second launch: the bytes of A that all blocks read, and one.
constexpr int64_t kBothBytes = 10 << 20, kBothBlock = 256 << 10;

constexpr int kBothWaves = 8;

int32_t both_columns(int32_t ydtype) { return kBothWaves * 16 * (ydtype == DAMOE_BF16 ? 8 : 4); }

bool both_pays(int32_t T, int32_t L, int32_t rp, int32_t K, int32_t N, int32_t ydtype, int32_t wdtype) {
  const int32_t cols = both_columns(ydtype);
  const int64_t one = (int64_t)rp * K * (wdtype == DAMOE_BF16 ? 2 : 4);
  return rp <= 64 && one <= kBothBlock && one * most_tiles(T, L, 16) * ((N + cols - 1) / cols) <= kBothBytes;
}

hipError_t both(DownArgs a, const UpArgs& b, int32_t xdtype, int32_t wdtype, int32_t ydtype, hipStream_t stream) {
  a.places = 16;
  a.units = (a.C + kUnit - 1) / kUnit;
  const int32_t cols = both_columns(ydtype);
  const dim3 grid((unsigned)most_tiles(a.T, a.L, 16), (b.C + cols - 1) / cols);
  const auto go = [&](auto rb) {
    return by_types(xdtype, wdtype, [&](auto xb, auto wb) {
      constexpr int RB = decltype(rb)::value, W = kBothWaves;
      constexpr bool XB = decltype(xb)::value, WB = decltype(wb)::value;
      const auto kernel = ydtype == DAMOE_BF16 ? k_adapter_both<XB, true, WB, RB, W> : k_adapter_both<XB, false, WB, RB, W>;
      hipLaunchKernelGGL(kernel, grid, dim3(W * kWave), 0, stream, a, b);
      return hipGetLastError();
    });
  };
  return a.r <= 8 ? go(std::integral_constant<int, 0>{}) : by_rank<4>(a.rp, go);
}

}  // namespace
}  // namespace damoe

using namespace damoe;

extern "C" {

size_t damoe_adapters_workspace_size(int32_t T_max, int32_t L, int32_t r, int32_t K, int32_t N) {
  if (check(T_max, L, r, K, N, DAMOE_F32, DAMOE_F32, DAMOE_F32)) return 0;
  const int32_t rp = padded_rank(r);
  return 256 + std::max(most_parts(T_max, K, rp), ready_bytes(T_max, rp) + kSpare);
}

damoe_status damoe_adapters(const void* x, int32_t xdtype, int64_t ldx, const int32_t* perm, const int32_t* offsets, int32_t T,
                            int32_t L, const void* a, const void* b, int32_t wdtype, int32_t r, int32_t K, int32_t N,
                            const float* scale, const void* add, int64_t ld_add, void* y, int32_t ydtype, int64_t ldy, float* u,
                            void* ws, size_t ws_bytes, hipStream_t stream) {
  if (const damoe_status s = check(T, L, r, K, N, xdtype, wdtype, ydtype)) return s;
  if (T == 0) return DAMOE_OK;
  if (!matrix_ok(x, ldx, K, xdtype) || !matrix_ok(y, ldy, N, ydtype) || (add && !matrix_ok(add, ld_add, N, ydtype)) ||
      (add == y && ld_add != ldy) || !offsets || !a || !b || !aligned(a, wdtype) || !aligned(b, wdtype) || !aligned(perm, DAMOE_F32) ||
      !aligned(offsets, DAMOE_F32) || !aligned(scale, DAMOE_F32) || !aligned(u, DAMOE_F32) || !ws ||
      reinterpret_cast<uintptr_t>(ws) % 16)
    return DAMOE_ERR_INVALID_ARG;
  const int32_t rp = padded_rank(r);
  if (both_pays(T, L, rp, K, N, ydtype, wdtype)) {
    const DownArgs da{x, ldx, a, perm, offsets, nullptr, nullptr, nullptr, u, L, T, K, r, rp, 0, 0};
    const UpArgs ua{nullptr, nullptr, 1, nullptr, b, scale, perm, offsets, add, ld_add, y, ldy, nullptr, L, T, N, r, rp, 0};
    return both(da, ua, xdtype, wdtype, ydtype, stream) == hipSuccess ? DAMOE_OK : DAMOE_ERR_HIP;
  }
  const DownPlan d = down_plan(T, K);
  const bool join = T < kManyRows;
  if (ws_bytes < (join ? part_bytes(d, T, rp) : ready_bytes(T, rp) + kSpare)) return DAMOE_ERR_WORKSPACE;
  float* part = join ? static_cast<float*>(ws) : nullptr;
  const DownArgs da{x, ldx, a, perm, offsets, nullptr, part, ws, u, L, T, K, r, rp, 0, 0};
  // `up` takes thirds where the weights are bf16, `down` leaves them there too.
  if (down<false>(da, d, xdtype, wdtype, stream) != hipSuccess) return DAMOE_ERR_HIP;
  const UpArgs ua{part, ws, d.parts, u, b, scale, perm, offsets, add, ld_add, y, ldy, static_cast<char*>(ws) + ready_bytes(T, rp),
                  L, T, N, r, rp, 0};
  const hipError_t e = join ? up<false, true>(ua, ydtype, wdtype, stream) : up<false, false>(ua, ydtype, wdtype, stream);
  return e == hipSuccess ? DAMOE_OK : DAMOE_ERR_HIP;
}

}  // extern "C"
