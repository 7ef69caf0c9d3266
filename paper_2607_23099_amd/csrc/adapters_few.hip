// damoe_adapters for few places, in one launch.
#include "adapters.h"

namespace damoe {
namespace {

// Few places: `down` and `up` in one launch.  A block takes a tile of at most 16 places and W x Up::kCols columns of y, and
// has the tile's u for itself, by W waves over K; blocks of other columns make it again.  Bound by one CU's loads of A: one row
// of 7168 to 4096 columns at rank 16 9.4 us, of 512 to 512 4.5.
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

// Whether the u that blocks make again costs less than a second launch, by the bytes of A that all blocks read and that one
// does.  Captured calls in one launch / in two, us: L = 48, r = 16, 7168 x 2048, 16 rows (7 MB) 6.6 / 8.4, 61 rows (22 MB) 12.0 /
// 9.4; L = 4, r = 32, 2048 x 2048, 256 rows (5 MB) 9.5 / 10.5, 2048 rows (34 MB) 20.0 / 17.5; L = 8, r = 16, 4096 x 7168, 61
// rows (10 MB) 13.7 / 8.3, one row (229 KB a block) 10.0 / 7.8, which a launch of 3 us on the host turns round (9.3 / 11.0 from
// Python).  B and the rows are not counted: L = 1, r = 16, 64 x 4096, 2048 rows 14.4 / 14.2, 8192 rows (4 MB of A) 55.6 / 31.5.
constexpr int64_t kBothBytes = 8 << 20, kBothBlock = 256 << 10;

constexpr int kBothWaves = 8;

int32_t both_columns(int32_t ydtype) { return kBothWaves * 16 * (ydtype == DAMOE_BF16 ? 8 : 4); }

}  // namespace

bool adapters_few(int32_t T, int32_t L, int32_t rp, int32_t K, int32_t N, int32_t ydtype, int32_t wdtype) {
  const int32_t cols = both_columns(ydtype);
  const int64_t one = (int64_t)rp * K * (wdtype == DAMOE_BF16 ? 2 : 4);
  return rp <= 64 && one <= kBothBlock && one * most_tiles(T, L, 16) * ((N + cols - 1) / cols) <= kBothBytes;
}

hipError_t adapters_in_one(DownArgs a, const UpArgs& b, int32_t xdtype, int32_t wdtype, int32_t ydtype, hipStream_t stream) {
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

}  // namespace damoe
