// damoe_adapters_grad's dx, dA and dB in one launch: for few rows behind `down`, else behind `sums`.
#include "adapters_outer.h"

namespace damoe {
namespace {

// Rows up to which a segment is one chunk of `outer`, so that nothing is left to be joined, and g's parts are added where
// they are used.  So / in chunks behind `sums`, us, bf16, 7168 to 4096: one adapter of rank 32, 512 rows 23.4 / 25.5, 1024 36.0 / 34.7,
// 2048 72.7 / 53.3; of rank 8, 1024 rows 24.9 / 30.0, 2048 53.4 / 42.4; 8 adapters of rank 32, 2048 rows 55.7 / 65.5.  2048 to 2048,
// one adapter of rank 32: 300 rows 18.1 / 18.0, 1024 33.4 / 20.8.
constexpr int32_t kFewRows = 1024;

// dB and dA (tiles of columns x tiles of places x blocks of ranks), dx (tiles of places x columns), and of few rows the zeros
// of segments without any.
struct RestArgs {
  OuterArgs b, a;
  UpArgs x;
  int32_t columns_b, columns_a, columns_x;  // tiles of columns
  int32_t ranks;                            // blocks of ranks
  int32_t blocks_b, outer, blocks_x;        // blocks of dB, of dB and dA, of dx
  int32_t zero_blocks;                      // of a segment
};

constexpr int kZeros = 32 * kOuterWaves * kWave;  // elements of a block

__device__ __forceinline__ void clear(float* p, int64_t size, int64_t at) {
  const int64_t end = min(size, at + kZeros);
  for (int64_t i = at + threadIdx.x; i < end; i += kOuterWaves * kWave) p[i] = 0.f;
}

// FEW: a segment is one chunk, and g's parts are added where they are used.  Else u and g are as `sums` laid them out.  One
// launch, so that the last blocks of a kind, which add up their waves' sums, run beside the next kind's streams: 8192 rows of
// 7168 and 4096 columns at rank 32 94 us, 107 in three launches (4.5 TB/s; blocks of the kinds in turn 96).
template <bool BF, bool WB, int RB, bool FEW>
__global__ void __launch_bounds__(kOuterWaves* kWave, FEW ? 1 : 2) k_adapter_grad_rest(RestArgs r) {
  constexpr int OR = RB >= 2 ? 2 : 1;  // blocks of 16 ranks of `outer`
  typedef Outer<BF, true, OR, false, FEW> B;
  typedef Outer<BF, false, OR, false, FEW> A;
  typedef UpJoin<BF, WB, true, RB> Join;
  typedef UpStream<BF, WB, true, RB> Stream;
  constexpr int kBytes = FEW ? std::max<int>(B::kLds * 4, Join::kSums + kUpWaves * Join::kRuns) : B::kLds * 4;
  __shared__ __align__(16) char lds[kBytes];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int n = blockIdx.x;
  const bool x = n >= r.outer;
  n -= x ? r.outer : 0;
  Tile tile;
  if (!x) {
    const bool is_b = n < r.blocks_b;
    const int columns = is_b ? r.columns_b : r.columns_a;
    n -= is_b ? 0 : r.blocks_b;
    const int column = n % columns, rest = n / columns;
    if (!find_tile<!FEW>(r.a.off, r.a.L, r.a.T, is_b ? r.b.chunk : r.a.chunk, rest / r.ranks, tile)) return;
    const int b0 = column * OuterTile<BF>::kCols, r0 = rest % r.ranks * 16 * OR;
    if (is_b) B::run(r.b, tile, b0, r0, reinterpret_cast<float*>(lds));
    else A::run(r.a, tile, b0, r0, reinterpret_cast<float*>(lds));
  } else if (n < r.blocks_x) {
    if (!find_tile<false>(r.x.off, r.x.L, r.x.T, r.x.places, n / r.columns_x, tile)) return;
    const int c0 = (n % r.columns_x * kUpWaves + wave) * Stream::U::kCols;
    if constexpr (FEW) Join::run(r.x, tile, c0, false, lds);
    else Stream::run(r.x, tile, c0, nullptr);
  } else {
    n -= r.blocks_x;
    const int l = n / r.zero_blocks;
    const Length s(r.a.off, r.a.L, r.a.T, 1, l);
    if (s.n) return;
    const int64_t size_a = (int64_t)r.a.r * r.a.C, size_b = (int64_t)r.b.r * r.b.C, at = (int64_t)(n % r.zero_blocks) * kZeros;
    clear(r.a.out + l * size_a, size_a, at);
    clear(r.b.out + l * size_b, size_b, at);
  }
}

// Blocks of 256 threads that one grid may have.
constexpr int64_t kMostBlocks = 1 << 22;

}  // namespace

bool adapters_grad_few(int32_t T, int32_t L, int32_t r, int32_t K, int32_t N, int32_t xdtype, int32_t ydtype) {
  // `outer` takes 16 bytes of a row at least.
  const int64_t zeros = ((int64_t)r * std::max(K, N) / kZeros + 1) * L, tiles = (int64_t)((K + N) / 64 + 2) * std::min(T, L) * 2;
  return T <= kFewRows && r <= 64 && xdtype == ydtype && std::min(K, N) >= 8 && zeros + tiles <= kMostBlocks;
}

bool adapters_grad_joined(int32_t T, int32_t L, int32_t r, int32_t K, int32_t N, int32_t xdtype, int32_t ydtype) {
  const int64_t tiles = (int64_t)((K + N) / 64 + 2) * (most_tiles(T, L, 128) + most_tiles(T, L, up_places(T)));
  return r <= 32 && xdtype == ydtype && std::min(K, N) >= 8 && tiles <= kMostBlocks;
}

hipError_t adapters_grad_in_one(const OuterArgs& b, const OuterArgs& a, UpArgs x, bool few, int32_t dtype, int32_t wdtype,
                                hipStream_t stream) {
  const auto go = [&](auto rb, auto is_few) {
    return by_types(dtype, wdtype, [&](auto bf, auto wb) {
      constexpr bool BF = decltype(bf)::value, WB = decltype(wb)::value, FEW = decltype(is_few)::value;
      constexpr int RB = decltype(rb)::value;
      constexpr int kCols = OuterTile<BF>::kCols, kUp = kUpWaves * Up<BF, WB, RB>::kCols;
      const auto tiles = [](int32_t n, int32_t per) { return (n + per - 1) / per; };
      RestArgs r{b, a, x};
      r.x.places = FEW ? 16 : up_places(a.T);
      r.columns_b = tiles(b.C, kCols), r.columns_a = tiles(a.C, kCols), r.columns_x = tiles(a.C, kUp);
      r.ranks = tiles(a.r, RB >= 2 ? 32 : 16);
      r.blocks_b = r.columns_b * (int32_t)most_tiles(a.T, a.L, b.chunk) * r.ranks;
      r.outer = r.blocks_b + r.columns_a * (int32_t)most_tiles(a.T, a.L, a.chunk) * r.ranks;
      r.blocks_x = x.y ? r.columns_x * (int32_t)most_tiles(a.T, a.L, r.x.places) : 0;
      r.zero_blocks = (int32_t)(((int64_t)a.r * std::max(a.C, b.C) + kZeros - 1) / kZeros);
      const unsigned zeros = !FEW || a.accumulate ? 0 : (unsigned)r.zero_blocks * a.L;
      hipLaunchKernelGGL((k_adapter_grad_rest<BF, WB, RB, FEW>), dim3(r.outer + r.blocks_x + zeros), dim3(kOuterWaves * kWave), 0, stream,
                         r);
      return hipGetLastError();
    });
  };
  const std::integral_constant<int, 0> eight;
  const std::integral_constant<int, 1> one;
  const std::integral_constant<int, 2> two;
  if (few) {
    const auto g = [&](auto rb) { return go(rb, std::true_type{}); };
    return a.r <= 8 ? g(eight) : by_rank<4>(a.rp, g);
  }
  const std::false_type many;
  return a.r <= 8 ? go(eight, many) : a.r <= 16 ? go(one, many) : go(two, many);
}

}  // namespace damoe
