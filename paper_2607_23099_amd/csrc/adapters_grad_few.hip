// damoe_adapters_grad for few rows: dx, dA and dB in one launch behind `down`.
#include "adapters_outer.h"

namespace damoe {
namespace {

// Rows up to which a segment is one chunk of `outer`, so that nothing is left to be joined, and g's parts are added where
// they are used.
constexpr int32_t kFewRows = 1024;

// Blocks in turn: dB and dA (tiles of columns x segments x blocks of ranks), dx (tiles of places x columns), and for the
// zeros of segments without rows.
struct RestArgs {
  OuterArgs b, a;
  UpArgs x;
  int32_t columns_b, columns_a, columns_x;  // tiles
  int32_t segments, ranks;                  // of each matrix: segments with rows at most, blocks of ranks
  int32_t end_b, end_a, end_x;              // numbers of blocks, each with those before it
  int32_t zero_blocks;                      // of a segment
};

constexpr int kZeros = 32 * kOuterWaves * kWave;  // elements of a block

__device__ __forceinline__ void clear(float* p, int64_t size, int64_t at) {
  const int64_t end = min(size, at + kZeros);
  for (int64_t i = at + threadIdx.x; i < end; i += kOuterWaves * kWave) p[i] = 0.f;
}

template <bool BF, bool WB, int RB>
__global__ void __launch_bounds__(kOuterWaves* kWave) k_adapter_grad_rest(RestArgs r) {
  constexpr int OR = RB >= 2 ? 2 : 1;  // blocks of 16 ranks of `outer`
  typedef Outer<BF, true, OR, false, true> B;
  typedef Outer<BF, false, OR, false, true> A;
  typedef UpJoin<BF, WB, true, RB> X;
  constexpr int kBytes = std::max<int>(B::kLds * 4, X::kSums + kUpWaves * X::kRuns);
  __shared__ __align__(16) char lds[kBytes];
  int n = blockIdx.x;
  Tile tile;
  if (n < r.end_a) {
    const bool is_b = n < r.end_b;
    const OuterArgs& o = is_b ? r.b : r.a;
    const int columns = is_b ? r.columns_b : r.columns_a;
    n -= is_b ? 0 : r.end_b;
    const int column = n % columns, rest = n / columns;
    if (!find_tile<false>(o.off, o.L, o.T, o.chunk, rest / r.ranks, tile)) return;
    const int b0 = column * OuterTile<BF>::kCols, r0 = rest % r.ranks * 16 * OR;
    if (is_b) B::run(r.b, tile, b0, r0, reinterpret_cast<float*>(lds));
    else A::run(r.a, tile, b0, r0, reinterpret_cast<float*>(lds));
  } else if (n < r.end_x) {
    n -= r.end_a;
    if (!find_tile<false>(r.x.off, r.x.L, r.x.T, 16, n / r.columns_x, tile)) return;
    const int c0 = (n % r.columns_x * kUpWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6)) * X::U::kCols;
    X::run(r.x, tile, c0, false, lds);
  } else {
    n -= r.end_x;
    const int l = n / r.zero_blocks;
    const Length s(r.a.off, r.a.L, r.a.T, 1, l);
    if (s.n) return;
    const int64_t size_a = (int64_t)r.a.r * r.a.C, size_b = (int64_t)r.b.r * r.b.C, at = (int64_t)(n % r.zero_blocks) * kZeros;
    clear(r.a.out + l * size_a, size_a, at);
    clear(r.b.out + l * size_b, size_b, at);
  }
}

}  // namespace

bool adapters_grad_few(int32_t T, int32_t L, int32_t r, int32_t K, int32_t N, int32_t xdtype, int32_t ydtype) {
  // `outer` takes 16 bytes of a row at least; one grid has all blocks.
  const int64_t zeros = ((int64_t)r * std::max(K, N) / kZeros + 1) * L, tiles = (int64_t)((K + N) / 64 + 2) * std::min(T, L) * 2;
  return T <= kFewRows && r <= 64 && xdtype == ydtype && std::min(K, N) >= 8 && zeros + tiles <= 1 << 22;
}

hipError_t adapters_grad_in_one(const OuterArgs& b, const OuterArgs& a, UpArgs x, int32_t dtype, int32_t wdtype, hipStream_t stream) {
  const auto go = [&](auto rb) {
    return by_types(dtype, wdtype, [&](auto bf, auto wb) {
      constexpr bool BF = decltype(bf)::value, WB = decltype(wb)::value;
      constexpr int RB = decltype(rb)::value;
      constexpr int kCols = OuterTile<BF>::kCols, kUp = kUpWaves * Up<BF, WB, RB>::kCols;
      const auto tiles = [](int32_t n, int32_t per) { return (n + per - 1) / per; };
      RestArgs r{b, a, x};
      r.columns_b = tiles(b.C, kCols), r.columns_a = tiles(a.C, kCols), r.columns_x = tiles(a.C, kUp);
      r.segments = std::min(a.T, a.L), r.ranks = tiles(a.r, RB >= 2 ? 32 : 16);
      r.end_b = r.columns_b * r.segments * r.ranks;
      r.end_a = r.end_b + r.columns_a * r.segments * r.ranks;
      r.end_x = r.end_a + (x.y ? r.columns_x * (int32_t)most_tiles(a.T, a.L, 16) : 0);
      r.zero_blocks = (int32_t)(((int64_t)a.r * std::max(a.C, b.C) + kZeros - 1) / kZeros);
      const unsigned zeros = a.accumulate ? 0 : (unsigned)r.zero_blocks * a.L;
      hipLaunchKernelGGL((k_adapter_grad_rest<BF, WB, RB>), dim3(r.end_x + zeros), dim3(kOuterWaves * kWave), 0, stream, r);
      return hipGetLastError();
    });
  };
  return a.r <= 8 ? go(std::integral_constant<int, 0>{}) : by_rank<4>(a.rp, go);
}

}  // namespace damoe
