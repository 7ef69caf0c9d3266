// damoe_adapters_grad: the gradient of y = add + s B (A x) with respect to x, A and B of each segment.
#include "adapters_outer.h"

namespace damoe {
namespace {

// ---------------------------------------------------------------- sums

// Sum of the parts of one value, in order, with eight loads in flight.
__device__ __forceinline__ float add_parts(const float* p, int64_t apart, int n) {
  float v = 0.f;
  for (int k = 0; k < n; k += 8) {
    float q[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) q[j] = k + j < n ? p[(k + j) * apart] : 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) v += q[j];
  }
  return v;
}

// u and the joined g of every place for the kernels after it: g for `up` (Ready), and both by ranks for `outer`, in pieces of
// eight places: [piece][3][rp][8] thirds in bf16, or [piece][2][rp][4] fp32.  A segment's places begin with a piece of their own.
struct SumsArgs {
  const float* part;  // g [parts][T][rp]
  const float* u;     // [T][r]
  const int32_t* off;
  void* ready;        // or NULL
  void* by_rank[2];   // g, u
  int32_t bf_ready, bf_rank[2];
  int32_t parts, L, T, r, rp;
};

constexpr int kSumsPlaces = 32;

// 8192 places at rank 32 from one part: 5.6 us.
__global__ void __launch_bounds__(256) k_adapter_sums(SumsArgs a) {
  __shared__ float lds[kMaxRank][kSumsPlaces + 1];
  const int which = blockIdx.y, quads = a.rp / 4;
  Tile tile;
  if (!find_tile<false>(a.off, a.L, a.T, kSumsPlaces, blockIdx.x, tile)) return;
  const int n = tile.hi - tile.lo;
  for (int e = threadIdx.x; e < kSumsPlaces * quads; e += 256) {
    const int p = e / quads, rho = 4 * (e - p * quads);
    floatx4 v = {0.f, 0.f, 0.f, 0.f};
    if (p < n && which == 0) {
      const float* part = a.part + (int64_t)(tile.lo + p) * a.rp + rho;
      for (int k = 0; k < a.parts; ++k) v += *reinterpret_cast<const floatx4*>(part + (int64_t)k * a.T * a.rp);
      if (a.ready) {
        const int i = p % 16, first = tile.lo + p - i, m = min(16, tile.hi - first);
        if (a.bf_ready) Ready<true>::put(Ready<true>::group(a.ready, first, a.rp), m, i, rho, a.rp, v);
        else Ready<false>::put(Ready<false>::group(a.ready, first, a.rp), m, i, rho, a.rp, v);
      }
    } else if (p < n) {
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (rho + k < a.r) v[k] = a.u[(int64_t)(tile.lo + p) * a.r + rho + k];
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) lds[rho + k][p] = v[k];
  }
  __syncthreads();
  const int64_t piece = (first_by_rank(tile.lo - tile.index * kSumsPlaces, tile.l) + tile.index * kSumsPlaces) / 8;
  for (int e = threadIdx.x; e < kSumsPlaces / 8 * a.rp; e += 256) {
    const int b = e / a.rp, rho = e - b * a.rp;
    if (8 * b >= n) break;
    float v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = lds[rho][8 * b + k];
    uint4* out = static_cast<uint4*>(a.by_rank[which]) + (piece + b) * (a.bf_rank[which] ? 3 : 2) * a.rp + rho;
    if (a.bf_rank[which]) {
      uint4 q[3];
      thirds(v, q);
#pragma unroll
      for (int h = 0; h < 3; ++h) out[h * a.rp] = q[h];
    } else {
      uint4 q[2];
      thirds(v, q);
#pragma unroll
      for (int h = 0; h < 2; ++h) out[h * a.rp] = q[h];
    }
  }
}

// ---------------------------------------------------------------- outer

template <bool BF, bool ACROSS, int RB, bool SMALL>
__global__ void __launch_bounds__(kOuterWaves* kWave, 2) k_adapter_outer(OuterArgs a) {
  typedef Outer<BF, ACROSS, RB, SMALL, false> O;
  __shared__ __align__(16) float sums[O::kLds];
  Tile tile;
  if (find_tile<true>(a.off, a.L, a.T, a.chunk, blockIdx.y, tile)) O::run(a, tile, blockIdx.x * OuterTile<BF>::kCols, blockIdx.z * 16 * RB, sums);
}

// The parts of segments of several chunks, in order, and zeros for empty segments.  9 chunks of 32 x 7168 and 16 of 32 x 4096:
// 5.5 us (16 MB that the caches hold).
struct JoinArgs {
  const int32_t* off;
  float* out[2];
  const float* slots[2];
  int64_t size[2];
  int32_t chunk[2], n_slots[2], L, T, accumulate, per;  // per: elements of a block
};

__global__ void __launch_bounds__(256) k_adapter_join(JoinArgs a) {
  const int l = blockIdx.y, m = blockIdx.z, lane = threadIdx.x & 63;
  const int64_t size = a.size[m], end = min(size, (int64_t)(blockIdx.x + 1) * a.per);
  if ((int64_t)blockIdx.x * a.per >= size) return;
  const Length seg(a.off, a.L, a.T, a.chunk[m], l);
  if (seg.n == 1 || (seg.n == 0 && a.accumulate)) return;
  int before = 0;
  for (int k = lane; k < l; k += 64) before += Length(a.off, a.L, a.T, a.chunk[m], k).split();
#pragma unroll
  for (int d = 32; d; d >>= 1) before += __shfl_xor(before, d);
  if (seg.n && before + seg.n > a.n_slots[m]) return;  // offsets that decrease
  float* out = a.out[m] + l * size;
  const float* slots = a.slots[m] + (int64_t)before * size;
  for (int64_t i = (int64_t)blockIdx.x * a.per + threadIdx.x; i < end; i += 256) {
    const float v = seg.n ? add_parts(slots + i, size, seg.n) : 0.f;
    out[i] = a.accumulate ? out[i] + v : v;
  }
}

// ---------------------------------------------------------------- launches

// Places of a chunk of `outer`: blocks for every CU twice over the matrix, of at least 128 places.
int32_t outer_chunk(int32_t T, int32_t C, int32_t dtype) {
  const int32_t cols = dtype == DAMOE_BF16 ? OuterTile<true>::kCols : OuterTile<false>::kCols;
  const int32_t tiles = (C + cols - 1) / cols;
  const int32_t chunks = std::max(1, std::min((T + 127) / 128, 512 / tiles));
  return ((T + chunks - 1) / chunks + 31) / 32 * 32;  // whole steps
}

// Slots of `outer`: a segment of n > 1 chunks has more than (n - 1) chunk places, so n is at most twice the chunks they fill.
int64_t slots_of(int32_t T, int32_t chunk) { return chunk >= T ? 0 : 2 * (int64_t)((T + chunk - 1) / chunk); }

hipError_t outer(const OuterArgs& a, int32_t dtype, bool across, hipStream_t stream) {
  using std::false_type;
  using std::true_type;
  const auto go = [&](auto bf, auto ac, auto rb, auto small) {
    constexpr bool BF = decltype(bf)::value;
    constexpr int RB = decltype(rb)::value;
    typedef OuterTile<BF> O;
    const dim3 grid((a.C + O::kCols - 1) / O::kCols, (unsigned)most_tiles(a.T, a.L, a.chunk), (a.r + 16 * RB - 1) / (16 * RB));
    hipLaunchKernelGGL((k_adapter_outer<BF, decltype(ac)::value, RB, decltype(small)::value>), grid, dim3(kOuterWaves * kWave), 0, stream,
                       a);
    return hipGetLastError();
  };
  const auto ranked = [&](auto bf, auto ac) {
    if (a.C < OuterTile<decltype(bf)::value>::kPer) return go(bf, ac, std::integral_constant<int, 1>{}, true_type{});
    return a.r <= 16 ? go(bf, ac, std::integral_constant<int, 1>{}, false_type{})
                     : go(bf, ac, std::integral_constant<int, 2>{}, false_type{});
  };
  if (dtype == DAMOE_BF16) return across ? ranked(true_type{}, true_type{}) : ranked(true_type{}, false_type{});
  return across ? ranked(false_type{}, true_type{}) : ranked(false_type{}, false_type{});
}

// By ranks; slots.
size_t rank_bytes(int32_t T, int32_t L, int32_t rp) { return up256(pieces_by_rank(T, L) * rp * 48); }
size_t slot_bytes(int64_t slots, int32_t r, int32_t C) { return up256((size_t)slots * r * C * 4); }

// The most that slots_of is: there are never more chunks than 128-place ones, nor than the blocks allow.
int64_t most_slots(int32_t T_max, int32_t C) {
  const int64_t tiles = (C + OuterTile<true>::kCols - 1) / OuterTile<true>::kCols;
  return T_max <= 128 ? 0 : 2 * std::min<int64_t>((T_max + 127) / 128, std::max<int64_t>(1, 512 / tiles));
}

}  // namespace
}  // namespace damoe

using namespace damoe;

extern "C" {

size_t damoe_adapters_grad_workspace_size(int32_t T_max, int32_t L, int32_t r, int32_t K, int32_t N) {
  if (check(T_max, L, r, K, N, DAMOE_F32, DAMOE_F32, DAMOE_F32)) return 0;
  const int32_t rp = padded_rank(r);
  return 256 + most_parts(T_max, N, rp) + ready_bytes(T_max, rp) + kSpare + 2 * rank_bytes(T_max, L, rp) + slot_bytes(most_slots(T_max, K), r, K) +
         slot_bytes(most_slots(T_max, N), r, N);
}

damoe_status damoe_adapters_grad(const void* x, int32_t xdtype, int64_t ldx, const void* dy, int32_t ydtype, int64_t ldy, const float* u,
                                 const int32_t* perm, const int32_t* offsets, int32_t T, int32_t L, const void* a, const void* b,
                                 int32_t wdtype, int32_t r, int32_t K, int32_t N, const float* scale, const void* add, int64_t ld_add,
                                 void* dx, int64_t ld_dx, float* da, float* db, int32_t accumulate, void* ws, size_t ws_bytes,
                                 hipStream_t stream) {
  if (const damoe_status s = check(T, L, r, K, N, xdtype, wdtype, ydtype)) return s;
  if (!da || !db || !offsets || !aligned(da, DAMOE_F32) || !aligned(db, DAMOE_F32) || !aligned(offsets, DAMOE_F32) ||
      (accumulate != 0 && accumulate != 1))
    return DAMOE_ERR_INVALID_ARG;
  if (T > 0 && (!matrix_ok(x, ldx, K, xdtype) || !matrix_ok(dy, ldy, N, ydtype) || !u || !aligned(u, DAMOE_F32) ||
                (dx && !matrix_ok(dx, ld_dx, K, xdtype)) || (dx && add && !matrix_ok(add, ld_add, K, xdtype)) ||
                (dx && add == dx && ld_add != ld_dx) || !a || !b || !aligned(a, wdtype) || !aligned(b, wdtype) ||
                !aligned(perm, DAMOE_F32) || !aligned(scale, DAMOE_F32) || !ws || reinterpret_cast<uintptr_t>(ws) % 16))
    return DAMOE_ERR_INVALID_ARG;
  const int32_t rp = padded_rank(r);
  const bool few = T > 0 && adapters_grad_few(T, L, r, K, N, xdtype, ydtype);  // then a segment is one chunk
  const int32_t ck = few || !T ? std::max(T, 1) : outer_chunk(T, K, xdtype), cn = few || !T ? std::max(T, 1) : outer_chunk(T, N, ydtype);
  const int32_t n_a = T ? (int32_t)slots_of(T, ck) : 0, n_b = T ? (int32_t)slots_of(T, cn) : 0;
  char* base = static_cast<char*>(ws);
  float *slots_a = nullptr, *slots_b = nullptr;
  if (T > 0) {
    const DownPlan d = down_plan(T, N);
    size_t end = 0;
    const auto piece = [&](size_t n) {
      char* p = base + end;
      end += n;
      return p;
    };
    float* part = reinterpret_cast<float*>(piece(part_bytes(d, T, rp)));
    void* ready = piece(ready_bytes(T, rp));
    char* spare = piece(kSpare);
    void* g_rank = piece(rank_bytes(T, L, rp));
    void* u_rank = piece(rank_bytes(T, L, rp));
    slots_a = reinterpret_cast<float*>(piece(slot_bytes(n_a, r, K)));
    slots_b = reinterpret_cast<float*>(piece(slot_bytes(n_b, r, N)));
    if (ws_bytes < end) return DAMOE_ERR_WORKSPACE;
    const DownArgs ga{dy, ldy, b, perm, offsets, scale, part, nullptr, nullptr, L, T, N, r, rp, 0, 0};
    if (down<true>(ga, d, ydtype, wdtype, stream) != hipSuccess) return DAMOE_ERR_HIP;
    // dB first: it reads what `down` has just read.
    const OuterArgs ob{dy, ldy, u_rank, u, 1, r, scale, perm, offsets, db, slots_b, n_b, L, T, N, r, rp, cn, accumulate};
    const OuterArgs oa{x, ldx, g_rank, part, d.parts, rp, nullptr, perm, offsets, da, slots_a, n_a, L, T, K, r, rp, ck, accumulate};
    const UpArgs xa{part, ready, d.parts, nullptr, a, nullptr, perm, offsets, add, ld_add, dx, ld_dx, spare, L, T, K, r, rp, 0};
    if (few) return adapters_grad_in_one(ob, oa, xa, true, xdtype, wdtype, stream) == hipSuccess ? DAMOE_OK : DAMOE_ERR_HIP;
    const SumsArgs sa{part, u, offsets, dx ? ready : nullptr, {g_rank, u_rank}, wdtype == DAMOE_BF16,
                      {xdtype == DAMOE_BF16, ydtype == DAMOE_BF16}, d.parts, L, T, r, rp};
    hipLaunchKernelGGL(k_adapter_sums, dim3((unsigned)most_tiles(T, L, kSumsPlaces), 2), dim3(256), 0, stream, sa);
    if (hipGetLastError() != hipSuccess) return DAMOE_ERR_HIP;
    if (adapters_grad_joined(T, L, r, K, N, xdtype, ydtype)) {
      if (adapters_grad_in_one(ob, oa, xa, false, xdtype, wdtype, stream) != hipSuccess) return DAMOE_ERR_HIP;
    } else {
      if (outer(ob, ydtype, true, stream) != hipSuccess) return DAMOE_ERR_HIP;
      if (outer(oa, xdtype, false, stream) != hipSuccess) return DAMOE_ERR_HIP;
      if (dx && up<true, false>(xa, xdtype, wdtype, stream) != hipSuccess) return DAMOE_ERR_HIP;
    }
  }
  JoinArgs j{offsets, {da, db}, {slots_a, slots_b}, {(int64_t)r * K, (int64_t)r * N}, {ck, cn}, {n_a, n_b}, L, T, accumulate, 256};
  const int64_t all = std::max(j.size[0], j.size[1]);
  while ((all + j.per - 1) / j.per * L > 2048 && j.per < all) j.per *= 2;
  hipLaunchKernelGGL(k_adapter_join, dim3((unsigned)((all + j.per - 1) / j.per), L, 2), dim3(256), 0, stream, j);
  return hipGetLastError() == hipSuccess ? DAMOE_OK : DAMOE_ERR_HIP;
}

}  // extern "C"
