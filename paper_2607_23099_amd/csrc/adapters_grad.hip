// damoe_adapters_grad: the gradient of y = add + s B (A x) with respect to x, A and B of each segment.
#include "adapters.h"

namespace damoe {
namespace {

constexpr int kOuterWaves = 4;

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

// Place of the by-rank pieces that segment l's first place, lo, has; and the pieces that there are of T places.
__host__ __device__ __forceinline__ int first_by_rank(int lo, int l) { return (lo + 7) / 8 * 8 + 16 * l; }
inline size_t pieces_by_rank(int32_t T, int32_t L) { return (size_t)(T + 7) / 8 + 2 * L + 8; }  // loads go up to 31 places past the last

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
#pragma unroll
      for (int h = 0; h < 3; ++h) {
        uint32_t q[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const uint32_t lo = take_third(v[2 * k]);
          q[k] = lo | (uint32_t)take_third(v[2 * k + 1]) << 16;
        }
        out[h * a.rp] = uint4{q[0], q[1], q[2], q[3]};
      }
    } else {
#pragma unroll
      for (int h = 0; h < 2; ++h)
        out[h * a.rp] = uint4{__float_as_uint(v[4 * h]), __float_as_uint(v[4 * h + 1]), __float_as_uint(v[4 * h + 2]), __float_as_uint(v[4 * h + 3])};
    }
  }
}

// ---------------------------------------------------------------- outer

struct OuterArgs {
  const void* x;       // rows (x, dy)
  int64_t ldx;
  const void* by_rank; // the other factor, of `sums`
  const float* scale;  // of a segment's sums, or NULL
  const int32_t* perm;
  const int32_t* off;
  float* out;          // dA [L][r][C], or dB [L][C][r]
  float* slots;        // parts of segments of several chunks, laid out as the output
  int32_t L, T, C, r, rp, chunk, accumulate;
};

template <bool BF>
struct OuterTile {
  // Columns of a lane's 16 bytes; a wave's tile of 32 places x 16 lanes of them.
  static constexpr int kPer = Elem<BF>::kPer16, kCols = 16 * kPer;
};

// Bits 8 g .. + 7 of a mask of places: whether place k of the lane's eight counts.
__device__ __forceinline__ bool counts(uint32_t mask, int g, int k) { return mask >> (8 * g + k) & 1; }

// A block has 128 (bf16) or 64 (fp32) columns and a chunk of a segment's places, in steps of 32 by its waves in turn.
// Lane (i, g) loads 16 bytes of places 8 g .. + 7 each, columns P i .. + P - 1 (P = 8 or 4), so a row's piece is 256 bytes
// side by side.  bf16: the eight pieces are turned in registers into the operands of P MFMAs over 32 places, the r factors
// are three thirds in bf16: products are exact.  fp32: element k of every lane is multiplied by an fp32 MFMA of its own.
// MFMA j has column P i + j as row i.  The next step's rows are loaded while one is multiplied.  Lanes past the last column
// take the last P again; SMALL: there are fewer than P, each is loaded for itself.
template <bool BF, bool ACROSS, int RB, bool SMALL>
__global__ void __launch_bounds__(kOuterWaves* kWave, 2) k_adapter_outer(OuterArgs a) {
  typedef OuterTile<BF> O;
  typedef typename Elem<BF>::T X;
  constexpr int P = O::kPer, F = BF ? 3 : 2;
  constexpr int kPlane = 64 * 4 + 4;  // floats of a wave's MFMA in LDS
  __shared__ __align__(16) float sums[kOuterWaves * P * kPlane];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int i = lane & 15, g = lane >> 4;
  const int r0 = blockIdx.z * 16 * RB, b0 = blockIdx.x * O::kCols;
  const int c = SMALL ? P * i : min(b0 + P * i, a.C - P);
  Tile tile;
  if (!find_tile<true>(a.off, a.L, a.T, a.chunk, blockIdx.y, tile)) return;
  floatx4 acc[P][RB];
#pragma unroll
  for (int j = 0; j < P; ++j)
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) acc[j][rb] = floatx4{0.f, 0.f, 0.f, 0.f};
  struct Rows {
    uint4 v[8];
    uint4 u[RB][F];
    uint32_t mask;  // of places
  };
  const Places places(a.perm, a.off);
  constexpr int kStep = 32 * kOuterWaves;
  const int first = tile.lo + 32 * wave, steps = first < tile.hi ? (tile.hi - first + kStep - 1) / kStep : 0;
  const int begin = tile.lo - tile.index * a.chunk, shift = first_by_rank(begin, tile.l) - begin;
  const auto at = [&](int s) { return first + min(s, steps - 1) * kStep; };
  // Lane by lane the row of place p + lane % 32.
  const auto place = [&](int s) { return places.load(min(at(s) + (lane & 31), tile.hi - 1)); };
  const auto load = [&](Rows& s, int loaded, int step) {
    const int p = at(step), mine = p + (lane & 31), t = places.row(loaded, min(mine, tile.hi - 1));
    const bool ok = mine < tile.hi && (uint32_t)t < (uint32_t)a.T;
    s.mask = (uint32_t)__ballot(ok);
    const int valid = ok ? t : 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const X* x = static_cast<const X*>(a.x) + __shfl(valid, 8 * g + k) * a.ldx + c;
      if constexpr (SMALL) {
        s.v[k] = uint4{0, 0, 0, 0};
        if (i == 0) s.v[k] = load_some<BF>(x, a.C);
      } else {
        s.v[k] = load16_at<Elem<BF>::kBytes>(x);
      }
    }
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
      for (int h = 0; h < F; ++h)
        s.u[rb][h] = static_cast<const uint4*>(a.by_rank)[((int64_t)((p + shift) / 8 + g) * F + h) * a.rp + r0 + 16 * rb + i];
  };
  const auto work = [&](Rows& s) {
    if (s.mask != ~0u) {  // nothing of places that do not count: their rows are others', their factors were never written
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (!counts(s.mask, g, k)) s.v[k] = uint4{0, 0, 0, 0};
#pragma unroll
      for (int rb = 0; rb < RB; ++rb)
#pragma unroll
        for (int h = 0; h < F; ++h) {
          uint32_t* q = reinterpret_cast<uint32_t*>(&s.u[rb][h]);
#pragma unroll
          for (int d = 0; d < 4; ++d) {
            if constexpr (BF) q[d] &= (counts(s.mask, g, 2 * d) ? 0xFFFFu : 0u) | (counts(s.mask, g, 2 * d + 1) ? 0xFFFF0000u : 0u);
            else q[d] = counts(s.mask, g, 4 * h + d) ? q[d] : 0u;
          }
        }
    }
    if constexpr (BF) {
      // Dword d of place k holds its columns 2 d and 2 d + 1; operand j wants column j of all places.
      uint4 x[P];
#pragma unroll
      for (int d = 0; d < P / 2; ++d) {
        uint32_t q[8], lo[4], hi[4];
#pragma unroll
        for (int k = 0; k < 8; ++k) q[k] = d == 0 ? s.v[k].x : d == 1 ? s.v[k].y : d == 2 ? s.v[k].z : s.v[k].w;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          lo[k] = __builtin_amdgcn_perm(q[2 * k + 1], q[2 * k], 0x05040100u);
          hi[k] = __builtin_amdgcn_perm(q[2 * k + 1], q[2 * k], 0x07060302u);
        }
        x[2 * d] = uint4{lo[0], lo[1], lo[2], lo[3]}, x[2 * d + 1] = uint4{hi[0], hi[1], hi[2], hi[3]};
      }
      // A sum's instructions are P RB apart, longer than one takes.
#pragma unroll
      for (int h = 0; h < F; ++h)
#pragma unroll
        for (int j = 0; j < P; ++j)
#pragma unroll
          for (int rb = 0; rb < RB; ++rb) acc[j][rb] = mfma16x16x32(x[j], s.u[rb][h], acc[j][rb]);
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const uint32_t q[4] = {s.v[k].x, s.v[k].y, s.v[k].z, s.v[k].w};
#pragma unroll
        for (int j = 0; j < P; ++j)
#pragma unroll
          for (int rb = 0; rb < RB; ++rb) acc[j][rb] = mma4(q[j], reinterpret_cast<const uint32_t*>(&s.u[rb][k / 4])[k % 4], acc[j][rb]);
      }
    }
  };
  if (steps == 1) {
    Rows s;
    load(s, place(0), 0);
    work(s);
  } else if (steps > 1) {
    Rows s[2];
    int loaded[2] = {place(0), place(1)};
    load(s[0], loaded[0], 0);
    for (int step = 0; step < steps; step += 2) {
      loaded[0] = place(step + 2);
      load(s[1], loaded[1], step + 1);
      work(s[0]);
      loaded[1] = place(step + 3);
      load(s[0], loaded[0], step + 2);
      if (step + 1 < steps) work(s[1]);
    }
  }
  // The waves' sums in order, through LDS, where threads side by side take elements side by side of the output.  Lane (i, g)
  // holds rank i of each block and, of MFMA j and register e, column P (4 g + e) + j of the lanes' columns.
  const int64_t size = (int64_t)a.r * a.C;
  float* out = tile.whole ? a.out + tile.l * size : a.slots + tile.slot * size;
  const float scale = a.scale ? a.scale[tile.l] : 1.f;
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    if (rb) __syncthreads();
#pragma unroll
    for (int j = 0; j < P; ++j) *reinterpret_cast<floatx4*>(sums + (wave * P + j) * kPlane + lane * 4) = acc[j][rb];
    __syncthreads();
#pragma unroll 4
    for (int e = threadIdx.x; e < 16 * O::kCols; e += kOuterWaves * kWave) {
      const int rank = ACROSS ? e % 16 : e / O::kCols, col = ACROSS ? e / 16 : e % O::kCols, rho = r0 + 16 * rb + rank;
      if (rho >= a.r || b0 + col >= a.C) continue;
      const int x = col / P, j = col % P + (SMALL ? 0 : max(0, b0 + P * x + P - a.C));
      const float* v = sums + j * kPlane + (rank + 16 * (x / 4)) * 4 + x % 4;
      float f = v[0];
#pragma unroll
      for (int w = 1; w < kOuterWaves; ++w) f += v[w * P * kPlane];
      f *= scale;
      float* o = out + (ACROSS ? (int64_t)(b0 + col) * a.r + rho : (int64_t)rho * a.C + b0 + col);
      *o = tile.whole && a.accumulate ? *o + f : f;
    }
  }
}

// The parts of segments of several chunks, in order, and zeros for empty segments.
struct JoinArgs {
  const int32_t* off;
  float* out[2];
  const float* slots[2];
  int64_t size[2];
  int32_t chunk[2], L, T, accumulate, per;  // per: elements of a block
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
  const int32_t ck = T ? outer_chunk(T, K, xdtype) : 1, cn = T ? outer_chunk(T, N, ydtype) : 1;
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
    slots_a = reinterpret_cast<float*>(piece(slot_bytes(slots_of(T, ck), r, K)));
    slots_b = reinterpret_cast<float*>(piece(slot_bytes(slots_of(T, cn), r, N)));
    if (ws_bytes < end) return DAMOE_ERR_WORKSPACE;
    const DownArgs ga{dy, ldy, b, perm, offsets, scale, part, nullptr, nullptr, L, T, N, r, rp, 0, 0};
    if (down<true>(ga, d, ydtype, wdtype, stream) != hipSuccess) return DAMOE_ERR_HIP;
    const SumsArgs sa{part, u, offsets, dx ? ready : nullptr, {g_rank, u_rank}, wdtype == DAMOE_BF16,
                      {xdtype == DAMOE_BF16, ydtype == DAMOE_BF16}, d.parts, L, T, r, rp};
    hipLaunchKernelGGL(k_adapter_sums, dim3((unsigned)most_tiles(T, L, kSumsPlaces), 2), dim3(256), 0, stream, sa);
    if (hipGetLastError() != hipSuccess) return DAMOE_ERR_HIP;
    // dB first: it reads what `down` has just read.
    const OuterArgs ob{dy, ldy, u_rank, scale, perm, offsets, db, slots_b, L, T, N, r, rp, cn, accumulate};
    if (outer(ob, ydtype, true, stream) != hipSuccess) return DAMOE_ERR_HIP;
    const OuterArgs oa{x, ldx, g_rank, nullptr, perm, offsets, da, slots_a, L, T, K, r, rp, ck, accumulate};
    if (outer(oa, xdtype, false, stream) != hipSuccess) return DAMOE_ERR_HIP;
    if (dx) {
      const UpArgs xa{nullptr, ready, 1, nullptr, a, nullptr, perm, offsets, add, ld_add, dx, ld_dx, spare, L, T, K, r, rp, 0};
      if (up<true, false>(xa, xdtype, wdtype, stream) != hipSuccess) return DAMOE_ERR_HIP;
    }
  }
  JoinArgs j{offsets, {da, db}, {slots_a, slots_b}, {(int64_t)r * K, (int64_t)r * N}, {ck, cn}, L, T, accumulate, 256};
  const int64_t all = std::max(j.size[0], j.size[1]);
  while ((all + j.per - 1) / j.per * L > 2048 && j.per < all) j.per *= 2;
  hipLaunchKernelGGL(k_adapter_join, dim3((unsigned)((all + j.per - 1) / j.per), L, 2), dim3(256), 0, stream, j);
  return hipGetLastError() == hipSuccess ? DAMOE_OK : DAMOE_ERR_HIP;
}

}  // extern "C"
