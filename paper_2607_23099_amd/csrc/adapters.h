// Low-rank adapters of many segments of rows at once: what damoe_adapters and its gradient share.
//
// Segment l is the places [off[l], off[l + 1]) and place p holds row t = perm[p] (p itself without perm).  With A_l [r][K],
// B_l [N][r] and s_l:
//   u_p = A_l x_t            y_t = add_t + s_l B_l u_p
//   g_p = s_l B_l^T dy_t     dx_t = add_t + A_l^T g_p     dA_l = sum_p g_p x_t^T     dB_l = s_l sum_p dy_t u_p^T
// r is small, so all of it is bound by the rows (x, dy, y, dx), or by the weights where few rows share an adapter.  Kernels,
// each a pass over one of these matrices:
//   down    rows of r sums over many columns (u, g): columns split over a block's waves, for few rows over blocks too
//   up      many columns of r products each (y, dx)
//   outer   r x columns sums over a segment's places (dA, dB), split over chunks of places whose parts `join` adds
// and `sums`, which lays u and g out for `up` and `outer` between them.  A block has places of one segment: it finds them by
// a scan over the segments' lengths, so no list of tiles has to be made and nothing depends on timing.
//
// Loops that stream rows have no branch around a load: vector loads complete in order and are counted, so where two paths
// with different numbers of them meet, a wave waits for all of them.  Places past the end load the last one again, and a
// row's partial unit of columns has code of its own behind the loop.  perm is read two steps ahead, before the rows of the
// step between, so that its value is there when the next rows are asked for.
#pragma once

#include "vec.h"

namespace damoe {
namespace {

constexpr int kMaxRank = DAMOE_MAX_RANK;
constexpr int kUpWaves = 4;

// ---------------------------------------------------------------- segments

// Places [lo, hi) of segment l, tile number `index` of its; `slot`: the number of tiles before it that belong to segments of
// several tiles.
struct Tile {
  int l, lo, hi, index, slot;
  bool whole;  // the segment's only tile
};

// Segment l's places and tiles; none from L on.
struct Length {
  int s, e, n;
  __device__ __forceinline__ Length(int begin, int end, int T, int P) {
    s = min(max(begin, 0), T);
    e = min(max(end, s), T);
    n = (int)((uint32_t)(e - s + P - 1) / (uint32_t)P);
  }
  __device__ __forceinline__ Length(const int32_t* off, int L, int T, int P, int l)
      : Length(off[min(l, L)], off[min(l + 1, L)], T, P) {}
  __device__ __forceinline__ int split() const { return n > 1 ? n : 0; }
};

// Inclusive sum over the wave's lanes: within rows of 16 by shifts, then each row's last lane to the rows behind it.
__device__ __forceinline__ int scan(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);
  return v;
}

// Tile number b of all, segments in order, each in tiles of P places; false past the last.  By each wave for itself: lane i
// counts segments i S .. + S - 1, and (L > 64) the lanes then the segments of the one that has the tile.
template <bool SLOTS>
__device__ __forceinline__ bool find_tile(const int32_t* off, int L, int T, int P, int b, Tile& t) {
  const int lane = threadIdx.x & 63, S = (L + 63) / 64;
  Length x(off, L, T, P, lane * S);
  int n = x.n, m = x.split();
  for (int j = 1; j < S; j += 4) {
    int at[5];
#pragma unroll
    for (int q = 0; q < 5; ++q) at[q] = off[min(lane * S + min(j + q, S), L)];
#pragma unroll
    for (int q = 0; q < 4; ++q) {  // past S: both ends are one
      const Length y(at[q], at[q + 1], T, P);
      n += y.n;
      if constexpr (SLOTS) m += y.split();
    }
  }
  int base = 0, slots = 0, l = 0;
  for (int level = 0;; ++level) {
    const int sum = scan(n);
    const int split = SLOTS ? scan(m) : 0;
    const uint64_t hit = __ballot(sum > b - base);
    if (!hit) return false;
    const int w = __builtin_amdgcn_readfirstlane(__builtin_ctzll(hit));
    base += __builtin_amdgcn_readlane(sum - n, w);
    if constexpr (SLOTS) slots += __builtin_amdgcn_readlane(split - m, w);
    l += w;
    if (S == 1 || level == 1) {
      t.l = l;
      t.index = b - base;
      t.slot = slots + t.index;
      t.whole = __builtin_amdgcn_readlane(x.n, w) == 1;
      t.lo = __builtin_amdgcn_readlane(x.s, w) + t.index * P;
      t.hi = min(t.lo + P, __builtin_amdgcn_readlane(x.e, w));
      return true;
    }
    l *= S;
    x = Length(off, L, T, P, lane < S ? l + lane : L);
    n = x.n, m = x.split();
  }
}

// Tiles of P places that T places in L segments have at most.
inline int64_t most_tiles(int32_t T, int32_t L, int32_t P) {
  const int64_t n = std::min(T, L);
  return (T + n * (P - 1)) / P;
}

// Rows of places by a load that is there with and without perm (then of a word that is not used).
struct Places {
  const int32_t* list;
  bool mapped;
  __device__ __forceinline__ Places(const int32_t* perm, const int32_t* off) : list(perm ? perm : off), mapped(perm != nullptr) {}
  __device__ __forceinline__ int load(int p) const { return list[mapped ? p : 0]; }
  __device__ __forceinline__ int row(int loaded, int p) const { return mapped ? loaded : p; }
};

// ---------------------------------------------------------------- operands

// Eight elements side by side as they lie in memory: bf16 (SRC) or fp32.
template <bool SRC>
struct Raw {
  uint32_t q[SRC ? 4 : 8];

  __device__ __forceinline__ void load(const void* base, int64_t i) {
    typedef Elem<SRC> E;
    const typename E::T* p = static_cast<const typename E::T*>(base) + i;
#pragma unroll
    for (int h = 0; h < (SRC ? 1 : 2); ++h) {
      const uint4 v = load16_at<E::kBytes>(p + 4 * h);
      q[4 * h] = v.x, q[4 * h + 1] = v.y, q[4 * h + 2] = v.z, q[4 * h + 3] = v.w;
    }
  }
  // n of them are the row's, the others 0.
  __device__ __forceinline__ void load_some(const void* base, int64_t i, int n) {
    const typename Elem<SRC>::T* p = static_cast<const typename Elem<SRC>::T*>(base) + i;
    if (n >= 8) return load(base, i);
#pragma unroll
    for (uint32_t& e : q) e = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < n) {
        if constexpr (SRC) q[j / 2] |= (uint32_t)p[j] << (16 * (j & 1));
        else q[j] = __float_as_uint(p[j]);
      }
  }
};

// Eight elements of one row of an MFMA operand: lane i + 16 g has row i, and g's eight of the 32 that are multiplied.
template <bool BF>
struct Frag {
  uint32_t q[BF ? 4 : 8];
};

template <bool BF, bool SRC>
__device__ __forceinline__ Frag<BF> frag(const Raw<SRC>& r) {
  static_assert(SRC || !BF, "fp32 is not rounded to bf16");
  Frag<BF> f;
#pragma unroll
  for (int j = 0; j < (BF ? 4 : 8); ++j) f.q[j] = BF || !SRC ? r.q[j] : j & 1 ? r.q[j / 2] & 0xFFFF0000u : r.q[j / 2] << 16;
  return f;
}

__device__ __forceinline__ floatx4 mma4(uint32_t a, uint32_t b, const floatx4& c) {
  return __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a), __uint_as_float(b), c, 0, 0, 0);
}

// c += rows x rows over 32: one bf16 instruction, or eight fp32 ones (instruction j multiplies element j of every lane).
__device__ __forceinline__ floatx4 mma(const Frag<true>& a, const Frag<true>& b, const floatx4& c) {
  return mfma16x16x32(uint4{a.q[0], a.q[1], a.q[2], a.q[3]}, uint4{b.q[0], b.q[1], b.q[2], b.q[3]}, c);
}
__device__ __forceinline__ floatx4 mma(const Frag<false>& a, const Frag<false>& b, floatx4 c) {
#pragma unroll
  for (int j = 0; j < 8; ++j) c = mma4(a.q[j], b.q[j], c);
  return c;
}

// A third of an fp32 value in bf16: the leading 8 bits of its significand, cut off and not rounded, so that the three
// thirds add up to all 24 and the first does not overflow.  An infinity or NaN is its own first third, without others.
__device__ __forceinline__ uint16_t take_third(float& v) {
  const uint32_t b = __float_as_uint(v), hi = b & 0xFFFF0000u;
  const bool finite = (b & 0x7F800000u) != 0x7F800000u;
  v = finite ? v - __uint_as_float(hi) : 0.f;
  return (uint16_t)(hi >> 16 | (!finite && (b & 0xFFFFu) ? 1u : 0u));  // a NaN whose leading bits are an infinity's stays one
}

// ---------------------------------------------------------------- down

// How the weights lie for `down`: rows of columns (A), or columns of ranks (B), there read one rank a lane, or (bf16, r even)
// two side by side, which are the same row of two blocks of 16 ranks.
enum Lie { kRows, kAcross, kPairs };

struct DownArgs {
  const void* x;   // rows that are contracted (x, dy)
  int64_t ldx;
  const void* w;   // A [L][r][C], or B [L][C][r]
  const int32_t* perm;
  const int32_t* off;
  const float* scale;  // of a segment's sums, or NULL
  float* part;     // [parts][T][rp], or NULL: with one part, what `up` takes and u are written
  void* ready;     // [3][T][rp] thirds in bf16, or [T][rp] fp32
  float* u;        // [T][r] or NULL
  int32_t L, T, C, r, rp;
  int32_t places;  // of a block
  int32_t units;   // of 64 columns that a block takes
};

// Eight columns from c on of the lane's ranks, lane % 16 of each block of 16.
template <bool WB, Lie LIE, int RB>
struct Weights8 {
  static constexpr int kSets = LIE == kPairs ? RB / 2 : RB, kWords = LIE == kRows && WB ? 4 : 8;
  uint32_t q[kSets][kWords];

  // n of the columns are the matrix's, the others 0.
  template <bool FULL>
  __device__ __forceinline__ void load(const DownArgs& a, int64_t slab, int r0, int i, int c, int n) {
    typedef typename Elem<WB>::T T;
    struct __attribute__((packed, aligned(2))) Two {
      uint32_t v;
    };
#pragma unroll
    for (int s = 0; s < kSets; ++s) {
      if constexpr (LIE == kRows) {
        Raw<WB> f;
        const int64_t at = slab + (int64_t)min(r0 + 16 * s + i, a.r - 1) * a.C + c;
        if constexpr (FULL) f.load(a.w, at);
        else f.load_some(a.w, at, n);
#pragma unroll
        for (int j = 0; j < kWords; ++j) q[s][j] = f.q[j];
      } else {
        const int rho = LIE == kPairs ? min(r0 + 32 * s + 2 * i, a.r - 2) : min(r0 + 16 * s + i, a.r - 1);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const T* p = static_cast<const T*>(a.w) + slab + (int64_t)(FULL ? c + j : min(c + j, a.C - 1)) * a.r + rho;
          if constexpr (LIE == kPairs) q[s][j] = reinterpret_cast<const Two*>(p)->v;
          else if constexpr (WB) q[s][j] = *p;
          else q[s][j] = __float_as_uint(*p);
          if (!FULL && j >= n) q[s][j] = 0;
        }
      }
    }
  }
  template <bool BF>
  __device__ __forceinline__ Frag<BF> get(int rb) const {
    if constexpr (LIE == kRows) {
      Raw<WB> f;
#pragma unroll
      for (int j = 0; j < kWords; ++j) f.q[j] = q[rb][j];
      return frag<BF>(f);
    } else {
      Frag<BF> f;
      if constexpr (LIE == kPairs) {
        const uint32_t(&v)[8] = q[rb / 2];
#pragma unroll
        for (int j = 0; j < (BF ? 4 : 8); ++j) {
          if constexpr (BF) f.q[j] = __builtin_amdgcn_perm(v[2 * j + 1], v[2 * j], rb & 1 ? 0x07060302u : 0x05040100u);
          else f.q[j] = rb & 1 ? v[j] & 0xFFFF0000u : v[j] << 16;
        }
      } else {
#pragma unroll
        for (int j = 0; j < (BF ? 4 : 8); ++j) f.q[j] = BF ? q[rb][2 * j] | q[rb][2 * j + 1] << 16 : WB ? q[rb][j] << 16 : q[rb][j];
      }
      return f;
    }
  }
};

// Sums over units of 64 columns by W waves in turn, RB blocks of 16 ranks from r0 on and M of 16 places.  A unit is two MFMA
// steps: lane (i, g) takes columns 16 g .. + 7 of it in the first and 16 g + 8 .. + 15 in the second, so that its loads of a
// row are 32 bytes (bf16) side by side.  D units are in flight.
template <bool XB, bool WB, Lie LIE, int RB, int M, int W>
struct Down {
  static constexpr bool BF = XB && WB;
  struct Unit {
    Raw<XB> x[2][M];
    Weights8<WB, LIE, RB> w[2];
  };
  static constexpr int kRegs = sizeof(Unit) / 4, D = kRegs <= 16 ? 4 : kRegs <= 32 ? 3 : 2;
  floatx4 acc[M][RB];

  __device__ __forceinline__ void multiply(const Unit& v, bool second) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      Frag<BF> w[RB];
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) w[rb] = v.w[h].template get<BF>(rb);
#pragma unroll
      for (int m = 0; m < M; ++m) {
        if (!BF && m && !second) continue;  // fp32 instructions are long: none for places that the tile does not have
        const Frag<BF> x = frag<BF>(v.x[h][m]);
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) acc[m][rb] = mma(w[rb], x, acc[m][rb]);
      }
    }
  }

  __device__ __forceinline__ void run(const DownArgs& a, const Tile& tile, int u0, int u1, int r0) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int i = lane & 15, g = lane >> 4;
    const Places places(a.perm, a.off);
    const bool second = tile.hi - tile.lo > 16;
    int64_t row[M];
#pragma unroll
    for (int m = 0; m < M; ++m) {
      const int p = min(tile.lo + 16 * m + i, tile.hi - 1), t = places.row(places.load(p), p);
      row[m] = (int64_t)((uint32_t)t < (uint32_t)a.T ? t : 0) * a.ldx;
    }
    const int64_t slab = (int64_t)tile.l * a.r * a.C;
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) acc[m][rb] = floatx4{0.f, 0.f, 0.f, 0.f};
    const auto load = [&](Unit& v, int u) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int c = u * 64 + 16 * g + 8 * h;
#pragma unroll
        for (int m = 0; m < M; ++m) v.x[h][m].load(a.x, row[m] + c);
        v.w[h].template load<true>(a, slab, r0, i, c, 8);
      }
    };
    const int whole = a.C / 64;  // units
    int left = min(u1, whole) - u0 - wave;
    left = left > 0 ? (left + W - 1) / W : 0;
    if (left > 0) {
      Unit v[D];
      int u = u0 + wave;
      const int last = u + (left - 1) * W;
#pragma unroll
      for (int d = 0; d < D; ++d) load(v[d], min(u + d * W, last));
      for (u += D * W; left >= 2 * D; left -= D) {
#pragma unroll
        for (int d = 0; d < D; ++d, u += W) {
          multiply(v[d], second);
          load(v[d], u);
        }
      }
#pragma unroll
      for (int d = 0; d < D; ++d, u += W) {
        if (d < left) multiply(v[d], second);
        if (d + D < left) load(v[d], u);
      }
#pragma unroll
      for (int d = 0; d < D - 1; ++d)
        if (d + D < left) multiply(v[d], second);
    }
    if (whole >= u0 && whole < u1 && (whole - u0) % W == wave) {
      Unit v;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int c = whole * 64 + 16 * g + 8 * h;
#pragma unroll
        for (int m = 0; m < M; ++m) v.x[h][m].load_some(a.x, row[m] + c, a.C - c);
        v.w[h].template load<false>(a, slab, r0, i, c, a.C - c);
      }
      multiply(v, second);
    }
  }

  // The waves' sums through LDS [W][M RB][64], added in order by value().
  static constexpr int kLds = W * M * RB * 64;  // of 16 bytes
  __device__ __forceinline__ void put(floatx4* red) const {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) red[(wave * M * RB + m * RB + rb) * 64 + lane] = acc[m][rb];
  }
  // Sums of place `p` of the tile, ranks 4 q .. + 3 from r0 on.  Lane (i, g) holds place i, rows 4 g .. + 3 of each block.
  static __device__ __forceinline__ floatx4 value(const floatx4* red, int p, int q) {
    floatx4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const floatx4* r = red + (w * M + p / 16) * RB * 64 + p % 16;
      if constexpr (LIE != kPairs) {
        v += r[q / 4 * 64 + 16 * (q % 4)];
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) {  // rank 32 h + 2 s + b is row s of block 2 h + b
          const int s = (4 * (q % 8) + k) / 2;
          v[k] += reinterpret_cast<const float*>(r + (2 * (q / 8) + (k & 1)) * 64 + 16 * (s / 4))[s % 4];
        }
      }
    }
    return v;
  }
};

// Rows of the sums that `up` takes: thirds in bf16 for bf16 weights, else fp32.
template <bool WB>
__device__ __forceinline__ void put_ready(void* ready, int64_t plane, int64_t at, floatx4 v) {
  if constexpr (WB) {
#pragma unroll
    for (int h = 0; h < 3; ++h) {
      uint16_t q[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        float f = v[k];
        q[k] = take_third(f);
        v[k] = f;
      }
      *reinterpret_cast<uint2*>(static_cast<uint16_t*>(ready) + h * plane + at) =
          uint2{q[0] | (uint32_t)q[1] << 16, q[2] | (uint32_t)q[3] << 16};
    }
  } else {
    *reinterpret_cast<floatx4*>(static_cast<float*>(ready) + at) = v;
  }
}

constexpr int kDownWaves = 8;

// More than 64 ranks take a block of the grid for each 64.
template <bool XB, bool WB, Lie LIE, int RB, int M>
__global__ void __launch_bounds__(kDownWaves* kWave) k_adapter_down(DownArgs a) {
  typedef Down<XB, WB, LIE, RB, M, kDownWaves> D;
  extern __shared__ floatx4 red[];
  const int u0 = blockIdx.y * a.units, u1 = min(u0 + a.units, (a.C + 63) / 64);
  const int r0 = blockIdx.z * 16 * RB;
  Tile tile;
  if (!find_tile<false>(a.off, a.L, a.T, a.places, blockIdx.x, tile)) return;
  D d;
  d.run(a, tile, u0, u1, r0);
  d.put(red);
  __syncthreads();
  const float s = a.scale ? a.scale[tile.l] : 1.f;
  for (int e = threadIdx.x; e < M * 16 * 4 * RB; e += kDownWaves * kWave) {
    const int q = e % (4 * RB), p = tile.lo + e / (4 * RB), rho = r0 + 4 * q;
    if (p >= tile.hi) continue;
    floatx4 v = D::value(red, e / (4 * RB), q);
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = rho + k < a.r ? s * v[k] : 0.f;
    if (a.part) {
      *reinterpret_cast<floatx4*>(a.part + ((int64_t)blockIdx.y * a.T + p) * a.rp + rho) = v;
      continue;
    }
    if (a.u) {
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (rho + k < a.r) a.u[(int64_t)p * a.r + rho + k] = v[k];
    }
    put_ready<WB>(a.ready, (int64_t)a.T * a.rp, (int64_t)p * a.rp + rho, v);
  }
}

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

// ---------------------------------------------------------------- up

struct UpArgs {
  const float* part;  // [parts][T][rp] (JOIN), joined here
  const void* ready;  // else: [3][T][rp] thirds in bf16, or [T][rp] fp32
  int32_t parts;
  float* u;           // JOIN: NULL, or the joined sums [T][r]
  const void* w;      // B [L][C][r], or A [L][r][C]
  const float* scale;
  const int32_t* perm;
  const int32_t* off;
  const void* add;
  int64_t lda;
  void* y;
  int64_t ldy;
  int32_t L, T, C, r, rp, places;
};

constexpr int kUpCols = 64;  // columns of a wave

// The sums of 16 places as MFMA operands, and the weights that they meet: RB blocks of 16 ranks, or (RB = 0) 8 ranks.
// bf16 weights: three thirds, whose products are exact, an operand each; of 16 ranks two in one operand over the same weights
// twice, of 8 ranks all three.  fp32: instruction j multiplies rank kPer g + j of lane (i, g).
template <bool WB, int RB>
struct Sums {
  static constexpr int kPlanes = WB ? 3 : 1;
  static constexpr int kPer = WB ? 8 : RB ? 4 * RB : 2;         // ranks of a lane in an operand
  static constexpr int kBlocks = WB && RB > 2 ? RB / 2 : 1;     // operands for the ranks
  static constexpr int kOps = !WB ? 1 : RB >= 2 ? 3 : RB ? 2 : 1;  // of each: for the thirds
  static constexpr int kWords = WB ? 4 : kPer;
  static constexpr int kStride = 16 * (RB ? RB : 1) + (WB ? 8 : 4);  // in LDS, of a place
  typedef typename std::conditional<WB, uint16_t, float>::type T;
  uint32_t q[kBlocks][kOps][kWords];

  // First rank of lane group g in block kb.
  static __device__ __forceinline__ int rank(int kb, int g) {
    if constexpr (!WB) return kPer * g;
    return RB >= 2 ? 32 * kb + 8 * g : RB ? 8 * (g & 1) : 0;
  }
  static __device__ __forceinline__ int third(int h, int g) {
    if constexpr (!WB) return 0;
    return RB >= 2 ? h : RB ? 2 * h + g / 2 : g;
  }

  // Row p of planes `plane` elements apart, rows of `stride`.
  __device__ __forceinline__ void load(const T* base, int64_t plane, int64_t p, int stride, int g) {
#pragma unroll
    for (int kb = 0; kb < kBlocks; ++kb)
#pragma unroll
      for (int h = 0; h < kOps; ++h) {
        const T* s = base + min(third(h, g), kPlanes - 1) * plane + p * stride + rank(kb, g);
        if constexpr (kWords == 2) {
          const uint2 v = *reinterpret_cast<const uint2*>(s);
          q[kb][h][0] = v.x, q[kb][h][1] = v.y;
        } else {
#pragma unroll
          for (int e = 0; e < kWords; e += 4) {
            const uint4 v = *reinterpret_cast<const uint4*>(s + (WB ? 0 : e));
            q[kb][h][e] = v.x, q[kb][h][e + 1] = v.y, q[kb][h][e + 2] = v.z, q[kb][h][e + 3] = v.w;
          }
        }
      }
  }
  static __device__ __forceinline__ void put(T* lds, int places, int p, int rho, float v) {
    if constexpr (WB) {
#pragma unroll
      for (int h = 0; h < 3; ++h) lds[(h * places + p) * kStride + rho] = take_third(v);
    } else {
      lds[p * kStride + rho] = v;
    }
  }
};

template <bool WB, int RB>
struct UpWeights {
  typedef Sums<WB, RB> S;
  uint32_t q[4][S::kBlocks][S::kWords];

  // Ranks of column c; ACROSS: `apart` elements from one to the next.  Ranks from r on are 0.
  template <bool ACROSS>
  static __device__ __forceinline__ void ranks(uint32_t (&q)[S::kWords], const void* base, int64_t i, int64_t apart, int n) {
    typedef Elem<WB> E;
    const typename E::T* p = static_cast<const typename E::T*>(base) + i;
    if (!ACROSS && n >= S::kPer) {
      if constexpr (S::kWords == 2) {
        q[0] = __float_as_uint(p[0]), q[1] = __float_as_uint(p[1]);
      } else {
#pragma unroll
        for (int e = 0; e < S::kWords; e += 4) {
          const uint4 v = load16_at<E::kBytes>(p + (WB ? 0 : e));
          q[e] = v.x, q[e + 1] = v.y, q[e + 2] = v.z, q[e + 3] = v.w;
        }
      }
      return;
    }
    uint32_t v[S::kPer];
#pragma unroll
    for (int j = 0; j < S::kPer; ++j) {  // past the last rank: that one again, and not used
      const typename E::T* at = p + (ACROSS ? min(j, n - 1) * apart : min(j, n - 1));
      if constexpr (WB) v[j] = *at;
      else v[j] = __float_as_uint(*at);
      if (j >= n) v[j] = 0;
    }
#pragma unroll
    for (int e = 0; e < S::kWords; ++e) q[e] = WB ? v[2 * e % S::kPer] | v[(2 * e + 1) % S::kPer] << 16 : v[e % S::kPer];
  }

  // Four MFMA blocks of 16 columns from c0 on: row i of block 2 q + m is column 32 q + 8 (i / 4) + 4 m + i % 4, so that a
  // lane's results of a pair are eight columns side by side of its place.
  template <bool ACROSS>
  __device__ __forceinline__ void load(const UpArgs& a, int64_t slab, int c0) {
    const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      const int c = min(c0 + 32 * (b / 2) + 8 * (i / 4) + 4 * (b & 1) + i % 4, a.C - 1);
#pragma unroll
      for (int kb = 0; kb < S::kBlocks; ++kb) {
        const int rho = S::rank(kb, g);
        ranks<ACROSS>(q[b][kb], a.w, slab + (ACROSS ? (int64_t)rho * a.C + c : (int64_t)c * a.r + rho), a.C, a.r - rho);
      }
    }
  }
};

// 16 places by 64 columns of a wave: what is added, the product, the result.
template <bool YB, bool WB, int RB>
struct Up {
  typedef Sums<WB, RB> S;
  typedef Elem<YB> E;
  typedef typename E::T Y;
  static constexpr int P = 8 / E::kPer16;  // 16-byte pieces of eight columns
  S u;
  uint4 add[2][P];

  // FULL: all of the wave's columns are the matrix's and there is something to add (or `zero`, a buffer that is read and not
  // used); t is a row.
  template <bool FULL>
  __device__ __forceinline__ void load_add(const UpArgs& a, const void* zero, int t, int c0) {
    const int g = (threadIdx.x & 63) >> 4;
    const void* base = FULL && !a.add ? zero : a.add;
    const int64_t row = FULL && !a.add ? 0 : t * a.lda;
#pragma unroll
    for (int q = 0; q < 2; ++q)
#pragma unroll
      for (int h = 0; h < P; ++h) {
        const int c = c0 + 32 * q + 8 * g + h * E::kPer16, n = a.C - c;
        const Y* p = static_cast<const Y*>(base) + row + (FULL && !a.add ? 0 : c);
        if constexpr (FULL) {
          add[q][h] = load16_at<E::kBytes>(p);
        } else {
          add[q][h] = uint4{0, 0, 0, 0};
          if (a.add && t >= 0 && n > 0) add[q][h] = load_some<YB>(p, n);
        }
      }
  }

  // Row t, if it is one, is add + s times the product.
  template <bool FULL>
  __device__ __forceinline__ void work(const UpArgs& a, const UpWeights<WB, RB>& w, int t, int c0, float s) {
    const int g = (threadIdx.x & 63) >> 4;
    floatx4 acc[4];
#pragma unroll
    for (int b = 0; b < 4; ++b) acc[b] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int kb = 0; kb < S::kBlocks; ++kb)
#pragma unroll
      for (int h = 0; h < S::kOps; ++h) {
        if constexpr (WB) {
          const bool none = S::third(h, g) >= 3;
          const uint32_t(&v)[S::kWords] = u.q[kb][h];
          const uint4 f = none ? uint4{0, 0, 0, 0} : uint4{v[0], v[1], v[2], v[3]};
#pragma unroll
          for (int b = 0; b < 4; ++b) {
            const uint32_t(&x)[S::kWords] = w.q[b][kb];
            acc[b] = mfma16x16x32(uint4{x[0], x[1], x[2], x[3]}, f, acc[b]);
          }
        } else {
#pragma unroll
          for (int j = 0; j < S::kWords; ++j)
#pragma unroll
            for (int b = 0; b < 4; ++b) acc[b] = mma4(w.q[b][kb][j], u.q[kb][h][j], acc[b]);
        }
      }
    if (t < 0) return;
#pragma unroll
    for (int q = 0; q < 2; ++q)
#pragma unroll
      for (int h = 0; h < P; ++h) {
        const int c = c0 + 32 * q + 8 * g + h * E::kPer16, n = a.C - c;
        if (!FULL && n <= 0) continue;
        float f[E::kPer16];
        unpack16<YB>(FULL && !a.add ? uint4{0, 0, 0, 0} : add[q][h], f);
#pragma unroll
        for (int e = 0; e < E::kPer16; ++e) f[e] = fmaf(s, acc[2 * q + (h * E::kPer16 + e) / 4][(h * E::kPer16 + e) % 4], f[e]);
        Y* p = static_cast<Y*>(a.y) + t * a.ldy + c;
        if constexpr (FULL) store16_at<E::kBytes>(p, pack16<YB>(f));
        else store_some<YB>(p, n, pack16<YB>(f));
      }
  }
};

// JOIN: at most 16 places, whose parts are added here, in LDS for the block's waves.
template <bool YB, bool WB, bool ACROSS, int RB, bool JOIN>
__global__ void __launch_bounds__(kUpWaves* kWave) k_adapter_up(UpArgs a) {
  typedef Sums<WB, RB> S;
  __shared__ __align__(16) typename S::T lds[JOIN ? S::kPlanes * 16 * S::kStride : 8];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int i = lane & 15, g = lane >> 4;
  Tile tile;
  if (!find_tile<false>(a.off, a.L, a.T, a.places, blockIdx.x, tile)) return;
  const int c0 = (blockIdx.y * kUpWaves + wave) * kUpCols;
  const bool full = c0 + kUpCols <= a.C;
  const int64_t slab = (int64_t)tile.l * a.r * a.C;
  const float s = a.scale ? a.scale[tile.l] : 1.f;
  const Places places(a.perm, a.off);
  const auto place = [&](int step) { return places.load(min(tile.lo + 16 * step + i, tile.hi - 1)); };
  const auto row = [&](int loaded, int step) {  // -1: none
    const int p = tile.lo + 16 * step + i, t = places.row(loaded, p);
    return p < tile.hi && (uint32_t)t < (uint32_t)a.T ? t : -1;
  };
  UpWeights<WB, RB> w;
  if constexpr (JOIN) {
    const int t = row(place(0), 0);
    w.template load<ACROSS>(a, slab, c0);
    Up<YB, WB, RB> v;
    v.template load_add<false>(a, nullptr, t, c0);
    const int n = tile.hi - tile.lo;
    for (int e = threadIdx.x; e < 16 * a.rp; e += kUpWaves * kWave) {
      const int p = e / a.rp, rho = e % a.rp;
      float f = 0.f;
      if (p < n) {
        f = add_parts(a.part + (int64_t)(tile.lo + p) * a.rp + rho, (int64_t)a.T * a.rp, a.parts);
        if (a.u && blockIdx.y == 0 && rho < a.r) a.u[(int64_t)(tile.lo + p) * a.r + rho] = f;
      }
      S::put(lds, 16, p, rho, f);
    }
    __syncthreads();
    v.u.load(lds, 16 * S::kStride, i, S::kStride, g);
    v.template work<false>(a, w, t, c0, s);
  } else {
    if (c0 >= a.C) return;
    const int steps = (tile.hi - tile.lo + 15) / 16;
    const auto load = [&](auto all, Up<YB, WB, RB>& v, int t, int step) {
      v.template load_add<decltype(all)::value>(a, a.ready, decltype(all)::value ? max(t, 0) : t, c0);
      v.u.load(static_cast<const typename S::T*>(a.ready), (int64_t)a.T * a.rp, min(tile.lo + 16 * step + i, tile.hi - 1), a.rp, g);
    };
    const std::true_type yes;
    const std::false_type no;
    if (full && steps > 1) {
      Up<YB, WB, RB> v[2];
      int loaded[2] = {place(0), place(1)}, t[2];
      w.template load<ACROSS>(a, slab, c0);
      t[0] = row(loaded[0], 0);
      load(yes, v[0], t[0], 0);
      for (int step = 0; step < steps; step += 2) {
        loaded[0] = place(step + 2);
        t[1] = row(loaded[1], step + 1);
        load(yes, v[1], t[1], step + 1);
        v[0].template work<true>(a, w, t[0], c0, s);
        if (step + 1 >= steps) break;
        loaded[1] = place(step + 3);
        t[0] = row(loaded[0], step + 2);
        load(yes, v[0], t[0], step + 2);
        v[1].template work<true>(a, w, t[1], c0, s);
      }
      return;
    }
    const int first = place(0);
    w.template load<ACROSS>(a, slab, c0);
    if (full) {
      Up<YB, WB, RB> v;
      const int t = row(first, 0);
      load(yes, v, t, 0);
      v.template work<true>(a, w, t, c0, s);
      return;
    }
    for (int step = 0; step < steps; ++step) {
      Up<YB, WB, RB> v;
      const int t = row(place(step), step);
      load(no, v, t, step);
      v.template work<false>(a, w, t, c0, s);
    }
  }
}

// ---------------------------------------------------------------- launches

constexpr size_t up256(size_t v) { return (v + 255) / 256 * 256; }

inline int32_t padded_rank(int32_t r) { return r <= 16 ? 16 : r <= 32 ? 32 : r <= 64 ? 64 : 128; }

// f of the number of 16-rank blocks, at most MAX (4 or 8).
template <int MAX, class F>
hipError_t by_rank(int32_t rp, F f) {
  using std::integral_constant;
  return rp == 16              ? f(integral_constant<int, 1>{})
         : rp == 32            ? f(integral_constant<int, 2>{})
         : rp == 64 || MAX < 8 ? f(integral_constant<int, 4>{})
                               : f(integral_constant<int, MAX>{});
}

template <class F>
hipError_t by_types(int32_t d0, int32_t d1, F f) {
  using std::false_type;
  using std::true_type;
  if (d0 == DAMOE_BF16) return d1 == DAMOE_BF16 ? f(true_type{}, true_type{}) : f(true_type{}, false_type{});
  return d1 == DAMOE_BF16 ? f(false_type{}, true_type{}) : f(false_type{}, false_type{});
}

// How `down` is split: places of a block, blocks over the columns and each one's units.  From kManyRows rows on there are
// blocks enough without a split over the columns, and what it leaves is what `up` takes.
constexpr int32_t kManyRows = 4096;

struct DownPlan {
  int32_t places, parts, units;
};

inline DownPlan down_plan(int32_t T, int32_t C) {
  DownPlan d;
  d.places = T < kManyRows ? 16 : 32;
  const int32_t blocks = (T + d.places - 1) / d.places, units = (C + 63) / 64;
  d.parts = T >= kManyRows ? 1 : std::max(1, std::min(512 / std::max(blocks, 1), (units + kDownWaves - 1) / kDownWaves));
  d.units = (units + d.parts - 1) / d.parts;
  d.parts = (units + d.units - 1) / d.units;
  return d;
}

template <bool ACROSS>
hipError_t down(DownArgs a, const DownPlan& d, int32_t xdtype, int32_t wdtype, hipStream_t stream) {
  a.places = d.places;
  a.units = d.units;
  return by_rank<4>(a.rp, [&](auto rb) {
    return by_types(xdtype, wdtype, [&](auto xb, auto wb) {
      constexpr int RB = decltype(rb)::value;
      constexpr bool XB = decltype(xb)::value, WB = decltype(wb)::value;
      const auto go = [&](auto lie, auto m) {
        constexpr int M = decltype(m)::value;
        constexpr Lie LIE = decltype(lie)::value;
        const dim3 grid((unsigned)most_tiles(a.T, a.L, a.places), d.parts, a.rp / (16 * RB));
        constexpr size_t lds = Down<XB, WB, LIE, RB, M, kDownWaves>::kLds * sizeof(floatx4);
        hipLaunchKernelGGL((k_adapter_down<XB, WB, LIE, RB, M>), grid, dim3(kDownWaves * kWave), lds, stream, a);
        return hipGetLastError();
      };
      // fp32 operands of 64 ranks leave no registers for more than 16 places.
      const std::integral_constant<int, 1> one;
      const std::integral_constant<int, RB == 4 && !(XB && WB) ? 1 : 2> most;
      a.places = std::min(a.places, 16 * most.value);
      const auto sized = [&](auto lie) { return a.places <= 16 ? go(lie, one) : go(lie, most); };
      if constexpr (!ACROSS) {
        return sized(std::integral_constant<Lie, kRows>{});
      } else {
        if constexpr (WB && RB >= 2)
          if (a.r % 2 == 0) return sized(std::integral_constant<Lie, kPairs>{});
        return sized(std::integral_constant<Lie, kAcross>{});
      }
    });
  });
}

// JOIN: from a.part, else from a.ready.
template <bool ACROSS, bool JOIN>
hipError_t up(UpArgs a, int32_t ydtype, int32_t wdtype, hipStream_t stream) {
  a.places = JOIN || a.T < kManyRows ? 16 : 128;
  const dim3 grid((unsigned)most_tiles(a.T, a.L, a.places), (a.C + kUpWaves * kUpCols - 1) / (kUpWaves * kUpCols));
  const auto go = [&](auto rb) {
    return by_types(ydtype, wdtype, [&](auto yb, auto wb) {
      hipLaunchKernelGGL((k_adapter_up<decltype(yb)::value, decltype(wb)::value, ACROSS, decltype(rb)::value, JOIN>), grid,
                         dim3(kUpWaves * kWave), 0, stream, a);
      return hipGetLastError();
    });
  };
  return a.r <= 8 ? go(std::integral_constant<int, 0>{}) : by_rank<8>(a.rp, go);
}

inline bool sizes_ok(int32_t T, int32_t L, int32_t r, int32_t K, int32_t N) {
  return T >= 0 && T <= DAMOE_MAX_T && L >= 1 && L <= DAMOE_MAX_E && r >= 1 && K >= 1 && N >= 1;
}

inline damoe_status check(int32_t T, int32_t L, int32_t r, int32_t K, int32_t N, int32_t d0, int32_t d1, int32_t d2) {
  if (!sizes_ok(T, L, r, K, N)) return DAMOE_ERR_INVALID_ARG;
  for (const int32_t d : {d0, d1, d2})
    if (d != DAMOE_BF16 && d != DAMOE_F32) return DAMOE_ERR_UNSUPPORTED;
  return r > kMaxRank || K > DAMOE_MAX_COLS || N > DAMOE_MAX_COLS ? DAMOE_ERR_UNSUPPORTED : DAMOE_OK;
}

inline bool aligned(const void* p, int32_t dtype) { return reinterpret_cast<uintptr_t>(p) % (dtype == DAMOE_BF16 ? 2 : 4) == 0; }

inline bool matrix_ok(const void* p, int64_t ld, int32_t cols, int32_t dtype) { return p && ld >= cols && aligned(p, dtype); }

// Bytes of pieces of the workspaces: fp32 parts; what `up` takes.
inline size_t part_bytes(const DownPlan& d, int32_t T, int32_t rp) { return up256((size_t)d.parts * T * rp * 4); }
inline size_t ready_bytes(int32_t T, int32_t rp) { return up256((size_t)T * rp * 6); }

// The most that part_bytes is for up to T_max rows: blocks times parts is at most 512, or the blocks themselves.
inline size_t most_parts(int32_t T_max, int32_t C, int32_t rp) {
  size_t most = 0;
  for (const int32_t t : {kManyRows - 1, T_max}) {
    const int32_t T = std::min(t, T_max), places = down_plan(T, C).places;
    const int32_t parts = ((C + 63) / 64 + kDownWaves - 1) / kDownWaves;
    most = std::max(most, std::min((size_t)T * parts, std::max<size_t>((size_t)T, (size_t)512 * places)) * rp * 4);
  }
  return up256(most);
}

}  // namespace
}  // namespace damoe
