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

#include "adapters_args.h"
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

// Lanes 4 b + a hold of register h element (h, a) of a 4 x 4 block of their own; after it element (a, h).
__device__ __forceinline__ void transpose4(uint32_t& r0, uint32_t& r1, uint32_t& r2, uint32_t& r3) {
  const int lane = threadIdx.x;
  const auto exchange = [](bool upper, auto other, uint32_t& x, uint32_t& y) {
    const uint32_t a = other(y), b = other(x);  // by all lanes
    x = upper ? a : x, y = upper ? y : b;
  };
  const auto one = [](uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xf, 0xf, true); };  // lane ^ 1
  const auto two = [](uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xf, 0xf, true); };  // lane ^ 2
  exchange(lane & 1, one, r0, r1);
  exchange(lane & 1, one, r2, r3);
  exchange(lane & 2, two, r0, r2);
  exchange(lane & 2, two, r1, r3);
}

constexpr int kUnit = 128;  // columns

// 16 rows of a unit of columns.  As operands lane (i, g) needs row i, but 16 lanes that load from 16 rows cost the address
// units a cycle each; four side by side that share 64 bytes cost one together.  So lane 16 g + 4 b + a loads piece a of rows
// 4 b + h, h = 0 .. 3, and four lanes exchange what they have.  Lane (i, g) then has columns 32 g .. + 31 of row i.
template <bool SRC>
struct Rows16 {
  static constexpr int kSets = SRC ? 1 : 2;  // of four pieces of 16 bytes
  uint32_t q[kSets * 4][4];

  // The lane's row number h of those that it loads.
  static __device__ __forceinline__ int mine(int h) { return (threadIdx.x >> 2 & 3) * 4 + h; }

  // at(h): the first element of row mine(h); c: the unit's first column.  Rows from n on are 0 where none of a load's counts.
  template <bool NT = false, class F>
  __device__ __forceinline__ void load(const void* base, F at, int c, int n = 16) {
    typedef Elem<SRC> E;
    const int g = (threadIdx.x & 63) >> 4, a = threadIdx.x & 3;
#pragma unroll
    for (int s = 0; s < kSets; ++s)
#pragma unroll
      for (int h = 0; h < 4; ++h) {
        uint4 v = {0, 0, 0, 0};
        if (h < n) v = load16_at<E::kBytes, NT>(static_cast<const typename E::T*>(base) + (at(h) + (c + 32 * g + (4 * s + a) * E::kPer16)));
        uint32_t(&d)[4] = q[4 * s + h];
        d[0] = v.x, d[1] = v.y, d[2] = v.z, d[3] = v.w;
      }
  }
  __device__ __forceinline__ void exchange() {
#pragma unroll
    for (int s = 0; s < kSets; ++s)
#pragma unroll
      for (int d = 0; d < 4; ++d) transpose4(q[4 * s][d], q[4 * s + 1][d], q[4 * s + 2][d], q[4 * s + 3][d]);
  }
  // Row i, from element `at` on, of which n columns from the lane's first are the row's; no exchange after it.
  __device__ __forceinline__ void load_some(const void* base, int64_t at, int n) {
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      Raw<SRC> f;
      f.load_some(base, at + 8 * t, n - 8 * t);
      put(t, f);
    }
  }
  // Columns 8 t .. + 7 of the lane's.
  __device__ __forceinline__ void put(int t, const Raw<SRC>& f) {
#pragma unroll
    for (int j = 0; j < (SRC ? 4 : 8); ++j) q[SRC ? t : 2 * t + j / 4][j % 4] = f.q[j];
  }
  __device__ __forceinline__ Raw<SRC> get(int t) const {
    Raw<SRC> f;
#pragma unroll
    for (int j = 0; j < (SRC ? 4 : 8); ++j) f.q[j] = q[SRC ? t : 2 * t + j / 4][j % 4];
    return f;
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
// thirds add up to all 24 and the first does not overflow (from 2^-110 on: bf16's smallest step is 2^-133, and what lies below
// it is in none).  An infinity or NaN is its own first third, without others.
__device__ __forceinline__ uint16_t take_third(float& v) {
  const uint32_t b = __float_as_uint(v), hi = b & 0xFFFF0000u;
  const bool finite = (b & 0x7F800000u) != 0x7F800000u;
  v = finite ? v - __uint_as_float(hi) : 0.f;
  return (uint16_t)(hi >> 16 | (!finite && (b & 0xFFFFu) ? 1u : 0u));  // a NaN whose leading bits are an infinity's stays one
}

// Eight values' thirds as operands.  An infinity has one third, a NaN is one in the second.
__device__ __forceinline__ void thirds(const uint32_t (&v)[8], uint4 (&out)[3]) {
  float f[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) f[k] = __uint_as_float(v[k]);
#pragma unroll
  for (int h = 0; h < 3; ++h) {
    uint32_t q[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) q[k] = __builtin_amdgcn_perm(__float_as_uint(f[2 * k + 1]), __float_as_uint(f[2 * k]), 0x07060302u);
    out[h] = uint4{q[0], q[1], q[2], q[3]};
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float rest = f[k] - __uint_as_float(__float_as_uint(f[k]) & 0xFFFF0000u);
      f[k] = h == 0 && __builtin_amdgcn_classf(f[k], 0x204) ? 0.f : rest;
    }
  }
}

// ---------------------------------------------------------------- down

// How the weights lie for `down`: rows of columns (A), or columns of ranks (B), there read one rank a lane, or (bf16, r even)
// two side by side, which are the same row of two blocks of 16 ranks.
enum Lie { kRows, kAcross, kPairs };

// A unit of columns of RB blocks of 16 ranks from r0 on, lane (i, g)'s columns as those of Rows16.
template <bool WB, Lie LIE, int RB>
struct Weights {
  static constexpr int kSets = LIE == kPairs ? RB / 2 : RB;
  typename std::conditional<LIE == kRows, Rows16<WB>[kSets], uint32_t[kSets][4][8]>::type q;

  // The weights from the segment's first on.  `columns` of the unit are the matrix's, the others 0.
  template <bool FULL>
  __device__ __forceinline__ void load(const DownArgs& a, const void* slab, int r0, int c, int columns) {
    typedef typename Elem<WB>::T T;
    struct __attribute__((packed, aligned(2))) Two {
      uint32_t v;
    };
    const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
#pragma unroll
    for (int s = 0; s < kSets; ++s) {
      if constexpr (LIE == kRows) {
        if constexpr (FULL) q[s].load(slab, [&](int h) { return min(r0 + 16 * s + Rows16<WB>::mine(h), a.r - 1) * a.C; }, c);
        else q[s].load_some(slab, min(r0 + 16 * s + i, a.r - 1) * a.C + c + 32 * g, columns - 32 * g);
      } else {
        const int rho = LIE == kPairs ? min(r0 + 32 * s + 2 * i, a.r - 2) : min(r0 + 16 * s + i, a.r - 1);
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const int k = 32 * g + 8 * t + j;
            const T* p = static_cast<const T*>(slab) + (FULL ? c + k : min(c + k, a.C - 1)) * a.r + rho;
            uint32_t& v = q[s][t][j];
            if constexpr (LIE == kPairs) v = reinterpret_cast<const Two*>(p)->v;
            else if constexpr (WB) v = *p;
            else v = __float_as_uint(*p);
            if (!FULL && k >= columns) v = 0;
          }
      }
    }
  }
  __device__ __forceinline__ void exchange() {
    if constexpr (LIE == kRows) {
#pragma unroll
      for (int s = 0; s < kSets; ++s) q[s].exchange();
    }
  }
  template <bool BF>
  __device__ __forceinline__ Frag<BF> get(int rb, int t) const {
    if constexpr (LIE == kRows) {
      return frag<BF>(q[rb].get(t));
    } else {
      const uint32_t(&v)[8] = q[LIE == kPairs ? rb / 2 : rb][t];
      Frag<BF> f;
#pragma unroll
      for (int j = 0; j < (BF ? 4 : 8); ++j) {
        if constexpr (LIE == kPairs) {
          if constexpr (BF) f.q[j] = __builtin_amdgcn_perm(v[2 * j + 1], v[2 * j], rb & 1 ? 0x07060302u : 0x05040100u);
          else f.q[j] = rb & 1 ? v[j] & 0xFFFF0000u : v[j] << 16;
        } else {
          if constexpr (BF) f.q[j] = v[2 * j] | v[2 * j + 1] << 16;
          else f.q[j] = WB ? v[j] << 16 : v[j];
        }
      }
      return f;
    }
  }
};

// Sums over units of columns by W waves in turn, RB blocks of 16 ranks from r0 on and M of 16 places.  A unit is four MFMA
// steps, of each lane's columns 8 t .. + 7.  D units are in flight.
template <bool XB, bool WB, Lie LIE, int RB, int M, int W>
struct Down {
  static constexpr bool BF = XB && WB;
  // fp32 weights of bf16 rows: three thirds of a weight in bf16, whose products are exact, take 48 cycles where 32 fp32
  // instructions for the same columns take 256, and the splitting about 60.
  static constexpr bool kThirds = XB && !WB;
  struct Unit {
    Rows16<XB> x[M];
    Weights<WB, LIE, RB> w;
  };
  static constexpr int kRegs = sizeof(Unit) / 4, D = W > 8 ? (kRegs <= 32 ? 2 : 1) : kRegs <= 32 ? 3 : kRegs <= 72 ? 2 : 1;
  floatx4 acc[M][RB];

  __device__ __forceinline__ void multiply(const Unit& v, bool second) {
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      if constexpr (kThirds) {
        uint4 w[RB][3];
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) thirds(v.w.template get<false>(rb, t).q, w[rb]);
#pragma unroll
        for (int h = 0; h < 3; ++h)
#pragma unroll
          for (int m = 0; m < M; ++m) {
            const Raw<XB> x = v.x[m].get(t);
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) acc[m][rb] = mfma16x16x32(w[rb][h], uint4{x.q[0], x.q[1], x.q[2], x.q[3]}, acc[m][rb]);
          }
        continue;
      }
      Frag<BF> w[RB];
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) w[rb] = v.w.template get<BF>(rb, t);
#pragma unroll
      for (int m = 0; m < M; ++m) {
        if (!BF && m && !second) continue;  // fp32 instructions are long: none for places that the tile does not have
        const Frag<BF> x = frag<BF>(v.x[m].get(t));
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) acc[m][rb] = mma(w[rb], x, acc[m][rb]);
      }
    }
  }
  __device__ __forceinline__ void exchange(Unit& v) {
#pragma unroll
    for (int m = 0; m < M; ++m) v.x[m].exchange();
    v.w.exchange();
  }

  __device__ __forceinline__ void run(const DownArgs& a, const Tile& tile, int u0, int u1, int r0) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Places places(a.perm, a.off);
    const bool second = tile.hi - tile.lo > 16;
    const auto at = [&](int place) { return min(tile.lo + place, tile.hi - 1); };  // past the end the last one
    const auto row = [&](int loaded, int place) {  // its first element
      const int t = places.row(loaded, at(place));
      return (int64_t)((uint32_t)t < (uint32_t)a.T ? t : 0) * a.ldx;
    };
    const char* slab = static_cast<const char*>(a.w) + (int64_t)tile.l * a.r * a.C * Elem<WB>::kBytes;
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) acc[m][rb] = floatx4{0.f, 0.f, 0.f, 0.f};
    const int whole = a.C / kUnit;  // units
    int left = min(u1, whole) - u0 - wave;
    left = left > 0 ? (left + W - 1) / W : 0;
    if (left > 0) {
      int loaded[M][4];
      int64_t rows[M][4];
      const auto load_w = [&](Unit& v, int u) { v.w.template load<true>(a, slab, r0, u * kUnit, kUnit); };
      const auto load_x = [&](Unit& v, int u) {
#pragma unroll
        for (int m = 0; m < M; ++m)
          v.x[m].template load<LIE == kRows>(a.x, [&](int h) { return rows[m][h]; }, u * kUnit, M == 1 ? tile.hi - tile.lo : 16);
      };
      const auto load = [&](Unit& v, int u) {
        load_w(v, u);
        load_x(v, u);
      };
      Unit v[D];
      int u = u0 + wave;
      // The first weights are asked for before perm's entries have come.
#pragma unroll
      for (int m = 0; m < M; ++m)
#pragma unroll
        for (int h = 0; h < 4; ++h) loaded[m][h] = places.load(at(16 * m + Rows16<XB>::mine(h)));
#pragma unroll
      for (int d = 0; d < D; ++d)
        if (d < left) load_w(v[d], u + d * W);
#pragma unroll
      for (int m = 0; m < M; ++m)
#pragma unroll
        for (int h = 0; h < 4; ++h) rows[m][h] = row(loaded[m][h], 16 * m + Rows16<XB>::mine(h));
#pragma unroll
      for (int d = 0; d < D; ++d)
        if (d < left) load_x(v[d], u + d * W);
      for (u += D * W; left >= 2 * D; left -= D) {
#pragma unroll
        for (int d = 0; d < D; ++d, u += W) {
          exchange(v[d]);
          multiply(v[d], second);
          load(v[d], u);
          __builtin_amdgcn_sched_barrier(0);  // or the loads are put behind the next unit's work
        }
      }
#pragma unroll
      for (int d = 0; d < D; ++d, u += W) {
        if (d < left) {
          exchange(v[d]);
          multiply(v[d], second);
        }
        if (d + D < left) load(v[d], u);
      }
#pragma unroll
      for (int d = 0; d < D - 1; ++d)
        if (d + D < left) {
          exchange(v[d]);
          multiply(v[d], second);
        }
    }
    if (whole >= u0 && whole < u1 && (whole - u0) % W == wave) {
      Unit v;
      const int c = whole * kUnit, i = lane & 15, g = lane >> 4;
#pragma unroll
      for (int m = 0; m < M; ++m) v.x[m].load_some(a.x, row(places.load(at(16 * m + i)), 16 * m + i) + c + 32 * g, a.C - c - 32 * g);
      v.w.template load<false>(a, slab, r0, c, a.C - c);
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

// The sums as `up` takes them: thirds in bf16 for bf16 weights, else fp32, in pieces of 16 bytes.  Groups of n <= 16 places
// have piece by piece those of their places side by side, which is how a wave loads an operand: piece b of place i lies at
// 16 (b n + i) of its group.  Piece: 8 ranks of a third, or 4 ranks.
template <bool WB>
struct Ready {
  static constexpr int kBytes = WB ? 6 : 4;  // of a place and rank

  static __device__ __forceinline__ char* group(void* base, int p, int rp) { return static_cast<char*>(base) + (int64_t)p * rp * kBytes; }
  static __device__ __forceinline__ int piece(int third, int rho, int rp) { return WB ? (third * rp + rho) / 8 : rho / 4; }

  // Ranks rho .. + 3 (rho a multiple of 4) of place i.
  static __device__ __forceinline__ void put(char* group, int n, int i, int rho, int rp, floatx4 v) {
#pragma unroll
    for (int h = 0; h < (WB ? 3 : 1); ++h) {
      char* p = group + 16 * (piece(h, rho, rp) * n + i);
      if constexpr (WB) {
        uint16_t q[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          float f = v[k];
          q[k] = take_third(f);
          v[k] = f;
        }
        *reinterpret_cast<uint2*>(p + 2 * (rho % 8)) = uint2{q[0] | (uint32_t)q[1] << 16, q[2] | (uint32_t)q[3] << 16};
      } else {
        *reinterpret_cast<floatx4*>(p) = v;
      }
    }
  }
};

constexpr int kDownWaves = 8;

// More than 64 ranks take a block of the grid for each 64.  Bound by x, which is read past the caches, as what `up` adds
// is (A keeps its place in them), and by the time in which a block finds its tile and adds up its waves, of which there is one a
// CU: 7168 rows of 7168 bf16 at rank 32 30 us (3.4 TB/s; 45 when 16 lanes loaded from 16 rows, 36 with plain loads); 4096
// rows over 256 segments at rank 8, fp32, 27 us for as many bytes of A as of x (4.3 TB/s).  Eight waves of two units in
// flight: sixteen of one took 39 us for 32, three units 37.
template <bool XB, bool WB, Lie LIE, int RB, int M>
__global__ void __launch_bounds__(kDownWaves* kWave) k_adapter_down(DownArgs a) {
  typedef Down<XB, WB, LIE, RB, M, kDownWaves> D;
  extern __shared__ floatx4 red[];
  const int u0 = blockIdx.y * a.units, u1 = min(u0 + a.units, (a.C + kUnit - 1) / kUnit);
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
    const int i = (p - tile.lo) % 16, first = p - i;
    Ready<WB>::put(Ready<WB>::group(a.ready, first, a.rp), min(16, tile.hi - first), i, rho, a.rp, v);
  }
}

// ---------------------------------------------------------------- up

constexpr size_t kSpare = 64 * 16;

// The sums of 16 places as MFMA operands: RB blocks of 16 ranks, or (RB = 0) 8 ranks.  bf16 weights: three thirds, whose
// products are exact, an operand each; of 16 ranks two in one operand over the same weights twice, of 8 ranks all three.
// fp32: instruction j multiplies rank kPer g + j of lane (i, g).
template <bool WB, int RB>
struct Sums {
  static constexpr int kPer = WB ? 8 : RB ? 4 * RB : 2;            // ranks of a lane in an operand
  static constexpr int kBlocks = WB && RB > 2 ? RB / 2 : 1;        // operands for the ranks
  static constexpr int kOps = !WB ? 1 : RB >= 2 ? 3 : RB ? 2 : 1;  // of each: for the thirds
  static constexpr int kWords = WB ? 4 : kPer;
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

  // Place i (at most n - 1) of a group of n.
  __device__ __forceinline__ void load(const char* group, int n, int i, int rp, int g) {
#pragma unroll
    for (int kb = 0; kb < kBlocks; ++kb)
#pragma unroll
      for (int h = 0; h < kOps; ++h) {
        const int rho = rank(kb, g), b = Ready<WB>::piece(min(third(h, g), 2), rho, rp);
        if constexpr (kWords == 2) {
          const uint2 v = *reinterpret_cast<const uint2*>(group + 16 * (b * n + i) + 4 * (rho % 4));
          q[kb][h][0] = v.x, q[kb][h][1] = v.y;
        } else {
#pragma unroll
          for (int e = 0; e < kWords / 4; ++e) {
            const uint4 v = *reinterpret_cast<const uint4*>(group + 16 * ((b + e) * n + i));
            uint32_t* d = &q[kb][h][4 * e];
            d[0] = v.x, d[1] = v.y, d[2] = v.z, d[3] = v.w;
          }
        }
      }
  }
};

// N elements side by side, of 8 to 32 bytes (stores: up to 16).
template <bool YB, int N>
struct Side {
  typedef Elem<YB> E;
  static constexpr int kWords = N * E::kBytes / 4;
  uint32_t q[kWords];

  template <bool NT = false>
  __device__ __forceinline__ void load(const typename E::T* p) {
    if constexpr (kWords >= 4) {
#pragma unroll
      for (int h = 0; h < kWords; h += 4) {
        const uint4 v = load16_at<E::kBytes, NT>(p + h / 4 * E::kPer16);
        q[h] = v.x, q[h + 1] = v.y, q[h + 2] = v.z, q[h + 3] = v.w;
      }
    } else {
      __builtin_memcpy(q, p, sizeof q);
    }
  }
  __device__ __forceinline__ void store(typename E::T* p) const {
    if constexpr (kWords == 4) store16_at<E::kBytes>(p, uint4{q[0], q[1], q[2], q[3]});
    else __builtin_memcpy(p, q, sizeof q);
  }
  // The first n elements are the row's; the others are 0, or left.
  __device__ __forceinline__ void load_some(const typename E::T* p, int n) {
    if (n >= N) return load(p);
#pragma unroll
    for (uint32_t& e : q) e = 0;
#pragma unroll
    for (int j = 0; j < N; ++j)
      if (j < n) {
        if constexpr (YB) q[j / 2] |= (uint32_t)p[j] << (16 * (j & 1));
        else q[j] = __float_as_uint(p[j]);
      }
  }
  __device__ __forceinline__ void store_some(typename E::T* p, int n) const {
    if (n >= N) return store(p);
#pragma unroll
    for (int j = 0; j < N; ++j)
      if (j < n) {
        if constexpr (YB) p[j] = (uint16_t)(q[j / 2] >> (16 * (j & 1)));
        else p[j] = __uint_as_float(q[j]);
      }
  }
  __device__ __forceinline__ float get(int j) const {
    if constexpr (YB) return __uint_as_float(j & 1 ? q[j / 2] & 0xFFFF0000u : q[j / 2] << 16);
    else return __uint_as_float(q[j]);
  }
  __device__ __forceinline__ void put(const float (&f)[N]) {
#pragma unroll
    for (int j = 0; j < kWords; ++j) {
      if constexpr (YB) q[j] = pack_bf16x2(f[2 * j], f[2 * j + 1]);
      else q[j] = __float_as_uint(f[j]);
    }
  }
};

// 16 places by 16 NB columns of a wave.  MFMA b has column NB i + b as its column i, so that lane (i, g) has NB columns side by
// side of places 4 g .. + 3, and 16 lanes 16 NB: rows are read and written in pieces of 128 to 256 bytes.
template <bool YB, bool WB, int RB>
struct Up {
  typedef Sums<WB, RB> S;
  typedef Elem<YB> E;
  typedef typename E::T Y;
  // 8 blocks of 128 fp32 ranks would take all registers.
  static constexpr int NB = !WB && RB == 8 ? 4 : E::kPer16, kCols = 16 * NB;

  // The weights of the wave's columns from c0 on, 0 for ranks from r on.
  struct Weights {
    uint32_t q[NB][S::kBlocks][S::kWords];

    // n ranks from element i on; ACROSS: `apart` elements from one to the next.
    template <bool ACROSS>
    static __device__ __forceinline__ void ranks(uint32_t (&q)[S::kWords], const void* base, int64_t i, int64_t apart, int n) {
      typedef Elem<WB> F;
      const typename F::T* p = static_cast<const typename F::T*>(base) + i;
      if (!ACROSS && n >= S::kPer) {
        if constexpr (S::kWords == 2) {
          q[0] = __float_as_uint(p[0]), q[1] = __float_as_uint(p[1]);
        } else {
#pragma unroll
          for (int e = 0; e < S::kWords; e += 4) {
            const uint4 v = load16_at<F::kBytes>(p + (WB ? 0 : e));
            q[e] = v.x, q[e + 1] = v.y, q[e + 2] = v.z, q[e + 3] = v.w;
          }
        }
        return;
      }
      uint32_t v[S::kPer];
#pragma unroll
      for (int j = 0; j < S::kPer; ++j) {  // past the last rank: that one again, and not used
        const typename F::T* at = p + (ACROSS ? min(j, n - 1) * apart : min(j, n - 1));
        if constexpr (WB) v[j] = *at;
        else v[j] = __float_as_uint(*at);
        if (j >= n) v[j] = 0;
      }
#pragma unroll
      for (int e = 0; e < S::kWords; ++e) q[e] = WB ? v[2 * e % S::kPer] | v[(2 * e + 1) % S::kPer] << 16 : v[e % S::kPer];
    }

    // Columns of ranks: 16 lanes that load from a column each would cost the address units 16 times.  The wave reads runs of
    // the lanes' columns, 256 bytes from 16 lanes, and its operands come from LDS; CB of a lane's NB columns at a time.
    static constexpr int kPadded = WB ? (RB ? 16 * RB : 8) : 4 * S::kPer, kColumn = kPadded * Elem<WB>::kBytes;
    static constexpr bool kStaged = kColumn <= 256;
    static constexpr int CB = kColumn * NB <= 256 ? NB : 256 / kColumn, kRun = CB * kColumn + 16;  // 16 bytes against bank conflicts
    static constexpr int kLds = kStaged ? 16 * kRun : 16;  // bytes of a wave

    __device__ __forceinline__ void load_runs(const UpArgs& a, int64_t slab, int c0, char* lds) {
      typedef Elem<WB> F;
      typedef typename F::T T;
      const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
      const T* w = static_cast<const T*>(a.w) + slab + (int64_t)c0 * a.r;
#pragma unroll
      for (int b0 = 0; b0 < NB; b0 += CB) {
        if (a.r % F::kPer16 == 0) {
          const int pieces = a.r / F::kPer16, run = CB * pieces;  // of 16 bytes; at most 16 a run
          const float per_run = 1.f / run, per_column = 1.f / pieces;
          uint4 v[4];
          int to[4];
#pragma unroll
          for (int y = 0; y < 4; ++y) {  // past the last one that one again
            const int e = min(64 * y + lane, 16 * run - 1);
            const int lane_of = (int)((e + 0.5f) * per_run), k = e - lane_of * run, column = (int)((k + 0.5f) * per_column);
            v[y] = load16_at<F::kBytes>(w + (NB * lane_of + b0) * a.r + k * F::kPer16);
            to[y] = lane_of * kRun + column * kColumn + (k - column * pieces) * 16;
          }
#pragma unroll
          for (int y = 0; y < 4; ++y) *reinterpret_cast<uint4*>(lds + to[y]) = v[y];
        } else {
          const int run = CB * a.r;
#pragma unroll 4
          for (int e = lane; e < 16 * run; e += 64) {
            const int lane_of = e / run, k = e - lane_of * run, column = k / a.r;
            *reinterpret_cast<T*>(lds + lane_of * kRun + column * kColumn + (k - column * a.r) * F::kBytes) =
                w[(NB * lane_of + b0) * a.r + k];
          }
        }
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int b = 0; b < CB; ++b)
#pragma unroll
          for (int kb = 0; kb < S::kBlocks; ++kb) {
            const int rho = S::rank(kb, g), n = a.r - rho;
            uint32_t(&d)[S::kWords] = q[b0 + b][kb];
            const char* from = lds + i * kRun + b * kColumn + rho * F::kBytes;
            if constexpr (S::kWords == 2) {
              const uint2 v = *reinterpret_cast<const uint2*>(from);
              d[0] = v.x, d[1] = v.y;
            } else {
#pragma unroll
              for (int e = 0; e < S::kWords; e += 4) {
                const uint4 v = *reinterpret_cast<const uint4*>(from + 4 * e);
                d[e] = v.x, d[e + 1] = v.y, d[e + 2] = v.z, d[e + 3] = v.w;
              }
            }
#pragma unroll
            for (int e = 0; e < S::kWords; ++e) {
              if constexpr (WB) d[e] &= (2 * e < n ? 0xFFFFu : 0u) | (2 * e + 1 < n ? 0xFFFF0000u : 0u);
              else d[e] = e < n ? d[e] : 0u;
            }
          }
        __builtin_amdgcn_wave_barrier();
      }
    }

    // lds: kLds bytes of the wave.
    template <bool ACROSS>
    __device__ __forceinline__ void load(const UpArgs& a, int l, int c0, char* lds) {
      const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
      const int64_t slab = (int64_t)l * a.r * a.C;
      if constexpr (!ACROSS && kStaged) {
        if (c0 + kCols <= a.C) return load_runs(a, slab, c0, lds);
      }
      if (ACROSS && c0 + kCols <= a.C) {  // the lane's columns of a rank are side by side
#pragma unroll
        for (int kb = 0; kb < S::kBlocks; ++kb) {
          const int rho = S::rank(kb, g), n = a.r - rho;
          Side<WB, NB> v[S::kPer];
#pragma unroll
          for (int j = 0; j < S::kPer; ++j)
            v[j].load(static_cast<const typename Elem<WB>::T*>(a.w) + slab + (int64_t)(rho + min(j, n - 1)) * a.C + c0 + NB * i);
#pragma unroll
          for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int e = 0; e < S::kWords; ++e) {
              if constexpr (WB) {
                const uint32_t two = __builtin_amdgcn_perm(v[2 * e + 1].q[b / 2], v[2 * e].q[b / 2], b & 1 ? 0x07060302u : 0x05040100u);
                q[b][kb][e] = two & ((2 * e < n ? 0xFFFFu : 0u) | (2 * e + 1 < n ? 0xFFFF0000u : 0u));
              } else {
                q[b][kb][e] = e < n ? v[e].q[b] : 0u;
              }
            }
        }
        return;
      }
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        const int c = min(c0 + NB * i + b, a.C - 1);
#pragma unroll
        for (int kb = 0; kb < S::kBlocks; ++kb) {
          const int rho = S::rank(kb, g);
          ranks<ACROSS>(q[b][kb], a.w, slab + (ACROSS ? (int64_t)rho * a.C + c : (int64_t)c * a.r + rho), a.C, a.r - rho);
        }
      }
    }
  };

  S u;
  Side<YB, NB> add[4];
  int t[4];  // rows of places 4 g .. + 3, -1: none

  // Lane by lane the row of place i of the group, -1: none.
  __device__ __forceinline__ void rows(int row) {
    const int g = (threadIdx.x & 63) >> 4;
#pragma unroll
    for (int e = 0; e < 4; ++e) t[e] = __shfl(row, 4 * g + e);
  }
  // FULL: all of the wave's columns are the matrix's.  `zero`: a buffer that is read where there is nothing to add, and not used.
  template <bool FULL>
  __device__ __forceinline__ void load_add(const UpArgs& a, const void* zero, int c0) {
    const int c = c0 + NB * (threadIdx.x & 15), n = a.C - c;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (FULL) {
        const Y* base = static_cast<const Y*>(a.add ? a.add : zero);
        add[e].template load<true>(base + (a.add ? max(t[e], 0) * a.lda + c : 0));
      } else {
        add[e] = Side<YB, NB>{};
        if (a.add && t[e] >= 0 && n > 0) add[e].load_some(static_cast<const Y*>(a.add) + t[e] * a.lda + c, n);
      }
    }
  }

  // The rows are add + s times the product.
  template <bool FULL>
  __device__ __forceinline__ void work(const UpArgs& a, const Weights& w, int c0, float s) {
    const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
    floatx4 acc[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) acc[b] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int kb = 0; kb < S::kBlocks; ++kb)
#pragma unroll
      for (int h = 0; h < S::kOps; ++h) {
        const uint32_t(&v)[S::kWords] = u.q[kb][h];
        if constexpr (WB) {
          const bool none = S::third(h, g) >= 3;
          const uint4 f = none ? uint4{0, 0, 0, 0} : uint4{v[0], v[1], v[2], v[3]};
#pragma unroll
          for (int b = 0; b < NB; ++b) {
            const uint32_t(&x)[S::kWords] = w.q[b][kb];
            acc[b] = mfma16x16x32(f, uint4{x[0], x[1], x[2], x[3]}, acc[b]);
          }
        } else {
#pragma unroll
          for (int j = 0; j < S::kWords; ++j)
#pragma unroll
            for (int b = 0; b < NB; ++b) acc[b] = mma4(v[j], w.q[b][kb][j], acc[b]);
        }
      }
    const int c = c0 + NB * i;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (!FULL && (t[e] < 0 || c >= a.C)) continue;
      float f[NB];
#pragma unroll
      for (int b = 0; b < NB; ++b) f[b] = fmaf(s, acc[b][e], FULL && !a.add ? 0.f : add[e].get(b));
      Side<YB, NB> v;
      v.put(f);
      Y* p = static_cast<Y*>(a.y) + t[e] * a.ldy + c;
      // The store is there for places without a row too, so that the wait for the next loads can count it.
      if constexpr (FULL) v.store(t[e] < 0 ? reinterpret_cast<Y*>(a.spare + 16 * lane) : p);
      else v.store_some(p, a.C - c);
    }
  }
};

// Few rows: bound by the chain of a launch, the tile, the parts, the product (61 rows of 48 segments, 7168 columns, rank 16: 5.5 us).
// A tile of at most 16 places whose parts are added here, in LDS for the block's waves; c0: the wave's columns.  `first`: the
// block that keeps u.
template <bool YB, bool WB, bool ACROSS, int RB>
struct UpJoin {
  typedef Up<YB, WB, RB> U;
  typedef Ready<WB> R;
  static constexpr int kRanks = RB ? 16 * RB : 16, kSums = 16 * kRanks * R::kBytes;
  static constexpr int kRuns = ACROSS ? 0 : U::Weights::kLds;  // bytes of LDS for a wave, behind kSums of the block

  static __device__ __forceinline__ void run(const UpArgs& a, const Tile& tile, int c0, bool first, char* lds) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int i = lane & 15, g = lane >> 4;
    const float s = a.scale ? a.scale[tile.l] : 1.f;
    const Places places(a.perm, a.off);
    const int p = min(tile.lo + i, tile.hi - 1), row = places.row(places.load(p), p);
    const int n = tile.hi - tile.lo;
    const auto part = [&](int e, int k) {
      const int at = min(e / (kRanks / 4), n - 1), rho = 4 * (e % (kRanks / 4));
      return *reinterpret_cast<const floatx4*>(a.part + ((int64_t)min(k, a.parts - 1) * a.T + tile.lo + at) * a.rp + rho);
    };
    floatx4 q[4];  // of the thread's first sums, asked for before the weights are waited for
#pragma unroll
    for (int j = 0; j < 4; ++j) q[j] = part(threadIdx.x, j);
    U v;
    typename U::Weights w;
    if (c0 < a.C) {
      w.template load<ACROSS>(a, tile.l, c0, lds + kSums + wave * kRuns);
      v.rows(tile.lo + i < tile.hi && (uint32_t)row < (uint32_t)a.T ? row : -1);
      v.template load_add<false>(a, nullptr, c0);
    }
    for (int e = threadIdx.x; e < 16 * kRanks / 4; e += kUpWaves * kWave) {
      const int at = e / (kRanks / 4), rho = 4 * (e % (kRanks / 4));
      floatx4 f = {0.f, 0.f, 0.f, 0.f};
      for (int k = 0; k < a.parts; k += 4) {  // in order, four loads in flight
        if (k || e != (int)threadIdx.x) {
#pragma unroll
          for (int j = 0; j < 4; ++j) q[j] = part(e, k + j);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (k + j < a.parts) f += q[j];
      }
      if (at >= n) f = floatx4{0.f, 0.f, 0.f, 0.f};
      if (a.u && first && at < n) {
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (rho + k < a.r) a.u[(int64_t)(tile.lo + at) * a.r + rho + k] = f[k];
      }
      R::put(lds, 16, at, rho, kRanks, f);
    }
    __syncthreads();
    if (c0 >= a.C) return;
    v.u.load(lds, 16, i, kRanks, g);
    v.template work<false>(a, w, c0, s);
  }
};

template <bool YB, bool WB, int RB>
__global__ void __launch_bounds__(kUpWaves* kWave) k_adapter_up_join(UpArgs a) {
  typedef UpJoin<YB, WB, false, RB> J;
  __shared__ __align__(16) char lds[J::kSums + kUpWaves * J::kRuns];
  Tile tile;
  if (!find_tile<false>(a.off, a.L, a.T, a.places, blockIdx.x, tile)) return;
  J::run(a, tile, (blockIdx.y * kUpWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6)) * J::U::kCols, blockIdx.y == 0, lds);
}

// A tile of any places, in steps of 16, whose sums are a.ready's; c0: the wave's columns.  Bound by what is added and written:
// 7168 rows of 4096 bf16 at rank 32 28 us (4.2 TB/s; 38 in pieces of 64 bytes), a tile of 128 places being as long as 1024
// blocks at once allow (64 places 31 us).
template <bool YB, bool WB, bool ACROSS, int RB>
struct UpStream {
  typedef Up<YB, WB, RB> U;
  typedef Ready<WB> R;
  static constexpr int kRuns = ACROSS ? 0 : U::Weights::kLds;  // bytes of LDS for a wave

  static __device__ __forceinline__ void run(const UpArgs& a, const Tile& tile, int c0, char* mine) {
    if (c0 >= a.C) return;
    const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
    const bool full = c0 + U::kCols <= a.C;
    const float s = a.scale ? a.scale[tile.l] : 1.f;
    const Places places(a.perm, a.off);
    const auto place = [&](int step) { return places.load(min(tile.lo + 16 * step + i, tile.hi - 1)); };
    const auto row = [&](int loaded, int step) {  // -1: none
      const int p = tile.lo + 16 * step + i, t = places.row(loaded, p);
      return p < tile.hi && (uint32_t)t < (uint32_t)a.T ? t : -1;
    };
    typename U::Weights w;
    const int steps = (tile.hi - tile.lo + 15) / 16;
    const auto load = [&](auto all, U& v, int t, int step) {
      const int p = tile.lo + 16 * min(step, steps - 1), n = min(16, tile.hi - p);
      v.u.load(R::group(a.ready, p, a.rp), n, min(i, n - 1), a.rp, g);
      v.rows(t);
      v.template load_add<decltype(all)::value>(a, a.ready, c0);
    };
    const std::true_type yes;
    const std::false_type no;
    constexpr bool kAhead = RB < 8;  // of 128 ranks there are no registers for a second step
    if (full && kAhead && steps > 1) {
      U v[2];
      int loaded[2] = {place(0), place(1)};
      w.template load<ACROSS>(a, tile.l, c0, mine);
      load(yes, v[0], row(loaded[0], 0), 0);
      for (int step = 0; step < steps; step += 2) {
        loaded[0] = place(step + 2);
        load(yes, v[1], row(loaded[1], step + 1), step + 1);
        v[0].template work<true>(a, w, c0, s);
        loaded[1] = place(step + 3);
        load(yes, v[0], row(loaded[0], step + 2), step + 2);
        if (step + 1 < steps) v[1].template work<true>(a, w, c0, s);
      }
      return;
    }
    const int first = place(0);
    w.template load<ACROSS>(a, tile.l, c0, mine);
    for (int step = 0; step < steps; ++step) {
      U v;
      const int t = row(step ? place(step) : first, step);
      if (full) {
        load(yes, v, t, step);
        v.template work<true>(a, w, c0, s);
      } else {
        load(no, v, t, step);
        v.template work<false>(a, w, c0, s);
      }
    }
  }
};

template <bool YB, bool WB, bool ACROSS, int RB>
__global__ void __launch_bounds__(kUpWaves* kWave) k_adapter_up(UpArgs a) {
  typedef UpStream<YB, WB, ACROSS, RB> S;
  __shared__ __align__(16) char runs[ACROSS ? 16 : kUpWaves * S::kRuns];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  Tile tile;
  if (find_tile<false>(a.off, a.L, a.T, a.places, blockIdx.x, tile))
    S::run(a, tile, (blockIdx.y * kUpWaves + wave) * S::U::kCols, runs + wave * S::kRuns);
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
// blocks enough without a split over the columns, and what it leaves is what `up` takes.  Parts joined / streamed, us, rows in
// random order, bf16, 7168 to 4096: 8 adapters of rank 16, 2048 rows 26.4 / 29.6, 3000 29.4 / 31.2, 4096 39.2 / 38.5, 6000 51.5 /
// 43.3; 48 of rank 32, 2048 rows 38.4 / 39.0, 3000 44.4 / 42.6, 4096 58.8 / 46.8; of rank 64 from 2048 rows on (56.5 / 52.5) streams
// are faster; 2048 to 2048, 48 of rank 16, 4096 rows 23.1 / 25.7.
constexpr int32_t kManyRows = 4096;

struct DownPlan {
  int32_t places, parts, units;
};

inline DownPlan down_plan(int32_t T, int32_t C) {
  DownPlan d;
  d.places = T < kManyRows ? 16 : 32;
  const int32_t blocks = (T + d.places - 1) / d.places, units = (C + kUnit - 1) / kUnit;
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

inline int32_t up_places(int32_t T) { return T < kManyRows ? 16 : 128; }

// JOIN: from a.part, else from a.ready.
template <bool ACROSS, bool JOIN>
hipError_t up(UpArgs a, int32_t ydtype, int32_t wdtype, hipStream_t stream) {
  a.places = JOIN ? 16 : up_places(a.T);
  dim3 grid((unsigned)most_tiles(a.T, a.L, a.places));
  const auto go = [&](auto rb) {
    return by_types(ydtype, wdtype, [&](auto yb, auto wb) {
      constexpr bool YB = decltype(yb)::value, WB = decltype(wb)::value;
      constexpr int RB = decltype(rb)::value, kCols = kUpWaves * Up<YB, WB, RB>::kCols;
      grid.y = (a.C + kCols - 1) / kCols;
      if constexpr (JOIN) hipLaunchKernelGGL((k_adapter_up_join<YB, WB, RB>), grid, dim3(kUpWaves * kWave), 0, stream, a);
      else hipLaunchKernelGGL((k_adapter_up<YB, WB, ACROSS, RB>), grid, dim3(kUpWaves * kWave), 0, stream, a);
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
    const int32_t parts = ((C + kUnit - 1) / kUnit + kDownWaves - 1) / kDownWaves;
    most = std::max(most, std::min((size_t)T * parts, std::max<size_t>((size_t)T, (size_t)512 * places)) * rp * 4);
  }
  return up256(most);
}

}  // namespace
}  // namespace damoe
