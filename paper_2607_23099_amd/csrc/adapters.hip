// Low-rank adapters of many segments of rows at once: damoe_adapters and its gradient.
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
#include "vec.h"

namespace damoe {
namespace {

constexpr int kMaxRank = DAMOE_MAX_RANK;
constexpr int kDownWaves = 8, kUpWaves = 4, kOuterWaves = 4;

// ---------------------------------------------------------------- segments

// Places [lo, hi) of segment l, tile number `index` of its; `slot`: the number of tiles before it that belong to segments of
// several tiles.
struct Tile {
  int l, lo, hi, index, slot;
  bool whole;  // the segment's only tile
};

// Tiles of the segment that lane's number l names.
struct Length {
  int s, n;
  int e;
  __device__ __forceinline__ Length(const int32_t* off, int L, int T, int P, int l) {
    s = l < L ? min(max(off[l], 0), T) : 0;
    e = l < L ? min(max(off[l + 1], s), T) : 0;
    n = (int)((uint32_t)(e - s + P - 1) / (uint32_t)P);
  }
  __device__ __forceinline__ int split() const { return n > 1 ? n : 0; }
};

__device__ __forceinline__ int scan(int v, int lane) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int u = __shfl_up(v, d);
    if (lane >= d) v += u;
  }
  return v;
}

// Tile number b of all, segments in order, each in tiles of P places; false past the last.  By each wave for itself: lane i
// counts segments i S .. + S - 1, and (L > 64) the lanes then the segments of the one that has the tile.
template <bool SLOTS>
__device__ __forceinline__ bool find_tile(const int32_t* off, int L, int T, int P, int b, Tile& t) {
  const int lane = threadIdx.x & 63, S = (L + 63) / 64;
  Length x(off, L, T, P, lane * S);
  int n = x.n, m = x.split();
  for (int j = 1; j < S; ++j) {
    const Length y(off, L, T, P, lane * S + j);
    n += y.n;
    if constexpr (SLOTS) m += y.split();
  }
  int base = 0, slots = 0, l = 0;
  for (int level = 0;; ++level) {
    const int sum = scan(n, lane);
    const int split = SLOTS ? scan(m, lane) : 0;
    const uint64_t hit = __ballot(sum > b - base);
    if (!hit) return false;
    const int w = __builtin_amdgcn_readfirstlane(__builtin_ctzll(hit));
    base += __builtin_amdgcn_readlane(sum - n, w);
    slots += __builtin_amdgcn_readlane(split - m, w);
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
int64_t most_tiles(int32_t T, int32_t L, int32_t P) {
  const int64_t n = std::min(T, L);
  return (T + n * (P - 1)) / P;
}

__device__ __forceinline__ int row_at(const int32_t* perm, int p) { return perm ? perm[p] : p; }

// ---------------------------------------------------------------- operands

// Eight elements of one row of an MFMA operand: lane i + 16 g has row i, and g's eight of the 32 that are multiplied.
template <bool BF>
struct Frag;
template <>
struct Frag<true> {
  uint32_t q[4] = {0, 0, 0, 0};
  __device__ __forceinline__ void set(int j, uint16_t v) { q[j / 2] |= (uint32_t)v << (16 * (j & 1)); }
};
template <>
struct Frag<false> {
  float q[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  __device__ __forceinline__ void set(int j, float v) { q[j] = v; }
  __device__ __forceinline__ void set(int j, uint16_t v) { q[j] = bf16_to_f32(v); }
};

// c += rows x rows over 32: one bf16 instruction, or eight fp32 ones (instruction j multiplies element j of every lane).
__device__ __forceinline__ floatx4 mma(const Frag<true>& a, const Frag<true>& b, const floatx4& c) {
  return mfma16x16x32(uint4{a.q[0], a.q[1], a.q[2], a.q[3]}, uint4{b.q[0], b.q[1], b.q[2], b.q[3]}, c);
}
__device__ __forceinline__ floatx4 mma(const Frag<false>& a, const Frag<false>& b, floatx4 c) {
#pragma unroll
  for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.q[j], b.q[j], c, 0, 0, 0);
  return c;
}

// Eight elements side by side, of which n are the row's (the others 0).  SRC: bf16 in memory.  FULL: n is at least 8.
template <bool SRC, bool BF, bool FULL>
__device__ __forceinline__ void load8(Frag<BF>& f, const void* base, int64_t i, int n) {
  static_assert(SRC || !BF, "fp32 is not rounded to bf16");
  typedef typename Elem<SRC>::T T;
  const T* p = static_cast<const T*>(base) + i;
  if (FULL || n >= 8) {
    if constexpr (SRC) {
      const uint4 v = load16_at<2>(p);
      if constexpr (BF) {
        f.q[0] = v.x, f.q[1] = v.y, f.q[2] = v.z, f.q[3] = v.w;
      } else {
        unpack16<true>(v, f.q);
      }
    } else {
      const uint4 a = load16_at<4>(p), b = load16_at<4>(p + 4);
      f.q[0] = __uint_as_float(a.x), f.q[1] = __uint_as_float(a.y), f.q[2] = __uint_as_float(a.z), f.q[3] = __uint_as_float(a.w);
      f.q[4] = __uint_as_float(b.x), f.q[5] = __uint_as_float(b.y), f.q[6] = __uint_as_float(b.z), f.q[7] = __uint_as_float(b.w);
    }
  } else {
    f = Frag<BF>{};
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < n) f.set(j, p[j]);
  }
}

// The same of eight elements `step` apart.
template <bool SRC, bool BF, bool FULL>
__device__ __forceinline__ void load8_apart(Frag<BF>& f, const void* base, int64_t i, int64_t step, int n) {
  typedef typename Elem<SRC>::T T;
  const T* p = static_cast<const T*>(base) + i;
  f = Frag<BF>{};
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (FULL || j < n) f.set(j, p[j * step]);
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

// Weight rows rho = lane % 16 of block rb: 8 columns from c on.  ACROSS: the weights lie column by column (B).
template <bool WB, bool BF, bool ACROSS, bool FULL>
__device__ __forceinline__ void weight8(Frag<BF>& f, const DownArgs& a, int64_t slab, int rho, int c, int n) {
  if constexpr (ACROSS) load8_apart<WB, BF, FULL>(f, a.w, slab + (int64_t)c * a.r + rho, a.r, n);
  else load8<WB, BF, FULL>(f, a.w, slab + (int64_t)rho * a.C + c, n);
}

// RB blocks of 16 ranks (more than 64 take a block of the grid each), M of 16 places.  A unit of 64 columns is two MFMA
// steps: lane (i, g) takes columns 16 g .. + 7 of it in the first and 16 g + 8 .. + 15 in the second, so that its loads of a
// row are 32 bytes (bf16) side by side.  The operands of a unit are loaded while the one before is multiplied.
template <bool XB, bool WB, bool ACROSS, int RB, int M>
__global__ void __launch_bounds__(kDownWaves* kWave) k_adapter_down(DownArgs a) {
  constexpr bool BF = XB && WB;
  extern __shared__ floatx4 red[];  // [kDownWaves][M RB][64]
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int i = lane & 15, g = lane >> 4;
  const int u0 = blockIdx.y * a.units, u1 = min(u0 + a.units, (a.C + 63) / 64);
  const int r0 = blockIdx.z * 16 * RB;
  Tile tile;
  if (!find_tile<false>(a.off, a.L, a.T, a.places, blockIdx.x, tile)) return;
  int64_t row[M];
#pragma unroll
  for (int m = 0; m < M; ++m) {
    const int p = tile.lo + 16 * m + i, t = row_at(a.perm, p < tile.hi ? p : tile.lo);
    row[m] = (int64_t)((uint32_t)t < (uint32_t)a.T ? t : 0) * a.ldx;
  }
  const int64_t slab = (int64_t)tile.l * a.r * a.C;
  floatx4 acc[M][RB];
#pragma unroll
  for (int m = 0; m < M; ++m)
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) acc[m][rb] = floatx4{0.f, 0.f, 0.f, 0.f};
  Frag<BF> fx[2][2][M], fw[2][2][RB];
  const auto load = [&](auto buf, int u) {
    constexpr int b = decltype(buf)::value;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int c = u * 64 + 16 * g + 8 * h, n = a.C - c;
      if (u * 64 + 64 <= a.C) {
#pragma unroll
        for (int m = 0; m < M; ++m) load8<XB, BF, true>(fx[b][h][m], a.x, row[m] + c, 8);
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) weight8<WB, BF, ACROSS, true>(fw[b][h][rb], a, slab, min(r0 + 16 * rb + i, a.r - 1), c, 8);
      } else {
#pragma unroll
        for (int m = 0; m < M; ++m) load8<XB, BF, false>(fx[b][h][m], a.x, row[m] + c, n);
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) weight8<WB, BF, ACROSS, false>(fw[b][h][rb], a, slab, min(r0 + 16 * rb + i, a.r - 1), c, n);
      }
    }
  };
  const auto multiply = [&](auto buf) {
    constexpr int b = decltype(buf)::value;
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int m = 0; m < M; ++m)
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) acc[m][rb] = mma(fw[b][h][rb], fx[b][h][m], acc[m][rb]);
  };
  const std::integral_constant<int, 0> even;
  const std::integral_constant<int, 1> odd;
  int u = u0 + wave;
  if (u < u1) load(even, u);
  for (; u < u1; u += 2 * kDownWaves) {
    if (u + kDownWaves < u1) load(odd, u + kDownWaves);
    multiply(even);
    if (u + 2 * kDownWaves < u1) load(even, u + 2 * kDownWaves);
    if (u + kDownWaves < u1) multiply(odd);
  }
  // The waves' sums in order.  Lane (i, g) holds place i, ranks 4 g .. + 3 of each block.
#pragma unroll
  for (int m = 0; m < M; ++m)
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) red[(wave * M * RB + m * RB + rb) * 64 + lane] = acc[m][rb];
  __syncthreads();
  const float s = a.scale ? a.scale[tile.l] : 1.f;
  for (int e = threadIdx.x; e < M * RB * 64; e += kDownWaves * kWave) {
    floatx4 v = red[e];
#pragma unroll
    for (int w = 1; w < kDownWaves; ++w) v += red[w * M * RB * 64 + e];
    const int p = tile.lo + 16 * (e / (64 * RB)) + (e & 15), rho = r0 + 16 * (e / 64 % RB) + 4 * (e / 16 % 4);
    if (p >= tile.hi) continue;
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
        *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.ready) + ((int64_t)h * a.T + p) * a.rp + rho) =
            uint2{q[0] | (uint32_t)q[1] << 16, q[2] | (uint32_t)q[3] << 16};
      }
    } else {
      *reinterpret_cast<floatx4*>(static_cast<float*>(a.ready) + (int64_t)p * a.rp + rho) = v;
    }
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

// The r sums of 16 places as MFMA operands.  bf16 weights: three thirds, whose products are exact, one an operand (of 16
// ranks two in one operand, over the same weights twice); else fp32.
template <bool WB, int RB>
struct Sums {
  static constexpr bool kTwo = WB && RB == 1;
  static constexpr int kBlocks = (RB + 1) / 2;  // of 32 ranks
  static constexpr int kFrags = !WB ? 1 : kTwo ? 2 : 3;
  static constexpr int kPlanes = WB ? 3 : 1;
  static constexpr int kStride = 16 * RB + (WB ? 8 : 4);  // in LDS, of a place
  typedef typename std::conditional<WB, uint16_t, float>::type T;
  Frag<WB> f[kBlocks][kFrags];

  // Row p of planes `plane` elements apart, rows of `stride`.
  __device__ __forceinline__ void load(const T* base, int64_t plane, int64_t p, int stride, int g) {
#pragma unroll
    for (int kb = 0; kb < kBlocks; ++kb)
#pragma unroll
      for (int h = 0; h < kFrags; ++h) {
        const int third = kTwo ? 2 * h + g / 2 : h, rho = 32 * kb + 8 * (kTwo ? g & 1 : g);
        f[kb][h] = Frag<WB>{};
        if (third >= kPlanes || rho >= 16 * RB) continue;
        const uint4* s = reinterpret_cast<const uint4*>(base + third * plane + p * stride + rho);
        const uint4 v = s[0];
        if constexpr (WB) {
          f[kb][h].q[0] = v.x, f[kb][h].q[1] = v.y, f[kb][h].q[2] = v.z, f[kb][h].q[3] = v.w;
        } else {
          unpack16<false>(v, *reinterpret_cast<float(*)[4]>(f[kb][h].q));
          unpack16<false>(s[1], *reinterpret_cast<float(*)[4]>(f[kb][h].q + 4));
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

// A wave has 64 columns, as four MFMA blocks of 16: row i of block 2 q + m is column 32 q + 8 (i / 4) + 4 m + i % 4, so that
// a lane's results of a pair are eight columns side by side of its place.  JOIN: at most 16 places, whose parts are added
// here, in LDS for the block's waves.
template <bool YB, bool WB, bool ACROSS, int RB, bool JOIN>
__global__ void __launch_bounds__(kUpWaves* kWave) k_adapter_up(UpArgs a) {
  typedef Sums<WB, RB> S;
  typedef Elem<YB> E;
  typedef typename E::T Y;
  constexpr int KB = S::kBlocks, P = 8 / E::kPer16;  // blocks of 32 ranks, 16-byte pieces of eight columns
  __shared__ __align__(16) typename S::T lds[JOIN ? S::kPlanes * 16 * S::kStride : 8];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int i = lane & 15, g = lane >> 4;
  Tile tile;
  if (!find_tile<false>(a.off, a.L, a.T, a.places, blockIdx.x, tile)) return;
  const int c0 = (blockIdx.y * kUpWaves + wave) * kUpCols;
  const int64_t slab = (int64_t)tile.l * a.r * a.C;
  const float s = a.scale ? a.scale[tile.l] : 1.f;
  Frag<WB> fw[4][KB];
#pragma unroll
  for (int b = 0; b < 4; ++b) {
    const int c = min(c0 + 32 * (b / 2) + 8 * (i / 4) + 4 * (b & 1) + i % 4, a.C - 1);
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      const int rho = 32 * kb + 8 * (S::kTwo ? g & 1 : g);
      if constexpr (ACROSS) load8_apart<WB, WB, false>(fw[b][kb], a.w, slab + (int64_t)rho * a.C + c, a.C, a.r - rho);
      else load8<WB, WB, false>(fw[b][kb], a.w, slab + (int64_t)c * a.r + rho, a.r - rho);
    }
  }
  struct Rows {
    int t;
    S u;
    uint4 add[2][P];
  };
  const auto load = [&](Rows& v, int p0) {
    const int p = p0 + i;
    v.t = p < tile.hi ? row_at(a.perm, p) : -1;
    if ((uint32_t)v.t >= (uint32_t)a.T) v.t = -1;
    if constexpr (!JOIN) v.u.load(static_cast<const typename S::T*>(a.ready), (int64_t)a.T * a.rp, min(p, tile.hi - 1), 16 * RB, g);
#pragma unroll
    for (int q = 0; q < 2; ++q)
#pragma unroll
      for (int h = 0; h < P; ++h) {
        v.add[q][h] = uint4{0, 0, 0, 0};
        const int c = c0 + 32 * q + 8 * g + h * E::kPer16, n = a.C - c;
        if (a.add && v.t >= 0 && n > 0) v.add[q][h] = load_some<YB>(static_cast<const Y*>(a.add) + v.t * a.lda + c, n);
      }
  };
  const auto work = [&](const Rows& v) {
    floatx4 acc[4];
#pragma unroll
    for (int b = 0; b < 4; ++b) acc[b] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int h = 0; h < S::kFrags; ++h)
#pragma unroll
        for (int b = 0; b < 4; ++b) acc[b] = mma(fw[b][kb], v.u.f[kb][h], acc[b]);
    if (v.t < 0) return;
#pragma unroll
    for (int q = 0; q < 2; ++q)
#pragma unroll
      for (int h = 0; h < P; ++h) {
        const int c = c0 + 32 * q + 8 * g + h * E::kPer16, n = a.C - c;
        if (n <= 0) continue;
        float f[E::kPer16];
        unpack16<YB>(v.add[q][h], f);
#pragma unroll
        for (int e = 0; e < E::kPer16; ++e) f[e] = fmaf(s, acc[2 * q + (h * E::kPer16 + e) / 4][(h * E::kPer16 + e) % 4], f[e]);
        store_some<YB>(static_cast<Y*>(a.y) + v.t * a.ldy + c, n, pack16<YB>(f));
      }
  };
  if constexpr (JOIN) {
    Rows v;
    load(v, tile.lo);
    const int n = tile.hi - tile.lo;
    for (int e = threadIdx.x; e < 16 * a.rp; e += kUpWaves * kWave) {
      const int p = e / (16 * RB), rho = e % (16 * RB);
      float f = 0.f;
      if (p < n) {
        f = add_parts(a.part + (int64_t)(tile.lo + p) * a.rp + rho, (int64_t)a.T * a.rp, a.parts);
        if (a.u && blockIdx.y == 0 && rho < a.r) a.u[(int64_t)(tile.lo + p) * a.r + rho] = f;
      }
      S::put(lds, 16, p, rho, f);
    }
    __syncthreads();
    v.u.load(lds, 16 * S::kStride, i, S::kStride, g);
    work(v);
  } else {
    if (c0 >= a.C) return;
    Rows v[2];
    load(v[0], tile.lo);
    for (int p = tile.lo; p < tile.hi; p += 32) {
      if (p + 16 < tile.hi) load(v[1], p + 16);
      work(v[0]);
      if (p + 16 >= tile.hi) break;
      if (p + 32 < tile.hi) load(v[0], p + 32);
      work(v[1]);
    }
  }
}

// ---------------------------------------------------------------- sums

// u and the joined g of every place for the kernels after it: g by places for `up` (thirds in bf16, or fp32), and both by
// ranks for `outer`: [3][rp][Tp] thirds in bf16, or [rp][Tp] fp32.
struct SumsArgs {
  const float* part;  // g [parts][T][rp]
  const float* u;     // [T][r]
  void* ready;
  void* by_rank[2];   // g, u
  int32_t bf_ready, bf_rank[2];
  int32_t parts, T, Tp, r, rp;
};

constexpr int kSumsPlaces = 32;

__device__ __forceinline__ void put_thirds(void* base, bool bf, int64_t plane, int64_t at, float v) {
  if (!bf) {
    static_cast<float*>(base)[at] = v;
    return;
  }
#pragma unroll
  for (int h = 0; h < 3; ++h) static_cast<uint16_t*>(base)[h * plane + at] = take_third(v);
}

__global__ void __launch_bounds__(256) k_adapter_sums(SumsArgs a) {
  __shared__ float tile[kMaxRank][kSumsPlaces + 1];
  const int p0 = blockIdx.x * kSumsPlaces, which = blockIdx.y, n = min(kSumsPlaces, a.T - p0);
  for (int e = threadIdx.x; e < n * a.rp; e += 256) {
    const int p = e / a.rp, rho = e - p * a.rp;
    float v = 0.f;
    if (which == 0) {
      const int64_t at = (int64_t)(p0 + p) * a.rp + rho;
      v = add_parts(a.part + at, (int64_t)a.T * a.rp, a.parts);
      if (a.ready) put_thirds(a.ready, a.bf_ready, (int64_t)a.T * a.rp, at, v);
    } else if (rho < a.r) {
      v = a.u[(int64_t)(p0 + p) * a.r + rho];
    }
    tile[rho][p] = v;
  }
  __syncthreads();
  for (int e = threadIdx.x; e < kSumsPlaces * a.rp; e += 256) {
    const int p = e % kSumsPlaces, rho = e / kSumsPlaces;
    if (p < n) put_thirds(a.by_rank[which], a.bf_rank[which], (int64_t)a.rp * a.Tp, (int64_t)rho * a.Tp + p0 + p, tile[rho][p]);
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
  int32_t L, T, Tp, C, r, rp, chunk, accumulate;
};

template <bool BF>
struct OuterTile {
  // Columns of a lane's 16 bytes; a wave's tile of 32 places x 16 lanes of them.
  static constexpr int kPer = Elem<BF>::kPer16, kCols = 16 * kPer;
};

// Eight places' values of a rank, places at or past n as 0 (what lies there is another segment's, or nothing).
__device__ __forceinline__ void keep_first(Frag<true>& f, int n) {
#pragma unroll
  for (int d = 0; d < 4; ++d) f.q[d] = n >= 2 * d + 2 ? f.q[d] : n == 2 * d + 1 ? f.q[d] & 0xFFFFu : 0u;
}
__device__ __forceinline__ void keep_first(Frag<false>& f, int n) {
#pragma unroll
  for (int k = 0; k < 8; ++k) f.q[k] = k < n ? f.q[k] : 0.f;
}

// A block has 128 (bf16) or 64 (fp32) columns and a chunk of a segment's places, in steps of 32 by its waves in turn.
// Lane (i, g) loads 16 bytes of places 8 g .. + 7 each, columns P i .. + P - 1 (P = 8 or 4), so a row's piece is 256 bytes
// side by side.  bf16: the eight pieces are turned in registers into the operands of P MFMAs over 32 places, the r factors
// are three thirds in bf16: products are exact.  fp32: element k of every lane is multiplied by an fp32 MFMA of its own.
// MFMA j has column P i + j as row i.  The next step's rows are loaded while one is multiplied.
template <bool BF, bool ACROSS, int RB>
__global__ void __launch_bounds__(kOuterWaves* kWave) k_adapter_outer(OuterArgs a) {
  typedef OuterTile<BF> O;
  typedef typename Elem<BF>::T X;
  typedef typename std::conditional<BF, uint16_t, float>::type U;
  constexpr int P = O::kPer, F = BF ? 3 : 1;
  constexpr int kPlane = 64 * 4 + 4;  // floats of a wave's MFMA in LDS
  __shared__ __align__(16) float sums[kOuterWaves * P * kPlane];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int i = lane & 15, g = lane >> 4;
  const int r0 = blockIdx.z * 16 * RB;
  const int c = blockIdx.x * O::kCols + P * i, n_c = a.C - c;
  Tile tile;
  if (!find_tile<true>(a.off, a.L, a.T, a.chunk, blockIdx.y, tile)) return;
  floatx4 acc[P][RB];
#pragma unroll
  for (int j = 0; j < P; ++j)
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) acc[j][rb] = floatx4{0.f, 0.f, 0.f, 0.f};
  struct Rows {
    uint4 v[8];
    Frag<BF> u[RB][F];
  };
  const auto load = [&](Rows& s, int p) {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int q = p + 8 * g + k;
      s.v[k] = uint4{0, 0, 0, 0};
      if (q < tile.hi && n_c > 0) {
        const int t = row_at(a.perm, q);
        if ((uint32_t)t < (uint32_t)a.T) s.v[k] = load_some<BF>(static_cast<const X*>(a.x) + t * a.ldx + c, n_c);
      }
    }
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
      for (int h = 0; h < F; ++h)
        load8<BF, BF, true>(s.u[rb][h], a.by_rank, ((int64_t)h * a.rp + r0 + 16 * rb + i) * a.Tp + p + 8 * g, 8);
  };
  const auto work = [&](Rows& s, int p) {
    if (p + 32 > tile.hi) {
#pragma unroll
      for (int rb = 0; rb < RB; ++rb)
#pragma unroll
        for (int h = 0; h < F; ++h) keep_first(s.u[rb][h], tile.hi - p - 8 * g);
    }
    if constexpr (BF) {
      // Dword d of place k holds its columns 2 d and 2 d + 1; operand j wants column j of all places.
#pragma unroll
      for (int d = 0; d < P / 2; ++d) {
        uint32_t q[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) q[k] = d == 0 ? s.v[k].x : d == 1 ? s.v[k].y : d == 2 ? s.v[k].z : s.v[k].w;
        Frag<true> lo, hi;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          lo.q[k] = __builtin_amdgcn_perm(q[2 * k + 1], q[2 * k], 0x05040100u);
          hi.q[k] = __builtin_amdgcn_perm(q[2 * k + 1], q[2 * k], 0x07060302u);
        }
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
#pragma unroll
          for (int h = 0; h < F; ++h) {
            acc[2 * d][rb] = mma(lo, s.u[rb][h], acc[2 * d][rb]);
            acc[2 * d + 1][rb] = mma(hi, s.u[rb][h], acc[2 * d + 1][rb]);
          }
      }
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        float q[4];
        unpack16<false>(s.v[k], q);
#pragma unroll
        for (int j = 0; j < P; ++j)
#pragma unroll
          for (int rb = 0; rb < RB; ++rb)
            acc[j][rb] = __builtin_amdgcn_mfma_f32_16x16x4f32(q[j], s.u[rb][0].q[k], acc[j][rb], 0, 0, 0);
      }
    }
  };
  constexpr int kStep = 32 * kOuterWaves;
  Rows s[2];
  int p = tile.lo + 32 * wave;
  if (p < tile.hi) load(s[0], p);
  for (; p < tile.hi; p += 2 * kStep) {
    if (p + kStep < tile.hi) load(s[1], p + kStep);
    work(s[0], p);
    if (p + kStep >= tile.hi) break;
    if (p + 2 * kStep < tile.hi) load(s[0], p + 2 * kStep);
    work(s[1], p + kStep);
  }
  // The waves' sums in order, through LDS, where threads side by side take elements side by side of the output.  Lane (i, g)
  // holds rank i of each block and, of MFMA j and register e, column P (4 g + e) + j.
  const int64_t size = (int64_t)a.r * a.C;
  float* out = tile.whole ? a.out + tile.l * size : a.slots + tile.slot * size;
  const float scale = a.scale ? a.scale[tile.l] : 1.f;
  const int b0 = blockIdx.x * O::kCols;
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
      const int j = col % P, x = col / P;
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

constexpr size_t up256(size_t v) { return (v + 255) / 256 * 256; }

int32_t padded_rank(int32_t r) { return r <= 16 ? 16 : r <= 32 ? 32 : r <= 64 ? 64 : 128; }

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

DownPlan down_plan(int32_t T, int32_t C) {
  DownPlan d;
  d.places = T <= 64 ? 1 : T <= 256 ? 4 : T < kManyRows ? 16 : 32;
  const int32_t blocks = (T + d.places - 1) / d.places, units = (C + 63) / 64;
  d.parts = T >= kManyRows ? 1 : std::max(1, std::min(512 / std::max(blocks, 1), (units + kDownWaves - 1) / kDownWaves));
  d.units = (units + d.parts - 1) / d.parts;
  d.parts = (units + d.units - 1) / d.units;
  return d;
}

int32_t up_places(int32_t T) { return T <= 64 ? 1 : T <= 256 ? 4 : T < kManyRows ? 16 : 128; }

// Places of a chunk of `outer`: blocks for every CU twice over the matrix, of at least 128 places.
int32_t outer_chunk(int32_t T, int32_t C, int32_t dtype) {
  const int32_t cols = dtype == DAMOE_BF16 ? OuterTile<true>::kCols : OuterTile<false>::kCols;
  const int32_t tiles = (C + cols - 1) / cols;
  const int32_t chunks = std::max(1, std::min((T + 127) / 128, 512 / tiles));
  return (T + chunks - 1) / chunks;
}

// Slots of `outer`: a segment of n > 1 chunks has more than (n - 1) chunk places, so n is at most twice the chunks they fill.
int64_t slots_of(int32_t T, int32_t chunk) { return chunk >= T ? 0 : 2 * (int64_t)((T + chunk - 1) / chunk); }

hipError_t down(DownArgs a, const DownPlan& d, int32_t xdtype, int32_t wdtype, bool across, hipStream_t stream) {
  a.places = d.places;
  a.units = d.units;
  return by_rank<4>(a.rp, [&](auto rb) {
    return by_types(xdtype, wdtype, [&](auto xb, auto wb) {
      constexpr int RB = decltype(rb)::value;
      constexpr bool XB = decltype(xb)::value, WB = decltype(wb)::value;
      const auto go = [&](auto ac, auto m) {
        constexpr int M = decltype(m)::value;
        const dim3 grid((unsigned)most_tiles(a.T, a.L, a.places), d.parts, a.rp / (16 * RB));
        hipLaunchKernelGGL((k_adapter_down<XB, WB, decltype(ac)::value, RB, M>), grid, dim3(kDownWaves * kWave),
                           kDownWaves * M * RB * 64 * sizeof(floatx4), stream, a);
        return hipGetLastError();
      };
      // fp32 operands of 64 ranks leave no registers for more than 16 places.
      const std::integral_constant<int, 1> one;
      const std::integral_constant<int, RB == 4 && !(XB && WB) ? 1 : 2> most;
      a.places = std::min(a.places, 16 * most.value);
      if (across) return a.places <= 16 ? go(std::true_type{}, one) : go(std::true_type{}, most);
      return a.places <= 16 ? go(std::false_type{}, one) : go(std::false_type{}, most);
    });
  });
}

// join: from a.part, else from a.ready.
hipError_t up(UpArgs a, int32_t ydtype, int32_t wdtype, bool across, bool join, hipStream_t stream) {
  a.places = up_places(a.T);
  const dim3 grid((unsigned)most_tiles(a.T, a.L, a.places), (a.C + kUpWaves * kUpCols - 1) / (kUpWaves * kUpCols));
  return by_rank<8>(a.rp, [&](auto rb) {
    return by_types(ydtype, wdtype, [&](auto yb, auto wb) {
      constexpr int RB = decltype(rb)::value;
      constexpr bool YB = decltype(yb)::value, WB = decltype(wb)::value;
      using std::false_type;
      using std::true_type;
      const auto go = [&](auto ac, auto jn) {
        hipLaunchKernelGGL((k_adapter_up<YB, WB, decltype(ac)::value, RB, decltype(jn)::value>), grid, dim3(kUpWaves * kWave), 0, stream,
                           a);
        return hipGetLastError();
      };
      return across ? go(true_type{}, false_type{}) : join ? go(false_type{}, true_type{}) : go(false_type{}, false_type{});
    });
  });
}

hipError_t outer(const OuterArgs& a, int32_t dtype, bool across, hipStream_t stream) {
  const auto go = [&](auto bf, auto ac, auto rb) {
    constexpr bool BF = decltype(bf)::value;
    constexpr int RB = decltype(rb)::value;
    typedef OuterTile<BF> O;
    const dim3 grid((a.C + O::kCols - 1) / O::kCols, (unsigned)most_tiles(a.T, a.L, a.chunk), (a.r + 16 * RB - 1) / (16 * RB));
    hipLaunchKernelGGL((k_adapter_outer<BF, decltype(ac)::value, RB>), grid, dim3(kOuterWaves * kWave), 0, stream, a);
    return hipGetLastError();
  };
  const auto ranked = [&](auto bf, auto ac) {
    return a.r <= 16 ? go(bf, ac, std::integral_constant<int, 1>{}) : go(bf, ac, std::integral_constant<int, 2>{});
  };
  using std::false_type;
  using std::true_type;
  if (dtype == DAMOE_BF16) return across ? ranked(true_type{}, true_type{}) : ranked(true_type{}, false_type{});
  return across ? ranked(false_type{}, true_type{}) : ranked(false_type{}, false_type{});
}

bool sizes_ok(int32_t T, int32_t L, int32_t r, int32_t K, int32_t N) {
  return T >= 0 && T <= DAMOE_MAX_T && L >= 1 && L <= DAMOE_MAX_E && r >= 1 && K >= 1 && N >= 1;
}

damoe_status check(int32_t T, int32_t L, int32_t r, int32_t K, int32_t N, int32_t d0, int32_t d1, int32_t d2) {
  if (!sizes_ok(T, L, r, K, N)) return DAMOE_ERR_INVALID_ARG;
  for (const int32_t d : {d0, d1, d2})
    if (d != DAMOE_BF16 && d != DAMOE_F32) return DAMOE_ERR_UNSUPPORTED;
  return r > kMaxRank || K > DAMOE_MAX_COLS || N > DAMOE_MAX_COLS ? DAMOE_ERR_UNSUPPORTED : DAMOE_OK;
}

bool aligned(const void* p, int32_t dtype) { return reinterpret_cast<uintptr_t>(p) % (dtype == DAMOE_BF16 ? 2 : 4) == 0; }

bool matrix_ok(const void* p, int64_t ld, int32_t cols, int32_t dtype) { return p && ld >= cols && aligned(p, dtype); }

// Rows of what `sums` lays out by ranks: loads of `outer` go up to 31 places past the last.
int32_t row_by_rank(int32_t T) { return (T + 7) / 8 * 8 + 64; }

// Bytes of each piece of the workspaces: fp32 parts; what `up` takes; by ranks; slots.
size_t part_bytes(const DownPlan& d, int32_t T, int32_t rp) { return up256((size_t)d.parts * T * rp * 4); }
size_t ready_bytes(int32_t T, int32_t rp) { return up256((size_t)T * rp * 6); }
size_t rank_bytes(int32_t T, int32_t rp) { return up256((size_t)row_by_rank(T) * rp * 6); }
size_t slot_bytes(int64_t slots, int32_t r, int32_t C) { return up256((size_t)slots * r * C * 4); }

// The most that part_bytes is for up to T_max rows: blocks times parts is at most 512, or the blocks themselves.
size_t most_parts(int32_t T_max, int32_t C, int32_t rp) {
  size_t most = 0;
  for (const int32_t t : {64, 256, kManyRows - 1, T_max}) {
    const int32_t T = std::min(t, T_max), places = down_plan(T, C).places;
    const int32_t parts = ((C + 63) / 64 + kDownWaves - 1) / kDownWaves;
    most = std::max(most, std::min((size_t)T * parts, std::max<size_t>((size_t)T, (size_t)512 * places)) * rp * 4);
  }
  return up256(most);
}

// The most that slots_of is: there are never more chunks than 128-place ones, nor than the blocks allow.
int64_t most_slots(int32_t T_max, int32_t C) {
  const int64_t tiles = (C + OuterTile<true>::kCols - 1) / OuterTile<true>::kCols;
  return T_max <= 128 ? 0 : 2 * std::min<int64_t>((T_max + 127) / 128, std::max<int64_t>(1, 512 / tiles));
}

}  // namespace
}  // namespace damoe

using namespace damoe;

extern "C" {

size_t damoe_adapters_workspace_size(int32_t T_max, int32_t L, int32_t r, int32_t K, int32_t N) {
  if (check(T_max, L, r, K, N, DAMOE_F32, DAMOE_F32, DAMOE_F32)) return 0;
  const int32_t rp = padded_rank(r);
  return 256 + std::max(most_parts(T_max, K, rp), ready_bytes(T_max, rp));
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
  const DownPlan d = down_plan(T, K);
  const bool join = T < kManyRows;
  if (ws_bytes < (join ? part_bytes(d, T, rp) : ready_bytes(T, rp))) return DAMOE_ERR_WORKSPACE;
  float* part = join ? static_cast<float*>(ws) : nullptr;
  const DownArgs da{x, ldx, a, perm, offsets, nullptr, part, ws, u, L, T, K, r, rp, 0, 0};
  // `up` takes thirds where the weights are bf16, `down` leaves them there too.
  if (down(da, d, xdtype, wdtype, false, stream) != hipSuccess) return DAMOE_ERR_HIP;
  const UpArgs ua{part, ws, d.parts, u, b, scale, perm, offsets, add, ld_add, y, ldy, L, T, N, r, rp, 0};
  return up(ua, ydtype, wdtype, false, join, stream) == hipSuccess ? DAMOE_OK : DAMOE_ERR_HIP;
}

size_t damoe_adapters_grad_workspace_size(int32_t T_max, int32_t L, int32_t r, int32_t K, int32_t N) {
  if (check(T_max, L, r, K, N, DAMOE_F32, DAMOE_F32, DAMOE_F32)) return 0;
  const int32_t rp = padded_rank(r);
  return 256 + most_parts(T_max, N, rp) + ready_bytes(T_max, rp) + 2 * rank_bytes(T_max, rp) + slot_bytes(most_slots(T_max, K), r, K) +
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
    void* g_rank = piece(rank_bytes(T, rp));
    void* u_rank = piece(rank_bytes(T, rp));
    slots_a = reinterpret_cast<float*>(piece(slot_bytes(slots_of(T, ck), r, K)));
    slots_b = reinterpret_cast<float*>(piece(slot_bytes(slots_of(T, cn), r, N)));
    if (ws_bytes < end) return DAMOE_ERR_WORKSPACE;
    const int32_t Tp = row_by_rank(T);
    const DownArgs ga{dy, ldy, b, perm, offsets, scale, part, nullptr, nullptr, L, T, N, r, rp, 0, 0};
    if (down(ga, d, ydtype, wdtype, true, stream) != hipSuccess) return DAMOE_ERR_HIP;
    const SumsArgs sa{part, u, dx ? ready : nullptr, {g_rank, u_rank}, wdtype == DAMOE_BF16, {xdtype == DAMOE_BF16, ydtype == DAMOE_BF16},
                      d.parts, T, Tp, r, rp};
    hipLaunchKernelGGL(k_adapter_sums, dim3((T + kSumsPlaces - 1) / kSumsPlaces, 2), dim3(256), 0, stream, sa);
    if (hipGetLastError() != hipSuccess) return DAMOE_ERR_HIP;
    // dB first: it reads what `down` has just read.
    const OuterArgs ob{dy, ldy, u_rank, scale, perm, offsets, db, slots_b, L, T, Tp, N, r, rp, cn, accumulate};
    if (outer(ob, ydtype, true, stream) != hipSuccess) return DAMOE_ERR_HIP;
    const OuterArgs oa{x, ldx, g_rank, nullptr, perm, offsets, da, slots_a, L, T, Tp, K, r, rp, ck, accumulate};
    if (outer(oa, xdtype, false, stream) != hipSuccess) return DAMOE_ERR_HIP;
    if (dx) {
      const UpArgs xa{nullptr, ready, 1, nullptr, a, nullptr, perm, offsets, add, ld_add, dx, ld_dx, L, T, K, r, rp, 0};
      if (up(xa, xdtype, wdtype, true, false, stream) != hipSuccess) return DAMOE_ERR_HIP;
    }
  }
  JoinArgs j{offsets, {da, db}, {slots_a, slots_b}, {(int64_t)r * K, (int64_t)r * N}, {ck, cn}, L, T, accumulate, 256};
  const int64_t all = std::max(j.size[0], j.size[1]);
  while ((all + j.per - 1) / j.per * L > 2048 && j.per < all) j.per *= 2;
  hipLaunchKernelGGL(k_adapter_join, dim3((unsigned)((all + j.per - 1) / j.per), L, 2), dim3(256), 0, stream, j);
  return hipGetLastError() == hipSuccess ? DAMOE_OK : DAMOE_ERR_HIP;
}

}  // extern "C"
