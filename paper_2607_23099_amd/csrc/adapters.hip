// Low-rank adapters of many segments of rows at once: damoe_adapters and its gradient.
//
// Segment l is the places [off[l], off[l + 1]) and place p holds row t = perm[p] (p itself without perm).  With A_l [r][K],
// B_l [N][r] and s_l:
//   u_p = A_l x_t            y_t = add_t + s_l B_l u_p
//   g_p = s_l B_l^T dy_t     dx_t = add_t + A_l^T g_p     dA_l = sum_p g_p x_t^T     dB_l = s_l sum_p dy_t u_p^T
// r is small, so all of it is bound by the rows (x, dy, y, dx), or by the weights where few rows share an adapter.  Three
// kernels make it up, each a pass over one of these matrices:
//   down    rows of r sums over many columns (u, g): columns split over a block's waves and over blocks
//   up      many columns of r products each (y, dx), which joins down's parts
//   outer   r x columns sums over a segment's places (dA, dB), split over chunks of places whose parts `join` adds
// Blocks take places at fixed distances, whatever the segments are, and go over the segments that they hold; so no list
// of tiles has to be made, and a segment's sums do not depend on timing.
#include "vec.h"

namespace damoe {
namespace {

constexpr int kMaxRank = DAMOE_MAX_RANK;
constexpr int kDownWaves = 8, kUpWaves = 4, kOuterWaves = 4;

// ---------------------------------------------------------------- segments

// End of each segment in turn, by a wave: 64 ends in its lanes.
struct Segments {
  const int32_t* off;
  int32_t L, T, base, ends;

  __device__ __forceinline__ void load(int l) {
    base = l;
    ends = off[1 + min(l + (int)(threadIdx.x & 63), L - 1)];
  }
  // Number of segments that end at or before place p: the one that holds it, L past the last.
  __device__ __forceinline__ int first(const int32_t* offsets, int32_t n, int32_t places, int32_t p) {
    off = offsets, L = n, T = places;
    int c = 0;
    for (int l = 0; l < L; l += 64) {
      load(l);
      c += __popcll(__ballot(l + (int)(threadIdx.x & 63) < L && ends <= p));
    }
    c = __builtin_amdgcn_readfirstlane(c);
    if (L > 64 && c < L) load(c);
    return c;
  }
  __device__ __forceinline__ int end(int l) {
    if (l - base >= 64) load(l);
    return min(__builtin_amdgcn_readlane(ends, l - base), T);
  }
};

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
  float* part;     // [parts][T][rp]
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

// RB blocks of 16 ranks (more than 64 take a block of the grid each), M of 16 places.  A unit of 64 columns is two MFMA steps: lane (i, g) takes columns 16 g .. + 7 of
// it in the first and 16 g + 8 .. + 15 in the second, so that its loads of a row are 32 bytes (bf16) side by side.  The
// operands of a unit are loaded while the one before is multiplied.
template <bool XB, bool WB, bool ACROSS, int RB, int M>
__global__ void __launch_bounds__(kDownWaves* kWave) k_adapter_down(DownArgs a) {
  constexpr bool BF = XB && WB;
  extern __shared__ floatx4 red[];  // [kDownWaves][M RB][64]
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int i = lane & 15, g = lane >> 4;
  const int p0 = blockIdx.x * a.places, p1 = min(p0 + a.places, a.T);
  const int u0 = blockIdx.y * a.units, u1 = min(u0 + a.units, (a.C + 63) / 64);
  const int r0 = blockIdx.z * 16 * RB;
  Segments seg;
  int l = seg.first(a.off, a.L, a.T, p0);
  if (l >= a.L) return;
  int64_t row[M];
#pragma unroll
  for (int m = 0; m < M; ++m) {
    const int p = p0 + 16 * m + i, t = row_at(a.perm, p < p1 ? p : p0);
    row[m] = (int64_t)((uint32_t)t < (uint32_t)a.T ? t : 0) * a.ldx;
  }
  for (int lo = p0; l < a.L && lo < p1; ++l) {
    const int hi = min(seg.end(l), p1);
    if (hi <= lo) continue;
    const int64_t slab = (int64_t)l * a.r * a.C;
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
    const float s = a.scale ? a.scale[l] : 1.f;
    for (int e = threadIdx.x; e < M * RB * 64; e += kDownWaves * kWave) {
      floatx4 v = red[e];
#pragma unroll
      for (int w = 1; w < kDownWaves; ++w) v += red[w * M * RB * 64 + e];
      const int p = p0 + 16 * (e / (64 * RB)) + (e & 15), rho = r0 + 16 * (e / 64 % RB) + 4 * (e / 16 % 4);
      if (p < lo || p >= hi) continue;
      float* out = a.part + ((int64_t)blockIdx.y * a.T + p) * a.rp + rho;
      float4 o;
      o.x = rho < a.r ? s * v[0] : 0.f;
      o.y = rho + 1 < a.r ? s * v[1] : 0.f;
      o.z = rho + 2 < a.r ? s * v[2] : 0.f;
      o.w = rho + 3 < a.r ? s * v[3] : 0.f;
      *reinterpret_cast<float4*>(out) = o;
    }
    __syncthreads();
    lo = hi;
  }
}

// ---------------------------------------------------------------- up

struct UpArgs {
  const float* part;  // [parts][T][rp]
  int32_t parts;
  float* u;           // NULL, or the joined sums [T][r]
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

// The joined sums of a block's places in LDS: three bf16 thirds with bf16 weights, whose products are exact; else fp32.
template <bool WB, int RB>
struct Sums {
  static constexpr int kStride = 16 * RB + (WB ? 8 : 4);
  typedef typename std::conditional<WB, uint16_t, float>::type T;
  static constexpr int kPlanes = WB ? 3 : 1;

  static __device__ __forceinline__ void put(T* lds, int places, int p, int rho, float v) {
    if constexpr (WB) {
#pragma unroll
      for (int h = 0; h < 3; ++h) lds[(h * places + p) * kStride + rho] = take_third(v);
    } else {
      lds[p * kStride + rho] = v;
    }
  }
  // Eight ranks from rho on (a multiple of 8) of place p, third h.
  static __device__ __forceinline__ void get(Frag<WB>& f, const T* lds, int places, int h, int p, int rho) {
    const uint4* s = reinterpret_cast<const uint4*>(lds + (h * places + p) * kStride + rho);
    const uint4 v = s[0];
    if constexpr (WB) {
      f.q[0] = v.x, f.q[1] = v.y, f.q[2] = v.z, f.q[3] = v.w;
    } else {
      const uint4 w = s[1];
      f.q[0] = __uint_as_float(v.x), f.q[1] = __uint_as_float(v.y), f.q[2] = __uint_as_float(v.z), f.q[3] = __uint_as_float(v.w);
      f.q[4] = __uint_as_float(w.x), f.q[5] = __uint_as_float(w.y), f.q[6] = __uint_as_float(w.z), f.q[7] = __uint_as_float(w.w);
    }
  }
};

// A wave has 64 columns, as four MFMA blocks of 16: row i of block 2 q + m is column 32 q + 8 (i / 4) + 4 m + i % 4, so that
// a lane's results of a pair are eight columns side by side of its place.
template <bool YB, bool WB, bool ACROSS, int RB>
__global__ void __launch_bounds__(kUpWaves* kWave) k_adapter_up(UpArgs a) {
  typedef Sums<WB, RB> S;
  typedef typename Elem<YB>::T Y;
  constexpr int KB = (RB + 1) / 2;  // blocks of 32 ranks
  extern __shared__ char lds_raw[];
  typename S::T* lds = reinterpret_cast<typename S::T*>(lds_raw);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int i = lane & 15, g = lane >> 4;
  const int p0 = blockIdx.x * a.places, p1 = min(p0 + a.places, a.T);
  const int padded = (a.places + 15) & ~15;
  Segments seg;
  int l = seg.first(a.off, a.L, a.T, p0);
  if (l >= a.L) return;
  const int covered = min(p1, max(p0, min(a.off[a.L], a.T)));
  for (int e = threadIdx.x; e < padded * a.rp; e += kUpWaves * kWave) {
    const int p = e / a.rp, rho = e - p * a.rp;
    float v = 0.f;
    if (p0 + p < covered) {
      const float* s = a.part + (int64_t)(p0 + p) * a.rp + rho;
      for (int k = 0; k < a.parts; ++k) v += s[(int64_t)k * a.T * a.rp];
      if (a.u && blockIdx.y == 0 && rho < a.r) a.u[(int64_t)(p0 + p) * a.r + rho] = v;
    }
    S::put(lds, padded, p, rho, v);
  }
  __syncthreads();
  const int c0 = (blockIdx.y * kUpWaves + wave) * kUpCols;
  if (c0 >= a.C) return;
  for (int lo = p0; l < a.L && lo < p1; ++l) {
    const int hi = min(seg.end(l), p1);
    if (hi <= lo) continue;
    const int64_t slab = (int64_t)l * a.r * a.C;
    const float s = a.scale ? a.scale[l] : 1.f;
    Frag<WB> fw[4][KB];
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      const int c = min(c0 + 32 * (b / 2) + 8 * (i / 4) + 4 * (b & 1) + i % 4, a.C - 1);
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
        // One block of 16 ranks: bf16 takes two of the thirds in one instruction, over the same weights.
        const int rho = 32 * kb + 8 * (RB == 1 && WB ? g & 1 : g);
        if constexpr (ACROSS) load8_apart<WB, WB, false>(fw[b][kb], a.w, slab + (int64_t)rho * a.C + c, a.C, a.r - rho);
        else load8<WB, WB, false>(fw[b][kb], a.w, slab + (int64_t)c * a.r + rho, a.r - rho);
      }
    }
    for (int m = (lo - p0) / 16; p0 + 16 * m < hi; ++m) {
      const int p = p0 + 16 * m + i;
      int t = p >= lo && p < hi ? row_at(a.perm, p) : -1;
      if ((uint32_t)t >= (uint32_t)a.T) t = -1;
      constexpr int P = 8 / Elem<YB>::kPer16;  // 16-byte pieces of eight columns
      uint4 add[2][P];
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const int c = c0 + 32 * q + 8 * g;
#pragma unroll
        for (int h = 0; h < P; ++h) {
          add[q][h] = uint4{0, 0, 0, 0};
          const int n = a.C - c - h * Elem<YB>::kPer16;
          if (a.add && t >= 0 && n > 0)
            add[q][h] = load_some<YB>(static_cast<const Y*>(a.add) + t * a.lda + c + h * Elem<YB>::kPer16, n);
        }
      }
      floatx4 acc[4];
#pragma unroll
      for (int b = 0; b < 4; ++b) acc[b] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
        if constexpr (WB && RB == 1) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {  // thirds 0 and 1, then 2 and none
            Frag<true> fu;
            if (2 * h + g / 2 < 3) S::get(fu, lds, padded, 2 * h + g / 2, 16 * m + i, 8 * (g & 1));
#pragma unroll
            for (int b = 0; b < 4; ++b) acc[b] = mma(fw[b][0], fu, acc[b]);
          }
        } else if constexpr (WB) {
#pragma unroll
          for (int h = 0; h < 3; ++h) {
            Frag<true> fu;
            S::get(fu, lds, padded, h, 16 * m + i, 32 * kb + 8 * g);
#pragma unroll
            for (int b = 0; b < 4; ++b) acc[b] = mma(fw[b][kb], fu, acc[b]);
          }
        } else {
          Frag<false> fu;
          if (32 * kb + 8 * g < a.rp) S::get(fu, lds, padded, 0, 16 * m + i, 32 * kb + 8 * g);
#pragma unroll
          for (int b = 0; b < 4; ++b) acc[b] = mma(fw[b][kb], fu, acc[b]);
        }
      }
      if (t < 0) continue;
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const int c = c0 + 32 * q + 8 * g;
#pragma unroll
        for (int h = 0; h < P; ++h) {
          constexpr int E = Elem<YB>::kPer16;
          const int n = a.C - c - h * E;
          if (n <= 0) continue;
          float f[E];
          unpack16<YB>(add[q][h], f);
#pragma unroll
          for (int e = 0; e < E; ++e) f[e] = fmaf(s, acc[2 * q + (h * E + e) / 4][(h * E + e) % 4], f[e]);
          store_some<YB>(static_cast<Y*>(a.y) + t * a.ldy + c + h * E, n, pack16<YB>(f));
        }
      }
    }
    lo = hi;
  }
}

// ---------------------------------------------------------------- outer

struct OuterArgs {
  const void* x;       // rows (x, dy)
  int64_t ldx;
  const float* u;      // the other factor: [parts][T][ldu], r of its columns used
  int32_t parts, ldu;
  const float* scale;  // of a segment's sums, or NULL
  const int32_t* perm;
  const int32_t* off;
  float* out;          // dA [L][r][C], or dB [L][C][r]
  float* slots;        // parts of segments that lie in several chunks, [2 chunks][r C], laid out as the output
  int32_t L, T, C, r, chunk, accumulate;
};

template <bool BF>
struct OuterTile {
  // Columns of a lane's 16 bytes; a wave's tile of 32 places x 16 lanes of them.
  static constexpr int kPer = Elem<BF>::kPer16, kCols = 16 * kPer;
};

// A block has 128 (bf16) or 64 (fp32) columns and a chunk of places, a segment's places in steps of 32 by its waves in
// turn.  Lane (i, g) loads 16 bytes at a time, columns P i .. + P - 1 (P = 8 or 4) of one place, so a row's piece is 256
// bytes side by side.  bf16: of places 8 g .. + 7, and the eight pieces are turned in registers into the operands of P
// MFMAs over 32 places, the r factors as three thirds in bf16: products are exact.  fp32: of places 4 s + g, which are the
// operands of fp32 MFMAs as they are.  MFMA j has column P i + j as row i.
template <bool BF, bool ACROSS, int RB>
__global__ void __launch_bounds__(kOuterWaves* kWave) k_adapter_outer(OuterArgs a) {
  typedef OuterTile<BF> O;
  typedef typename Elem<BF>::T X;
  constexpr int P = O::kPer;
  extern __shared__ floatx4 red[];  // [kOuterWaves / 2][P RB][64]
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int i = lane & 15, g = lane >> 4;
  const int r0 = blockIdx.z * 16 * RB;
  const int q0 = blockIdx.y * a.chunk, q1 = min(q0 + a.chunk, a.T);
  const int c = blockIdx.x * O::kCols + P * i, n_c = a.C - c;
  Segments seg;
  int l = seg.first(a.off, a.L, a.T, q0);
  if (l >= a.L) return;
  bool before = l > 0 ? a.off[l] < q0 : q0 > 0;
  for (int lo = q0; l < a.L && lo < q1; ++l) {
    const int end = seg.end(l), hi = min(end, q1);
    if (hi <= lo) continue;
    floatx4 acc[P][RB];
#pragma unroll
    for (int j = 0; j < P; ++j)
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) acc[j][rb] = floatx4{0.f, 0.f, 0.f, 0.f};
    for (int p = lo + 32 * wave; p < hi; p += 32 * kOuterWaves) {
      uint4 v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int q = p + (BF ? 8 * g + k : 4 * k + g);
        v[k] = uint4{0, 0, 0, 0};
        if (q < hi && n_c > 0) {
          const int t = row_at(a.perm, q);
          if ((uint32_t)t < (uint32_t)a.T) v[k] = load_some<BF>(static_cast<const X*>(a.x) + t * a.ldx + c, n_c);
        }
      }
      float f[RB][8];
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        const int rho = r0 + 16 * rb + i;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const int q = p + (BF ? 8 * g + k : 4 * k + g);
          f[rb][k] = 0.f;
          if (q < hi && rho < a.r)
            for (int z = 0; z < a.parts; ++z) f[rb][k] += a.u[((int64_t)z * a.T + q) * a.ldu + rho];
        }
      }
      if constexpr (BF) {
        Frag<true> fx[P];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const uint32_t q[4] = {v[k].x, v[k].y, v[k].z, v[k].w};
#pragma unroll
          for (int j = 0; j < P; ++j) fx[j].set(k, (uint16_t)(q[j / 2] >> (16 * (j & 1))));
        }
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
#pragma unroll
          for (int h = 0; h < 3; ++h) {
            Frag<true> fu;
#pragma unroll
            for (int k = 0; k < 8; ++k) fu.set(k, take_third(f[rb][k]));
#pragma unroll
            for (int j = 0; j < P; ++j) acc[j][rb] = mma(fx[j], fu, acc[j][rb]);
          }
      } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const float q[4] = {__uint_as_float(v[k].x), __uint_as_float(v[k].y), __uint_as_float(v[k].z), __uint_as_float(v[k].w)};
#pragma unroll
          for (int j = 0; j < P; ++j)
#pragma unroll
            for (int rb = 0; rb < RB; ++rb)
              acc[j][rb] = __builtin_amdgcn_mfma_f32_16x16x4f32(q[j], f[rb][k], acc[j][rb], 0, 0, 0);
        }
      }
    }
    // The waves' sums: the upper half of them added to the lower, in the same order always.
#pragma unroll
    for (int half = kOuterWaves / 2; half; half >>= 1) {
      if (wave >= half && wave < 2 * half) {
#pragma unroll
        for (int e = 0; e < P * RB; ++e) red[((wave - half) * P * RB + e) * 64 + lane] = acc[e / RB][e % RB];
      }
      __syncthreads();
      if (wave < half) {
#pragma unroll
        for (int e = 0; e < P * RB; ++e) acc[e / RB][e % RB] += red[(wave * P * RB + e) * 64 + lane];
      }
      __syncthreads();
    }
    if (wave == 0) {
      const bool whole = !before && end <= q1;
      const int64_t size = (int64_t)a.r * a.C;
      float* out = whole ? a.out + l * size : a.slots + (2 * (int64_t)blockIdx.y + (before ? 0 : 1)) * size;
      const float s = a.scale ? a.scale[l] : 1.f;
      // Lane (i, g) has rank i of each block and, of MFMA j and register e, column P (4 g + e) + j.
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        const int rho = r0 + 16 * rb + i;
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int j = 0; j < P; ++j) {
            const int col = blockIdx.x * O::kCols + P * (4 * g + e) + j;
            if (rho >= a.r || col >= a.C) continue;
            float* o = out + (ACROSS ? (int64_t)col * a.r + rho : (int64_t)rho * a.C + col);
            const float v = s * acc[j][rb][e];
            *o = whole && a.accumulate ? *o + v : v;
          }
      }
    }
    before = false;
    lo = hi;
  }
}

// The parts of segments that lie in several chunks, in order, and zeros for empty segments.
struct JoinArgs {
  const int32_t* off;
  float* out[2];
  const float* slots[2];
  int64_t size[2];
  int32_t chunk[2], L, T, accumulate, per;  // per: elements of a block
};

__global__ void __launch_bounds__(256) k_adapter_join(JoinArgs a) {
  const int l = blockIdx.y;
  const int32_t s = l ? a.off[l] : 0, e = min(a.off[l + 1], a.T);
  const bool empty = e <= s;
  if (empty && a.accumulate) return;
  const int64_t all = a.size[0] + a.size[1];
  const int64_t end = min(all, (int64_t)(blockIdx.x + 1) * a.per);
  for (int64_t at = (int64_t)blockIdx.x * a.per + threadIdx.x; at < end; at += 256) {
    const int m = at >= a.size[0];
    const int64_t i = at - (m ? a.size[0] : 0), size = a.size[m];
    float* o = a.out[m] + l * size + i;
    if (empty) {
      *o = 0.f;
      continue;
    }
    const int c0 = s / a.chunk[m], c1 = (e - 1) / a.chunk[m];
    if (c0 == c1) continue;
    float v = a.accumulate ? *o : 0.f;
    v += a.slots[m][(2 * (int64_t)c0 + 1) * size + i];
    for (int k = c0 + 1; k <= c1; ++k) v += a.slots[m][2 * (int64_t)k * size + i];
    *o = v;
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

// How `down` is split: places of a block, blocks over the columns and each one's units.
struct DownPlan {
  int32_t places, parts, units;
};

DownPlan down_plan(int32_t T, int32_t C) {
  DownPlan d;
  d.places = T <= 64 ? 1 : T <= 256 ? 4 : T < 2048 ? 16 : 32;
  const int32_t blocks = (T + d.places - 1) / d.places, units = (C + 63) / 64;
  d.parts = std::max(1, std::min(512 / std::max(blocks, 1), (units + kDownWaves - 1) / kDownWaves));
  d.units = (units + d.parts - 1) / d.parts;
  d.parts = (units + d.units - 1) / d.units;
  return d;
}

int32_t up_places(int32_t T) { return T <= 64 ? 1 : T <= 256 ? 4 : T < 2048 ? 16 : 64; }

// Places of a chunk of `outer`: enough chunks that the blocks fill the card twice, of at least 128 places.
int32_t outer_chunk(int32_t T, int32_t C, int32_t dtype) {
  const int32_t cols = dtype == DAMOE_BF16 ? OuterTile<true>::kCols : OuterTile<false>::kCols;
  const int32_t tiles = (C + cols - 1) / cols;
  const int32_t chunks = std::max(1, std::min((T + 127) / 128, 1024 / std::max(tiles, 1)));
  return (T + chunks - 1) / chunks;
}

hipError_t down(DownArgs a, const DownPlan& d, int32_t xdtype, int32_t wdtype, bool across, hipStream_t stream) {
  a.places = d.places;
  a.units = d.units;
  return by_rank<4>(a.rp, [&](auto rb) {
    return by_types(xdtype, wdtype, [&](auto xb, auto wb) {
      constexpr int RB = decltype(rb)::value;
      constexpr bool XB = decltype(xb)::value, WB = decltype(wb)::value;
      const auto go = [&](auto ac, auto m) {
        constexpr int M = decltype(m)::value;
        const dim3 grid((a.T + a.places - 1) / a.places, d.parts, a.rp / (16 * RB));
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

hipError_t up(UpArgs a, int32_t ydtype, int32_t wdtype, bool across, hipStream_t stream) {
  a.places = up_places(a.T);
  const dim3 grid((a.T + a.places - 1) / a.places, (a.C + kUpWaves * kUpCols - 1) / (kUpWaves * kUpCols));
  return by_rank<8>(a.rp, [&](auto rb) {
    return by_types(ydtype, wdtype, [&](auto yb, auto wb) {
      typedef Sums<decltype(wb)::value, decltype(rb)::value> S;
      const size_t lds = (size_t)S::kPlanes * ((a.places + 15) & ~15) * S::kStride * sizeof(typename S::T);
      const auto go = [&](auto ac) {
        hipLaunchKernelGGL((k_adapter_up<decltype(yb)::value, decltype(wb)::value, decltype(ac)::value, decltype(rb)::value>), grid,
                           dim3(kUpWaves * kWave), lds, stream, a);
        return hipGetLastError();
      };
      return across ? go(std::true_type{}) : go(std::false_type{});
    });
  });
}

hipError_t outer(const OuterArgs& a, int32_t dtype, bool across, hipStream_t stream) {
  const auto go = [&](auto bf, auto ac, auto rb) {
    constexpr bool BF = decltype(bf)::value;
    constexpr int RB = decltype(rb)::value;
    typedef OuterTile<BF> O;
    const dim3 grid((a.C + O::kCols - 1) / O::kCols, (a.T + a.chunk - 1) / a.chunk, (a.r + 16 * RB - 1) / (16 * RB));
    hipLaunchKernelGGL((k_adapter_outer<BF, decltype(ac)::value, RB>), grid, dim3(kOuterWaves * kWave),
                       (kOuterWaves / 2) * O::kPer * RB * 64 * sizeof(floatx4), stream, a);
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

size_t part_bytes(const DownPlan& d, int32_t T, int32_t rp) { return up256((size_t)d.parts * T * rp * 4); }

// Most parts x places over the calls of up to T_max rows: the parts grow only where T does not, so the largest T of each
// number of places is the most.
size_t most_parts(int32_t T_max, int32_t C, int32_t rp) {
  size_t most = 0;
  for (const int32_t t : {64, 256, 2047, T_max}) {
    const int32_t T = std::min(t, T_max);
    // Blocks times parts is at most 512, or the blocks themselves.
    const int32_t parts = ((C + 63) / 64 + kDownWaves - 1) / kDownWaves, places = down_plan(T, C).places;
    most = std::max(most, std::min((size_t)T * parts, std::max<size_t>((size_t)T, (size_t)512 * places)) * rp * 4);
  }
  return up256(most);
}

// Chunks of `outer` at most for up to T_max rows.
int64_t most_chunks(int32_t T_max, int32_t C) {
  const int64_t tiles = (C + OuterTile<true>::kCols - 1) / OuterTile<true>::kCols;
  return std::min<int64_t>((T_max + 127) / 128, std::max<int64_t>(1, 1024 / tiles));
}

size_t slot_bytes(int64_t chunks, int32_t r, int32_t C) { return up256((size_t)(2 * chunks) * r * C * 4); }

}  // namespace
}  // namespace damoe

using namespace damoe;

extern "C" {

size_t damoe_adapters_workspace_size(int32_t T_max, int32_t L, int32_t r, int32_t K, int32_t N) {
  if (check(T_max, L, r, K, N, DAMOE_F32, DAMOE_F32, DAMOE_F32)) return 0;
  return 256 + most_parts(T_max, K, padded_rank(r));
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
  if (ws_bytes < part_bytes(d, T, rp)) return DAMOE_ERR_WORKSPACE;
  float* part = static_cast<float*>(ws);
  const DownArgs da{x, ldx, a, perm, offsets, nullptr, part, L, T, K, r, rp, 0, 0};
  if (down(da, d, xdtype, wdtype, false, stream) != hipSuccess) return DAMOE_ERR_HIP;
  const UpArgs ua{part, d.parts, u, b, scale, perm, offsets, add, ld_add, y, ldy, L, T, N, r, rp, 0};
  return up(ua, ydtype, wdtype, false, stream) == hipSuccess ? DAMOE_OK : DAMOE_ERR_HIP;
}

size_t damoe_adapters_grad_workspace_size(int32_t T_max, int32_t L, int32_t r, int32_t K, int32_t N) {
  if (check(T_max, L, r, K, N, DAMOE_F32, DAMOE_F32, DAMOE_F32)) return 0;
  return 256 + most_parts(T_max, N, padded_rank(r)) + slot_bytes(most_chunks(T_max, K), r, K) + slot_bytes(most_chunks(T_max, N), r, N);
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
  float *part = nullptr, *slots_a = nullptr, *slots_b = nullptr;
  if (T > 0) {
    const DownPlan d = down_plan(T, N);
    const size_t at_a = part_bytes(d, T, rp), at_b = at_a + slot_bytes((T + ck - 1) / ck, r, K);
    if (ws_bytes < at_b + slot_bytes((T + cn - 1) / cn, r, N)) return DAMOE_ERR_WORKSPACE;
    part = reinterpret_cast<float*>(base);
    slots_a = reinterpret_cast<float*>(base + at_a);
    slots_b = reinterpret_cast<float*>(base + at_b);
    const DownArgs ga{dy, ldy, b, perm, offsets, scale, part, L, T, N, r, rp, 0, 0};
    if (down(ga, d, ydtype, wdtype, true, stream) != hipSuccess) return DAMOE_ERR_HIP;
    if (dx) {
      const UpArgs xa{part, d.parts, nullptr, a, nullptr, perm, offsets, add, ld_add, dx, ld_dx, L, T, K, r, rp, 0};
      if (up(xa, xdtype, wdtype, true, stream) != hipSuccess) return DAMOE_ERR_HIP;
    }
    const OuterArgs oa{x, ldx, part, d.parts, rp, nullptr, perm, offsets, da, slots_a, L, T, K, r, ck, accumulate};
    if (outer(oa, xdtype, false, stream) != hipSuccess) return DAMOE_ERR_HIP;
    const OuterArgs ob{dy, ldy, u, 1, r, scale, perm, offsets, db, slots_b, L, T, N, r, cn, accumulate};
    if (outer(ob, ydtype, true, stream) != hipSuccess) return DAMOE_ERR_HIP;
  }
  JoinArgs j{offsets, {da, db}, {slots_a, slots_b}, {(int64_t)r * K, (int64_t)r * N}, {ck, cn}, L, T, accumulate, 1024};
  const int64_t all = j.size[0] + j.size[1];
  while ((all + j.per - 1) / j.per * L > 4096 && j.per < all) j.per *= 2;
  hipLaunchKernelGGL(k_adapter_join, dim3((unsigned)((all + j.per - 1) / j.per), L), dim3(256), 0, stream, j);
  return hipGetLastError() == hipSuccess ? DAMOE_OK : DAMOE_ERR_HIP;
}

}  // extern "C"
