// Sums over places of r x columns products (dA, dB): what damoe_adapters_grad's files share.
#pragma once

#include "adapters.h"

namespace damoe {
namespace {

constexpr int kOuterWaves = 4;

// Place of the by-rank pieces that segment l's first place, lo, has; and the pieces that there are of T places.
__host__ __device__ __forceinline__ int first_by_rank(int lo, int l) { return (lo + 7) / 8 * 8 + 16 * l; }
inline size_t pieces_by_rank(int32_t T, int32_t L) { return (size_t)(T + 7) / 8 + 2 * L + 8; }  // loads go up to 31 places past the last

// Eight places' values of a rank as operands: three thirds in bf16, or two halves of four in fp32.
__device__ __forceinline__ void thirds(const float (&v)[8], uint4 (&out)[3]) {
  uint32_t q[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) q[k] = __float_as_uint(v[k]);
  thirds(q, out);
}
__device__ __forceinline__ void thirds(const float (&v)[8], uint4 (&out)[2]) {
#pragma unroll
  for (int h = 0; h < 2; ++h)
    out[h] = uint4{__float_as_uint(v[4 * h]), __float_as_uint(v[4 * h + 1]), __float_as_uint(v[4 * h + 2]), __float_as_uint(v[4 * h + 3])};
}

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
// MFMA j has column P i + j as row i.  8192 rows of 7168 at rank 32 alone: 40 us, 20 of them the tile's search, the products
// and the joining of waves and chunks, which do not overlap a block's own stream.  The next step's rows are loaded while one is multiplied.  Lanes past the last column
// take the last P again; SMALL: there are fewer than P, each is loaded for itself.
// DIRECT: the r factors are a.part's, whose thirds are made here; a step's rows are then waited for.
template <bool BF, bool ACROSS, int RB, bool SMALL, bool DIRECT>
struct Outer {
  typedef OuterTile<BF> O;
  typedef typename Elem<BF>::T X;
  static constexpr int P = O::kPer, F = BF ? 3 : 2;
  static constexpr int kPlane = 64 * 4 + 4;  // floats of a wave's MFMA in LDS
  static constexpr int kLds = kOuterWaves * P * kPlane;

  static __device__ __forceinline__ void run(const OuterArgs& a, const Tile& tile, int b0, int r0, float* sums) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int i = lane & 15, g = lane >> 4;
    const int c = SMALL ? P * i : min(b0 + P * i, a.C - P);
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
          if constexpr (!DIRECT) s.u[rb][h] = static_cast<const uint4*>(a.by_rank)[((int64_t)((p + shift) / 8 + g) * F + h) * a.rp + r0 + 16 * rb + i];
      if constexpr (DIRECT) {
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
          float f[8] = {};
          const float* part = a.part + min(r0 + 16 * rb + i, a.r - 1);
          if (a.parts == 1) {
#pragma unroll
            for (int k = 0; k < 8; ++k) f[k] = part[(int64_t)min(p + 8 * g + k, tile.hi - 1) * a.ld];
          }
          for (int n = a.parts == 1 ? 1 : 0; n < a.parts; n += 4) {  // in order, four parts' loads in flight
            float q[4][8];
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
              for (int k = 0; k < 8; ++k)
                q[j][k] = part[((int64_t)min(n + j, a.parts - 1) * a.T + min(p + 8 * g + k, tile.hi - 1)) * a.ld];
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
              for (int k = 0; k < 8; ++k)
                if (n + j < a.parts) f[k] += q[j][k];
          }
          thirds(f, s.u[rb]);
        }
      }
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
    if (DIRECT || steps == 1) {
      for (int step = 0; step < steps; ++step) {
        Rows s;
        load(s, place(step), step);
        work(s);
      }
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
    if (!tile.whole && tile.slot >= a.n_slots) return;  // offsets that decrease
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
};

}  // namespace
}  // namespace damoe
