// The dense MXFP4 product y = add + Q(x) W^T on the scaled fp4 matrix instructions.
//
// Both operands are in DAMOE_LAYOUT_TILE32: W as the caller holds it, Q(x) quantised into the workspace by
// the call.  v_mfma_scale_f32_32x32x64_f8f6f4 multiplies a step of 64 columns: lane 32 h + r holds row r,
// columns 32 h .. + 31, one scale block, and takes its scale from a byte of a register.  Products and scales
// are exact (a product is a multiple of 2^-2 times the scales, at most 36), the sums are fp32.
#include <type_traits>

#include "common.h"
#include "device.h"
#include "mxfp4.h"

namespace damoe {
namespace {

typedef int v8i __attribute__((ext_vector_type(8)));

struct LinearArgs {
  const uint8_t* w;   // tiles of N x K
  const uint8_t* x;   // tiles of T x K
  const void* add;
  void* y;
  int64_t ld_add, ldy;
  int32_t T, N, nk;   // nk: tiles along K
  int32_t y_bf;
  int32_t vec;        // rows of y and add start at 16 bytes, N is whole eights, 32 rows lie within 2^31 bytes
  int32_t tiles_r;    // row tiles of W (the kernel of many tokens)
};

// Both operands' fp4 codes fill the lower half of the instruction's 8-register operands.
template <int J>
__device__ __forceinline__ floatx16 mfma_fp4(const uint4& a, uint32_t sa, const uint4& b, uint32_t sb, const floatx16& c) {
  const v8i av = {(int)a.x, (int)a.y, (int)a.z, (int)a.w, 0, 0, 0, 0};
  const v8i bv = {(int)b.x, (int)b.y, (int)b.z, (int)b.w, 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(av, bv, c, 4, 4, J, (int)sa, J, (int)sb);
}

__device__ __forceinline__ float load_elem(const void* p, int64_t i, bool bf) {
  return bf ? bf16_to_f32(static_cast<const uint16_t*>(p)[i]) : static_cast<const float*>(p)[i];
}

// ---------------------------------------------------------------- many tokens
//
// A workgroup of four waves takes tiles of 128 MA rows of W x 32 NB tokens, one after the other: a wave has 32 MA rows
// (MA blocks) and all the tokens, MA NB accumulator blocks.  A stage, 256 columns, is 4 MA NB MFMAs a wave.  A CU loads
// about 100 GB/s, which bounds the small tiles, so they are as near to square as whole waves of rows allow, and
// two workgroups of 128 rows share a CU, one's start and end beside the other's stages (256 x 32 / 128 x 64, 256 x 64 /
// 128 x 96: 15.0 / 12.5 and 17.7 / 14.2 us at T = 300, 4096 x 7168; 49.9 / 43.4 and 45.0 / 40.7 at 4096, 7168 x 2048).
//   W      straight into registers, every fragment read by one wave: the registers of a step are loaded for a
//          stage D ahead as soon as its MFMAs have read them.
//   tokens through LDS, which the four waves share: global -> registers (D stages ahead) -> LDS (the wave's quarter
//          of the stage), in a ring of three stages.  The operand layout makes every LDS access one contiguous 1 KB.
// One barrier a stage, in its middle: it makes the next stage's tokens visible, so that the first operands of
// the next stage can be read before this one's last MFMAs, and with three buffers the one being filled is
// that of the stage before last.  Reads, writes and loads stand one at a time behind pairs of MFMAs.  The stages of a
// workgroup's tiles run on without a gap: the last stages of a tile load the first of the next one, whose results
// leave while those loads are in flight.
constexpr int wait_lgkm(int n) { return 15 | (7 << 4) | (n << 8) | (3 << 14); }

typedef __attribute__((address_space(3))) uint8_t lds_t;
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint4 lds_read16(const lds_t* p) {
  return __builtin_bit_cast(uint4, *reinterpret_cast<const __attribute__((address_space(3))) u32x4*>(p));
}
__device__ __forceinline__ uint32_t lds_read4(const lds_t* p) {
  return *reinterpret_cast<const __attribute__((address_space(3))) uint32_t*>(p);
}
__device__ __forceinline__ void lds_write16(lds_t* p, uint4 v) {
  *reinterpret_cast<__attribute__((address_space(3))) u32x4*>(p) = __builtin_bit_cast(u32x4, v);
}
__device__ __forceinline__ void lds_write4(lds_t* p, uint32_t v) {
  *reinterpret_cast<__attribute__((address_space(3))) uint32_t*>(p) = v;
}

// Tiles of a workgroup.  Workgroups b, b + 8, ... share an XCD and its L2: each XCD takes a run of the tiles in bands of
// kBand row tiles, so that the 32 tiles it works on at a time are about 4 x 8 and read 12 rows of tiles, not 18 or 33.
constexpr int kBand = 4;

struct TileWalk {
  int n, per, first, step, tiles_r, tiles_t;

  __device__ __forceinline__ TileWalk(const LinearArgs& a, int tiles_t_) : tiles_r(a.tiles_r), tiles_t(tiles_t_) {
    n = tiles_r * tiles_t;
    per = (n + 7) / 8;
    first = blockIdx.x >> 3;
    step = gridDim.x >> 3;
  }

  // The workgroup's tile number `turn`; false past its last.
  __device__ __forceinline__ bool tile(int turn, int& rt, int& tt) const {
    const int i = first + turn * step, l = (blockIdx.x & 7) * per + i;
    if (i >= per || l >= n) return false;
    const int band = l / (kBand * tiles_t), in = l - band * kBand * tiles_t;
    const int width = min(kBand, tiles_r - band * kBand);
    rt = band * kBand + in % width;
    tt = in / width;
    return true;
  }
};

// A wave's 32 tokens x 32 MA columns of results on their way through LDS, so that stores fill whole 128-byte lines (a lane
// of the accumulators holds four columns of one token): rows of bf16 where nothing is added, of fp32 otherwise, 16
// bytes apart.  LDS carries out a wave's accesses in order, so only the compiler is held back between them.
constexpr uint32_t out_bytes(int MA) { return 32 * (32 * MA * 4 + 16); }

__device__ __forceinline__ void wave_lds_fence() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_wave_barrier();
}

template <int MA, bool YBF, bool ADD>
struct Out {
  static constexpr bool kHalf = YBF && !ADD;             // bf16 rows in LDS
  static constexpr uint32_t kElem = kHalf ? 2 : 4, kCols = 32 * MA, kPitch = kCols * kElem + 16;
  static constexpr int kLanes = kCols * kElem / 16;         // lanes of a row, 16 bytes each
  static constexpr int kRowsAt = 64 / kLanes, kTrips = 32 / kRowsAt;
  uint4 v[kTrips];

  // Register 4 q + i of lane 32 g + r of block m is column 32 m + 8 q + 4 g + i of token r.
  static __device__ __forceinline__ void put(lds_t* out, floatx16 c, int m, int lane) {
    if constexpr (kHalf) asm volatile("" : "+v"(c));  // converted here and not, all blocks at once, ahead of the loop
    lds_t* p = out + (uint32_t)(lane & 31) * kPitch + (32u * m + 4u * (lane >> 5)) * kElem;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      if constexpr (kHalf) {
        const u32x2 h = {pack_bf16x2(c[4 * q], c[4 * q + 1]), pack_bf16x2(c[4 * q + 2], c[4 * q + 3])};
        *reinterpret_cast<__attribute__((address_space(3))) u32x2*>(p + 16 * q) = h;
      } else {
        lds_write16(p + 32 * q, make_uint4(__float_as_uint(c[4 * q]), __float_as_uint(c[4 * q + 1]),
                                           __float_as_uint(c[4 * q + 2]), __float_as_uint(c[4 * q + 3])));
      }
    }
  }

  __device__ __forceinline__ void get(const lds_t* out, int lane) {
    const lds_t* p = out + (uint32_t)(lane / kLanes) * kPitch + 16u * (lane % kLanes);
#pragma unroll
    for (int i = 0; i < kTrips; ++i) v[i] = lds_read16(p + i * kRowsAt * kPitch);
  }

  // The rows of tokens t0 .. t0 + 31, columns n0 .. + kCols - 1, where a.vec: whole lanes in or out of range, rows within 32-bit
  // offsets of the block's first.  A store's offset is all in its vector register: behind a 16-byte store with one in a
  // scalar register the compiler lets the next instruction write the store's data, which reached memory now and then
  // (an address in place of a sum, fp32 with `add`); behind one without it puts the wait that is needed.
  __device__ __forceinline__ void store(const LinearArgs& a, int64_t t0, int n0, int lane) const {
    constexpr uint32_t es = YBF ? 2 : 4;
    const int n = 16 / (int)kElem * (lane % kLanes), r0 = lane / kLanes;
    const int rows = n0 + n < a.N ? (int)min((int64_t)32, a.T - t0) - r0 : 0;
    const __amdgpu_buffer_rsrc_t ry = make_rsrc(static_cast<char*>(a.y) + (t0 * a.ldy + n0) * es, kOobOffset);
    const uint32_t ldy = (uint32_t)a.ldy * es, yo = (uint32_t)r0 * ldy + (uint32_t)n * es;
#pragma unroll
    for (int i = 0; i < kTrips; ++i) {
      const bool in = i * kRowsAt < rows;
      const uint32_t o = in ? yo + (uint32_t)(i * kRowsAt) * ldy : kOobOffset;
      if constexpr (kHalf) {
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v[i]), ry, o, 0, 0);
        continue;
      }
      float f[4] = {__uint_as_float(v[i].x), __uint_as_float(v[i].y), __uint_as_float(v[i].z), __uint_as_float(v[i].w)};
      if constexpr (ADD) {
        const __amdgpu_buffer_rsrc_t ra = make_rsrc(static_cast<const char*>(a.add) + (t0 * a.ld_add + n0) * es, kOobOffset);
        const uint32_t lda = (uint32_t)a.ld_add * es;
        const uint32_t p = in ? (uint32_t)r0 * lda + (uint32_t)n * es : kOobOffset, sp = (uint32_t)(i * kRowsAt) * lda;
        if constexpr (YBF) {
          const uint2 d = buf_load<uint2, 0>(ra, p, sp);
          f[0] += __uint_as_float(d.x << 16), f[1] += __uint_as_float(d.x & 0xFFFF0000u);
          f[2] += __uint_as_float(d.y << 16), f[3] += __uint_as_float(d.y & 0xFFFF0000u);
        } else {
          const uint4 d = buf_load<uint4, 0>(ra, p, sp);
          f[0] += __uint_as_float(d.x), f[1] += __uint_as_float(d.y);
          f[2] += __uint_as_float(d.z), f[3] += __uint_as_float(d.w);
        }
      }
      if constexpr (YBF) {
        const u32x2 h = {pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3])};
        __builtin_amdgcn_raw_buffer_store_b64(h, ry, o, 0, 0);
      } else {
        const u32x4 h = {__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])};
        __builtin_amdgcn_raw_buffer_store_b128(h, ry, o, 0, 0);
      }
    }
  }

  // The same for any strides, alignment and N: global accesses of whole lanes at an element's alignment, and the
  // elements of a row's last lane one by one (60 calls with odd N take 0.76 to 0.88 of the time that a column a lane, an
  // element at a time, took; where `store` applies it is 3% faster).
  __device__ __forceinline__ void store_any(const LinearArgs& a, int64_t t0, int n0, int lane) const {
    constexpr int kN = 16 / (int)kElem;
    typedef std::conditional_t<YBF, uint16_t, float> T;
    typedef uint32_t Words __attribute__((ext_vector_type(kN * sizeof(T) / 4), aligned(sizeof(T))));
    const int n = n0 + kN * (lane % kLanes), r0 = lane / kLanes;
    const int rows = (int)min((int64_t)32, a.T - t0) - r0, cols = min(kN, a.N - n);
    T* y = static_cast<T*>(a.y) + (t0 + r0) * a.ldy + n;
    const T* add = static_cast<const T*>(a.add) + (t0 + r0) * a.ld_add + n;
#pragma unroll
    for (int i = 0; i < kTrips; ++i, y += kRowsAt * a.ldy, add += kRowsAt * a.ld_add) {
      if (i * kRowsAt >= rows || cols <= 0) continue;
      union {
        Words w;
        T e[kN];
      } o, d;
      const uint32_t u[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
      if constexpr (ADD) {
        if (cols == kN) d.w = *reinterpret_cast<const Words*>(add);
        else
          for (int e = 0; e < kN; ++e) d.e[e] = e < cols ? add[e] : T(0);
      }
      if constexpr (kHalf) {
#pragma unroll
        for (int e = 0; e < 4; ++e) o.w[e] = u[e];
      } else {
#pragma unroll
        for (int e = 0; e < kN; ++e) {
          float f = __uint_as_float(u[e]);
          if constexpr (ADD && YBF) f += bf16_to_f32(d.e[e]);
          if constexpr (ADD && !YBF) f += d.e[e];
          if constexpr (YBF) o.e[e] = __builtin_bit_cast(uint16_t, (__bf16)f);
          else o.e[e] = f;
        }
      }
      if (cols == kN) {
        *reinterpret_cast<Words*>(y) = o.w;
      } else {
#pragma unroll
        for (int e = 0; e < kN; ++e)
          if (e < cols) y[e] = o.e[e];
      }
    }
  }
};

template <int MA, int NB, bool YBF, bool ADD>
__global__ void __launch_bounds__(256, 3 - MA) k_mxfp4_gemm(LinearArgs a) {
  constexpr uint32_t kStage = NB * kTileBytes;
  // Token operands read ahead of their MFMAs; reads of the next stage's start behind the barrier, in step 2.
  constexpr int kAhead = NB >= 2 ? 4 : 2;
  constexpr int D = 2;  // stages ahead that weights and tokens are loaded (4 is no faster, and its code starts colder)
  constexpr int kScaleMoves = (NB + 3) / 4;  // a wave's 256 B pieces of a stage (its 1 KB pieces: NB)
  extern __shared__ __attribute__((aligned(1024))) uint8_t gemm_smem[];
  lds_t* const lds = (lds_t*)gemm_smem;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  lds_t* const mine = lds + 3 * kStage + w * out_bytes(MA);
  const int nrb = (a.N + 31) / 32, ntb = (a.T + 31) / 32, nk = a.nk;
  // Stages of a tile: whole turns of the D sets of registers, and two at least (a stage's loads reach into the next
  // tile at most); stages past nk multiply zero weights.
  const int ns = max(2 * D, (nk + D - 1) / D * D);
  const TileWalk walk(a, (ntb + NB - 1) / NB);
  int rt, tt, turn = 0;
  if (!walk.tile(0, rt, tt)) return;

  const __amdgpu_buffer_rsrc_t rw = make_rsrc(a.w, (uint32_t)nrb * (uint32_t)nk * kTileBytes);
  const __amdgpu_buffer_rsrc_t rx = make_rsrc(a.x, (uint32_t)ntb * (uint32_t)nk * kTileBytes);
  const uint32_t row_bytes = (uint32_t)nk * kTileBytes;  // of a row of tiles
  const uint32_t l16 = 16u * lane, l4 = 4u * lane;

  // Where a tile's weights and tokens start: row and token blocks past the last repeat it, and their results are not
  // stored.
  struct Base {
    uint32_t w[MA], x[NB], xs[kScaleMoves];
  };
  auto base_of = [&](int rt_, int tt_) __attribute__((always_inline)) {
    Base b;
#pragma unroll
    for (int m = 0; m < MA; ++m) b.w[m] = (uint32_t)min((rt_ * 4 + w) * MA + m, nrb - 1) * row_bytes;
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      const int piece = w * NB + i;
      b.x[i] = (uint32_t)min(tt_ * NB + (piece >> 2), ntb - 1) * row_bytes + 1024u * (piece & 3);
    }
#pragma unroll
    for (int i = 0; i < kScaleMoves; ++i)
      b.xs[i] = (uint32_t)min(tt_ * NB + min(w * kScaleMoves + i, NB - 1), ntb - 1) * row_bytes + kTileCodes;
    return b;
  };
  Base cur = base_of(rt, tt), nxt = cur;

  // Sets by the stage modulo D, of scales from LDS modulo 2.
  uint4 wq[D][MA][4], st[D][NB], xr[kAhead];
  uint32_t wsc[D][MA], sts[D][kScaleMoves], xs[2][NB];
  floatx16 acc[MA][NB];

  // Loads of stage t of the current tile, or t - ns of the next.
  auto at = [&](int t) __attribute__((always_inline)) { return (uint32_t)min(t < ns ? t : t - ns, nk - 1) * kTileBytes; };
  auto load_w = [&](int t, int p, int j, int m) __attribute__((always_inline)) {
    const uint32_t o = (t < ns ? t : t - ns) < nk ? l16 : kOobOffset;  // out of range: zero codes
    wq[p][m][j] = buf_load<uint4, 0>(rw, o + 1024u * j, (t < ns ? cur.w[m] : nxt.w[m]) + at(t));
  };
  auto load_ws = [&](int t, int p, int m) __attribute__((always_inline)) {
    wsc[p][m] = buf_load<uint32_t, 0>(rw, l4, (t < ns ? cur.w[m] : nxt.w[m]) + at(t) + kTileCodes);
  };
  auto load_x = [&](int t, int p, int i) __attribute__((always_inline)) {
    st[p][i] = buf_load<uint4, 0>(rx, l16, (t < ns ? cur.x[i] : nxt.x[i]) + at(t));
  };
  auto load_xs = [&](int t, int p, int i) __attribute__((always_inline)) {
    sts[p][i] = buf_load<uint32_t, 0>(rx, l4, (t < ns ? cur.xs[i] : nxt.xs[i]) + at(t));
  };
  auto write_x = [&](lds_t* buf, int p, int i) __attribute__((always_inline)) {
    const int piece = w * NB + i;
    lds_write16(buf + (piece >> 2) * kTileBytes + 1024 * (piece & 3) + l16, st[p][i]);
  };
  auto write_xs = [&](lds_t* buf, int p, int i) __attribute__((always_inline)) {
    lds_write4(buf + min(w * kScaleMoves + i, NB - 1) * kTileBytes + kTileCodes + l4, sts[p][i]);
  };
  // Token operand i of a stage: step i / NB, token block i % NB.
  auto read_x = [&](const lds_t* buf, int i) __attribute__((always_inline)) {
    return lds_read16(buf + (i % NB) * kTileBytes + 1024 * (i / NB) + l16);
  };
  auto read_xs = [&](const lds_t* buf, int p, int n) __attribute__((always_inline)) {
    xs[p][n] = lds_read4(buf + n * kTileBytes + kTileCodes + l4);
  };
  // MFMAs of step J of stage t in buf (next: the buffer of the stage after it), and behind each pair one or two of the
  // stage's other accesses: step 0 writes the next stage's tokens, step 1 loads those of stage t + 1 + D into the
  // registers that became free, step 2 reads the next stage's scales; every step loads the weights of the step before
  // it again, for D stages on.
  auto step = [&](const lds_t* buf, lds_t* next, int t, auto p, auto j) __attribute__((always_inline)) {
    constexpr int P = decltype(p)::value, J = decltype(j)::value;  // P: t modulo D
    constexpr int Q = (P + 1) % D, R = (P + D - 1) % D;
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      const int i = J * NB + n, f = i + kAhead;
#pragma unroll
      for (int m = 0; m < MA; ++m) acc[m][n] = mfma_fp4<J>(wq[P][m][J], wsc[P][m], xr[i % kAhead], xs[P % 2][n], acc[m][n]);
      xr[i % kAhead] = f < 4 * NB ? read_x(buf, f) : read_x(next, f - 4 * NB);
      if constexpr (J == 0) {
        write_x(next, Q, n);
        if (n < kScaleMoves) write_xs(next, Q, n);
      } else if constexpr (J == 1) {
        load_x(t + 1 + D, Q, n);
        if (n < kScaleMoves) load_xs(t + 1 + D, Q, n);
      } else if constexpr (J == 2) {
        read_xs(next, 1 - P % 2, n);
      }
#pragma unroll
      for (int m = 0; m < MA; ++m) {
        if (n != (m + 1) * NB / 3) continue;
        if constexpr (J == 0) {
          load_w(t - 1 + D, R, 3, m);
          load_ws(t - 1 + D, R, m);
        } else {
          load_w(t + D, P, J - 1, m);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  using std::integral_constant;
  auto barrier = [&]() __attribute__((always_inline)) {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  auto stage = [&](int t, const lds_t* buf, lds_t* next, auto p) __attribute__((always_inline)) {
    step(buf, next, t, p, integral_constant<int, 0>{});
    step(buf, next, t, p, integral_constant<int, 1>{});
    // Step 0's writes are older than step 1's NB operand reads, and LDS answers a wave in order.
    __builtin_amdgcn_s_waitcnt(wait_lgkm(NB < kAhead ? 0 : kAhead - 1));
    barrier();
    step(buf, next, t, p, integral_constant<int, 2>{});
    step(buf, next, t, p, integral_constant<int, 3>{});
  };

#pragma unroll
  for (int p = 0; p < D; ++p) {
#pragma unroll
    for (int i = 0; i < NB; ++i) load_x(p, p, i);
#pragma unroll
    for (int i = 0; i < kScaleMoves; ++i) load_xs(p, p, i);
#pragma unroll
    for (int m = 0; m < MA; ++m) {
#pragma unroll
      for (int j = 0; j < 4; ++j) load_w(p, p, j, m);
      load_ws(p, p, m);
    }
  }
#pragma unroll
  for (int i = 0; i < NB; ++i) write_x(lds, 0, i);
#pragma unroll
  for (int i = 0; i < kScaleMoves; ++i) write_xs(lds, 0, i);
#pragma unroll
  for (int i = 0; i < NB; ++i) load_x(D, 0, i);
#pragma unroll
  for (int i = 0; i < kScaleMoves; ++i) load_xs(D, 0, i);
  __builtin_amdgcn_s_waitcnt(wait_lgkm(0));
  barrier();
#pragma unroll
  for (int n = 0; n < NB; ++n) read_xs(lds, 0, n);
#pragma unroll
  for (int i = 0; i < kAhead; ++i) xr[i] = read_x(lds, i);
  uint32_t b0 = 0, b1 = kStage, b2 = 2 * kStage;
  for (;;) {
    int rt1 = rt, tt1 = tt;
    const bool more = walk.tile(++turn, rt1, tt1);
    nxt = base_of(rt1, tt1);  // with no next tile, the loads repeat this one's
#pragma unroll
    for (int m = 0; m < MA; ++m)
#pragma unroll
      for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[m][n][i] = 0.f;
    const auto turn_of = [&](int t, auto p) __attribute__((always_inline)) {
      stage(t + decltype(p)::value, lds + b0, lds + b1, p);
      const uint32_t o = b0;
      b0 = b1, b1 = b2, b2 = o;
    };
    for (int t = 0; t < ns; t += D) {
      turn_of(t, integral_constant<int, 0>{});
      turn_of(t, integral_constant<int, 1>{});
    }
    // Results, a token block at a time through LDS of the wave's own; a block's stores go out while the next one's
    // values come back from LDS.
    using O = Out<MA, YBF, ADD>;
    O o[2];
    const int nb = min(NB, ntb - tt * NB), n0 = (rt * 4 + w) * 32 * MA;
#pragma unroll
    for (int n = 0; n <= NB; ++n) {
      if (n < NB && n < nb) {
#pragma unroll
        for (int m = 0; m < MA; ++m) O::put(mine, acc[m][n], m, lane);
        wave_lds_fence();
        o[n & 1].get(mine, lane);
        wave_lds_fence();
      }
      if (n > 0 && n <= nb) {
        const int64_t t0 = (int64_t)(tt * NB + n - 1) * 32;
        if (a.vec) o[(n - 1) & 1].store(a, t0, n0, lane);
        else o[(n - 1) & 1].store_any(a, t0, n0, lane);
      }
    }
    if (!more) break;
    rt = rt1, tt = tt1;
    cur = nxt;
  }
}

template <int MA, int NB>
constexpr size_t gemm_lds() {
  return 3 * NB * kTileBytes + 4 * out_bytes(MA);
}

// ---------------------------------------------------------------- few tokens
//
// A workgroup of eight waves takes 16 MR rows of W and 16 NT tokens, and its waves the tiles of 256 columns in turn, so
// that even a short row keeps every wave's loads in flight at once; the waves' sums meet in LDS and are added in
// order.  The weight stream is the traffic (latency at few rows), so nothing is staged: a wave reads both operands
// straight into registers.
//
// v_mfma_scale_f32_16x16x128_f8f6f4: lane 16 b + i holds row i, columns 32 b .. + 31, one scale block.  In a tile that is
// the piece of step b / 2 (+ 2 for the second 128 columns), half b % 2, and byte b / 2 (+ 2) of its scales.  The
// result has D[4 (l / 16) + i][l % 16] in register i.
constexpr int kRowsThreads = 512, kRowsWaves = kRowsThreads / kWave;

struct RowsArgs {
  LinearArgs l;
  const void* x;  // rows to quantise here (XT: bf16 or fp32), 16-byte aligned; or unused
  int64_t ldx;
  int32_t K;
};

// 16 rows of a tile in operand form.
struct Half {
  uint4 q[2];
  uint32_t s;

  // off: the lane's offset in the tile, soff its scales'.
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t r, uint32_t tile, uint32_t off, uint32_t soff) {
    q[0] = buf_load<uint4, 0>(r, off, tile);
    q[1] = buf_load<uint4, 0>(r, off + 2048u, tile);
    s = buf_load<uint32_t, 0>(r, soff, tile);
  }
  __device__ __forceinline__ void align(int lane) { s >>= 8 * (lane >> 5); }  // byte b / 2 to the front
};

// The same from 32 values a lane and 128 columns, quantised in the lane.
template <bool BF>
struct Raw {
  Eight<BF> e[2][4];

  __device__ __forceinline__ void load(const void* x, int64_t row, int c, int K) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (row >= 0 && c + 128 * h < K) e[h][i].template load<true>(x, row + c + 128 * h + 8 * i);
        else e[h][i].zero();
      }
  }
  __device__ __forceinline__ void quantise(Half& o) const {
    o.s = 0;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      uint32_t m = e[h][0].amax();
#pragma unroll
      for (int i = 1; i < 4; ++i) m = max(m, e[h][i].amax());
      const uint32_t s = fp4_scale_byte(m);
      o.q[h] = make_uint4(e[h][0].codes(s), e[h][1].codes(s), e[h][2].codes(s), e[h][3].codes(s));
      o.s |= s << (16 * h);
    }
  }
};

template <int H>
__device__ __forceinline__ floatx4 mfma_half(const Half& a, const Half& b, const floatx4& c) {
  const v8i av = {(int)a.q[H].x, (int)a.q[H].y, (int)a.q[H].z, (int)a.q[H].w, 0, 0, 0, 0};
  const v8i bv = {(int)b.q[H].x, (int)b.q[H].y, (int)b.q[H].z, (int)b.q[H].w, 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(av, bv, c, 4, 4, 2 * H, (int)a.s, 2 * H, (int)b.s);
}

// XT: 0 tokens quantised in the workspace, 1 bf16 and 2 fp32 rows quantised here (NT = 1).
template <int MR, int NT, int XT>
__global__ void __launch_bounds__(kRowsThreads, NT > 2 ? 2 : 4) k_mxfp4_rows(RowsArgs ra) {
  static_assert(MR * NT <= kRowsWaves, "a thread sums one lane's four values");
  const LinearArgs& a = ra.l;
  __shared__ floatx4 red[kRowsWaves][MR * NT][kWave];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int i16 = lane & 15, b = lane >> 4;
  const int nrb = (a.N + 31) / 32, ntb = (a.T + 31) / 32, nk = a.nk;
  const int row0 = blockIdx.x * 16 * MR, tok0 = blockIdx.y * 16 * NT;
  const uint32_t row_bytes = (uint32_t)nk * kTileBytes;
  const __amdgpu_buffer_rsrc_t rw = make_rsrc(a.w, (uint32_t)nrb * row_bytes);
  const __amdgpu_buffer_rsrc_t rx = make_rsrc(a.x, (uint32_t)ntb * row_bytes);
  // Lane offsets in a tile, of rows 0 .. 15 of it; the upper sixteen rows are 256 (scales: 64) bytes on.
  const uint32_t off = 1024u * (b >> 1) + 16u * (32 * (b & 1) + i16), soff = kTileCodes + 4u * (32 * (b & 1) + i16);
  uint32_t wbase[MR], xbase[NT], wup[MR], xup[NT];
#pragma unroll
  for (int m = 0; m < MR; ++m) {  // row blocks past the last repeat it; their results are not stored
    const int r = row0 + 16 * m;
    wbase[m] = (uint32_t)min(r >> 5, nrb - 1) * row_bytes;
    wup[m] = (r >> 4) & 1;
  }
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int t = tok0 + 16 * n;
    xbase[n] = (uint32_t)min(t >> 5, ntb - 1) * row_bytes;
    xup[n] = (t >> 4) & 1;
  }
  floatx4 acc[MR][NT];
#pragma unroll
  for (int m = 0; m < MR; ++m)
#pragma unroll
    for (int n = 0; n < NT; ++n) acc[m][n] = floatx4{0.f, 0.f, 0.f, 0.f};

  // Tiles whose weights a wave loads together, and tiles of raw tokens it holds at a time.
  constexpr int U = NT > 2 ? 2 : 4, UX = XT == 1 ? 2 : 1;
  for (int k0 = w; k0 < nk; k0 += U * kRowsWaves) {
    Half wf[U][MR], xf[U][NT];
    Raw<XT != 2> raw[UX];
    const auto load_raw = [&](int u) __attribute__((always_inline)) {
      const int k = k0 + u * kRowsWaves;
      if (k < nk) raw[u % UX].load(ra.x, tok0 + i16 < a.T ? (tok0 + i16) * ra.ldx : -1, 256 * k + 32 * b, ra.K);
    };
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = k0 + u * kRowsWaves;
      if (XT != 0 && u < UX) load_raw(u);
      if (k >= nk) continue;
      const uint32_t tile = (uint32_t)k * kTileBytes;
#pragma unroll
      for (int m = 0; m < MR; ++m) wf[u][m].load(rw, wbase[m] + tile, off + 256u * wup[m], soff + 64u * wup[m]);
      if constexpr (XT == 0) {
#pragma unroll
        for (int n = 0; n < NT; ++n) xf[u][n].load(rx, xbase[n] + tile, off + 256u * xup[n], soff + 64u * xup[n]);
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (k0 + u * kRowsWaves >= nk) continue;
#pragma unroll
      for (int m = 0; m < MR; ++m) wf[u][m].align(lane);
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        if constexpr (XT == 0) {
          xf[u][n].align(lane);
        } else {
          raw[u % UX].quantise(xf[u][n]);
          if (u + UX < U) load_raw(u + UX);
        }
#pragma unroll
        for (int m = 0; m < MR; ++m) {
          acc[m][n] = mfma_half<0>(wf[u][m], xf[u][n], acc[m][n]);
          acc[m][n] = mfma_half<1>(wf[u][m], xf[u][n], acc[m][n]);
        }
      }
    }
  }
#pragma unroll
  for (int m = 0; m < MR; ++m)
#pragma unroll
    for (int n = 0; n < NT; ++n) red[w][m * NT + n][lane] = acc[m][n];
  __syncthreads();
  if (w >= MR * NT) return;
  floatx4 v = red[0][w][lane];
#pragma unroll
  for (int i = 1; i < kRowsWaves; ++i) v += red[i][w][lane];
  const int64_t t = tok0 + 16 * (w % NT) + i16;
  const int n0 = row0 + 16 * (w / NT) + 4 * b;
  if (t >= a.T) return;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (n0 + i >= a.N) continue;
    float f = v[i];
    if (a.add) f += load_elem(a.add, t * a.ld_add + n0 + i, a.y_bf);
    if (a.y_bf) static_cast<uint16_t*>(a.y)[t * a.ldy + n0 + i] = __builtin_bit_cast(uint16_t, (__bf16)f);
    else static_cast<float*>(a.y)[t * a.ldy + n0 + i] = f;
  }
}

// Which kernel a call of more than 32 tokens takes: the one with the least estimated time, in us, fitted to
// 660 measured calls (random T = 33 to 8192, N = 100 to 8192, K = 256 to 8192; in 220 others the pick took at most
// 1.11 of the fastest kernel's time, 1.002 in the geometric mean).
// k_mxfp4_rows<2, 4> runs rounds of a workgroup a CU, each a start and its waves' tiles, and its XCDs take each tile from
// behind their L2s (`moved`, bytes).  k_mxfp4_gemm<MA, NB> runs rounds of tiles, each a fixed part, stages, which take the
// longer the more CUs share the caches and the card's power, and, where rows of y or add are unaligned, slower stores.
// A last round that is not full counts for the mean of a full one and its part where the CUs hold two workgroups.
// Fastest at T = 64 / 300 / 1000 / 4096: 4096 x 7168 rows 6.5, gemm<1, 2> 12.5 (rows 16.4), <1, 2> 21.3 (<1, 3> 23.0),
// <2, 8> 57.2 (<2, 4> 59.3); 7168 x 2048 rows 4.4, <1, 3> 6.8 (<1, 2> 7.6), <2, 4> 12.1 (<1, 3> 13.2), <1, 3> 40.7
// (<2, 4> 41.3).  Tiles of 128 x 128 would be up to 8% faster in 35 calls of 660.
enum Path { kRows, kGemm12, kGemm13, kGemm24, kGemm28 };

Path path_of(int32_t T, int32_t N, int32_t K, bool vec, int cus) {
  const double nk = (double)tiles_of(K, kTileCols);
  const double stages = std::max(4.0, nk + (double)(tiles_of(K, kTileCols) & 1));
  const auto rounds = [&](int64_t n) { return (double)((n + cus - 1) / cus); };
  const auto part_rounds = [&](int64_t n) { return 0.5 * (rounds(n) + std::max(1.0, (double)n / cus)); };
  const int64_t nb = tiles_of(N, 32), tb = tiles_of(T, 32);
  const double moved = (double)(tb * std::min<int64_t>(8, nb) + nb * std::min<int64_t>(8, (tb + 1) / 2)) * nk * kTileBytes;
  double best = 1.2 + part_rounds(nb * ((tb + 1) / 2)) * (2.4 + 0.1 * nk) + 0.04e-6 * moved;
  Path path = kRows;
  constexpr struct {
    Path path;
    int ma, nb;
    double stage, shared, fixed, any;
  } gemms[] = {{kGemm12, 1, 2, 0.28, 0.11, 0.3, 0.0},
               {kGemm13, 1, 3, 0.34, 0.14, 0.45, 0.3},
               {kGemm24, 2, 4, 0.52, 0.51, 2.2, 1.1},
               {kGemm28, 2, 8, 0.98, 0.9, 4.4, 2.5}};
  for (const auto& g : gemms) {
    const int64_t tiles = tiles_of(N, 128 * g.ma) * tiles_of(T, 32 * g.nb);
    const double stage = g.stage + g.shared * std::min(1.0, (double)tiles / cus);
    const double t = 2.95 + (g.ma == 1 ? part_rounds(tiles) : rounds(tiles)) * (stages * stage + g.fixed + (vec ? 0.0 : g.any));
    if (t < best) best = t, path = g.path;
  }
  return path;
}

// As many workgroups as the CUs hold: two a CU of the 128-row tiles (at most 256 registers), one of the others.
template <int MA, int NB>
hipError_t launch_gemm(LinearArgs a, int cus, hipStream_t stream) {
  a.tiles_r = (int32_t)tiles_of(a.N, 128 * MA);
  const int64_t tiles = a.tiles_r * tiles_of(a.T, 32 * NB);
  const dim3 grid((unsigned)std::min<int64_t>(tiles_of(tiles, 8), std::max(1, cus * (3 - MA) / 8)) * 8);
  const auto go = [&](void (*f)(LinearArgs)) { hipLaunchKernelGGL(f, grid, dim3(256), (gemm_lds<MA, NB>()), stream, a); };
  if (a.y_bf) go(a.add ? k_mxfp4_gemm<MA, NB, true, true> : k_mxfp4_gemm<MA, NB, true, false>);
  else go(a.add ? k_mxfp4_gemm<MA, NB, false, true> : k_mxfp4_gemm<MA, NB, false, false>);
  return hipGetLastError();
}

template <int MA, int NB>
hipError_t gemm_limits() {
  for (auto f : {k_mxfp4_gemm<MA, NB, false, false>, k_mxfp4_gemm<MA, NB, false, true>, k_mxfp4_gemm<MA, NB, true, false>,
                 k_mxfp4_gemm<MA, NB, true, true>}) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(f), hipFuncAttributeMaxDynamicSharedMemorySize,
                                             gemm_lds<MA, NB>());
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

constexpr int32_t kMaxDim = 1 << 20;

bool linear_shape_ok(int32_t T, int32_t N, int32_t K) { return T >= 0 && N > 0 && K > 0; }

bool linear_range_ok(int32_t T, int32_t N, int32_t K) {
  return T <= DAMOE_MAX_T && N <= kMaxDim && K <= kMaxDim && K % 32 == 0 &&
         tiles_of(T, 32) * tiles_of(K, kTileCols) * kTileBytes < (int64_t)1 << 31 &&
         tiles_of(N, 32) * tiles_of(K, kTileCols) * kTileBytes < (int64_t)1 << 31;
}

size_t x_tiles_bytes(int32_t T, int32_t K) {
  return (size_t)tiles_of(T, kTileRows) * tiles_of(K, kTileCols) * kTileBytes;
}

}  // namespace

hipError_t mxfp4_set_lds_limits() {
  for (const hipError_t e : {gemm_limits<1, 2>(), gemm_limits<1, 3>(), gemm_limits<2, 4>(), gemm_limits<2, 8>()})
    if (e != hipSuccess) return e;
  return hipSuccess;
}

}  // namespace damoe

using namespace damoe;

extern "C" {

size_t damoe_mxfp4_linear_workspace_size(int32_t T_max, int32_t N, int32_t K) {
  if (!linear_shape_ok(T_max, N, K) || !linear_range_ok(T_max, N, K)) return 0;
  return std::max<size_t>(256, (x_tiles_bytes(T_max, K) + 255) / 256 * 256);
}

damoe_status damoe_mxfp4_linear(const void* x, int32_t xdtype, int64_t ldx, int32_t T, int32_t K, const uint8_t* w,
                                int32_t N, const void* add, int64_t ld_add, void* y, int32_t ydtype, int64_t ldy,
                                void* ws, size_t ws_bytes, hipStream_t stream) {
  if (!linear_shape_ok(T, N, K)) return DAMOE_ERR_INVALID_ARG;
  if (!linear_range_ok(T, N, K)) return DAMOE_ERR_UNSUPPORTED;
  if ((xdtype != DAMOE_BF16 && xdtype != DAMOE_F32) || (ydtype != DAMOE_BF16 && ydtype != DAMOE_F32))
    return DAMOE_ERR_UNSUPPORTED;
  if (ldx < K || ldy < N || (add && ld_add < N)) return DAMOE_ERR_INVALID_ARG;
  if (T == 0) return DAMOE_OK;
  if (!x || !w || !y || !ws) return DAMOE_ERR_INVALID_ARG;
  const uintptr_t xs = xdtype == DAMOE_BF16 ? 2 : 4, ys = ydtype == DAMOE_BF16 ? 2 : 4;
  if (reinterpret_cast<uintptr_t>(x) % xs || reinterpret_cast<uintptr_t>(y) % ys || reinterpret_cast<uintptr_t>(add) % ys ||
      reinterpret_cast<uintptr_t>(w) % 16 || reinterpret_cast<uintptr_t>(ws) % 16)
    return DAMOE_ERR_INVALID_ARG;
  if (ws_bytes < x_tiles_bytes(T, K)) return DAMOE_ERR_WORKSPACE;
  uint8_t* xt = static_cast<uint8_t*>(ws);
  const bool x_bf = xdtype == DAMOE_BF16;
  const auto rows_ok = [&](const void* p, int64_t ld) {
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld * (int64_t)ys % 16 == 0 && ld * (int64_t)ys * 32 < (int64_t)1 << 31;
  };
  const bool vec = N % 8 == 0 && rows_ok(y, ldy) && (!add || rows_ok(add, ld_add));
  const LinearArgs a{w, xt, add, y, ld_add, ldy, T, N, (int32_t)tiles_of(K, kTileCols), ydtype == DAMOE_BF16, vec, 0};
  // Up to four tokens are quantised where they are used, which saves a launch of 2.9 us, unless the workgroups of a CU
  // (16 rows each, 256 CUs) go over so many tiles that doing it in each of them costs more.  T = 1, quantised in the kernel
  // / before it: 4096 x 7168 5.8 / 3.6 + 2.9 us, 7168 x 2048 4.6 / 3.2 + 2.9, 8192 x 8192 11.5 / 6.9 + 2.9; from T = 8 on the
  // reads of x cost more (4096 x 7168 7.5).
  const bool fused = T <= 4 && tiles_of(K, kTileCols) * tiles_of(N, 16 * 256) <= 36 &&
                     reinterpret_cast<uintptr_t>(x) % 16 == 0 && ldx * (int64_t)xs % 16 == 0;
  if (!fused && launch_quantise_tiles(x, x_bf, T, K, ldx, xt, stream) != hipSuccess) return DAMOE_ERR_HIP;
  int cus = 0;
  if (T > 32) {
    const damoe_status st = device_cus(&cus);
    if (st != DAMOE_OK) return st;
  }
  const RowsArgs r{a, x, ldx, K};
  const auto rows = [&](void (*f)(RowsArgs), int mr, int nt) {
    hipLaunchKernelGGL(f, dim3((unsigned)tiles_of(N, 16 * mr), (unsigned)tiles_of(T, 16 * nt)), dim3(kRowsThreads), 0, stream, r);
    return hipGetLastError();
  };
  hipError_t e;
  if (fused) e = rows(x_bf ? k_mxfp4_rows<1, 1, 1> : k_mxfp4_rows<1, 1, 2>, 1, 1);
  else if (T <= 16) e = rows(k_mxfp4_rows<1, 1, 0>, 1, 1);
  else if (T <= 32) e = rows(k_mxfp4_rows<1, 2, 0>, 1, 2);
  else switch (path_of(T, N, K, vec, cus)) {
    case kRows: e = rows(k_mxfp4_rows<2, 4, 0>, 2, 4); break;
    case kGemm12: e = launch_gemm<1, 2>(a, cus, stream); break;
    case kGemm13: e = launch_gemm<1, 3>(a, cus, stream); break;
    case kGemm24: e = launch_gemm<2, 4>(a, cus, stream); break;
    default: e = launch_gemm<2, 8>(a, cus, stream);
  }
  return e == hipSuccess ? DAMOE_OK : DAMOE_ERR_HIP;
}

}  // extern "C"
