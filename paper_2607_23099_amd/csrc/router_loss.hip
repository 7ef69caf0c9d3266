// Loss of a routed batch and its gradient: the balance loss per sequence, the z-loss, the counts and mean
// probabilities per expert, and the gradient of these and of the gates with respect to the logits.
//
// With p_te the score of expert e for token t (softmax, or sigmoid over its row's sum), c_se and n_s the
// assignments and valid tokens of sequence s, f_se = E c_se / (k n_s):
//   balance = 1/S' sum_s 1/n_s sum_{t in s} sum_e f_se p_te,   z = 1/N sum_t lse_t^2
// f holds counts, which have no gradient, so with g_t = alpha / (S' n_s)
//   d balance / d l_te = g_t p_te (f_se - sum_j f_sj p_tj)   (sigmoid: times 1 - sigmoid(l_te))
//   d z / d l_te       = 2 / N lse_t softmax(l_t)_e
//
// Both directions read each row of logits once, a wave a row, kept in registers: the row's maximum and sums
// are wave reductions.  Memory bound at many tokens (the logits, and the gradient on the way back), latency
// bound at few.
//
// Forward: a block (of one wave, where sequences are short) takes a chunk of tokens and, for each sequence that it
// meets, writes one slot of partial sums (probabilities and counts by expert, z, tokens).  Block b's slot of sequence s is
// b + s: the slots of a walk over the tokens, distinct while offsets do not decrease.  The next launch adds the slots of
// each sequence, 32 experts a block, in a fixed order, and a third one adds the sequences (the last block of the second
// could, found by an atomic count, which takes as long as the launch).  One block adds the slots of a single sequence where
// they are few, and a batch that fits one block takes one launch.
#include "common.h"

namespace damoe {
namespace {

constexpr int kLossThreads = 512;
constexpr int kOneThreads = 1024;  // of the block that takes a small batch alone
constexpr int kMaxChunks = 512;    // blocks of the forward pass: two per compute unit
constexpr int kMinChunk = 4 * kLossThreads / kWave;
constexpr int kGroup = 32;         // experts of a block that adds slots, where there are few sequences
constexpr int kFewSeqs = 16;       // below this many sequences their blocks have 1024 threads, else 256
constexpr int kManySeqs = 128;     // from here on a block adds all experts of a sequence
constexpr int kGradThreads = 256;
constexpr int kGradWaves = kGradThreads / kWave;

// Up to kWaveTokens tokens, in sequences of up to kWaveMean in the mean, blocks are single waves of up to four tokens: a
// block of eight goes over its sequences in turn, 1.7 us each.  Waves / blocks of eight, all launches, 256 experts: 40 tokens
// in 28 sequences 10.9 / 56 us, 512 in 512 12.5 / 77, 512 in 8 12.1 / 12.9, 4096 in 64 12.8 / 12.8, one of 3969 tokens and
// 127 of one 50 / 80; the slots of long sequences cost more (4096 in 2 15.6 / 13.1).  The bound on the tokens is right for
// means of 32 and more only: 16384 tokens in sequences of 1, 2, 4, 8, 32, 64 take 66 / 125, 40 / 69, 25 / 42, 21.5 / 25.6,
// 18.8 / 14.2, 16.9 / 13.8 us, 65536 take 252 / 485, 122 / 241, 69 / 131, 49 / 74, 34 / 31, 33 / 27.
constexpr int32_t kWaveTokens = 4096, kWaveMean = 64;

bool by_waves(int32_t T, int32_t S) { return T <= kWaveTokens && T <= (int64_t)S * kWaveMean; }

// Tokens of a block of the forward pass.
int32_t chunk_tokens(int32_t T, int32_t S) {
  if (by_waves(T, S)) return T < 2 * (int64_t)S ? 1 : T < 4 * (int64_t)S ? 2 : 4;
  const int32_t c = (T + kMaxChunks - 1) / kMaxChunks;
  return std::max((c + kMinChunk - 1) / kMinChunk * kMinChunk, kMinChunk);
}

struct LossArgs {
  const void* logits;
  int64_t ld;
  const int32_t* ids;
  const uint8_t* mask;
  const int32_t* off;  // NULL: one sequence of T tokens
  int32_t T, E, k, S;
  int32_t chunk, nb;   // tokens of a block, blocks
  int32_t* err;
  float2* part;        // [nb + S][Ep]: sum of p, bits of the count
  int32_t Ep;          // E rounded up to kGroup
  int32_t width;       // experts of a block that adds slots
  float2* part_zn;     // [nb + S]: sum of lse^2, bits of the valid tokens
  double* seq_l;       // [S][Ep / width]: sum over the group's experts of f P
  float* seq_z;        // [S]: sum of lse^2
  float alpha, z_coef;
  float* loss;
  int32_t* counts;
  float* probs;
  int32_t* tokens;
};

struct GradArgs {
  const void* logits;
  int64_t ld;
  const int32_t* ids;
  const float* w;
  const float* dw;
  const uint8_t* mask;
  const int32_t* off;
  const int32_t* counts;
  const int32_t* tokens;
  int32_t T, E, k, S;
  int32_t run;  // rows of a wave
  float alpha, z_coef;
  const float* dloss;
  void* dlogits;
  int64_t ldd;
};

// ---------------------------------------------------------------- wave reductions (every lane gets the result)

template <int CTRL>
__device__ __forceinline__ float dppf(float x) {
  return __uint_as_float(__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), CTRL, 0xF, 0xF, false));
}

template <class Op>
__device__ __forceinline__ float wave_all(float x, Op op) {
  x = op(x, dppf<0xB1>(x));   // quad_perm 1 0 3 2
  x = op(x, dppf<0x4E>(x));   // quad_perm 2 3 0 1
  x = op(x, dppf<0x141>(x));  // row_half_mirror
  x = op(x, dppf<0x140>(x));  // row_mirror
  const uint32_t a = __float_as_uint(x);
  const auto r = __builtin_amdgcn_permlane16_swap(a, a, false, false);
  x = op(__uint_as_float(r[0]), __uint_as_float(r[1]));
  const uint32_t b = __float_as_uint(x);
  const auto q = __builtin_amdgcn_permlane32_swap(b, b, false, false);
  return op(__uint_as_float(q[0]), __uint_as_float(q[1]));
}

__device__ __forceinline__ float wave_max(float x) {
  return wave_all(x, [](float a, float b) { return fmaxf(a, b); });
}
__device__ __forceinline__ float wave_sum(float x) {
  return wave_all(x, [](float a, float b) { return a + b; });
}

constexpr float kLog2e = 1.44269504088896f, kLn2 = 0.693147180559945f;

__device__ __forceinline__ float exp_f(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }

// LDS of a wave's own: what other lanes of the wave wrote before is read after it.
__device__ __forceinline__ void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// ---------------------------------------------------------------- rows

// A lane's V * NC values of a row: columns 64 V c + V lane + i.  V = 4 and 2 want rows of whole aligned fours or twos.
template <int V, int NC, bool BF>
struct Row {
  typedef float Vec __attribute__((ext_vector_type(V)));
  float v[V * NC];

  static __device__ __forceinline__ int col(int c, int lane) { return (c * kWave + lane) * V; }

  __device__ __forceinline__ void load(const void* base, int64_t row, int64_t ld, int E, int lane, float fill) {
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int e = col(c, lane);
      if (e < E) {
        if constexpr (BF) {
          const uint16_t* p = static_cast<const uint16_t*>(base) + row * ld + e;
          if constexpr (V == 1) {
            v[c] = bf16_to_f32(*p);
          } else {
            uint32_t q[V / 2];
            if constexpr (V == 4) {
              const uint2 u = *reinterpret_cast<const uint2*>(p);
              q[0] = u.x, q[1] = u.y;
            } else {
              q[0] = *reinterpret_cast<const uint32_t*>(p);
            }
#pragma unroll
            for (int i = 0; i < V; ++i) v[V * c + i] = __uint_as_float(i & 1 ? q[i / 2] & 0xFFFF0000u : q[i / 2] << 16);
          }
        } else {
          const Vec q = *reinterpret_cast<const Vec*>(static_cast<const float*>(base) + row * ld + e);
#pragma unroll
          for (int i = 0; i < V; ++i) v[V * c + i] = q[i];
        }
      } else {
#pragma unroll
        for (int i = 0; i < V; ++i) v[V * c + i] = fill;
      }
    }
  }

  __device__ __forceinline__ void fill(float x) {
#pragma unroll
    for (int i = 0; i < V * NC; ++i) v[i] = x;
  }

  // With the nontemporal hint, which is as fast or faster at every size (fp32, 256 experts: 16384 tokens 9.1 against
  // 11.7 us, 131072 52 against 59; three batches of 65536 x 384 in turn 46 against 53).
  __device__ __forceinline__ void store(void* base, int64_t row, int64_t ld, int E, int lane) const {
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int e = col(c, lane);
      if (e >= E) continue;
      if constexpr (BF) {
        uint16_t* p = static_cast<uint16_t*>(base) + row * ld + e;
        if constexpr (V == 1) {
          *p = bf16_of(v[c]);
        } else {
          uint32_t q[V / 2];
#pragma unroll
          for (int i = 0; i < V / 2; ++i) q[i] = (uint32_t)bf16_of(v[V * c + 2 * i]) | (uint32_t)bf16_of(v[V * c + 2 * i + 1]) << 16;
          typedef uint32_t Words __attribute__((ext_vector_type(V / 2)));
          Words d;
#pragma unroll
          for (int i = 0; i < V / 2; ++i) d[i] = q[i];
          __builtin_nontemporal_store(d, reinterpret_cast<Words*>(p));
        }
      } else {
        Vec q;
#pragma unroll
        for (int i = 0; i < V; ++i) q[i] = v[V * c + i];
        __builtin_nontemporal_store(q, reinterpret_cast<Vec*>(static_cast<float*>(base) + row * ld + e));
      }
    }
  }

  // One rounding to bf16, nearest even; a NaN stays one.
  static __device__ __forceinline__ uint16_t bf16_of(float f) { return __builtin_bit_cast(uint16_t, (__bf16)f); }

  __device__ __forceinline__ float max() const {
    float m = v[0];
#pragma unroll
    for (int i = 1; i < V * NC; ++i) m = fmaxf(m, v[i]);
    return m;
  }
};

// exp(l - m), m the row's maximum.  (l log2 e - m log2 e in one fma would be an instruction less, but is off by the
// rounding of m log2 e, which is anything at the type's largest magnitudes.)
__device__ __forceinline__ float shifted_exp(float l, float m) { return exp_f(l - m); }

__device__ __forceinline__ float lse_of(float m, float sum) { return m + __builtin_amdgcn_logf(sum) * kLn2; }

// Sigmoids of a row with maximum m: with e = exp(-|l|) and r = 1 / (1 + e), sigmoid(l) is r or e r and 1 - sigmoid(l)
// the other.  Where the whole row is negative, sigmoid(l) exp(-m) = exp(l - m) r takes its place: p is the same, and rows
// of very negative logits do not underflow.  ex: shifted_exp of l.
__device__ __forceinline__ float2 sigmoids(float l, float ex, float m) {
  const float e = exp_f(-fabsf(l)), r = __builtin_amdgcn_rcpf(1.f + e);
  const float big = r, small = e * r;
  return make_float2(m < 0.f ? ex * r : l >= 0.f ? big : small, l >= 0.f ? small : big);
}

// What a row's sigmoids are divided by: their sum, or NaN where the sum of the shifted exponentials is, since the sigmoid of
// +inf is a finite 1 (and a term of the gradient that a coefficient of 0 multiplies would be NaN in that column alone).
__device__ __forceinline__ float norm_of(float sigmoid_sum, float exp_sum) { return exp_sum == exp_sum ? sigmoid_sum : exp_sum; }

__device__ __forceinline__ int offset_at(const int32_t* off, int32_t s, int32_t T) {
  const int o = off ? off[s] : (s == 0 ? 0 : T);
  return min(max(o, 0), T);
}

// The first sequence from s on that ends behind token t, S if there is none; the same in every lane.  64 ends at a time,
// then, past a long run of empty sequences or from a start far ahead, 64 equal steps of what is left.  The result lies in
// [s, S] whatever the offsets hold.
__device__ __forceinline__ int seq_behind(const int32_t* off, int s, int S, int T, int t, int lane) {
  if (!off) return s == 0 && t < T ? 0 : S;
  int lo = s, hi = S;  // the result lies in [lo, hi]
  for (bool first = true;; first = false) {
    const uint64_t behind = __ballot(lo + lane >= hi || offset_at(off, lo + lane + 1, T) > t);
    if (behind || hi - lo <= kWave) return __builtin_amdgcn_readfirstlane(behind ? min(lo + (int)__builtin_ctzll(behind), hi) : hi);
    if (first) {
      lo += kWave;
    }
    while (hi - lo > kWave) {
      const int step = (hi - lo + kWave - 1) / kWave, i = lo + (lane + 1) * step - 1;
      const int n = __popcll(__ballot(i < hi && offset_at(off, i + 1, T) <= t));  // steps that end at or before t
      lo = min(lo + n * step, hi);
      hi = min(lo + step, hi);
    }
  }
}

// ---------------------------------------------------------------- forward

__device__ __forceinline__ void write_loss(const LossArgs& a, double balance, double z, int n_seq, int n_tok) {
  const float b = n_seq > 0 ? (float)(balance / n_seq) : 0.f;
  const float zz = n_tok > 0 ? (float)(z / n_tok) : 0.f;
  a.loss[0] = (a.alpha != 0.f ? a.alpha * b : 0.f) + (a.z_coef != 0.f ? a.z_coef * zz : 0.f);
  a.loss[1] = b;
  a.loss[2] = zz;
  a.tokens[a.S] = n_seq;
  a.tokens[a.S + 1] = n_tok;
}

constexpr int kAloneThreads = 1024, kTotalThreads = 256;

// Rows of sums that a block's waves leave in LDS.
constexpr int loss_rows(int threads) { return threads > kWave ? threads / kWave / 2 : 1; }

template <int THREADS>
struct SeqSmem {
  float4 p[THREADS];
  double l[THREADS / kWave];
  float z;
  int32_t n;
};

// Sequence s, `width` experts (an even number) from e0 on: its slots added in order, f, P and their product's sum, which
// thread 0 returns with z and n.  Thread lanes r + c adds every split-th slot from r on, two experts at a time (more
// than 512 experts: a block of 256 threads goes over them in turn).
template <int THREADS>
__device__ __forceinline__ double add_slots(const LossArgs& a, SeqSmem<THREADS>& sm, int s, int e0, int width) {
  const int tid = threadIdx.x, lanes = min(width / 2, THREADS), split = THREADS / lanes;
  const int r = tid / lanes, c = tid - r * lanes;
  const int o0 = offset_at(a.off, s, a.T), o1 = offset_at(a.off, s + 1, a.T);
  const int b0 = o0 / a.chunk;
  const int nslot = o1 > o0 ? min((o1 - 1) / a.chunk, a.nb - 1) - b0 + 1 : 0;
  const int64_t base = (int64_t)b0 + s;
  if (tid < kWave) {  // tokens and z of the sequence
    float z = 0.f;
    int n = 0;
    for (int i = tid; i < nslot; i += kWave) {
      const float2 q = a.part_zn[base + i];
      z += q.x;
      n += __float_as_int(q.y);
    }
    z = wave_sum(z);
    for (int d = 1; d < kWave; d <<= 1) n += __shfl_xor(n, d);
    if (tid == 0) {
      sm.z = z;
      sm.n = n;
    }
  }
  double l = 0.0;
  for (int w0 = 0; w0 < width; w0 += 2 * lanes) {
    float p0 = 0.f, p1 = 0.f;
    int c0 = 0, c1 = 0;
    const bool in = r < split && w0 + 2 * c < width;
    if (in) {
      const float4* q = reinterpret_cast<const float4*>(a.part + base * a.Ep + e0 + w0) + c;
#pragma unroll 8
      for (int i = r; i < nslot; i += split) {
        const float4 v = q[(int64_t)i * (a.Ep / 2)];
        p0 += v.x, p1 += v.z;
        c0 += __float_as_int(v.y), c1 += __float_as_int(v.w);
      }
    }
    sm.p[tid] = make_float4(p0, __int_as_float(c0), p1, __int_as_float(c1));
    __syncthreads();
    for (int m = split, h; m > 1; m = h) {  // the upper half's sums into the lower half's
      h = (m + 1) / 2;
      if (r < m - h) {
        float4 v = sm.p[tid];
        const float4 o = sm.p[tid + h * lanes];
        v.x += o.x, v.z += o.z;
        v.y = __int_as_float(__float_as_int(v.y) + __float_as_int(o.y));
        v.w = __int_as_float(__float_as_int(v.w) + __float_as_int(o.w));
        sm.p[tid] = v;
      }
      __syncthreads();
    }
    const int n = sm.n;
    if (r == 0 && in) {
      const float4 v = sm.p[tid];
      const float p[2] = {v.x, v.z};
      const int cnt[2] = {__float_as_int(v.y), __float_as_int(v.w)};
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int e = e0 + w0 + 2 * c + i;
        if (e >= a.E) continue;
        const float P = n > 0 ? p[i] / (float)n : 0.f;
        a.counts[(int64_t)s * a.E + e] = cnt[i];
        if (a.probs) a.probs[(int64_t)s * a.E + e] = P;
        if (n > 0) l += (double)a.E * cnt[i] / ((double)a.k * n) * P;
      }
    }
    __syncthreads();
  }
  for (int d = 1; d < kWave; d <<= 1) l += __shfl_xor(l, d);
  if ((tid & 63) == 0) sm.l[tid >> 6] = l;
  __syncthreads();
  if (tid == 0)
    for (int i = 1; i < THREADS / kWave; ++i) l += sm.l[i];
  return l;
}

// A block for a group of experts of a sequence.
template <int THREADS>
__global__ void __launch_bounds__(THREADS) k_router_loss_seq(LossArgs a) {
  __shared__ SeqSmem<THREADS> sm;
  const int G = a.Ep / a.width, s = blockIdx.x / G, g = blockIdx.x % G;
  const double l = add_slots(a, sm, s, g * a.width, a.width);
  if (threadIdx.x == 0) {
    a.seq_l[(int64_t)s * G + g] = l;
    if (g == 0) {
      a.seq_z[s] = sm.z;
      a.tokens[s] = sm.n;
    }
  }
}

// One block for all of a single sequence.
__global__ void __launch_bounds__(kAloneThreads) k_router_loss_alone(LossArgs a) {
  __shared__ SeqSmem<kAloneThreads> sm;
  const double l = add_slots(a, sm, 0, 0, a.Ep);
  if (threadIdx.x == 0) {
    a.tokens[0] = sm.n;
    write_loss(a, l, sm.z, sm.n > 0, sm.n);
  }
}

// The sum over sequences, by one block in a fixed order (what a sequence without tokens left is 0).
__global__ void __launch_bounds__(kTotalThreads) k_router_loss_total(LossArgs a) {
  __shared__ double red[kTotalThreads / kWave][4];
  const int tid = threadIdx.x;
  const int64_t m = (int64_t)a.S * (a.Ep / a.width);
  double l = 0, z = 0;
  int seqs = 0, n = 0;
#pragma unroll 4
  for (int64_t i = tid; i < m; i += kTotalThreads) l += a.seq_l[i];
#pragma unroll 4
  for (int s = tid; s < a.S; s += kTotalThreads) {
    const int ns = a.tokens[s];
    z += a.seq_z[s];
    seqs += ns > 0;
    n += ns;
  }
  for (int d = 1; d < kWave; d <<= 1) {
    l += __shfl_xor(l, d);
    z += __shfl_xor(z, d);
    seqs += __shfl_xor(seqs, d);
    n += __shfl_xor(n, d);
  }
  if ((tid & 63) == 0) {
    double* const q = red[tid >> 6];
    q[0] = l, q[1] = z, q[2] = seqs, q[3] = n;
  }
  __syncthreads();
  if (tid == 0) {
    for (int i = 1; i < kTotalThreads / kWave; ++i) {
      l += red[i][0];
      z += red[i][1];
      seqs += (int)red[i][2];
      n += (int)red[i][3];
    }
    write_loss(a, l, z, seqs, n);
  }
}

// ONE (kOneThreads): the batch is one block's, which has every sequence's sums and finishes them.
template <int V, int NC, bool BF, bool SIG, int kThreads>
__global__ void __launch_bounds__(kThreads) k_router_loss(LossArgs a) {
  constexpr bool ONE = kThreads == kOneThreads;
  constexpr int kWaves = kThreads / kWave, kRed = loss_rows(kThreads);
  // Rows of logits a wave holds at a time.
  constexpr int kRows = V * NC <= 4 ? 4 : V * NC <= 8 ? 2 : 1;
  extern __shared__ __attribute__((aligned(16))) float loss_smem[];
  float* const red = loss_smem;                                      // [kRed][E]
  int32_t* const hist = reinterpret_cast<int32_t*>(red + kRed * a.E);  // [E]
  __shared__ float z_red[kWaves];
  __shared__ int32_t n_red[kWaves];
  __shared__ double l_red[kWaves];
  double l_sum = 0.0, z_sum = 0.0;  // ONE, thread 0: over the sequences so far
  int seqs = 0, n_sum = 0;
  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int E = a.E, k = a.k;
  const int t0 = blockIdx.x * a.chunk, t1 = min(t0 + a.chunk, a.T);
  const float kNegInf = -__builtin_huge_valf();

  for (int e = tid; e < E; e += kThreads) hist[e] = 0;
  __syncthreads();
  // The sequences with tokens in the block (ONE: all, as those without have their zeros to write).
  int t_next = t0;
  for (int s = ONE ? 0 : seq_behind(a.off, 0, a.S, a.T, t0, lane); s < a.S;
       s = ONE ? s + 1 : seq_behind(a.off, s + 1, a.S, a.T, t_next, lane)) {
    const int b0 = offset_at(a.off, s, a.T), b1 = offset_at(a.off, s + 1, a.T);
    if (!ONE && b0 >= t1) break;
    const int lo = max(t0, b0), hi = min(t1, b1);
    if (!ONE && lo >= hi) continue;  // decreasing offsets
    t_next = hi;
    float acc[V * NC];
#pragma unroll
    for (int i = 0; i < V * NC; ++i) acc[i] = 0.f;
    float zsum = 0.f;
    int n = 0;
    // A wave's next rows are loaded before it works on the present ones.
    Row<V, NC, BF> next[kRows];
    uint32_t next_ok = 0;
    int next_id = -1;
    auto fetch = [&](int t) __attribute__((always_inline)) {
      next_ok = 0;
      next_id = -1;
      if (t >= hi) return;
      // The slots of the rows' tokens, one a lane (16 a row), and from them which tokens are valid.
      const int u = lane >> 4, j = lane & 15;
      const bool in = u < kRows && t + u < hi && (!a.mask || a.mask[t + u] != 0);
      if (in && j < k) next_id = a.ids[(int64_t)(t + u) * k + j];
      const uint64_t ok = __ballot(in);
#pragma unroll
      for (int q = 0; q < kRows; ++q) {
        if ((ok >> (16 * q)) & 1) {
          next_ok |= 1u << q;
          next[q].load(a.logits, t + q, a.ld, E, lane, kNegInf);
        } else {
          next[q].fill(0.f);
        }
      }
    };
    fetch(lo + w * kRows);
    for (int t = lo + w * kRows; t < hi; t += kWaves * kRows) {
      Row<V, NC, BF> r[kRows];
#pragma unroll
      for (int u = 0; u < kRows; ++u) r[u] = next[u];
      const uint32_t ok = next_ok;
      const int id = next_id;
      fetch(t + kWaves * kRows);
      if (id >= E) atomicOr(a.err, DAMOE_DEVERR_EXPERT_ID);
      else if (id >= 0) atomicAdd(&hist[id], 1);
      float m[kRows], sum[kRows], inv[kRows];
#pragma unroll
      for (int u = 0; u < kRows; ++u) m[u] = wave_max(r[u].max());
#pragma unroll
      for (int u = 0; u < kRows; ++u) {
        const float mm = m[u] == kNegInf ? 0.f : m[u];  // a row of -inf alone: every term 0
        sum[u] = 0.f;
        float sg = 0.f;
#pragma unroll
        for (int i = 0; i < V * NC; ++i) {
          const float l = r[u].v[i], x = shifted_exp(l, mm);
          sum[u] += x;
          if constexpr (SIG) {
            r[u].v[i] = sigmoids(l, x, mm).x;
            sg += r[u].v[i];
          } else {
            r[u].v[i] = x;
          }
        }
        inv[u] = sg;
      }
#pragma unroll
      for (int u = 0; u < kRows; ++u) {
        sum[u] = wave_sum(sum[u]);
        inv[u] = SIG ? norm_of(wave_sum(inv[u]), sum[u]) : sum[u];
      }
#pragma unroll
      for (int u = 0; u < kRows; ++u) {
        const bool live = ((ok >> u) & 1) && sum[u] != 0.f;  // 0: nothing but -inf (a NaN makes it NaN)
        n += (ok >> u) & 1;
        const float lse = lse_of(m[u], sum[u]), f = 1.f / inv[u];
        if (!live) continue;
        zsum += lse * lse;
#pragma unroll
        for (int i = 0; i < V * NC; ++i) acc[i] += r[u].v[i] * f;
      }
    }
    // The waves' sums by expert: the upper half's go to LDS and into the lower half's, whose go there next.
    auto put = [&](int row, bool add) __attribute__((always_inline)) {
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const int e = Row<V, NC, BF>::col(c, lane) + i;
          if (e < E) red[row * E + e] = add ? red[row * E + e] + acc[V * c + i] : acc[V * c + i];
        }
    };
    if (w >= kWaves / 2) put(w - kWaves / 2, false);
    if (lane == 0) {
      z_red[w] = zsum;
      n_red[w] = n;
    }
    __syncthreads();
    if (w < kWaves / 2) put(w, true);
    __syncthreads();
    float z = 0.f;
    int nn = 0;
    for (int i = 0; i < kWaves; ++i) {
      z += z_red[i];
      nn += n_red[i];
    }
    const int64_t slot = (int64_t)blockIdx.x + s;
    double l = 0.0;
    for (int e = tid; e < (ONE ? E : a.Ep); e += kThreads) {
      float p = 0.f;
      int cnt = 0;
      if (e < E) {
#pragma unroll
        for (int i = 0; i < kRed; ++i) p += red[i * E + e];
        cnt = hist[e];
        hist[e] = 0;
      }
      if constexpr (ONE) {
        const float P = nn > 0 ? p / (float)nn : 0.f;
        a.counts[(int64_t)s * E + e] = cnt;
        if (a.probs) a.probs[(int64_t)s * E + e] = P;
        if (nn > 0) l += (double)E * cnt / ((double)k * nn) * P;
      } else {
        a.part[slot * a.Ep + e] = make_float2(p, __int_as_float(cnt));
      }
    }
    if constexpr (ONE) {
      for (int d = 1; d < kWave; d <<= 1) l += __shfl_xor(l, d);
      if (lane == 0) l_red[w] = l;
    } else if (tid == 0) {
      a.part_zn[slot] = make_float2(z, __int_as_float(nn));
    }
    __syncthreads();
    if (ONE && tid == 0) {
      a.tokens[s] = nn;
      if (nn > 0) {
        for (int i = 0; i < kWaves; ++i) l_sum += l_red[i];
        z_sum += z;
        ++seqs;
        n_sum += nn;
      }
    }
  }
  if (ONE && tid == 0) write_loss(a, l_sum, z_sum, seqs, n_sum);
}

// ---------------------------------------------------------------- gradient

// Sum over the 16 lanes of a DPP row, in each of them.
__device__ __forceinline__ float row16_sum(float x) {
  x += dppf<0xB1>(x);
  x += dppf<0x4E>(x);
  x += dppf<0x141>(x);
  return x + dppf<0x140>(x);
}

template <int V, int NC, bool BF, bool SIG>
struct Grad {
  static constexpr int kVals = V * NC;
  // Rows a wave works on together where they lie in one sequence: fewer for sigmoids, whose registers would leave three
  // waves a SIMD (65536 tokens, 384 experts: 47 us with two rows, 58 with four).
  static constexpr int kRows = kVals <= 8 ? (SIG ? 2 : 4) : kVals <= 12 ? 2 : 1;
  const GradArgs& a;
  float* gate;  // LDS of the wave, [kRows][E], zero between rows
  int lane;
  float zc, bal;
  float f[kVals];

  // Rows t .. t + U - 1, all in the sequence of f and bal; those that are not valid get 0.
  template <int U>
  __device__ __forceinline__ void rows(int t) const {
    const int E = a.E, k = a.k;
    const float kNegInf = -__builtin_huge_valf();
    const int u16 = lane >> 4, j = lane & 15;
    const bool in = u16 < U && (!a.mask || a.mask[t + (u16 < U ? u16 : 0)] != 0);
    const uint64_t ok = __ballot(in);
    Row<V, NC, BF> r[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if ((ok >> (16 * u)) & 1) r[u].load(a.logits, t + u, a.ld, E, lane, kNegInf);
      else r[u].fill(0.f);
    }
    if (a.w) {
      // dw_j -> w_j (dw_j - sum_i w_i dw_i), added to the expert's column (twice for an id held twice).
      int id = -1;
      float wj = 0.f, dj = 0.f;
      if (in && j < k) {
        const int64_t i = (int64_t)(t + u16) * k + j;
        id = a.ids[i];
        if (id >= 0 && id < E) {
          wj = a.w[i];
          dj = a.dw[i];
        }
      }
      const float dot = row16_sum(wj * dj);
      wave_fence();
      if (id >= 0 && id < E) atomicAdd(&gate[u16 * E + id], wj * (dj - dot));
      wave_fence();
    }
    float m[U], sum[U], ps[U], fp[U], ex[U][kVals], p[SIG ? U : 1][kVals];
#pragma unroll
    for (int u = 0; u < U; ++u) m[u] = wave_max(r[u].max());
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const float mm = m[u] == kNegInf ? 0.f : m[u];
      sum[u] = ps[u] = fp[u] = 0.f;
#pragma unroll
      for (int i = 0; i < kVals; ++i) {
        ex[u][i] = shifted_exp(r[u].v[i], mm);
        sum[u] += ex[u][i];
        if constexpr (SIG) {
          const float2 sg = sigmoids(r[u].v[i], ex[u][i], mm);
          p[u][i] = sg.x;
          r[u].v[i] = sg.y;  // 1 - sigmoid
          ps[u] += p[u][i];
          fp[u] += p[u][i] * f[i];
        } else {
          fp[u] += ex[u][i] * f[i];
        }
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      sum[u] = wave_sum(sum[u]);
      ps[u] = SIG ? norm_of(wave_sum(ps[u]), sum[u]) : sum[u];
      fp[u] = wave_sum(fp[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const bool live = sum[u] != 0.f;
      const float ip = live ? 1.f / ps[u] : 0.f, dot = fp[u] * ip, b = bal * ip;
      const float zt = live && a.z_coef != 0.f ? zc * lse_of(m[u], sum[u]) / sum[u] : 0.f;
#pragma unroll
      for (int i = 0; i < kVals; ++i) {
        float d;
        if constexpr (SIG) d = b * p[u][i] * (f[i] - dot) * r[u].v[i] + zt * ex[u][i];
        else d = (b * (f[i] - dot) + zt) * ex[u][i];
        r[u].v[i] = d;
      }
      if (a.w) {
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          const int e = Row<V, NC, BF>::col(c, lane);
          if (e >= E) continue;
          typedef typename Row<V, NC, BF>::Vec Vec;
          Vec* const q = reinterpret_cast<Vec*>(gate + u * E + e);
          const Vec x = *q;
          *q = Vec(0.f);
#pragma unroll
          for (int i = 0; i < V; ++i) r[u].v[V * c + i] += x[i];
        }
      }
      if (!((ok >> (16 * u)) & 1)) r[u].fill(0.f);
      r[u].store(a.dlogits, t + u, a.ldd, E, lane);
    }
  }
};

template <int V, int NC, bool BF, bool SIG>
__global__ void __launch_bounds__(kGradThreads) k_router_loss_grad(GradArgs a) {
  using G = Grad<V, NC, BF, SIG>;
  extern __shared__ __attribute__((aligned(16))) float grad_smem[];  // [waves][kRows][E]: the gates' gradient of rows
  const int lane = threadIdx.x & 63;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int E = a.E;
  const int t0 = (blockIdx.x * kGradWaves + w) * a.run, t1 = min(t0 + a.run, a.T);
  if (t0 >= t1) return;
  G d{a, grad_smem + w * G::kRows * E, lane};
  if (a.w)
    for (int e = lane; e < G::kRows * E; e += kWave) d.gate[e] = 0.f;
  const float g = a.dloss ? *a.dloss : 1.f;
  const float n_seq = (float)a.tokens[a.S], n_tok = (float)a.tokens[a.S + 1];
  d.zc = a.z_coef != 0.f ? g * a.z_coef * 2.f / n_tok : 0.f;
  int s = -1, begin = 0, end = 0;  // the sequence that t is in or ahead of
  for (int t = t0; t < t1;) {
    if (s < a.S && (s < 0 || t >= end)) {
      s = seq_behind(a.off, s + 1, a.S, a.T, t, lane);
      begin = end = a.T;
      if (s < a.S) {
        begin = offset_at(a.off, s, a.T);
        end = offset_at(a.off, s + 1, a.T);
        const float n = (float)a.tokens[s];
        d.bal = a.alpha != 0.f ? g * a.alpha / (n_seq * n) : 0.f;
        const float fs = (float)E / ((float)a.k * n);
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int i = 0; i < V; ++i) {
            const int e = Row<V, NC, BF>::col(c, lane) + i;
            d.f[V * c + i] = e < E ? fs * (float)a.counts[(int64_t)s * E + e] : 0.f;
          }
      }
    }
    if (s >= a.S || t < begin) {  // in no sequence
      Row<V, NC, BF> r;
      r.fill(0.f);
      r.store(a.dlogits, t, a.ldd, E, lane);
      ++t;
    } else if (t + G::kRows <= min(t1, end)) {
      d.template rows<G::kRows>(t);
      t += G::kRows;
    } else {
      d.template rows<1>(t);
      ++t;
    }
  }
}

// ---------------------------------------------------------------- launches

// Columns a lane holds: fours where rows are whole aligned fours (twos where those leave no lane idle), else single
// ones; NC chunks of 64 V columns.
template <class F>
hipError_t by_columns(int32_t E, bool four, F f) {
  const auto go = [&](auto v, auto nc) { return f(v, nc); };
  using std::integral_constant;
  if (four) {
    const integral_constant<int, 4> v;
    if (E > 256 && E <= 384) return go(integral_constant<int, 2>{}, integral_constant<int, 3>{});
    return E <= 256   ? go(v, integral_constant<int, 1>{})
           : E <= 512 ? go(v, integral_constant<int, 2>{})
                      : go(v, integral_constant<int, 4>{});
  }
  const integral_constant<int, 1> v;
  return E <= 64    ? go(v, integral_constant<int, 1>{})
         : E <= 128 ? go(v, integral_constant<int, 2>{})
         : E <= 256 ? go(v, integral_constant<int, 4>{})
         : E <= 512 ? go(v, integral_constant<int, 8>{})
                    : go(v, integral_constant<int, 16>{});
}

// f of the logits' type and the score as integral constants.
template <class F>
hipError_t by_kind(int32_t dtype, int32_t score, F f) {
  using std::false_type;
  using std::true_type;
  const bool sig = score == DAMOE_SCORE_SIGMOID;
  if (dtype == DAMOE_BF16) return sig ? f(true_type{}, true_type{}) : f(true_type{}, false_type{});
  return sig ? f(false_type{}, true_type{}) : f(false_type{}, false_type{});
}

// Tokens and sequences that one block takes alone.
constexpr int32_t kOneTokens = 96, kOneSeqs = 2;
// Partial sums of a single sequence that one block adds.
constexpr size_t kAlonePartials = 65536;

size_t up256(size_t v) { return (v + 255) / 256 * 256; }

// Workspace: the control word, then the partial sums of nb + S slots, then the sequences'.
struct LossWs {
  size_t part, zn, seq_l, seq_z, total;
};

int32_t padded(int32_t E) { return (E + kGroup - 1) / kGroup * kGroup; }

LossWs loss_ws(int32_t T, int32_t E, int32_t S) {
  const int32_t chunk = chunk_tokens(T, S), Ep = padded(E);
  const size_t slots = (size_t)((T + chunk - 1) / chunk) + S;
  LossWs o;
  o.part = 256;
  o.zn = o.part + up256(slots * Ep * 8);
  o.seq_l = o.zn + up256(slots * 8);
  o.seq_z = o.seq_l + up256((size_t)S * (Ep / kGroup) * 8);
  o.total = o.seq_z + up256((size_t)S * 4);
  return o;
}

bool loss_shape_ok(int32_t T, int32_t E, int32_t k, int32_t S) {
  return T >= 0 && T <= DAMOE_MAX_T && E >= 1 && E <= DAMOE_MAX_E && k >= 1 && k <= DAMOE_MAX_K && k <= E && S >= 1 &&
         S <= DAMOE_MAX_T;
}

// Whether every row starts at whole aligned fours.
bool fours(const void* p, int64_t ld, int32_t E, int32_t dtype) {
  const size_t b = dtype == DAMOE_BF16 ? 8 : 16;
  return E % 4 == 0 && ld % 4 == 0 && reinterpret_cast<uintptr_t>(p) % b == 0;
}

}  // namespace
}  // namespace damoe

using namespace damoe;

extern "C" {

size_t damoe_router_loss_workspace_size(int32_t T_max, int32_t E, int32_t S) {
  if (!loss_shape_ok(T_max, E, 1, S)) return 0;
  // The chunk grows with T in steps, so a smaller T may take more blocks: never over kMaxChunks, or those of the last T
  // that waves take one, two or four tokens at a time.
  const size_t at = loss_ws(T_max, E, S).total;
  const int32_t full = std::min<int32_t>(T_max, kMaxChunks * kMinChunk);
  size_t most = std::max(at, loss_ws(full, E, S).total);
  for (const int64_t t : {2 * (int64_t)S - 1, 4 * (int64_t)S - 1, (int64_t)S * kWaveMean})
    most = std::max(most, loss_ws((int32_t)std::min<int64_t>({T_max, kWaveTokens, t}), E, S).total);
  return most;
}

damoe_status damoe_router_loss(const void* logits, int32_t dtype, int64_t ld, const int32_t* topk_ids,
                               const uint8_t* mask, const int32_t* seq_offsets, int32_t T, int32_t E, int32_t k,
                               int32_t S, int32_t score, float alpha, float z_coef, float* loss, int32_t* counts,
                               float* probs, int32_t* tokens, void* ws, size_t ws_bytes, hipStream_t stream) {
  if (!loss_shape_ok(T, E, k, S) || ld < E || (!seq_offsets && S != 1)) return DAMOE_ERR_INVALID_ARG;
  if (score != DAMOE_SCORE_SOFTMAX && score != DAMOE_SCORE_SIGMOID) return DAMOE_ERR_INVALID_ARG;
  if (dtype != DAMOE_BF16 && dtype != DAMOE_F32) return DAMOE_ERR_UNSUPPORTED;
  if (!loss || !counts || !tokens || !ws || (T > 0 && (!logits || !topk_ids))) return DAMOE_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(logits) % (dtype == DAMOE_BF16 ? 2 : 4)) return DAMOE_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(ws) % 16) return DAMOE_ERR_INVALID_ARG;
  const LossWs o = loss_ws(T, E, S);
  if (ws_bytes < o.total) return DAMOE_ERR_WORKSPACE;
  char* base = static_cast<char*>(ws);
  LossArgs a{};
  a.logits = logits;
  a.ld = ld;
  a.ids = topk_ids;
  a.mask = mask;
  a.off = seq_offsets;
  a.T = T;
  a.E = E;
  a.k = k;
  a.S = S;
  a.chunk = chunk_tokens(T, S);
  a.nb = (T + a.chunk - 1) / a.chunk;
  a.err = reinterpret_cast<int32_t*>(base);
  a.part = reinterpret_cast<float2*>(base + o.part);
  a.Ep = padded(E);
  a.width = S < kManySeqs ? kGroup : a.Ep;
  a.part_zn = reinterpret_cast<float2*>(base + o.zn);
  a.seq_l = reinterpret_cast<double*>(base + o.seq_l);
  a.seq_z = reinterpret_cast<float*>(base + o.seq_z);
  a.alpha = alpha;
  a.z_coef = z_coef;
  a.loss = loss;
  a.counts = counts;
  a.probs = probs;
  a.tokens = tokens;
  // One block does it all for up to kOneTokens tokens of a few sequences.
  const bool one = T <= kOneTokens && S <= kOneSeqs;
  if (one) a.chunk = std::max(T, 1), a.nb = 1;
  const bool waves = !one && by_waves(T, S);
  const size_t lds = (size_t)(loss_rows(one ? kOneThreads : waves ? kWave : kLossThreads) + 1) * E * 4;
  const dim3 grid(std::max(a.nb, 1));
  const hipError_t e = by_columns(E, fours(logits, ld, E, dtype), [&](auto v, auto nc) {
    return by_kind(dtype, score, [&](auto bf, auto sig) {
      constexpr int V = decltype(v)::value, NC = decltype(nc)::value;
      constexpr bool BF = decltype(bf)::value, SIG = decltype(sig)::value;
      if (one) hipLaunchKernelGGL((k_router_loss<V, NC, BF, SIG, kOneThreads>), grid, dim3(kOneThreads), lds, stream, a);
      else if (waves) hipLaunchKernelGGL((k_router_loss<V, NC, BF, SIG, kWave>), grid, dim3(kWave), lds, stream, a);
      else hipLaunchKernelGGL((k_router_loss<V, NC, BF, SIG, kLossThreads>), grid, dim3(kLossThreads), lds, stream, a);
      return hipGetLastError();
    });
  });
  if (e != hipSuccess) return DAMOE_ERR_HIP;
  if (!one && S == 1 && (size_t)a.nb * a.Ep <= kAlonePartials) {
    hipLaunchKernelGGL(k_router_loss_alone, dim3(1), dim3(kAloneThreads), 0, stream, a);
  } else if (!one) {
    const dim3 blocks((unsigned)S * (a.Ep / a.width));
    if (S < kFewSeqs) hipLaunchKernelGGL(k_router_loss_seq<1024>, blocks, dim3(1024), 0, stream, a);
    else hipLaunchKernelGGL(k_router_loss_seq<256>, blocks, dim3(256), 0, stream, a);
    hipLaunchKernelGGL(k_router_loss_total, dim3(1), dim3(kTotalThreads), 0, stream, a);
  }
  return hipGetLastError() == hipSuccess ? DAMOE_OK : DAMOE_ERR_HIP;
}

damoe_status damoe_router_loss_grad(const void* logits, int32_t dtype, int64_t ld, const int32_t* topk_ids,
                                    const float* topk_w, const float* dtopk_w, const uint8_t* mask,
                                    const int32_t* seq_offsets, const int32_t* counts, const int32_t* tokens,
                                    int32_t T, int32_t E, int32_t k, int32_t S, int32_t score, float alpha,
                                    float z_coef, const float* dloss, void* dlogits, int64_t ldd,
                                    hipStream_t stream) {
  if (!loss_shape_ok(T, E, k, S) || ld < E || ldd < E || (!seq_offsets && S != 1)) return DAMOE_ERR_INVALID_ARG;
  if (score != DAMOE_SCORE_SOFTMAX && score != DAMOE_SCORE_SIGMOID) return DAMOE_ERR_INVALID_ARG;
  if (dtype != DAMOE_BF16 && dtype != DAMOE_F32) return DAMOE_ERR_UNSUPPORTED;
  if (!counts || !tokens || (!topk_w) != (!dtopk_w)) return DAMOE_ERR_INVALID_ARG;
  if (T == 0) return DAMOE_OK;
  if (!logits || !dlogits || (topk_w && !topk_ids) || (dlogits == logits && ld != ldd)) return DAMOE_ERR_INVALID_ARG;
  const size_t es = dtype == DAMOE_BF16 ? 2 : 4;
  if (reinterpret_cast<uintptr_t>(logits) % es || reinterpret_cast<uintptr_t>(dlogits) % es) return DAMOE_ERR_INVALID_ARG;
  GradArgs a{logits, ld, topk_ids, topk_w, dtopk_w, mask, seq_offsets, counts, tokens, T, E, k, S, 0,
             alpha, z_coef, dloss, dlogits, ldd};
  a.run = std::max(1, std::min(16, (T + 4095) / 4096));
  const int waves = (T + a.run - 1) / a.run;
  const bool four = fours(logits, ld, E, dtype) && fours(dlogits, ldd, E, dtype);
  const hipError_t e = by_columns(E, four, [&](auto v, auto nc) {
    return by_kind(dtype, score, [&](auto bf, auto sig) {
      constexpr int V = decltype(v)::value, NC = decltype(nc)::value;
      constexpr bool BF = decltype(bf)::value, SIG = decltype(sig)::value;
      const size_t lds = topk_w ? (size_t)kGradWaves * Grad<V, NC, BF, SIG>::kRows * E * 4 : 0;
      hipLaunchKernelGGL((k_router_loss_grad<V, NC, BF, SIG>), dim3((waves + kGradWaves - 1) / kGradWaves),
                         dim3(kGradThreads), lds, stream, a);
      return hipGetLastError();
    });
  });
  return e == hipSuccess ? DAMOE_OK : DAMOE_ERR_HIP;
}

}  // extern "C"
