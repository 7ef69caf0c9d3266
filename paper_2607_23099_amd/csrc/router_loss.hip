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
// Forward: a block takes a chunk of tokens and, for each sequence that it meets, writes one slot of partial
// sums (probabilities, counts, z, tokens).  Block b's slot of sequence s is b + s: the slots of a walk over
// the tokens, distinct while offsets do not decrease.  A block per sequence then adds its slots in order, so
// the sums run in a fixed order, and a last block adds the sequences.
#include "common.h"

namespace damoe {
namespace {

constexpr int kRows = 4;          // rows of logits a wave holds at a time
constexpr int kLossThreads = 256;
constexpr int kLossWaves = kLossThreads / kWave;
constexpr int kMaxChunks = 512;   // blocks of the forward pass: two per compute unit
constexpr int kMinChunk = kRows * kLossWaves;

// Tokens of a block of the forward pass.
__host__ __device__ inline int32_t chunk_tokens(int32_t T) {
  const int32_t c = (T + kMaxChunks - 1) / kMaxChunks;
  return (c + kMinChunk - 1) / kMinChunk * kMinChunk;
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
  float* part_p;       // [nb + S][E]
  int32_t* part_c;     // [nb + S][E]
  float2* part_zn;     // [nb + S]: sum of lse^2, bits of the valid tokens
  float2* seq_lz;      // [S]: sum_e f P, sum of lse^2
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

__device__ __forceinline__ float exp_f(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504088896f); }

// LDS of a wave's own: what other lanes of the wave wrote before is read after it.
__device__ __forceinline__ void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// ---------------------------------------------------------------- rows

// A lane's V * NC values of a row: columns 64 V c + V lane + i.  V = 4 wants rows of whole aligned fours.
template <int V, int NC, bool BF>
struct Row {
  float v[V * NC];

  static __device__ __forceinline__ int col(int c, int lane) { return (c * kWave + lane) * V; }

  __device__ __forceinline__ void load(const void* base, int64_t row, int64_t ld, int E, int lane, float fill) {
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int e = col(c, lane);
      if (e < E) {
        if constexpr (BF) {
          const uint16_t* p = static_cast<const uint16_t*>(base) + row * ld + e;
          if constexpr (V == 4) {
            const uint2 q = *reinterpret_cast<const uint2*>(p);
            v[4 * c] = __uint_as_float(q.x << 16);
            v[4 * c + 1] = __uint_as_float(q.x & 0xFFFF0000u);
            v[4 * c + 2] = __uint_as_float(q.y << 16);
            v[4 * c + 3] = __uint_as_float(q.y & 0xFFFF0000u);
          } else {
            v[c] = bf16_to_f32(*p);
          }
        } else {
          const float* p = static_cast<const float*>(base) + row * ld + e;
          if constexpr (V == 4) {
            const float4 q = *reinterpret_cast<const float4*>(p);
            v[4 * c] = q.x;
            v[4 * c + 1] = q.y;
            v[4 * c + 2] = q.z;
            v[4 * c + 3] = q.w;
          } else {
            v[c] = *p;
          }
        }
      } else {
#pragma unroll
        for (int i = 0; i < V; ++i) v[V * c + i] = fill;
      }
    }
  }

  __device__ __forceinline__ void store(void* base, int64_t row, int64_t ld, int E, int lane) const {
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int e = col(c, lane);
      if (e >= E) continue;
      if constexpr (BF) {
        uint16_t* p = static_cast<uint16_t*>(base) + row * ld + e;
        if constexpr (V == 4) {
          uint2 q;
          q.x = (uint32_t)bf16_of(v[4 * c]) | (uint32_t)bf16_of(v[4 * c + 1]) << 16;
          q.y = (uint32_t)bf16_of(v[4 * c + 2]) | (uint32_t)bf16_of(v[4 * c + 3]) << 16;
          *reinterpret_cast<uint2*>(p) = q;
        } else {
          *p = bf16_of(v[c]);
        }
      } else {
        float* p = static_cast<float*>(base) + row * ld + e;
        if constexpr (V == 4) {
          *reinterpret_cast<float4*>(p) = make_float4(v[4 * c], v[4 * c + 1], v[4 * c + 2], v[4 * c + 3]);
        } else {
          *p = v[c];
        }
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

// exp(l - m) of a row with maximum m; all 0 where the row is -inf throughout (-inf - -inf would be NaN).
__device__ __forceinline__ float shifted_exp(float l, float m) { return exp_f(l - m); }

// sigmoid(l) over a common factor of the row with maximum m: sigmoid(l) = e^min(l, 0) / (1 + e^-|l|), and the
// row's largest keeps a numerator of 1, so that rows of very negative logits do not underflow.
__device__ __forceinline__ float shifted_sigmoid(float l, float m) {
  return exp_f(fminf(l, 0.f) - fminf(m, 0.f)) * __builtin_amdgcn_rcpf(1.f + exp_f(-fabsf(l)));
}

// 1 - sigmoid(l) = sigmoid(-l)
__device__ __forceinline__ float one_minus_sigmoid(float l) {
  return exp_f(fminf(-l, 0.f)) * __builtin_amdgcn_rcpf(1.f + exp_f(-fabsf(l)));
}

__device__ __forceinline__ int offset_at(const int32_t* off, int32_t s, int32_t T) {
  const int o = off ? off[s] : (s == 0 ? 0 : T);
  return min(max(o, 0), T);
}

// ---------------------------------------------------------------- forward

template <int V, int NC, bool BF, bool SIG>
__global__ void __launch_bounds__(kLossThreads) k_router_loss(LossArgs a) {
  extern __shared__ float loss_smem[];
  float* const red = loss_smem;                                                // [waves][E]
  int32_t* const hist = reinterpret_cast<int32_t*>(red + kLossWaves * a.E);    // [E]
  __shared__ float z_red[kLossWaves];
  __shared__ int32_t n_red[kLossWaves];
  __shared__ int32_t first;
  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int E = a.E, k = a.k;
  const int t0 = blockIdx.x * a.chunk, t1 = min(t0 + a.chunk, a.T);
  const float kNegInf = -__builtin_huge_valf();

  // The first sequence that may reach past t0: the number of ends at or before it.
  if (tid == 0) first = 0;
  for (int e = tid; e < E; e += kLossThreads) hist[e] = 0;
  __syncthreads();
  if (a.off) {
    int n = 0;
    for (int s = tid; s < a.S; s += kLossThreads) n += offset_at(a.off, s + 1, a.T) <= t0;
    if (n) atomicAdd(&first, n);
    __syncthreads();
  }
  for (int s = first; s < a.S; ++s) {
    const int b0 = offset_at(a.off, s, a.T), b1 = offset_at(a.off, s + 1, a.T);
    if (b0 >= t1) break;
    const int lo = max(t0, b0), hi = min(t1, b1);
    if (lo >= hi) continue;
    float acc[V * NC];
#pragma unroll
    for (int i = 0; i < V * NC; ++i) acc[i] = 0.f;
    float zsum = 0.f;
    int n = 0;
    for (int t = lo + w * kRows; t < hi; t += kLossWaves * kRows) {
      Row<V, NC, BF> r[kRows];
      bool ok[kRows];
#pragma unroll
      for (int u = 0; u < kRows; ++u) ok[u] = t + u < hi && (!a.mask || a.mask[t + u] != 0);
#pragma unroll
      for (int u = 0; u < kRows; ++u) {
        if (ok[u]) {
          r[u].load(a.logits, t + u, a.ld, E, lane, kNegInf);
        } else {
#pragma unroll
          for (int i = 0; i < V * NC; ++i) r[u].v[i] = 0.f;
        }
      }
      // The slots of the kRows tokens, one a lane (k <= 16).
      if (lane < kRows * k) {
        const int u = lane / k;
        if (t + u < hi && (!a.mask || a.mask[t + u] != 0)) {
          const int id = a.ids[(int64_t)t * k + lane];
          if (id >= E) atomicOr(a.err, DAMOE_DEVERR_EXPERT_ID);
          else if (id >= 0) atomicAdd(&hist[id], 1);
        }
      }
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
            r[u].v[i] = shifted_sigmoid(l, mm);
            sg += r[u].v[i];
          } else {
            r[u].v[i] = x;
          }
        }
        sum[u] = wave_sum(sum[u]);
        inv[u] = SIG ? wave_sum(sg) : sum[u];
      }
#pragma unroll
      for (int u = 0; u < kRows; ++u) {
        if (!ok[u]) continue;
        ++n;
        if (m[u] == kNegInf) continue;
        const float lse = m[u] + __logf(sum[u]);
        zsum += lse * lse;
        const float f = 1.f / inv[u];
#pragma unroll
        for (int i = 0; i < V * NC; ++i) acc[i] += r[u].v[i] * f;
      }
    }
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const int e = Row<V, NC, BF>::col(c, lane) + i;
        if (e < E) red[w * E + e] = acc[V * c + i];
      }
    if (lane == 0) {
      z_red[w] = zsum;
      n_red[w] = n;
    }
    __syncthreads();
    const int64_t slot = (int64_t)blockIdx.x + s;
    for (int e = tid; e < E; e += kLossThreads) {
      float p = 0.f;
#pragma unroll
      for (int i = 0; i < kLossWaves; ++i) p += red[i * E + e];
      a.part_p[slot * E + e] = p;
      a.part_c[slot * E + e] = hist[e];
      hist[e] = 0;
    }
    if (tid == 0) {
      float z = 0.f;
      int nn = 0;
      for (int i = 0; i < kLossWaves; ++i) {
        z += z_red[i];
        nn += n_red[i];
      }
      a.part_zn[slot] = make_float2(z, __int_as_float(nn));
    }
    __syncthreads();
  }
}

__device__ __forceinline__ void write_loss(const LossArgs& a, double balance, double z, int n_seq, int n_tok) {
  const float b = n_seq > 0 ? (float)(balance / n_seq) : 0.f;
  const float zz = n_tok > 0 ? (float)(z / n_tok) : 0.f;
  a.loss[0] = (a.alpha != 0.f ? a.alpha * b : 0.f) + (a.z_coef != 0.f ? a.z_coef * zz : 0.f);
  a.loss[1] = b;
  a.loss[2] = zz;
  a.tokens[a.S] = n_seq;
  a.tokens[a.S + 1] = n_tok;
}

constexpr int kSeqThreads = 1024;

// A block per sequence: its slots added in order, f and P, and their product's sum.
__global__ void __launch_bounds__(kSeqThreads) k_router_loss_seq(LossArgs a) {
  __shared__ float p_red[kSeqThreads];
  __shared__ int32_t c_red[kSeqThreads];
  __shared__ double lz[kSeqThreads / kWave];
  __shared__ float z_tot;
  __shared__ int32_t n_tot;
  const int tid = threadIdx.x, E = a.E, s = blockIdx.x;
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
      z_tot = z;
      n_tot = n;
      a.tokens[s] = n;
    }
  }
  __syncthreads();
  const int n = n_tot;
  double l = 0.0;
  // Columns in passes of `cols`; the threads of a column share its slots.
  const int cols = min((E + kWave - 1) / kWave * kWave, kSeqThreads), split = kSeqThreads / cols;
  const int c = tid % cols, g = tid / cols;
  for (int e0 = 0; e0 < E; e0 += cols) {
    const int e = e0 + c;
    float p = 0.f;
    int cnt = 0;
    if (e < E && g < split) {
      for (int i = g; i < nslot; i += split) {
        p += a.part_p[(base + i) * E + e];
        cnt += a.part_c[(base + i) * E + e];
      }
    }
    p_red[tid] = p;
    c_red[tid] = cnt;
    __syncthreads();
    if (g == 0 && e < E) {
      for (int i = 1; i < split; ++i) {
        p += p_red[i * cols + c];
        cnt += c_red[i * cols + c];
      }
      const float P = n > 0 ? p / (float)n : 0.f;
      a.counts[(int64_t)s * E + e] = cnt;
      if (a.probs) a.probs[(int64_t)s * E + e] = P;
      if (n > 0) l += (double)E * cnt / ((double)a.k * n) * P;
    }
    __syncthreads();
  }
  for (int d = 1; d < kWave; d <<= 1) l += __shfl_xor(l, d);
  if ((tid & 63) == 0) lz[tid >> 6] = l;
  __syncthreads();
  if (tid == 0) {
    l = 0.0;
    for (int i = 0; i < kSeqThreads / kWave; ++i) l += lz[i];
    if (a.S == 1) write_loss(a, l, z_tot, n > 0, n);
    else a.seq_lz[s] = make_float2((float)l, z_tot);
  }
}

// The sum over sequences, in a fixed order.
__global__ void __launch_bounds__(256) k_router_loss_total(LossArgs a) {
  __shared__ double red[3][4];
  __shared__ int64_t n_red[4];
  const int tid = threadIdx.x;
  double l = 0, z = 0;
  int64_t seqs = 0, n = 0;
  for (int s = tid; s < a.S; s += 256) {
    const int ns = a.tokens[s];
    if (ns <= 0) continue;
    const float2 q = a.seq_lz[s];
    l += q.x;
    z += q.y;
    ++seqs;
    n += ns;
  }
  for (int d = 1; d < kWave; d <<= 1) {
    l += __shfl_xor(l, d);
    z += __shfl_xor(z, d);
    seqs += __shfl_xor(seqs, d);
    n += __shfl_xor(n, d);
  }
  if ((tid & 63) == 0) {
    red[0][tid >> 6] = l;
    red[1][tid >> 6] = z;
    red[2][tid >> 6] = (double)seqs;
    n_red[tid >> 6] = n;
  }
  __syncthreads();
  if (tid == 0) {
    for (int i = 1; i < 4; ++i) {
      l += red[0][i];
      z += red[1][i];
      seqs += (int64_t)red[2][i];
      n += n_red[i];
    }
    write_loss(a, l, z, (int)seqs, (int)n);
  }
}

// ---------------------------------------------------------------- gradient

template <int V, int NC, bool BF, bool SIG>
__global__ void __launch_bounds__(kLossThreads) k_router_loss_grad(GradArgs a) {
  extern __shared__ float grad_smem[];  // [waves][E]: the gates' gradient of a row
  const int lane = threadIdx.x & 63;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int E = a.E, k = a.k;
  float* const gate = grad_smem + w * E;
  const int t0 = (blockIdx.x * kLossWaves + w) * a.run, t1 = min(t0 + a.run, a.T);
  if (t0 >= t1) return;
  const float kNegInf = -__builtin_huge_valf();
  for (int e = lane; e < E; e += kWave) gate[e] = 0.f;
  const float g = a.dloss ? *a.dloss : 1.f;
  const float n_seq = (float)a.tokens[a.S], n_tok = (float)a.tokens[a.S + 1];
  const float zc = a.z_coef != 0.f ? g * a.z_coef * 2.f / n_tok : 0.f;

  int s = 0;
  if (a.off) {
    for (int i = lane; i < a.S; i += kWave) s += offset_at(a.off, i + 1, a.T) <= t0;
    for (int d = 1; d < kWave; d <<= 1) s += __shfl_xor(s, d);
    s = __builtin_amdgcn_readfirstlane(s);
  }
  int begin = 0, end = -1, cur = -1;  // of sequence s once `cur` names it
  float f[V * NC], bal = 0.f;
  for (int t = t0; t < t1; ++t) {
    // The sequence of t; its f in registers.
    while (s < a.S && (cur != s || t >= end)) {
      if (cur == s) ++s;
      if (s >= a.S) break;
      cur = s;
      begin = offset_at(a.off, s, a.T);
      end = offset_at(a.off, s + 1, a.T);
      if (t < end) {
        const float n = (float)a.tokens[s];
        bal = a.alpha != 0.f ? g * a.alpha / (n_seq * n) : 0.f;
        const float fs = (float)E / ((float)k * n);
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int i = 0; i < V; ++i) {
            const int e = Row<V, NC, BF>::col(c, lane) + i;
            f[V * c + i] = e < E ? fs * (float)a.counts[(int64_t)s * E + e] : 0.f;
          }
      }
    }
    const bool ok = s < a.S && t >= begin && t < end && (!a.mask || a.mask[t] != 0);
    Row<V, NC, BF> r;
    if (!ok) {
#pragma unroll
      for (int i = 0; i < V * NC; ++i) r.v[i] = 0.f;
      r.store(a.dlogits, t, a.ldd, E, lane);
      continue;
    }
    r.load(a.logits, t, a.ld, E, lane, kNegInf);
    if (a.w) {
      // dw_j -> w_j (dw_j - sum_i w_i dw_i), added to the expert's column (twice for an id held twice).
      int id = -1;
      float wj = 0.f, dj = 0.f;
      if (lane < k) {
        id = a.ids[(int64_t)t * k + lane];
        if (id >= 0 && id < E) {
          wj = a.w[(int64_t)t * k + lane];
          dj = a.dw[(int64_t)t * k + lane];
        }
      }
      const float dot = wave_sum(wj * dj);
      wave_fence();
      if (id >= 0 && id < E) atomicAdd(&gate[id], wj * (dj - dot));
      wave_fence();
    }
    const float m = wave_max(r.max());
    const float mm = m == kNegInf ? 0.f : m;
    float sum = 0.f, ps = 0.f, fp = 0.f;
    float ex[V * NC], p[V * NC];
#pragma unroll
    for (int i = 0; i < V * NC; ++i) {
      ex[i] = shifted_exp(r.v[i], mm);
      p[i] = SIG ? shifted_sigmoid(r.v[i], mm) : ex[i];
      sum += ex[i];
      ps += p[i];
      fp += p[i] * f[i];
    }
    sum = wave_sum(sum);
    ps = SIG ? wave_sum(ps) : sum;
    fp = wave_sum(fp);
    const bool live = m != kNegInf;
    const float ip = live ? 1.f / ps : 0.f;
    const float dot = fp * ip;
    const float zt = live && a.z_coef != 0.f ? zc * (m + __logf(sum)) / sum : 0.f;
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const int j = V * c + i, e = Row<V, NC, BF>::col(c, lane) + i;
        float d = bal * p[j] * ip * (f[j] - dot);
        if constexpr (SIG) d *= one_minus_sigmoid(r.v[j]);
        d += zt * ex[j];
        if (a.w && e < E) {
          d += gate[e];
          gate[e] = 0.f;
        }
        r.v[j] = d;
      }
    r.store(a.dlogits, t, a.ldd, E, lane);
  }
}

// ---------------------------------------------------------------- launches

// Columns a lane holds: fours where rows are whole aligned fours, else single ones; NC chunks of 64 V columns.
template <template <int, int, bool, bool> class L, class A>
hipError_t pick(const A& a, bool four, bool bf, bool sig, dim3 grid, size_t lds, hipStream_t stream) {
  auto go = [&](auto v, auto nc) {
    constexpr int V = decltype(v)::value, NC = decltype(nc)::value;
    if (bf) return sig ? L<V, NC, true, true>::run(a, grid, lds, stream) : L<V, NC, true, false>::run(a, grid, lds, stream);
    return sig ? L<V, NC, false, true>::run(a, grid, lds, stream) : L<V, NC, false, false>::run(a, grid, lds, stream);
  };
  using std::integral_constant;
  const int E = a.E;
  if (four) {
    const integral_constant<int, 4> v;
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

template <int V, int NC, bool BF, bool SIG>
struct RunLoss {
  static hipError_t run(const LossArgs& a, dim3 grid, size_t lds, hipStream_t stream) {
    hipLaunchKernelGGL((k_router_loss<V, NC, BF, SIG>), grid, dim3(kLossThreads), lds, stream, a);
    return hipGetLastError();
  }
};

template <int V, int NC, bool BF, bool SIG>
struct RunGrad {
  static hipError_t run(const GradArgs& a, dim3 grid, size_t lds, hipStream_t stream) {
    hipLaunchKernelGGL((k_router_loss_grad<V, NC, BF, SIG>), grid, dim3(kLossThreads), lds, stream, a);
    return hipGetLastError();
  }
};

size_t up256(size_t v) { return (v + 255) / 256 * 256; }

// Workspace: control word, then the partial sums of nb + S slots, then the sequences'.
struct LossWs {
  size_t p, c, zn, seq, total;
};

LossWs loss_ws(int32_t T, int32_t E, int32_t S) {
  const int32_t chunk = std::max(chunk_tokens(T), kMinChunk);
  const size_t slots = (size_t)((T + chunk - 1) / chunk) + S;
  LossWs o;
  o.p = 256;
  o.c = o.p + up256(slots * E * 4);
  o.zn = o.c + up256(slots * E * 4);
  o.seq = o.zn + up256(slots * 8);
  o.total = o.seq + up256((size_t)S * 8);
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
  // The chunk grows with T in steps, so a smaller T may take more blocks, but never over kMaxChunks.
  const size_t at = loss_ws(T_max, E, S).total;
  const int32_t full = std::min<int32_t>(T_max, kMaxChunks * kMinChunk);
  return std::max({at, loss_ws(full, E, S).total, loss_ws(std::min(T_max, 1), E, S).total});
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
  a.chunk = std::max(chunk_tokens(T), kMinChunk);
  a.nb = (T + a.chunk - 1) / a.chunk;
  a.err = reinterpret_cast<int32_t*>(base);
  a.part_p = reinterpret_cast<float*>(base + o.p);
  a.part_c = reinterpret_cast<int32_t*>(base + o.c);
  a.part_zn = reinterpret_cast<float2*>(base + o.zn);
  a.seq_lz = reinterpret_cast<float2*>(base + o.seq);
  a.alpha = alpha;
  a.z_coef = z_coef;
  a.loss = loss;
  a.counts = counts;
  a.probs = probs;
  a.tokens = tokens;
  if (a.nb > 0) {
    const size_t lds = (size_t)(kLossWaves + 1) * E * 4;
    if (pick<RunLoss>(a, fours(logits, ld, E, dtype), dtype == DAMOE_BF16, score == DAMOE_SCORE_SIGMOID, dim3(a.nb),
                      lds, stream) != hipSuccess)
      return DAMOE_ERR_HIP;
  }
  hipLaunchKernelGGL(k_router_loss_seq, dim3(S), dim3(kSeqThreads), 0, stream, a);
  if (S > 1) hipLaunchKernelGGL(k_router_loss_total, dim3(1), dim3(256), 0, stream, a);
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
  return pick<RunGrad>(a, four, dtype == DAMOE_BF16, score == DAMOE_SCORE_SIGMOID,
                       dim3((waves + kLossWaves - 1) / kLossWaves), (size_t)kLossWaves * E * 4, stream) == hipSuccess
             ? DAMOE_OK
             : DAMOE_ERR_HIP;
}

}  // extern "C"
