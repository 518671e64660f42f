// Clipped policy loss over log-probabilities, with a KL term, and its gradient.  For a counted token with d = new - old,
// r = exp(d), advantage A and e = exp(ref - new) - 1:
//   clipped  <=>  A > 0 and r > 1 + high,  or  A < 0 and r < 1 - low
//   loss     =    -A r   (clipped: -A (1 + high), -A (1 - low))   + kl_weight (e - (ref - new))
//   d loss / d new  =  (clipped ? 0 : -A r) - kl_weight e,
// weighted by 1 / count, by 1 / (count of the row * rows with a count), or by 1.
//
// The weights need the counts before the first gradient can be written: where a mask or lengths are given,
// k_policy_count goes over them first (a quarter of a byte and less for a byte that the second pass moves).  k_policy then
// reads every value once.  Few values are done by one cluster in one launch (k_policy_small).  Differences are exact (two
// fp32 numbers), gains and sums 64 bits, in a fixed order; KL terms, which never cancel one another, and gradients 32 bits, or 64
// where fp32 does not hold them before they have their weight (far_values).  Large calls are
// bound by the arithmetic of a token and its loads, about alike (1M tokens with everything: 14.5 us, of which 2.6 us are bytes at
// HBM's rate), small ones by the launches (128 x 501: 7.3 us) and the length of one token's chain (64 values: 3.8 us).
#include "../../include/prunedctc.h"
#include "pctc_internal.h"

#include <cooperative_groups.h>

#include <cmath>
#include <math_constants.h>

namespace cg = cooperative_groups;

namespace pctc {
namespace {

constexpr int POLICY_THREADS = 256;
constexpr int POLICY_EACH = 4;                   // values of a group
constexpr long long POLICY_MANY = 148 * 4 * POLICY_THREADS * POLICY_EACH;   // more values than run at a time in groups of their
                                                 // own take two groups a thread (1M values: 14.6 -> 13.3 us; 64,000: 7.2 -> 9.1)
constexpr int POLICY_SMALL_THREADS = 512;
constexpr int POLICY_CLUSTER = 8;
constexpr long long POLICY_SMALL = 16384;        // up to so many values one cluster does all (15,000 values: 6.1 us against 9.4)
static_assert(POLICY_SMALL <= POLICY_CLUSTER * POLICY_SMALL_THREADS * POLICY_EACH, "one round");
constexpr int POLICY_SHORT_ROW = 32;             // masks of rows up to this length are counted by a thread each,
constexpr int POLICY_LONG_ROW = 2048;            // up to this one by a warp, longer ones by a block
constexpr int POLICY_COUNT_BLOCKS = 148;         // blocks that count, at most

struct Totals {                                  // fewer than 2^31 values
  int count;                                     // counted tokens
  int rows;                                      // rows that have one
};
struct PolicyHead {                              // start of the workspace
  unsigned ticket;
  unsigned blocks;                               // that have counted
  Totals totals[POLICY_COUNT_BLOCKS];            // of each of them
};

struct alignas(16) BlockSums {                   // the sums of a block's tokens
  double loss, kl;
  int count, clipped;
};

struct PolicyArgs {
  const float* logp;
  const float* old_logp;
  const float* ref;
  const float* adv;
  const unsigned char* mask;
  const int* lengths;
  float* grad;
  float* stats;                                  // [3] loss, mean KL, share of clipped tokens
  int* count_out;
  PolicyHead* head;
  int* row_count;                                // [N], made where the weights need it and a mask is given
  BlockSums* partial;                            // [blocks]
  long long N, T, total;
  long long ld_logp, ld_old, ld_ref, ld_adv, ld_mask, ld_grad;   // ld_adv 0: one advantage a row
  float2 log_low, log_high;                      // logarithms of where ratios are clipped, as a number and its rest
  double low, high;                              // the clipped ratios
  float kl_weight, sign;
  int reduction;
  int counting;                                  // counts come from k_policy_count
};

__device__ __forceinline__ int length_of(const PolicyArgs& a, long long n) {
  return a.lengths ? (int)min((long long)max(a.lengths[n], 0), a.T) : (int)a.T;
}

// The sums of a thread's few tokens.  Gains A r of both signs cancel, so they are 64 bits; the KL terms do not.
struct TokenSums {
  double gain = 0.0;
  float kl_loss = 0.f, kl = 0.f;                 // loss = kl_loss - gain
  float size = 0.f;                              // magnitudes of the gradients without their weights
  int clipped = 0, count = 0;
};

// a - b without a rounding: a number and its rest (Knuth's two-sum).  Where the difference is not finite the rest is 0.
__device__ __forceinline__ float2 difference(float a, float b) {
  const float s = __fsub_rn(a, b), back = __fsub_rn(s, a);
  const float rest = __fsub_rn(__fsub_rn(a, __fsub_rn(s, back)), __fadd_rn(b, back));
  return make_float2(s, fabsf(s) < CUDART_INF_F ? rest : 0.f);
}
__device__ __forceinline__ bool above(float2 a, float2 b) { return a.x > b.x || (a.x == b.x && a.y > b.y); }

// exp(d) - 1 - d for |d| < 1 by its series d^2 (1/2 + d/6 + ... + d^11 / 13!), where the difference would cancel (the next term
// is under 1e-10 of the sum).
__device__ __forceinline__ float exp_tail(float d) {
  constexpr float c[] = {1.f / 6227020800.f, 1.f / 479001600.f, 1.f / 39916800.f, 1.f / 3628800.f, 1.f / 362880.f, 1.f / 40320.f,
                         1.f / 5040.f, 1.f / 720.f, 1.f / 120.f, 1.f / 24.f, 1.f / 6.f, 1.f / 2.f};
  float s = c[0];
#pragma unroll
  for (int j = 1; j < 12; ++j) s = fmaf(d, s, c[j]);
  return d * d * s;
}
// exp(b - a) - 1 - (b - a) and exp(b - a) - 1; the rounding of a difference under 1 is one of 2^-24.
__device__ __forceinline__ void kl_terms(float a, float b, float& kl, float& e) {
  const float d = b - a;
  if (fabsf(d) < 1.f) {
    kl = exp_tail(d);
    e = d + kl;
  } else {
    const float2 f = difference(b, a);
    e = expm1f(f.x);
    if (!isinf(e)) e = fmaf(e + 1.f, f.y, e);
    kl = isinf(e) ? e : (e - f.x) - f.y;
  }
}

// One token: adds to the sums and returns its gradient before the weight w (wd: the same in 64 bits).  Values come with the
// sign of log-probabilities; what does not count comes as zeros with no advantage, and gives zeros.
__device__ __forceinline__ float policy_token(const PolicyArgs& a, float x, float x_old, float x_ref, float A, float w, double wd,
                                              TokenSums& s) {
  const float2 d = difference(x, x_old);         // exact: whether a ratio is clipped does not depend on a rounding
  const bool over = A > 0.f && above(d, a.log_high), under = A < 0.f && above(a.log_low, d), clipped = over || under;
  // below e the ratio is 1 + d in 64 bits and what is left, up to 0.72 (a hundredth where |d| < 0.14), in 32
  const double dd = (double)d.x + (double)d.y;
  const double r = fabsf(d.x) < 1.f ? (1.0 + dd) + (double)exp_tail(d.x) : exp(dd);
  const float r32 = (float)r;
  const bool none = A == 0.f && fabsf(d.x) < CUDART_INF_F;           // no 0 * inf where exp(d) overflows for a finite d
  float g = clipped || none ? 0.f : -A * r32;
  if (a.ref) {
    float kl, e;
    kl_terms(x, x_ref, kl, e);
    s.kl_loss = fmaf(w, a.kl_weight * kl, s.kl_loss);
    g = fmaf(-a.kl_weight, e, g);
    s.kl += kl;
  }
  if (!none) s.gain = fma(wd, (double)A * (over ? a.high : under ? a.low : r), s.gain);
  s.clipped += clipped ? 1 : 0;
  s.size += fabsf(g);
  return g;
}
// Whether fp32 held the gradients and KL terms of a thread's tokens without their weights with room to spare (not if one is NaN).
// Where it did not, far_values does them over; ratios, gains and what they add up to are 64 bits in either case.
constexpr float POLICY_FAR = 1.2676506e30f;      // 2^100
__device__ __forceinline__ bool held(const PolicyArgs& a, const TokenSums& s) {
  return s.size + (fabsf(a.kl_weight) + 1.f) * s.kl < POLICY_FAR;
}

// The weight of the tokens of a row with `count` of them, in 64 bits: 1 / n for a whole number n.
__device__ __forceinline__ double inverse(double n) {
  const float w = 1.f / (float)n;
  return fma((double)w, fma(-(double)w, n, 1.0), (double)w);      // one step of Newton's: 2^-48
}
__device__ __forceinline__ double weight_part(const PolicyArgs& a, const Totals& t) {
  return a.reduction == PCTC_POLICY_SUM ? 1.0 : a.reduction == PCTC_POLICY_TOKENS ? inverse((double)max(t.count, 1)) : (double)max(t.rows, 1);
}
__device__ __forceinline__ double weight_of(const PolicyArgs& a, double part, int count) {
  return a.reduction == PCTC_POLICY_SEQUENCES ? inverse((double)max(count, 1) * part) : part;
}

// How many of bytes 0 .. n - 1 are not zero, of the `lanes` threads' shares.
__device__ __forceinline__ int count_bytes(const unsigned char* m, int n, int lane, int lanes) {
  int c = 0;
  const int head = min((int)((16 - ((size_t)m & 15)) & 15), n), vecs = (n - head) / 16;
  for (int t = lane; t < head; t += lanes) c += m[t] != 0;
  const uint4* body = reinterpret_cast<const uint4*>(m + head);
#pragma unroll 4
  for (int i = lane; i < vecs; i += lanes) {
    const uint4 v = body[i];
    c += (__popc(__vcmpne4(v.x, 0u)) + __popc(__vcmpne4(v.y, 0u)) + __popc(__vcmpne4(v.z, 0u)) + __popc(__vcmpne4(v.w, 0u))) >> 3;
  }
  for (int t = head + vecs * 16 + lane; t < n; t += lanes) c += m[t] != 0;
  return c;
}
// Rows worker, worker + workers, ...: a worker is `lanes` threads (1, 32, or the block).
template <int THREADS>
__device__ __forceinline__ Totals count_rows(const PolicyArgs& a, int lanes, long long worker, long long workers) {
  __shared__ int scratch[THREADS / 32];
  Totals t{0, 0};
  const int lane = threadIdx.x & (lanes - 1);
  for (long long n = worker; n < a.N; n += workers) {
    int c = a.mask ? count_bytes(a.mask + n * a.ld_mask, length_of(a, n), lane, lanes) : lane == 0 ? length_of(a, n) : 0;
    if (lanes > 1) c = __reduce_add_sync(0xffffffffu, c);
    if (lanes > 32) {
      __syncthreads();
      if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = c;
      __syncthreads();
      c = 0;
      for (int i = 0; i < THREADS / 32; ++i) c += scratch[i];
    }
    if (lane != 0) continue;
    if (a.row_count) a.row_count[n] = c;
    t.count += c;
    t.rows += c > 0;
  }
  return t;
}

__device__ __forceinline__ Totals warp_sum(Totals t) {
  return Totals{__reduce_add_sync(0xffffffffu, t.count), __reduce_add_sync(0xffffffffu, t.rows)};
}
// Sums over a block, valid in thread 0.
template <int THREADS>
__device__ __forceinline__ Totals count_all(const PolicyArgs& a, int block, int blocks) {
  __shared__ Totals scratch[THREADS / 32];
  const int lanes = !a.mask || a.T <= POLICY_SHORT_ROW ? 1 : a.T <= POLICY_LONG_ROW ? 32 : THREADS, each = THREADS / lanes;
  Totals t = warp_sum(count_rows<THREADS>(a, lanes, (long long)block * each + threadIdx.x / lanes, (long long)blocks * each));
  if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = t;
  __syncthreads();
  if (threadIdx.x < 32) t = warp_sum(threadIdx.x < THREADS / 32 ? scratch[threadIdx.x] : Totals{0, 0});
  return t;
}
// The sums of tokens of a block, valid in thread 0.
template <int THREADS>
__device__ __forceinline__ BlockSums block_sum(double loss, double kl, int count, int clipped) {
  __shared__ BlockSums scratch[THREADS / 32];
  const auto warp = [&](int from) {
    for (int d = from; d > 0; d >>= 1) {
      loss += __shfl_xor_sync(0xffffffffu, loss, d);
      kl += __shfl_xor_sync(0xffffffffu, kl, d);
    }
    count = __reduce_add_sync(0xffffffffu, count);
    clipped = __reduce_add_sync(0xffffffffu, clipped);
  };
  warp(16);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = BlockSums{loss, kl, count, clipped};
  __syncthreads();
  if (threadIdx.x < 32) {
    const BlockSums s = threadIdx.x < THREADS / 32 ? scratch[threadIdx.x] : BlockSums{0.0, 0.0, 0, 0};
    loss = s.loss; kl = s.kl; count = s.count; clipped = s.clipped;
    warp(THREADS / 64);
  }
  return BlockSums{loss, kl, count, clipped};
}

__global__ void __launch_bounds__(POLICY_THREADS) k_policy_count(const PolicyArgs a) {
  launch_next();
  if (a.counting) {
    const Totals t = count_all<POLICY_THREADS>(a, blockIdx.x, gridDim.x);
    if (threadIdx.x == 0) a.head->totals[blockIdx.x] = t;
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    a.head->ticket = 0;
    a.head->blocks = gridDim.x;
  }
}

// Four values of a thread: those from `first` on, in one row and 16-byte aligned (VEC), or first, first + step, ...
template <bool VEC>
struct Values {
  static constexpr int ROWS = VEC ? 1 : POLICY_EACH;
  float x[POLICY_EACH], o[POLICY_EACH], q[POLICY_EACH], A[POLICY_EACH];
  int row[ROWS], col[ROWS], length[ROWS];        // length -1: behind the last value
  unsigned masks;                                // bit k: value k counts

  // All loads at once; what a mask leaves out is read, but not looked at.
  __device__ __forceinline__ void load(const PolicyArgs& a, long long first, long long step) {
    masks = 0;
#pragma unroll
    for (int k = 0; k < ROWS; ++k) {
      const long long i = first + k * step;
      row[k] = (int)((unsigned)i / (unsigned)a.T);                // fewer than 2^31 values
      col[k] = (int)(i - row[k] * a.T);
      length[k] = i < a.total ? length_of(a, row[k]) : -1;
    }
#pragma unroll
    for (int k = 0; k < ROWS; ++k) {
      if (col[k] >= length[k]) continue;
      const long long n = row[k];
      const int c = col[k];
      if constexpr (VEC) {
        const float4 fx = *reinterpret_cast<const float4*>(a.logp + n * a.ld_logp + c);
        const float4 fo = *reinterpret_cast<const float4*>(a.old_logp + n * a.ld_old + c);
        float4 fq = make_float4(0.f, 0.f, 0.f, 0.f), fa;
        if (a.ref) fq = *reinterpret_cast<const float4*>(a.ref + n * a.ld_ref + c);
        if (a.ld_adv) fa = *reinterpret_cast<const float4*>(a.adv + n * a.ld_adv + c);
        else fa.x = fa.y = fa.z = fa.w = a.adv[n];
        unsigned m = 0x01010101u;
        if (a.mask) m = *reinterpret_cast<const unsigned*>(a.mask + n * a.ld_mask + c);
        x[0] = fx.x; x[1] = fx.y; x[2] = fx.z; x[3] = fx.w;
        o[0] = fo.x; o[1] = fo.y; o[2] = fo.z; o[3] = fo.w;
        q[0] = fq.x; q[1] = fq.y; q[2] = fq.z; q[3] = fq.w;
        A[0] = fa.x; A[1] = fa.y; A[2] = fa.z; A[3] = fa.w;
#pragma unroll
        for (int j = 0; j < POLICY_EACH; ++j)
          if (((m >> (8 * j)) & 0xffu) != 0 && c + j < length[k]) masks |= 1u << j;
      } else {
        x[k] = a.logp[n * a.ld_logp + c];
        o[k] = a.old_logp[n * a.ld_old + c];
        q[k] = a.ref ? a.ref[n * a.ld_ref + c] : 0.f;
        A[k] = a.ld_adv ? a.adv[n * a.ld_adv + c] : a.adv[n];
        if (!a.mask || a.mask[n * a.ld_mask + c] != 0) masks |= 1u << k;
      }
    }
  }
  __device__ __forceinline__ void finish(const PolicyArgs& a, double part, TokenSums& s) const {
    float g[POLICY_EACH] = {};
    if (masks) {
      double wd = part;
#pragma unroll
      for (int k = 0; k < POLICY_EACH; ++k) {
        if (k < ROWS && a.reduction == PCTC_POLICY_SEQUENCES)
          wd = weight_of(a, part, !VEC && !(masks >> k & 1) ? 1 : a.mask ? a.row_count[row[k]] : length[k]);
        const bool on = masks >> k & 1;
        const float w = (float)wd;
        const float v = policy_token(a, on ? a.sign * x[k] : 0.f, on ? a.sign * o[k] : 0.f, on ? a.sign * q[k] : 0.f, on ? A[k] : 0.f, w, wd, s);
        g[k] = on ? a.sign * w * v : 0.f;
      }
    }
    s.count += __popc(masks);
    if (!a.grad) return;
    if constexpr (VEC) {
      if (length[0] >= 0) *reinterpret_cast<float4*>(a.grad + row[0] * a.ld_grad + col[0]) = make_float4(g[0], g[1], g[2], g[3]);
    } else {
#pragma unroll
      for (int k = 0; k < POLICY_EACH; ++k)
        if (length[k] >= 0) a.grad[row[k] * a.ld_grad + col[k]] = g[k];
    }
  }
};

// A thread's values first, first + step, ... (POLICY_EACH of each of `groups` groups that lie `group` apart) once more where fp32
// was too short for one of them, in 64 bits: gradients, and what the KL terms add to the loss and to their sum.
struct FarSums {
  double loss, kl;
};
__device__ __noinline__ FarSums far_values(const PolicyArgs& a, long long first, int groups, int group, int step, double part) {
  FarSums s{0.0, 0.0};
  for (int j = 0; j < groups * POLICY_EACH; ++j) {
    const long long i = first + (j / POLICY_EACH) * group + (j % POLICY_EACH) * step, n = i / a.T, c = i - n * a.T;
    if (i >= a.total || c >= length_of(a, n) || (a.mask && a.mask[n * a.ld_mask + c] == 0)) continue;
    const double wd = a.reduction == PCTC_POLICY_SEQUENCES ? weight_of(a, part, a.mask ? a.row_count[n] : length_of(a, n)) : part;
    const float x = a.sign * a.logp[n * a.ld_logp + c], A = a.ld_adv ? a.adv[n * a.ld_adv + c] : a.adv[n];
    const float2 d = difference(x, a.sign * a.old_logp[n * a.ld_old + c]);
    const bool none = (A > 0.f && above(d, a.log_high)) || (A < 0.f && above(a.log_low, d)) || (A == 0.f && fabsf(d.x) < CUDART_INF_F);
    double g = none ? 0.0 : -(double)A * exp((double)d.x + (double)d.y);
    if (a.ref) {
      const float x_ref = a.sign * a.ref[n * a.ld_ref + c];
      float kl32, e32;
      kl_terms(x, x_ref, kl32, e32);
      double kl = kl32, e = e32;
      if (!(fabsf(e32) < POLICY_FAR)) {
        const double f = (double)x_ref - (double)x;
        e = expm1(f);
        kl = isinf(e) ? e : e - f;
      }
      // (no 0 * inf where exp(f) overflows for a finite f)
      if (a.kl_weight != 0.f || !(fabsf(x) < CUDART_INF_F && fabsf(x_ref) < CUDART_INF_F)) {
        g -= a.kl_weight * e;
        s.loss += wd * (a.kl_weight * kl);
      }
      s.kl += kl;
    }
    if (a.grad) a.grad[n * a.ld_grad + c] = (float)(a.sign * wd * g);
  }
  return s;
}

__device__ __forceinline__ void write_stats(const PolicyArgs& a, const BlockSums& s) {
  const double n = (double)max(s.count, 1);
  a.stats[0] = (float)s.loss;
  a.stats[1] = (float)(s.kl / n);
  a.stats[2] = (float)((double)s.clipped / n);
  *a.count_out = s.count;
}

template <bool VEC, int GROUPS>
__global__ void __launch_bounds__(POLICY_THREADS) k_policy(const __grid_constant__ PolicyArgs a) {
  __shared__ double shared_part;
  __shared__ bool last;
  const long long tile = (long long)blockIdx.x * (POLICY_THREADS * POLICY_EACH * GROUPS);
  Values<VEC> v[GROUPS];
#pragma unroll
  for (int i = 0; i < GROUPS; ++i) {
    const long long first = tile + i * (POLICY_THREADS * POLICY_EACH);
    v[i].load(a, VEC ? first + threadIdx.x * POLICY_EACH : first + threadIdx.x, VEC ? 1 : POLICY_THREADS);
  }
  wait_for_previous();                           // the inputs are older than the launch before this one; the counts are its own
  Totals t{(int)a.total, (int)a.N};
  if (a.counting) {
    if (threadIdx.x < 32) {
      t = Totals{0, 0};
      const int blocks = a.head->blocks;
#pragma unroll
      for (int i = 0; i < (POLICY_COUNT_BLOCKS + 31) / 32; ++i)
        if (i * 32 + (int)threadIdx.x < blocks) {
          const Totals u = a.head->totals[i * 32 + threadIdx.x];
          t.count += u.count;
          t.rows += u.rows;
        }
      t = warp_sum(t);
      if (threadIdx.x == 0) shared_part = weight_part(a, t);
    }
    __syncthreads();
  }
  const double part = a.counting ? shared_part : weight_part(a, t);
  TokenSums s;
#pragma unroll
  for (int i = 0; i < GROUPS; ++i) v[i].finish(a, part, s);
  FarSums k{(double)s.kl_loss, (double)s.kl};
  if (!held(a, s))
    k = far_values(a, tile + threadIdx.x * (VEC ? POLICY_EACH : 1), GROUPS, POLICY_THREADS * POLICY_EACH, VEC ? 1 : POLICY_THREADS, part);
  BlockSums sums = block_sum<POLICY_THREADS>(k.loss - s.gain, k.kl, s.count, s.clipped);
  if (threadIdx.x == 0) {
    BlockSums* p = a.partial + blockIdx.x;
    __stcg(reinterpret_cast<double2*>(p), make_double2(sums.loss, sums.kl));
    __stcg(reinterpret_cast<int2*>(&p->count), make_int2(sums.count, sums.clipped));
    __threadfence();
    last = atomicAdd(&a.head->ticket, 1u) == gridDim.x - 1;
    __threadfence();
  }
  __syncthreads();
  if (!last) return;
  sums = BlockSums{0.0, 0.0, 0, 0};              // every thread the same blocks, whoever comes last
#pragma unroll 4
  for (long long b = threadIdx.x; b < gridDim.x; b += POLICY_THREADS) {
    const BlockSums* p = a.partial + b;
    const double2 u = __ldcg(reinterpret_cast<const double2*>(p));
    const int2 c = __ldcg(reinterpret_cast<const int2*>(&p->count));
    sums.loss += u.x;
    sums.kl += u.y;
    sums.count += c.x;
    sums.clipped += c.y;
  }
  sums = block_sum<POLICY_THREADS>(sums.loss, sums.kl, sums.count, sums.clipped);
  if (threadIdx.x == 0) write_stats(a, sums);
}

// All of it by one cluster (of one block or more): the counts and the sums cross shared memory.
template <bool VEC>
__global__ void __launch_bounds__(POLICY_SMALL_THREADS) k_policy_small(const __grid_constant__ PolicyArgs a) {
  __shared__ Totals counts;
  __shared__ double shared_part;
  __shared__ BlockSums block_sums;
  cg::cluster_group cluster = cg::this_cluster();
  const int blocks = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const long long thread = rank * POLICY_SMALL_THREADS + threadIdx.x, threads = blocks * POLICY_SMALL_THREADS;
  Values<VEC> v;
  v.load(a, VEC ? thread * POLICY_EACH : thread, VEC ? 1 : threads);
  Totals t{(int)a.total, (int)a.N};
  if (a.counting) {
    t = count_all<POLICY_SMALL_THREADS>(a, rank, blocks);
    if (threadIdx.x == 0) counts = t;
    cluster.sync();                              // the row counts in global memory are visible, too
    if (threadIdx.x < 32) {
      t = warp_sum((int)threadIdx.x < blocks ? *cluster.map_shared_rank(&counts, (int)threadIdx.x) : Totals{0, 0});
      if (threadIdx.x == 0) shared_part = weight_part(a, t);
    }
    __syncthreads();
  }
  TokenSums s;
  const double part = a.counting ? shared_part : weight_part(a, t);
  v.finish(a, part, s);
  FarSums k{(double)s.kl_loss, (double)s.kl};
  if (!held(a, s)) k = far_values(a, VEC ? thread * POLICY_EACH : thread, 1, 0, VEC ? 1 : (int)threads, part);
  BlockSums sums = block_sum<POLICY_SMALL_THREADS>(k.loss - s.gain, k.kl, s.count, s.clipped);
  if (blocks == 1) {
    if (threadIdx.x == 0) write_stats(a, sums);
    return;
  }
  if (threadIdx.x == 0) block_sums = sums;
  cluster.sync();
  if (rank == 0 && threadIdx.x == 0) {
    for (int b = 1; b < blocks; ++b) {
      const BlockSums* other = cluster.map_shared_rank(&block_sums, b);
      sums.loss += other->loss;
      sums.kl += other->kl;
      sums.count += other->count;
      sums.clipped += other->clipped;
    }
    write_stats(a, sums);
  }
  cluster.sync();                                // nobody leaves before all have been read
}

// ---------------------------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------------------------
struct PolicyPlan {
  bool many;
  long long blocks;
  size_t rows, partial, total;
};
PolicyPlan policy_plan(const pctc_policy_t* p) {
  PolicyPlan w;
  w.many = p->N * p->T > POLICY_MANY;
  const long long tile = POLICY_THREADS * POLICY_EACH * (w.many ? 2 : 1);
  w.blocks = (p->N * p->T + tile - 1) / tile;
  w.rows = (sizeof(PolicyHead) + 255) / 256 * 256;
  w.partial = w.rows + ((size_t)p->N * 4 + 255) / 256 * 256;
  w.total = w.partial + (size_t)w.blocks * sizeof(BlockSums);
  return w;
}
float2 number_and_rest(double v) {
  const float x = (float)v;
  return make_float2(x, std::isinf(x) ? 0.f : (float)(v - (double)x));
}
pctc_status_t check_policy(const pctc_policy_t* p) {
  if (!p || p->N < 1 || p->T < 1) return PCTC_ERR_INVALID_ARG;
  if (p->N > 0x7fffffffLL / p->T) return PCTC_ERR_UNSUPPORTED;
  if (!(p->clip_low >= 0.0 && p->clip_low <= 1.0) || !(p->clip_high >= 0.0) || !std::isfinite((float)p->kl_weight)) return PCTC_ERR_INVALID_ARG;
  if (p->reduction != PCTC_POLICY_TOKENS && p->reduction != PCTC_POLICY_SEQUENCES && p->reduction != PCTC_POLICY_SUM)
    return PCTC_ERR_INVALID_ARG;
  return PCTC_OK;
}

}  // namespace
}  // namespace pctc

using namespace pctc;

extern "C" {

pctc_status_t pctc_policy_workspace_bytes(const pctc_policy_t* p, size_t* bytes_out) {
  if (!bytes_out) return PCTC_ERR_INVALID_ARG;
  const pctc_status_t st = check_policy(p);
  if (st != PCTC_OK) return st;
  *bytes_out = policy_plan(p).total;
  return PCTC_OK;
}

pctc_status_t pctc_policy_loss(const pctc_policy_t* p, const float* logp, const float* old_logp, const float* ref_logp,
                               const float* advantages, const uint8_t* mask, const int32_t* lengths, float* grad,
                               float* stats, int32_t* count, void* workspace, size_t workspace_bytes, void* stream_v) {
  const pctc_status_t st = check_policy(p);
  if (st != PCTC_OK) return st;
  if (!logp || !old_logp || !advantages || !stats || !count || !workspace || ((size_t)workspace & 255)) return PCTC_ERR_INVALID_ARG;
  if (((size_t)logp | (size_t)old_logp | (size_t)ref_logp | (size_t)advantages | (size_t)lengths | (size_t)grad | (size_t)stats |
       (size_t)count) & 3)
    return PCTC_ERR_INVALID_ARG;
  const PolicyPlan w = policy_plan(p);
  if (workspace_bytes < w.total) return PCTC_ERR_WORKSPACE_TOO_SMALL;
  const Rows in[] = {{logp, p->N, p->ld_logp, p->T, 4},
                     {old_logp, p->N, p->ld_old, p->T, 4},
                     {ref_logp, p->N, p->ld_ref, p->T, 4},
                     {advantages, p->ld_adv ? p->N : 1, p->ld_adv ? p->ld_adv : p->N, p->ld_adv ? p->T : p->N, 4},
                     {mask, p->N, p->ld_mask, p->T, 1},
                     {lengths, 1, p->N, p->N, 4}};
  const Rows out[] = {{grad, p->N, p->ld_grad, p->T, 4},
                      {stats, 1, 3, 3, 4},
                      {count, 1, 1, 1, 4},
                      {workspace, 1, (long long)w.total, (long long)w.total, 1}};
  for (const Rows& r : in) {
    if (r.p && r.ld < r.cols && r.rows > 1) return PCTC_ERR_INVALID_ARG;
    if (r.p && r.ld > MAX_ELEMENTS / r.rows) return PCTC_ERR_UNSUPPORTED;
  }
  if (grad && p->ld_grad < p->T && p->N > 1) return PCTC_ERR_INVALID_ARG;
  if (grad && p->ld_grad > MAX_ELEMENTS / p->N) return PCTC_ERR_UNSUPPORTED;
  for (int i = 0; i < 4; ++i) {
    for (const Rows& r : in)
      if (out[i].overlaps(r)) return PCTC_ERR_INVALID_ARG;
    for (int j = 0; j < i; ++j)
      if (out[i].overlaps(out[j])) return PCTC_ERR_INVALID_ARG;
  }

  PolicyArgs a = {};
  a.logp = logp;
  a.old_logp = old_logp;
  a.ref = ref_logp;
  a.adv = advantages;
  a.mask = mask;
  a.lengths = lengths;
  a.grad = grad;
  a.stats = stats;
  a.count_out = count;
  a.head = (PolicyHead*)workspace;
  a.row_count = mask && p->reduction == PCTC_POLICY_SEQUENCES ? (int*)((char*)workspace + w.rows) : nullptr;
  a.partial = (BlockSums*)((char*)workspace + w.partial);
  a.N = p->N;
  a.T = p->T;
  a.total = p->N * p->T;
  a.ld_logp = p->ld_logp;
  a.ld_old = p->ld_old;
  a.ld_ref = p->ld_ref;
  a.ld_adv = p->ld_adv;
  a.ld_mask = p->ld_mask;
  a.ld_grad = p->ld_grad;
  a.log_low = number_and_rest(std::log1p(-p->clip_low));
  a.log_high = number_and_rest(std::log1p(p->clip_high));
  a.low = 1.0 - p->clip_low;
  a.high = 1.0 + p->clip_high;
  a.kl_weight = (float)p->kl_weight;
  a.sign = p->negated ? -1.f : 1.f;
  a.reduction = p->reduction;
  a.counting = (mask || lengths) && p->reduction != PCTC_POLICY_SUM;
  // groups of four values of one row, 16-byte aligned in every array
  const bool vec = p->T % 4 == 0 && (((size_t)logp | (size_t)old_logp | (size_t)ref_logp | (size_t)grad) & 15) == 0 && ((size_t)mask & 3) == 0 &&
                   ((p->ld_logp | p->ld_old | (ref_logp ? p->ld_ref : 0) | (mask ? p->ld_mask : 0) | (grad ? p->ld_grad : 0)) & 3) == 0 &&
                   (!p->ld_adv || (((size_t)advantages & 15) == 0 && (p->ld_adv & 3) == 0));
  cudaStream_t stream = (cudaStream_t)stream_v;
  if (a.total <= POLICY_SMALL) {
    auto kernel = vec ? k_policy_small<true> : k_policy_small<false>;
    if (a.total <= POLICY_SMALL_THREADS * POLICY_EACH) {           // a cluster of one
      kernel<<<1, POLICY_SMALL_THREADS, 0, stream>>>(a);
      return cudaGetLastError() == cudaSuccess ? PCTC_OK : PCTC_ERR_CUDA;
    }
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = POLICY_CLUSTER;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(POLICY_CLUSTER);
    cfg.blockDim = dim3(POLICY_SMALL_THREADS);
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, a) == cudaSuccess ? PCTC_OK : PCTC_ERR_CUDA;
  }
  const long long threads = !a.counting ? 1 : !mask || a.T <= POLICY_SHORT_ROW ? a.N : a.T <= POLICY_LONG_ROW ? a.N * 32 : a.N * POLICY_THREADS;
  const long long blocks = (threads + POLICY_THREADS - 1) / POLICY_THREADS;
  k_policy_count<<<(unsigned)(blocks < POLICY_COUNT_BLOCKS ? blocks : POLICY_COUNT_BLOCKS), POLICY_THREADS, 0, stream>>>(a);
  if (cudaGetLastError() != cudaSuccess) return PCTC_ERR_CUDA;
  auto kernel = w.many ? (vec ? k_policy<true, 2> : k_policy<false, 2>) : vec ? k_policy<true, 1> : k_policy<false, 1>;
  return launch_behind(kernel, (unsigned)w.blocks, POLICY_THREADS, 0, stream, a) == cudaSuccess ? PCTC_OK : PCTC_ERR_CUDA;
}

}  // extern "C"
