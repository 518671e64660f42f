// Clipped policy loss over log-probabilities, with a KL term, and its gradient.  For a counted token with d = new - old,
// r = exp(d), advantage A and e = exp(ref - new) - 1:
//   clipped  <=>  A > 0 and r > 1 + high,  or  A < 0 and r < 1 - low
//   loss     =    -A r   (clipped: -A (1 + high), -A (1 - low))   + kl_weight (e - (ref - new))
//   d loss / d new  =  (clipped ? 0 : -A r) - kl_weight e,
// weighted by 1 / count, by 1 / (count of the row * rows with a count), or by 1.
//
// The weights need the counts before the first gradient can be written: where a mask or lengths are given,
// k_policy_count goes over them first (a quarter of a byte and less for a byte that the second pass moves).  k_policy then
// reads every value once.  Few values are done by one cluster in one launch (k_policy_small).  Sums are 64 bits, in a fixed
// order.  Large calls are bound by HBM, small ones by the launch.
#include "../../include/prunedctc.h"
#include "pctc_internal.h"

#include <cooperative_groups.h>

#include <cmath>

namespace cg = cooperative_groups;

namespace pctc {
namespace {

constexpr int POLICY_THREADS = 256;
constexpr int POLICY_EACH = 4;                   // values a thread
constexpr int POLICY_SMALL_THREADS = 512;
constexpr int POLICY_CLUSTER = 8;
constexpr long long POLICY_SMALL = 32768;        // up to so many values one cluster does all
constexpr int POLICY_SHORT_ROW = 32;             // rows up to this length are counted by one thread each

struct Totals {
  long long count;                               // counted tokens
  long long rows;                                // rows that have one
};
struct PolicyHead {                              // start of the workspace
  Totals totals;
  unsigned ticket;
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
  double* partial;                               // [blocks][3]
  long long N, T, total;
  long long ld_logp, ld_old, ld_ref, ld_adv, ld_mask, ld_grad;   // ld_adv 0: one advantage a row
  double log_low, log_high;                      // where ratios are clipped
  float low, high, kl_weight, sign;
  int reduction;
  int counting;                                  // counts come from k_policy_count
};

__device__ __forceinline__ int length_of(const PolicyArgs& a, long long n) {
  return a.lengths ? (int)min((long long)max(a.lengths[n], 0), a.T) : (int)a.T;
}

// The sums of one token.
struct TokenSums {
  double loss = 0.0, kl = 0.0;
  int clipped = 0;
};

// exp(d) - 1 - d and exp(d) - 1.  Near 0 the first by its series (d^2 (1/2 + d/6 + ... + d^6/40320): the next term is under
// 1e-9 of the sum for |d| < 1/4), where the difference would cancel.
__device__ __forceinline__ void kl_terms(double d, float& kl, float& e) {
  const float hi = (float)d;
  const float lo = isinf(hi) ? 0.f : (float)(d - (double)hi);
  e = expm1f(hi);
  if (!isinf(e)) e = fmaf(e + 1.f, lo, e);
  if (fabsf(hi) < 0.25f) {
    float s = fmaf(hi, 1.f / 40320.f, 1.f / 5040.f);
    s = fmaf(hi, s, 1.f / 720.f);
    s = fmaf(hi, s, 1.f / 120.f);
    s = fmaf(hi, s, 1.f / 24.f);
    s = fmaf(hi, s, 1.f / 6.f);
    s = fmaf(hi, s, 0.5f);
    kl = hi * hi * s;
  } else {
    kl = isinf(e) ? e : (e - hi) - lo;
  }
}

// One counted token: adds to the sums and returns its gradient, both before the weight.
__device__ __forceinline__ float policy_token(const PolicyArgs& a, float x, float x_old, float x_ref, float A, double w,
                                              TokenSums& s) {
  // differences in 64 bits: whether a ratio is clipped does not depend on their rounding
  const double d = (double)a.sign * ((double)x - (double)x_old);
  const float hi = (float)d;
  const float lo = isinf(hi) ? 0.f : (float)(d - (double)hi);
  const float r0 = expf(hi), r = isinf(r0) ? r0 : fmaf(r0, lo, r0);
  const bool over = A > 0.f && d > a.log_high, under = A < 0.f && d < a.log_low, clipped = over || under;
  const float used = over ? a.high : under ? a.low : r;
  const float gain = A == 0.f ? (r == r ? 0.f : r) : A * used;   // no 0 * inf where the ratio overflows
  float loss = -gain, g = clipped ? 0.f : -gain;
  if (a.ref) {
    float kl, e;
    kl_terms((double)a.sign * ((double)x_ref - (double)x), kl, e);
    loss = fmaf(a.kl_weight, kl, loss);
    g = fmaf(-a.kl_weight, e, g);
    s.kl += (double)kl;
  }
  s.loss += w * (double)loss;
  s.clipped += clipped ? 1 : 0;
  return g;
}

// The weight of the tokens of a row with `count` of them.
__device__ __forceinline__ float weight_of(const PolicyArgs& a, const Totals& t, long long count) {
  if (a.reduction == PCTC_POLICY_SUM) return 1.f;
  if (a.reduction == PCTC_POLICY_TOKENS) return 1.f / (float)max(t.count, 1ll);
  return 1.f / ((float)max(count, 1ll) * (float)max(t.rows, 1ll));
}

// Counts the tokens of row n with `lanes` threads (1, or a warp).
template <int LANES>
__device__ __forceinline__ int count_row(const PolicyArgs& a, long long n) {
  const int len = length_of(a, n);
  if (!a.mask) return len;
  const unsigned char* m = a.mask + n * a.ld_mask;
  int c = 0;
  for (int t = LANES == 1 ? 0 : (int)(threadIdx.x & 31); t < len; t += LANES) c += m[t] != 0;
  return LANES == 1 ? c : __reduce_add_sync(0xffffffffu, c);
}
// Rows first, first + step, ...: `worker` is one of `workers` threads (or warps).
template <int LANES>
__device__ __forceinline__ Totals count_rows(const PolicyArgs& a, long long worker, long long workers) {
  Totals t{0, 0};
  const bool writes = LANES == 1 || (threadIdx.x & 31) == 0;
  for (long long n = worker; n < a.N; n += workers) {
    const int c = count_row<LANES>(a, n);
    if (!writes) continue;
    if (a.row_count) a.row_count[n] = c;
    t.count += c;
    t.rows += c > 0;
  }
  return t;
}

template <int THREADS, typename V>
__device__ __forceinline__ V block_sum(V v, V* scratch) {          // valid in thread 0; scratch [THREADS / 32]
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) v += __shfl_down_sync(0xffffffffu, v, d);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = v;
  __syncthreads();
  V sum = 0;
  if (threadIdx.x == 0)
    for (int i = 0; i < THREADS / 32; ++i) sum += scratch[i];
  return sum;
}

__global__ void __launch_bounds__(POLICY_THREADS) k_policy_count(const PolicyArgs a) {
  __shared__ long long scratch[POLICY_THREADS / 32];
  const long long thread = (long long)blockIdx.x * POLICY_THREADS + threadIdx.x, threads = (long long)gridDim.x * POLICY_THREADS;
  const Totals t = a.T <= POLICY_SHORT_ROW ? count_rows<1>(a, thread, threads) : count_rows<32>(a, thread >> 5, threads >> 5);
  const long long count = block_sum<POLICY_THREADS>(t.count, scratch), rows = block_sum<POLICY_THREADS>(t.rows, scratch);
  if (threadIdx.x == 0) {                        // whole numbers: their order does not matter
    atomicAdd((unsigned long long*)&a.head->totals.count, (unsigned long long)count);
    atomicAdd((unsigned long long*)&a.head->totals.rows, (unsigned long long)rows);
  }
}

// Values first, first + step, ... of the flattened array, `each` of them.
template <int EACH>
__device__ __forceinline__ void policy_values(const PolicyArgs& a, const Totals& t, long long first, long long step, TokenSums& s) {
  float x[EACH], o[EACH], q[EACH], A[EACH];
  bool counted[EACH], inside[EACH];
  long long rows[EACH];
  int cols[EACH];
#pragma unroll
  for (int k = 0; k < EACH; ++k) {
    const long long i = first + k * step;
    inside[k] = i < a.total;
    const long long n = (unsigned)i / (unsigned)a.T;         // fewer than 2^31 values
    rows[k] = n;
    cols[k] = (int)(i - n * a.T);
    counted[k] = inside[k] && cols[k] < length_of(a, n) && (!a.mask || a.mask[n * a.ld_mask + cols[k]] != 0);
    if (!counted[k]) continue;
    x[k] = a.logp[n * a.ld_logp + cols[k]];
    o[k] = a.old_logp[n * a.ld_old + cols[k]];
    if (a.ref) q[k] = a.ref[n * a.ld_ref + cols[k]];
    A[k] = a.ld_adv ? a.adv[n * a.ld_adv + cols[k]] : a.adv[n];
  }
#pragma unroll
  for (int k = 0; k < EACH; ++k) {
    if (!inside[k]) continue;
    float g = 0.f;
    if (counted[k]) {
      const float w = weight_of(a, t, a.reduction != PCTC_POLICY_SEQUENCES ? 0
                                      : a.mask ? a.row_count[rows[k]] : length_of(a, rows[k]));
      g = a.sign * w * policy_token(a, x[k], o[k], q[k], A[k], (double)w, s);
    }
    if (a.grad) a.grad[rows[k] * a.ld_grad + cols[k]] = g;
  }
}

__device__ __forceinline__ void write_stats(const PolicyArgs& a, const Totals& t, double loss, double kl, double clipped) {
  const double n = (double)max(t.count, 1ll);
  a.stats[0] = (float)loss;
  a.stats[1] = (float)(kl / n);
  a.stats[2] = (float)(clipped / n);
  *a.count_out = (int)t.count;
}

__global__ void __launch_bounds__(POLICY_THREADS) k_policy(const PolicyArgs a) {
  __shared__ double scratch[POLICY_THREADS / 32];
  __shared__ bool last;
  const Totals t = a.counting ? a.head->totals : Totals{a.total, a.N};
  TokenSums s;
  policy_values<POLICY_EACH>(a, t, (long long)blockIdx.x * (POLICY_THREADS * POLICY_EACH) + threadIdx.x, POLICY_THREADS, s);
  const double loss = block_sum<POLICY_THREADS>(s.loss, scratch), kl = block_sum<POLICY_THREADS>(s.kl, scratch),
               clipped = block_sum<POLICY_THREADS>((double)s.clipped, scratch);
  if (threadIdx.x == 0) {
    double* p = a.partial + 3ll * blockIdx.x;
    __stcg(p, loss);
    __stcg(p + 1, kl);
    __stcg(p + 2, clipped);
    __threadfence();
    last = atomicAdd(&a.head->ticket, 1u) == gridDim.x - 1;
    __threadfence();
  }
  __syncthreads();
  if (!last) return;
  double sum[3] = {0.0, 0.0, 0.0};               // every thread the same blocks, whoever comes last
  for (long long b = threadIdx.x; b < gridDim.x; b += POLICY_THREADS)
#pragma unroll
    for (int j = 0; j < 3; ++j) sum[j] += __ldcg(a.partial + 3 * b + j);
#pragma unroll
  for (int j = 0; j < 3; ++j) sum[j] = block_sum<POLICY_THREADS>(sum[j], scratch);
  if (threadIdx.x == 0) write_stats(a, t, sum[0], sum[1], sum[2]);
}

// All of it by one cluster (of one block or more): the counts and the sums cross shared memory.
__global__ void __launch_bounds__(POLICY_SMALL_THREADS) k_policy_small(const PolicyArgs a) {
  __shared__ double scratch[POLICY_SMALL_THREADS / 32];
  __shared__ long long whole[POLICY_SMALL_THREADS / 32];
  __shared__ Totals counts;
  __shared__ double sums[3];
  cg::cluster_group cluster = cg::this_cluster();
  const int blocks = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const long long thread = rank * POLICY_SMALL_THREADS + threadIdx.x, threads = blocks * POLICY_SMALL_THREADS;
  Totals t{a.total, a.N};
  if (a.counting) {
    const Totals mine = a.T <= POLICY_SHORT_ROW ? count_rows<1>(a, thread, threads) : count_rows<32>(a, thread >> 5, threads >> 5);
    const long long count = block_sum<POLICY_SMALL_THREADS>(mine.count, whole), rows = block_sum<POLICY_SMALL_THREADS>(mine.rows, whole);
    if (threadIdx.x == 0) counts = Totals{count, rows};
    cluster.sync();                              // the row counts in global memory are visible, too
    t = Totals{0, 0};
    for (int b = 0; b < blocks; ++b) {
      const Totals* other = cluster.map_shared_rank(&counts, b);
      t.count += other->count;
      t.rows += other->rows;
    }
  }
  TokenSums s;
  for (long long i = thread; i < a.total; i += threads * POLICY_EACH) policy_values<POLICY_EACH>(a, t, i, threads, s);
  const double loss = block_sum<POLICY_SMALL_THREADS>(s.loss, scratch), kl = block_sum<POLICY_SMALL_THREADS>(s.kl, scratch),
               clipped = block_sum<POLICY_SMALL_THREADS>((double)s.clipped, scratch);
  if (threadIdx.x == 0) {
    sums[0] = loss;
    sums[1] = kl;
    sums[2] = clipped;
  }
  cluster.sync();
  if (rank == 0 && threadIdx.x == 0) {
    double all[3] = {0.0, 0.0, 0.0};
    for (int b = 0; b < blocks; ++b) {
      const double* other = cluster.map_shared_rank(&sums[0], b);
      for (int j = 0; j < 3; ++j) all[j] += other[j];
    }
    write_stats(a, t, all[0], all[1], all[2]);
  }
  cluster.sync();                                // nobody leaves before all have been read
}

// ---------------------------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------------------------
struct PolicyPlan {
  long long blocks;
  size_t rows, partial, total;
};
PolicyPlan policy_plan(const pctc_policy_t* p) {
  PolicyPlan w;
  w.blocks = (p->N * p->T + POLICY_THREADS * POLICY_EACH - 1) / (POLICY_THREADS * POLICY_EACH);
  w.rows = 256;
  w.partial = w.rows + ((size_t)p->N * 4 + 255) / 256 * 256;
  w.total = w.partial + (size_t)w.blocks * 3 * sizeof(double);
  return w;
}
pctc_status_t check_policy(const pctc_policy_t* p) {
  if (!p || p->N < 1 || p->T < 1) return PCTC_ERR_INVALID_ARG;
  if (p->N > 0x7fffffffLL / p->T) return PCTC_ERR_UNSUPPORTED;
  if (!(p->clip_low >= 0.0 && p->clip_low <= 1.0) || !(p->clip_high >= 0.0) || !std::isfinite(p->kl_weight)) return PCTC_ERR_INVALID_ARG;
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
  a.partial = (double*)((char*)workspace + w.partial);
  a.N = p->N;
  a.T = p->T;
  a.total = p->N * p->T;
  a.ld_logp = p->ld_logp;
  a.ld_old = p->ld_old;
  a.ld_ref = p->ld_ref;
  a.ld_adv = p->ld_adv;
  a.ld_mask = p->ld_mask;
  a.ld_grad = p->ld_grad;
  a.log_low = std::log1p(-p->clip_low);
  a.log_high = std::log1p(p->clip_high);
  a.low = (float)(1.0 - p->clip_low);
  a.high = (float)(1.0 + p->clip_high);
  a.kl_weight = (float)p->kl_weight;
  a.sign = p->negated ? -1.f : 1.f;
  a.reduction = p->reduction;
  a.counting = mask || lengths;
  cudaStream_t stream = (cudaStream_t)stream_v;
  if (a.total <= POLICY_SMALL) {
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = a.total <= POLICY_SMALL_THREADS * POLICY_EACH ? 1 : POLICY_CLUSTER;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(attr[0].val.clusterDim.x);
    cfg.blockDim = dim3(POLICY_SMALL_THREADS);
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, k_policy_small, a) == cudaSuccess ? PCTC_OK : PCTC_ERR_CUDA;
  }
  if (cudaMemsetAsync(workspace, 0, sizeof(PolicyHead), stream) != cudaSuccess) return PCTC_ERR_CUDA;
  if (a.counting) {
    const long long workers = a.T <= POLICY_SHORT_ROW ? a.N : a.N * 32, blocks = (workers + POLICY_THREADS - 1) / POLICY_THREADS;
    k_policy_count<<<(unsigned)(blocks < 148 * 8 ? blocks : 148 * 8), POLICY_THREADS, 0, stream>>>(a);
    if (cudaGetLastError() != cudaSuccess) return PCTC_ERR_CUDA;
  }
  k_policy<<<(unsigned)w.blocks, POLICY_THREADS, 0, stream>>>(a);
  return cudaGetLastError() == cudaSuccess ? PCTC_OK : PCTC_ERR_CUDA;
}

}  // extern "C"
