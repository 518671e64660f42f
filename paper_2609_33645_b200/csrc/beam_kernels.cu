// Beam search's selection over beams and vocabulary, and the reordering of the states that go with it.
//
// Selection.  With lse_b the log-sum-exp of beam b's logits,
//   cand(b, v) = score_b + (x_bv - lse_b),
// and the K largest of an utterance's B * V candidates go on; among equals the lowest b * V + v.  Every logit
// has to be read once for lse_b, and a candidate can be judged only after that: what is kept of the one
// pass over HBM is the maximum of every 512 logits.  The K best candidates lie in the K blocks with the
// best maxima (K better ones stand against any other), so a few blocks are read again, from L2, and only there
// single logits are compared.
//
// Two launches.  k_beam_stream makes the pass: short CTAs of 4 warps, each for a stretch of one row, in any order and
// on any SM.  k_beam_select then needs the maxima only: one CTA of 16 warps an utterance (a cluster of up to 8 where they
// are many), which find the blocks that matter, read those, and rank the candidates.  A first version did both in one
// launch of a cluster per utterance; its clusters left SMs idle and all had their tails at the same time (utterances x
// beams x 151,936: 64 x 8 bf16 55 us against 41, 2 x 8 bf16 24.5 against 13.0, 1 x 4 fp32 14.4 against 11.1).
//
// Measured: 64 x 8 x 151,936 bf16 with a tenth of the beams ended, 140 MB: 41.7 us (21 at the rate of a copy), of which the
// stream takes 31 and the ranking 10; 1 x 4 fp32: 11.4 us, of which 3 and 8.  The stream is bound by no single thing:
// special function unit 60% busy (16 exponentials a cycle and SM are hardly more than the 12 bf16 logits that HBM
// delivers), issue slots 60%, HBM 64% of a copy's rate.  More blocks in flight, more or fewer warps a CTA, and longer
// stretches measured the same.  The ranking is a chain of about ten dependent steps of 0.3 to 1 us each.
//
// Exponentials and the sums of 16 of them are fp32, of differences from a running maximum (so that their errors are
// relative to the difference, not to the logit); everything after that, and every comparison of candidates, is 64
// bits.  So the order within a beam is that of its logits, and candidates of different beams are ordered as far as the
// log-sum-exps tell them apart (RunningSum: within 2e-7 measured, 6e-7 + 1.4e-7 ln V at most).  Scores are rounded to fp32 when
// they are stored.
#include "../../include/prunedctc.h"
#include "pctc_internal.h"

#include <cooperative_groups.h>
#include <math_constants.h>

#include <new>
#include <utility>

namespace cg = cooperative_groups;

namespace pctc {
namespace {

constexpr int SEL_MAX = 32;                       // beams in and out
constexpr int SEL_WARPS = 16, SEL_THREADS = SEL_WARPS * 32;
constexpr int SEL_MAX_CLUSTER = 8;
constexpr int STREAM_WARPS = 4;
constexpr int STREAM_CTAS = 4 * 148;              // CTAs of the first launch that are worth shorter stretches: four an SM
constexpr int SEL_BLOCK = 512;                    // logits per maximum: 16 a lane
constexpr int SEL_LANE = SEL_BLOCK / 32;
constexpr int SEL_MAX_BLOCKS = 512;               // blocks a CTA reads again
constexpr int SEL_MAX_CAND = 2048;
constexpr long long SEL_MAX_V = 1 << 21;
constexpr int SEL_MAX_DYN = SEL_MAX * (int)(SEL_MAX_V / SEL_BLOCK) / SEL_MAX_CLUSTER * 4;   // maxima of a CTA

struct SelArgs {
  const void* logits;
  long long stride_n, stride_b;                   // elements
  const float* scores;
  const unsigned char* finished;                  // or null
  int N, B, K, V, eos, nb;                        // nb: blocks a row
  float* scores_out;
  int *parents, *tokens;
  unsigned char* finished_out;
  int* flags;
  // what the first launch leaves for the second, by row (utterance, beam)
  float* maxima;                                  // [N * B, nb]
  float* part_m;                                  // [N * B, parts]: reference and sum of exponentials of each CTA's stretch
  double* part_s;
  int parts, per;                                 // CTAs a row, blocks a warp
};

struct Cand {
  double score;
  unsigned long long at;                          // b << 32 | v
};
__device__ __forceinline__ bool before(const Cand& a, const Cand& b) {
  return a.score > b.score || (a.score == b.score && a.at < b.at);
}

// Maxima here are NaN if an operand is: a block with a NaN shows by its maximum.
__device__ __forceinline__ float warp_max(float v) {
  float r;
  asm("redux.sync.max.NaN.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
  return r;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ __forceinline__ float lane_max(const float (&x)[SEL_LANE]) {
  float m = max3(x[0], x[1], x[2]), n = max3(x[3], x[4], x[5]);
#pragma unroll
  for (int e = 6; e + 3 < SEL_LANE; e += 4) {
    m = max3(m, x[e], x[e + 1]);
    n = max3(n, x[e + 2], x[e + 3]);
  }
  return max3(m, n, max3(x[SEL_LANE - 2], x[SEL_LANE - 1], x[SEL_LANE - 1]));
}
static_assert(SEL_LANE == 16, "lane_max");
__device__ __forceinline__ float exp2_approx(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

struct Pair { float a, b; };
__device__ __forceinline__ Pair add2(Pair x, Pair y) {
  Pair r;
  asm("{\n\t.reg .b64 u, v;\n\tmov.b64 u, {%2, %3};\n\tmov.b64 v, {%4, %5};\n\tadd.rn.f32x2 u, u, v;\n\tmov.b64 {%0, %1}, u;\n\t}"
      : "=f"(r.a), "=f"(r.b) : "f"(x.a), "f"(x.b), "f"(y.a), "f"(y.b));
  return r;
}
__device__ __forceinline__ Pair mul2(Pair x, Pair y) {
  Pair r;
  asm("{\n\t.reg .b64 u, v;\n\tmov.b64 u, {%2, %3};\n\tmov.b64 v, {%4, %5};\n\tmul.rn.f32x2 u, u, v;\n\tmov.b64 {%0, %1}, u;\n\t}"
      : "=f"(r.a), "=f"(r.b) : "f"(x.a), "f"(x.b), "f"(y.a), "f"(y.b));
  return r;
}
__device__ __forceinline__ Pair both(float v) { return Pair{v, v}; }

// Sum of exp(x_i - z) of a lane's values: packed differences, products and sums, one ex2 each.
__device__ __forceinline__ float lane_exp(const float (&x)[SEL_LANE], float z) {
  Pair acc0 = both(0.f), acc1 = both(0.f);
#pragma unroll
  for (int e = 0; e < SEL_LANE; e += 4) {
    const Pair y = mul2(add2(Pair{x[e], x[e + 1]}, both(-z)), both(1.44269504f));
    const Pair w = mul2(add2(Pair{x[e + 2], x[e + 3]}, both(-z)), both(1.44269504f));
    acc0 = add2(acc0, Pair{exp2_approx(y.a), exp2_approx(y.b)});
    acc1 = add2(acc1, Pair{exp2_approx(w.a), exp2_approx(w.b)});
  }
  acc0 = add2(acc0, acc1);
  return acc0.a + acc0.b;
}

// A lane's 16 of a block of 512 logits: 16-byte loads where every row starts on a 16-byte boundary, else one by one.
// load() takes the lane's first one; load_part() the block's first one, of which `left` exist (the others read -inf).
template <typename T, bool VEC>
struct Block;
template <>
struct Block<__nv_bfloat16, true> {
  uint4 r[2];
  static __device__ __forceinline__ int index(int lane, int e) { return (e < 8 ? 0 : 248) + lane * 8 + e; }
  static __device__ __forceinline__ int first(int lane) { return lane * 8; }
  __device__ __forceinline__ void load(const __nv_bfloat16* p) {
    r[0] = ((const uint4*)p)[0];
    r[1] = ((const uint4*)p)[32];
  }
  __device__ __forceinline__ void load_part(const __nv_bfloat16* p, int left, int lane) {
    unsigned w[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int i = index(lane, 2 * e);
      const unsigned lo = i < left ? ((const unsigned short*)p)[i] : 0xff80u;
      const unsigned hi = i + 1 < left ? ((const unsigned short*)p)[i + 1] : 0xff80u;
      w[e] = lo | hi << 16;
    }
    r[0] = make_uint4(w[0], w[1], w[2], w[3]);
    r[1] = make_uint4(w[4], w[5], w[6], w[7]);
  }
  __device__ __forceinline__ void get(float (&x)[SEL_LANE]) const {
    const unsigned w[8] = {r[0].x, r[0].y, r[0].z, r[0].w, r[1].x, r[1].y, r[1].z, r[1].w};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      x[2 * e] = __uint_as_float(w[e] << 16);
      x[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
    }
  }
};
template <>
struct Block<float, true> {
  float4 r[4];
  static __device__ __forceinline__ int index(int lane, int e) { return e / 4 * 128 + lane * 4 + e % 4; }
  static __device__ __forceinline__ int first(int lane) { return lane * 4; }
  __device__ __forceinline__ void load(const float* p) {
#pragma unroll
    for (int q = 0; q < 4; ++q) r[q] = ((const float4*)p)[32 * q];
  }
  static __device__ __forceinline__ float one(const float* p, int i, int left) { return i < left ? p[i] : -CUDART_INF_F; }
  __device__ __forceinline__ void load_part(const float* p, int left, int lane) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int i = index(lane, 4 * q);
      r[q] = make_float4(one(p, i, left), one(p, i + 1, left), one(p, i + 2, left), one(p, i + 3, left));
    }
  }
  __device__ __forceinline__ void get(float (&x)[SEL_LANE]) const {
#pragma unroll
    for (int q = 0; q < 4; ++q) { x[4 * q] = r[q].x; x[4 * q + 1] = r[q].y; x[4 * q + 2] = r[q].z; x[4 * q + 3] = r[q].w; }
  }
};
template <typename T>
struct Block<T, false> {
  T r[SEL_LANE];
  static __device__ __forceinline__ int index(int lane, int e) { return e * 32 + lane; }
  static __device__ __forceinline__ int first(int lane) { return lane; }
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int e = 0; e < SEL_LANE; ++e) r[e] = p[e * 32];
  }
  __device__ __forceinline__ void load_part(const T* p, int left, int lane) {
#pragma unroll
    for (int e = 0; e < SEL_LANE; ++e) r[e] = index(lane, e) < left ? p[index(lane, e)] : (T)(-CUDART_INF_F);
  }
  __device__ __forceinline__ void get(float (&x)[SEL_LANE]) const {
#pragma unroll
    for (int e = 0; e < SEL_LANE; ++e) x[e] = (float)r[e];
  }
};

// Running sum of exponentials of a lane, of differences from the running maximum `ref`.  A lane's 16 of a block are added
// in fp32; the sum over blocks and the factor that follows a new maximum are 64 bits.  The largest logit counts exactly 1, so
// a log-sum-exp is never below it.  Another one, d below it, is off by the rounding of the difference, of the product and of
// log2 e (together under 1.4e-7 |d|) and by the 2^-22 of ex2, times its share of the sum; the five roundings of the 16 add
// 5 x 2^-24.  A reference that was followed only when the maximum was 4 ahead measured the same time (64 x 8 bf16: 45.1 us),
// with errors of up to 6e-7 in rows of one peak, against 6e-8.
struct RunningSum {
  float ref;
  double sum;
  __device__ __forceinline__ void clear() { ref = -CUDART_INF_F; sum = 0.0; }
  // adds a lane's share of a block; m: the block's maximum
  __device__ __forceinline__ void add(const float (&x)[SEL_LANE], float m) {
    if (!(m <= ref)) {                           // a new maximum, or a NaN
      if (sum != 0.0) sum *= exp((double)ref - (double)m);
      ref = m;
    }
    sum += (double)lane_exp(x, ref == -CUDART_INF_F ? 0.f : ref);
  }
  __device__ __forceinline__ double total() const {
    double s = sum;
#pragma unroll
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    return s;
  }
};

struct SelShared {
  float score[SEL_MAX];
  unsigned char kind[SEL_MAX];                    // 0 dead, 1 live, 2 ended
  int rows[SEL_MAX];                              // the live rows, ascending
  int nlive, bad;
  double lse[SEL_MAX];                            // by row; NaN: the row gives no candidates
  double top[SEL_WARPS][32];                      // per warp and group of blocks
  double bound[SEL_MAX_CLUSTER];                  // per CTA: K of its candidates reach this score
  int warp_count[SEL_WARPS];
  int nblocks, nequal, ncand, overflow;
  long long raised;                               // a higher threshold that K candidates of a block reach (see there)
  int blocks[SEL_MAX_BLOCKS];
  Cand cand[SEL_MAX_CAND];
  Cand best[SEL_WARPS];
};

// (reference, sum) pairs of the lanes of a warp joined: m the largest, s = sum_i s_i exp(m_i - m), in 64 bits.
__device__ __forceinline__ void join(float& m, double& s) {
  const float mine = m;
#pragma unroll
  for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  if (mine != m && s != 0.0) s *= exp((double)mine - (double)m);
#pragma unroll
  for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
}

// The K best by K passes over all candidates, each for the best one behind the last: for inputs whose ties or
// order leave more candidates than the lists hold.  A thread meets its candidates in their order, so that one that ties
// with the last is the best it can find.  Called by all threads of one CTA.
// Measured: 8 x 32 x 151,936 bf16, K = 32, all logits equal: 1.5 ms (79 one logit at a time and to the end of every row).
template <typename T>
__device__ void select_by_passes(SelShared& sh, const SelArgs& a, const T* base) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  Cand last{CUDART_INF, 0};
  int found = 0;
  for (int k = 0; k < a.K; ++k) {
    Cand best{-CUDART_INF, ~0ull};
    for (int i = 0; i < sh.nlive && best.score != last.score; ++i) {
      const int b = sh.rows[i];
      const double score = sh.score[b], lse = sh.lse[b];
      if (isnan(lse)) continue;
      const T* row = base + b * a.stride_b;
      constexpr int AHEAD = 8;
      for (int v0 = tid; v0 < a.V && best.score != last.score; v0 += AHEAD * SEL_THREADS) {
        float x[AHEAD];
#pragma unroll
        for (int q = 0; q < AHEAD; ++q) x[q] = v0 + q * SEL_THREADS < a.V ? (float)row[v0 + q * SEL_THREADS] : -CUDART_INF_F;
#pragma unroll
        for (int q = 0; q < AHEAD; ++q) {
          const Cand c{score + ((double)x[q] - lse), (unsigned long long)b << 32 | (unsigned)(v0 + q * SEL_THREADS)};
          if (c.score > -CUDART_INF && before(last, c) && before(c, best)) best = c;
        }
      }
    }
    if (tid < a.B && sh.kind[tid] == 2) {
      const Cand c{(double)sh.score[tid], (unsigned long long)tid << 32 | (unsigned)a.eos};
      if (before(last, c) && before(c, best)) best = c;
    }
    for (int o = 16; o; o >>= 1) {
      const Cand c{__shfl_xor_sync(0xffffffffu, best.score, o), __shfl_xor_sync(0xffffffffu, best.at, o)};
      if (before(c, best)) best = c;
    }
    __syncthreads();
    if (lane == 0) sh.best[warp] = best;
    __syncthreads();
    best = sh.best[0];
    for (int w = 1; w < SEL_WARPS; ++w)
      if (before(sh.best[w], best)) best = sh.best[w];
    if (best.score == -CUDART_INF) break;
    if (tid == 0) sh.cand[k] = best;
    last = best;
    ++found;
  }
  __syncthreads();
  if (tid == 0) sh.ncand = found;
  __syncthreads();
}

// The pass over the logits: a CTA takes 4 * per blocks of one row.
template <typename T, bool VEC>
__global__ void __launch_bounds__(STREAM_WARPS * 32, 8) k_beam_stream(const SelArgs a) {
  __shared__ float sh_m[STREAM_WARPS];
  __shared__ double sh_s[STREAM_WARPS];
  const int row = blockIdx.x / a.parts, seg = blockIdx.x - row * a.parts;
  const int n = row / a.B, b = row - n * a.B, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int g0 = (seg * STREAM_WARPS + warp) * a.per, count = min(a.per, a.nb - g0);
  float* maxima = a.maxima + (long long)row * a.nb + g0;
  const T* p = (const T*)a.logits + n * a.stride_n + b * a.stride_b + (long long)g0 * SEL_BLOCK;
  const int left = a.V - g0 * SEL_BLOCK;          // logits from p on
  constexpr int AHEAD = VEC && sizeof(T) == 2 ? 2 : 1;      // blocks in flight: 2 KB a warp, 64 KB an SM
  Block<T, VEC> ring[AHEAD];
  auto fetch = [&](Block<T, VEC>& o, int i) {
    if (i >= count) return;
    if (left - i * SEL_BLOCK >= SEL_BLOCK) o.load(p + i * SEL_BLOCK + Block<T, VEC>::first(lane));
    else o.load_part(p + i * SEL_BLOCK, left - i * SEL_BLOCK, lane);
  };
#pragma unroll
  for (int u = 0; u < AHEAD; ++u) fetch(ring[u], u);
  // not waited for before the first loads: a dead or ended beam's logits count for nothing
  if (!isfinite(a.scores[row]) || (a.finished && a.finished[row])) return;
  RunningSum sum;
  sum.clear();
  for (int i0 = 0; i0 < count; i0 += AHEAD) {
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      if (u && i0 + u >= count) break;
      float x[SEL_LANE];
      ring[u].get(x);
      fetch(ring[u], i0 + u + AHEAD);
      const float m = warp_max(lane_max(x));
      if (lane == 0) maxima[i0 + u] = m;
      sum.add(x, m);
    }
  }
  const double s = sum.total();
  if (lane == 0) { sh_m[warp] = sum.ref; sh_s[warp] = s; }
  __syncthreads();
  if (warp == 0) {
    float m = lane < STREAM_WARPS ? sh_m[lane] : -CUDART_INF_F;
    double t = lane < STREAM_WARPS ? sh_s[lane] : 0.0;
    join(m, t);
    if (lane == 0) {
      a.part_m[(long long)row * a.parts + seg] = m;
      a.part_s[(long long)row * a.parts + seg] = t;
    }
  }
}

// Finds and ranks the candidates, from maxima and sums.
template <typename T, bool VEC>
__global__ void __launch_bounds__(SEL_THREADS, 2) k_beam_select(const SelArgs a) {
  __shared__ SelShared sh;
  extern __shared__ float bmax[];                 // [live rows][blocks of this CTA]
  cg::cluster_group cluster = cg::this_cluster();
  auto started = cluster.barrier_arrive();        // waited for before the first write to another CTA
  const int C = (int)cluster.num_blocks(), c = (int)cluster.block_rank();
  const int n = blockIdx.x / C;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const T* base = (const T*)a.logits + n * a.stride_n;
  const long long row0 = (long long)n * a.B;
  const int b0 = (int)((long long)a.nb * c / C), b1 = (int)((long long)a.nb * (c + 1) / C), nbl = b1 - b0;

  // every warp looks at all beams' scores; warp 0 writes down what it finds
  const float my_score = lane < a.B ? a.scores[row0 + lane] : -CUDART_INF_F;
  const bool done = lane < a.B && a.finished && a.finished[row0 + lane];
  const int kind = !isfinite(my_score) ? 0 : done ? 2 : 1;
  const unsigned live = __ballot_sync(0xffffffffu, kind == 1);
  const int nlive = __popc(live), place = __popc(live & ((1u << lane) - 1));     // of a live beam in the list of these
  if (warp == 0) {
    const unsigned bad = __ballot_sync(0xffffffffu, isnan(my_score) || my_score == CUDART_INF_F);
    if (lane < a.B) {
      sh.score[lane] = my_score;
      sh.kind[lane] = (unsigned char)kind;
    }
    if (kind == 1) sh.rows[place] = lane;
    if (lane == 0) {
      sh.nlive = nlive;
      sh.bad = bad != 0;
      sh.nblocks = sh.nequal = sh.ncand = sh.overflow = 0;
      sh.raised = (long long)0x8000000000000000ull;
    }
  }

  // ---- a warp (few rows: several) a row: its maxima to shared memory, its log-sum-exp, and the best block in each of
  // 32 groups ----
  // Block e of the list [live rows][blocks of this CTA] belongs to group e % 32, which is a lane here.
  int share = 1;                                  // warps a row
  while (share < SEL_WARPS && share * 2 * nlive <= SEL_WARPS) share *= 2;
  const int first_row = warp / share, row_step = SEL_WARPS / share, sub = warp % share;
  double top = -CUDART_INF;
  bool bad_row = false;
  for (int r = first_row; r < nlive; r += row_step) {
    const int b = __ffs(__ballot_sync(0xffffffffu, kind == 1 && place == r)) - 1;
    const long long row = row0 + b;
    float* mine = bmax + r * nbl;
    const int i0 = ((lane - r * nbl) & 31) + 32 * sub;
#pragma unroll 4
    for (int i = i0; i < nbl; i += 32 * share) mine[i] = a.maxima[row * a.nb + b0 + i];
    const float* pm = a.part_m + row * a.parts;
    const double* ps = a.part_s + row * a.parts;
    float m = -CUDART_INF_F;
#pragma unroll 2
    for (int i = lane; i < a.parts; i += 32) m = fmaxf(m, pm[i]);
#pragma unroll
    for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    double s = 0.0;
#pragma unroll 2
    for (int i = lane; i < a.parts; i += 32) {
      const double t = ps[i];
      s += t == 0.0 || pm[i] == m ? t : t * exp((double)pm[i] - (double)m);
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    // nothing allowed, or a NaN or +inf among the logits: no candidates
    const double lse = (double)m + log(s);
    const bool fine = isfinite(lse);
    bad_row = bad_row || isnan(s) || m == CUDART_INF_F;
    if (lane == 0 && sub == 0) sh.lse[b] = fine ? lse : CUDART_NAN;
    const double score = __shfl_sync(0xffffffffu, my_score, b);
    if (fine)
#pragma unroll 4
      for (int i = i0; i < nbl; i += 32 * share) top = fmax(top, score + ((double)mine[i] - lse));
  }
  sh.top[warp][lane] = top;
  __syncthreads();
  if (bad_row && lane == 0) atomicOr(&sh.bad, 1);
  const int items = nlive * nbl;

  // ---- the blocks that can hold one of the K best: those that reach the K-th best of the groups' maxima, of the CTA
  // of the cluster where that is highest ----
  auto block_score = [&](int r, int i) {
    const int b = sh.rows[r];
    const double s = (double)sh.score[b] + ((double)bmax[r * nbl + i] - sh.lse[b]);
    return isnan(s) ? -CUDART_INF : s;
  };
  cluster.barrier_wait(std::move(started));
  if (warp == 0) {
#pragma unroll
    for (int w = 1; w < SEL_WARPS; ++w) top = fmax(top, sh.top[w][lane]);
    sh.top[0][lane] = top;
    __syncwarp();
    int rank = 0;
#pragma unroll 8
    for (int i = 0; i < 32; ++i) {
      const double o = sh.top[0][i];
      rank += o > top || (o == top && i < lane);
    }
    const unsigned kth = __ballot_sync(0xffffffffu, rank == a.K - 1);
    const double bound = __shfl_sync(0xffffffffu, top, __ffs(kth) - 1);
    if (lane < C) cluster.map_shared_rank(&sh, lane)->bound[c] = bound;
  }
  cluster.sync();
  double thr = sh.bound[0];
  for (int o = 1; o < C; ++o) thr = fmax(thr, sh.bound[o]);
  for (int r = first_row; r < nlive; r += row_step)
#pragma unroll 4
    for (int i = lane + 32 * sub; i < nbl; i += 32 * share) {
      const double s = block_score(r, i);
      if (s > -CUDART_INF && s >= thr) {
        if (s == thr) atomicAdd(&sh.nequal, 1);
        const int p = atomicAdd(&sh.nblocks, 1);
        if (p < SEL_MAX_BLOCKS) sh.blocks[p] = r * nbl + i;
      }
    }
  __syncthreads();
  if (sh.nequal > a.K || sh.nblocks > SEL_MAX_BLOCKS) {   // of the blocks that tie with the threshold the first K will do
    __syncthreads();
    if (tid == 0) sh.nblocks = 0;
    int equal = 0;
    for (int e0 = 0; e0 < items; e0 += SEL_THREADS) {
      const int e = e0 + tid;
      const double s = e < items ? block_score(e / nbl, e % nbl) : -CUDART_INF;
      const bool some = s > -CUDART_INF;
      const unsigned eq = __ballot_sync(0xffffffffu, some && s == thr);
      if (lane == 0) sh.warp_count[warp] = __popc(eq);
      __syncthreads();
      int prior = equal, all = equal;
      for (int w = 0; w < SEL_WARPS; ++w) {
        if (w < warp) prior += sh.warp_count[w];
        all += sh.warp_count[w];
      }
      equal = all;
      if (some && (s > thr || (s == thr && prior + __popc(eq & ((1u << lane) - 1)) < a.K))) {
        const int p = atomicAdd(&sh.nblocks, 1);
        if (p < SEL_MAX_BLOCKS) sh.blocks[p] = e; else atomicOr(&cluster.map_shared_rank(&sh, 0)->overflow, 1);
      }
      __syncthreads();
    }
  }

  // ---- single logits of those blocks, to the first CTA's list ----
  const int nblk = sh.nblocks < SEL_MAX_BLOCKS ? sh.nblocks : SEL_MAX_BLOCKS;
  float x[SEL_LANE];
  int b = 0, v0 = 0, loaded = -1;                 // beam and first token of the block in x
  auto load_block = [&](int i) {
    if (loaded == i) return;
    const int e = sh.blocks[i], r = e / nbl;
    b = sh.rows[r];
    v0 = (b0 + e - r * nbl) * SEL_BLOCK;
    const T* p = base + b * a.stride_b + v0;
    Block<T, VEC> raw;
    if (v0 + SEL_BLOCK <= a.V) raw.load(p + Block<T, VEC>::first(lane)); else raw.load_part(p, a.V - v0, lane);
    raw.get(x);
    loaded = i;
  };
  auto cand = [&](int q) { return (double)sh.score[b] + ((double)x[q] - sh.lse[b]); };
  // A logit under this cannot reach `least` (64-bit rounding allowed for): single precision decides for nearly all.
  auto floor_of = [&](double least) {
    const double score = sh.score[b], lse = sh.lse[b], t = (least - score) + lse;
    return __double2float_rd(t - (fabs(t) + fabs(score) + fabs(lse)) * 1e-12);
  };
  auto reaching = [&](float least) {              // of the block's logits
    int n = 0;
#pragma unroll
    for (int q = 0; q < SEL_LANE; ++q) n += x[q] >= least && x[q] > -CUDART_INF_F;
    return (int)__reduce_add_sync(0xffffffffu, n);
  };
  // Where one beam is far ahead and a row has few blocks, these hold many logits that reach the threshold.  A block with
  // more than K of them raises it, to the K-th best of the 64 maxima of eight of its logits each (47 x 16 x 3,719, K = 16:
  // 20 us, 45 without; rows of many blocks have no need of it).
  bool raised = false;
  for (int i = warp; i < nblk && a.nb <= 2 * a.K; i += SEL_WARPS) {
    load_block(i);
    if (reaching(floor_of(thr)) <= a.K) continue;
    float h0 = x[0], h1 = x[8];
#pragma unroll
    for (int q = 1; q < 8; ++q) { h0 = fmaxf(h0, x[q]); h1 = fmaxf(h1, x[q + 8]); }
    int above0 = 0, above1 = 0;
#pragma unroll 8
    for (int l = 0; l < 32; ++l) {
      const float o0 = __shfl_sync(0xffffffffu, h0, l), o1 = __shfl_sync(0xffffffffu, h1, l);
      above0 += (o0 > h0) + (o1 > h0);
      above1 += (o0 > h1) + (o1 > h1);
    }
    const float kth = -warp_max(-fminf(above0 < a.K ? h0 : CUDART_INF_F, above1 < a.K ? h1 : CUDART_INF_F));
    const double bound = (double)sh.score[b] + ((double)kth - sh.lse[b]);
    if (kth > -CUDART_INF_F && bound > thr) {
      raised = true;
      // doubles in the order of integers
      long long key = __double_as_longlong(bound);
      key ^= (key >> 63) & 0x7fffffffffffffffll;
      if (lane == 0) atomicMax(&sh.raised, key);
    }
  }
  if (__syncthreads_or(raised)) {
    long long key = sh.raised;
    key ^= (key >> 63) & 0x7fffffffffffffffll;
    thr = __longlong_as_double(key);
  }
  SelShared* head = cluster.map_shared_rank(&sh, 0);
  auto found = [&](double score, int beam, int v) {
    const int p = atomicAdd(&head->ncand, 1);
    if (p < SEL_MAX_CAND) head->cand[p] = Cand{score, (unsigned long long)beam << 32 | (unsigned)v};
  };
  // backwards: the last one is in registers still
  for (int i = nblk > warp ? warp + (nblk - 1 - warp) / SEL_WARPS * SEL_WARPS : -1; i >= 0; i -= SEL_WARPS) {
    load_block(i);
    const float least = floor_of(thr);
    const int reach = reaching(least);
    if (reach == 0) continue;
    if (reach <= 2 * a.K) {
#pragma unroll
      for (int q = 0; q < SEL_LANE; ++q)
        if (x[q] >= least && x[q] > -CUDART_INF_F) {
          const double s = cand(q);
          if (s >= thr) found(s, b, v0 + Block<T, VEC>::index(lane, q));
        }
      continue;
    }
    unsigned used = 0;
    for (int k = 0; k < a.K; ++k) {               // ties: the K best of the block, one by one
      double best = -CUDART_INF;
      int at = 0x7fffffff, q0 = 0;
#pragma unroll
      for (int q = 0; q < SEL_LANE; ++q) {
        const double s = cand(q);
        const int v = v0 + Block<T, VEC>::index(lane, q);
        if (!(used >> q & 1) && (s > best || (s == best && s > -CUDART_INF && v < at))) {
          best = s;
          at = v;
          q0 = q;
        }
      }
      double all = best;
#pragma unroll
      for (int o = 16; o; o >>= 1) all = fmax(all, __shfl_xor_sync(0xffffffffu, all, o));
      const int first = (int)__reduce_min_sync(0xffffffffu, best == all ? (unsigned)at : 0x7fffffffu);
      if (best == all && at == first) {
        used |= 1u << q0;
        found(all, b, at);
      }
    }
  }
  cluster.sync();                                 // from here on nobody reads or writes another CTA's shared memory
  if (c != 0) return;

  // ---- the first CTA ranks what all have found ----
  if (tid < a.B && sh.kind[tid] == 2) found(sh.score[tid], tid, a.eos);
  __syncthreads();
  if (sh.overflow || sh.ncand > SEL_MAX_CAND) select_by_passes<T>(sh, a, base);
  const int nc = sh.ncand;
  auto put = [&](int k, double score, int parent, int token) {
    const int o = n * a.K + k;
    a.scores_out[o] = (float)score;
    a.parents[o] = parent;
    a.tokens[o] = token;
    if (a.finished_out) a.finished_out[o] = parent >= 0 && (sh.kind[parent] == 2 || token == a.eos);
  };
  int lanes = 1;                                  // that count for one candidate
  while (lanes < 32 && 2 * lanes * nc <= SEL_THREADS) lanes *= 2;
  for (int i0 = 0; i0 < nc; i0 += SEL_THREADS / lanes) {
    const int i = i0 + tid / lanes;
    const Cand x = sh.cand[min(i, nc - 1)];
    int rank = 0;
#pragma unroll 8
    for (int j = tid % lanes; j < nc; j += lanes) rank += before(sh.cand[j], x);
    for (int o = 1; o < lanes; o *= 2) rank += __shfl_xor_sync(0xffffffffu, rank, o);
    if (i < nc && tid % lanes == 0 && rank < a.K) put(rank, x.score, (int)(x.at >> 32), (int)(unsigned)x.at);
  }
  for (int k = nc + tid; k < a.K; k += SEL_THREADS) put(k, -CUDART_INF, -1, -1);
  if (tid == 0 && a.flags) a.flags[n] = sh.bad ? PCTC_UTT_NONFINITE : 0;
}

// Host checks: the rows of the beams of logits or of a state as byte ranges, base + i * outer + j * inner, i < N, j < rows, each `len` long.
struct RowSet {
  size_t base;
  long long outer, inner, len;
  int rows;
  bool write;
  size_t end(int N) const { return base + (size_t)((N - 1) * outer + (rows - 1) * inner + len); }
};
// One of the two levels of a pair of such sets: how often each repeats, and the stride that they have in common.
struct Level {
  long long na, nb, stride;
};
// Whether f(d + t * stride) holds for one of the shifts t that bring an extent of b, d behind a's, to a's extent.
template <typename F>
bool meets(const Level& l, long long d, long long extent_a, long long extent_b, F f) {
  if (l.na == 1 && l.nb == 1) return d < extent_a && -d < extent_b && f(d);
  if (l.stride <= 0) return true;
  const long long least = -extent_b - d, down = least / l.stride - (least % l.stride < 0);
  for (long long t = std::max(down + 1, 1 - l.na); t < l.nb && d + t * l.stride < extent_a; ++t)
    if (f(d + t * l.stride)) return true;
  return false;
}
// The level with the larger stride first.
template <typename F>
bool larger_first(const Level& x, const Level& y, F f) { return x.stride >= y.stride ? f(x, y) : f(y, x); }
// Whether a range shares a byte with one of the rows.
bool range_clash(const RowSet& r, int N, const Span& s) {
  if (r.end(N) <= s.lo || s.hi <= r.base) return false;
  const Level utts{r.outer ? N : 1, 1, r.outer}, beams{r.inner ? r.rows : 1, 1, r.inner};
  const long long len = (long long)(s.hi - s.lo);
  return larger_first(utts, beams, [&](const Level& big, const Level& small) {
    return meets(big, (long long)(s.lo - r.base), (small.na - 1) * small.stride + r.len, len,
                 [&](long long d) { return meets(small, d, r.len, len, [](long long) { return true; }); });
  });
}

pctc_status_t check(const pctc_beam_t* p) {
  if (!p) return PCTC_ERR_INVALID_ARG;
  if (p->N <= 0 || p->B <= 0 || p->K <= 0 || p->V <= 0) return PCTC_ERR_INVALID_ARG;
  if (p->dtype != PCTC_BF16 && p->dtype != PCTC_FP32) return PCTC_ERR_UNSUPPORTED;
  if (p->B > SEL_MAX || p->K > SEL_MAX || p->V > SEL_MAX_V) return PCTC_ERR_UNSUPPORTED;
  if (p->eos_id < -1 || (long long)p->eos_id >= p->V) return PCTC_ERR_INVALID_ARG;
  if (p->stride_b < p->V || p->stride_n < 0) return PCTC_ERR_INVALID_ARG;
  if ((long long)p->N * p->B * ((p->V + SEL_BLOCK - 1) / SEL_BLOCK) > 0x3fffffffLL) return PCTC_ERR_UNSUPPORTED;
  if ((long long)p->N * SEL_MAX > 0x3fffffffLL) return PCTC_ERR_UNSUPPORTED;
  return PCTC_OK;
}

struct SelWorkspace {
  size_t o_part_m, o_part_s, total;
  int nb, parts, per;
};
SelWorkspace workspace_of(const pctc_beam_t* p) {
  SelWorkspace w;
  w.nb = (int)((p->V + SEL_BLOCK - 1) / SEL_BLOCK);
  const size_t rows = (size_t)p->N * p->B;
  w.per = std::min(8, (w.nb + STREAM_WARPS - 1) / STREAM_WARPS);
  do w.parts = (w.nb + STREAM_WARPS * w.per - 1) / (STREAM_WARPS * w.per);
  while (rows * w.parts < STREAM_CTAS && w.per > 1 && (w.per /= 2));
  auto up = [](size_t x) { return (x + 255) / 256 * 256; };
  w.o_part_m = up(rows * w.nb * 4);
  w.o_part_s = w.o_part_m + up(rows * w.parts * 4);
  w.total = w.o_part_s + up(rows * w.parts * 8);
  return w;
}

// What the call writes may overlap nothing else that it takes; scores and finished may be written over as they are (K == B).
bool select_overlaps(const SelArgs& a, size_t es, size_t workspace_bytes) {
  const size_t in = (size_t)a.N * a.B, out = (size_t)a.N * a.K;
  Span s[8];
  size_t n = 0;
  auto add = [&](const void* p, size_t bytes, bool write) {
    if (p) s[n++] = Span{(size_t)p, (size_t)p + bytes, write};
  };
  add(a.maxima, workspace_bytes, true);
  add(a.scores_out, 4 * out, true);
  add(a.parents, 4 * out, true);
  add(a.tokens, 4 * out, true);
  add(a.finished_out, out, true);
  add(a.flags, 4 * (size_t)a.N, true);
  const RowSet logits{(size_t)a.logits, (long long)(a.stride_n * es), (long long)(a.stride_b * es), (long long)(a.V * es), a.B, false};
  for (size_t i = 0; i < n; ++i)
    if (range_clash(logits, a.N, s[i])) return true;
  if (a.scores != a.scores_out) add(a.scores, 4 * in, false);
  if (a.finished != a.finished_out) add(a.finished, in, false);
  return spans_conflict(s, n);
}

template <typename T, bool VEC>
cudaError_t launch_select(const SelArgs& a, cudaStream_t stream) {
  k_beam_stream<T, VEC><<<a.N * a.B * a.parts, STREAM_WARPS * 32, 0, stream>>>(a);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  int C = 1;
  while (C < SEL_MAX_CLUSTER && (long long)a.B * a.nb > 4096LL * C) C *= 2;
  const size_t dyn = (size_t)a.B * ((a.nb + C - 1) / C) * 4;
  auto kern = k_beam_select<T, VEC>;
  if (dyn + sizeof(SelShared) > 48 * 1024) {
    e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, SEL_MAX_DYN);
    if (e != cudaSuccess) return e;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(a.N * C);
  cfg.blockDim = dim3(SEL_THREADS);
  cfg.dynamicSmemBytes = dyn;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = C;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = C > 1 ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, kern, a);
}

}  // namespace
}  // namespace pctc

using namespace pctc;

extern "C" {

pctc_status_t pctc_beam_workspace_bytes(const pctc_beam_t* p, size_t* bytes_out) {
  const pctc_status_t st = check(p);
  if (st != PCTC_OK) return st;
  if (!bytes_out) return PCTC_ERR_INVALID_ARG;
  *bytes_out = workspace_of(p).total;
  return PCTC_OK;
}

pctc_status_t pctc_beam_select(const pctc_beam_t* p, const void* logits, const float* scores, const uint8_t* finished,
                               float* scores_out, int32_t* parents, int32_t* tokens, uint8_t* finished_out,
                               int32_t* utt_flags, void* workspace, size_t workspace_bytes, void* stream_v) {
  const pctc_status_t st = check(p);
  if (st != PCTC_OK) return st;
  const SelWorkspace w = workspace_of(p);
  if (!workspace || ((size_t)workspace & 255)) return PCTC_ERR_INVALID_ARG;
  if (workspace_bytes < w.total) return PCTC_ERR_WORKSPACE_TOO_SMALL;
  if (!logits || !scores || !scores_out || !parents || !tokens) return PCTC_ERR_INVALID_ARG;
  if (finished && p->eos_id < 0) return PCTC_ERR_INVALID_ARG;
  if (p->K != p->B && (scores_out == scores || (finished && finished_out == finished))) return PCTC_ERR_INVALID_ARG;
  const size_t es = p->dtype == PCTC_BF16 ? 2 : 4;
  if ((size_t)logits & (es - 1)) return PCTC_ERR_INVALID_ARG;
  if (((size_t)scores | (size_t)scores_out | (size_t)parents | (size_t)tokens | (size_t)utt_flags) & 3) return PCTC_ERR_INVALID_ARG;
  SelArgs a;
  a.logits = logits;
  a.stride_n = p->stride_n;
  a.stride_b = p->stride_b;
  a.scores = scores;
  a.finished = finished;
  a.N = p->N; a.B = p->B; a.K = p->K; a.V = (int)p->V; a.eos = p->eos_id;
  a.nb = w.nb;
  a.scores_out = scores_out;
  a.parents = parents;
  a.tokens = tokens;
  a.finished_out = finished_out;
  a.flags = utt_flags;
  a.maxima = (float*)workspace;
  a.part_m = (float*)((char*)workspace + w.o_part_m);
  a.part_s = (double*)((char*)workspace + w.o_part_s);
  a.parts = w.parts;
  a.per = w.per;
  if (select_overlaps(a, es, w.total)) return PCTC_ERR_INVALID_ARG;
  const bool vec = (((size_t)logits | (size_t)p->stride_n * es | (size_t)p->stride_b * es) & 15) == 0;
  cudaStream_t stream = (cudaStream_t)stream_v;
  const cudaError_t e = p->dtype == PCTC_BF16
      ? (vec ? launch_select<__nv_bfloat16, true>(a, stream) : launch_select<__nv_bfloat16, false>(a, stream))
      : (vec ? launch_select<float, true>(a, stream) : launch_select<float, false>(a, stream));
  return e == cudaSuccess ? PCTC_OK : PCTC_ERR_CUDA;
}

}  // extern "C"

// ---------------------------------------------------------------------------
// Reordering of states
// ---------------------------------------------------------------------------
//
// out[n, k] = in[n, parents[n, k]] for a list of states.  A state's row of one beam is `segments` pieces of
// `units` units each (the units of a time axis, of which only the first lengths[n] count).  A CTA owns a column:
// the same bytes of all beams of an utterance; a thread loads its 1 to 16 bytes of every parent before it
// stores any.  So a parent that several beams share is read once, and in place needs no second buffer: nobody
// else touches the column.  In place a beam that stays where it is moves nothing.
// Bound by HBM.  A CTA takes one tile of 4 KB columns: a persistent grid of such tiles, whose CTAs drift apart, was slower
// (16 caches [16, 8, 8, 151, 64] bf16: 83 us against 64; 12 caches [8, 4, 8, 2000, 64]: 252 against 194, 8 TB/s written
// and read as seen by the caller, since shared parents are read once; 12 caches [8, 4, 8, 300, 64] in place with half of
// the beams moving: 25 against 16).
namespace pctc {
namespace {

constexpr int MOVE_THREADS = 256;

struct MoveState {
  const char* src;
  char* dst;
  long long src_n, src_b, dst_n, dst_b;           // byte strides of utterances and beams
  long long seg;                                  // byte stride of segments
  long long unit;                                 // bytes of a unit
  int segments, units;                            // units: of the whole axis (lengths are cut to it)
  int tiles;                                      // tiles of one segment
  int timed;                                      // lengths apply
  int width;                                      // bytes a thread moves at a time: 16, 8, 4, 2 or 1
};
template <int LIM>
struct MoveTable {
  MoveState s[LIM];
  int tile0[LIM + 1];                             // tiles before state i
  int n;
};
constexpr int MOVE_SMALL = 32, MOVE_LARGE = 256;
static_assert(sizeof(MoveTable<MOVE_LARGE>) <= 32000, "kernel parameters");

// The parents of an utterance's slots: in registers, or, where 32 columns of 16 bytes need them all, in shared memory.
template <int KB>
struct Parents {
  int p[KB];
  __device__ __forceinline__ int operator[](int k) const { return p[k]; }
};
template <>
struct Parents<32> {
  const int* p;
  __device__ __forceinline__ int operator[](int k) const { return p[k]; }
};

// Pieces of a column that a thread moves: with few beams one is too little work for a CTA's index arithmetic (12 caches
// [8, 4, 8, 300, 64] in place: 20.5 us with one, 16.1 with two, 18.0 with four); with eight beams two took longer (73
// against 64 us for 16 caches [16, 8, 8, 151, 64]).
constexpr __host__ __device__ int move_rows(int KB) { return KB <= 4 ? 2 : 1; }

template <typename U, int KB>
__device__ __forceinline__ void move_tile(const MoveState& s, const Parents<KB>& par, long long bytes, int n, int seg,
                                          int tile) {
  constexpr int ROWS = move_rows(KB), STEP = MOVE_THREADS * (int)sizeof(U);
  const long long at = (long long)tile * ROWS * STEP + threadIdx.x * (int)sizeof(U);
  if (at >= bytes) return;
  const bool in_place = s.src == s.dst;
  const char* src = s.src + n * s.src_n + seg * s.seg + at;
  char* dst = s.dst + n * s.dst_n + seg * s.seg + at;
  U v[ROWS][KB];
#pragma unroll
  for (int k = 0; k < KB; ++k) {
    if (par[k] < 0 || (in_place && par[k] == k)) continue;
    const char* from = src + par[k] * s.src_b;
#pragma unroll
    for (int q = 0; q < ROWS; ++q)
      if (at + q * STEP < bytes) v[q][k] = *(const U*)(from + q * STEP);
  }
#pragma unroll
  for (int k = 0; k < KB; ++k) {
    if (par[k] < 0 || (in_place && par[k] == k)) continue;
    char* to = dst + k * s.dst_b;
#pragma unroll
    for (int q = 0; q < ROWS; ++q)
      if (at + q * STEP < bytes) *(U*)(to + q * STEP) = v[q][k];
  }
}

template <int LIM, int KB>
__global__ void __launch_bounds__(MOVE_THREADS) k_beam_move(const __grid_constant__ MoveTable<LIM> tab,
                                                            const int* __restrict__ parents,
                                                            const int* __restrict__ lengths, int N, int B, int K) {
  const int t = blockIdx.x;
  int lo = 0, hi = tab.n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (tab.tile0[mid] <= t) lo = mid; else hi = mid - 1;
  }
  const MoveState& s = tab.s[lo];
  const int local = t - tab.tile0[lo];
  const int ns = local / s.tiles, tile = local - ns * s.tiles, n = ns / s.segments, seg = ns - n * s.segments;
  auto parent = [&](int k) {
    const int p = k < K ? __ldg(parents + n * K + k) : -1;
    return p >= 0 && p < B ? p : -1;
  };
  Parents<KB> par;
  if constexpr (KB == 32) {
    __shared__ int shared[KB];
    if (threadIdx.x < KB) shared[threadIdx.x] = parent(threadIdx.x);
    __syncthreads();
    par.p = shared;
  } else {
#pragma unroll
    for (int k = 0; k < KB; ++k) par.p[k] = parent(k);
  }
  int units = s.units;
  if (s.timed) units = min(max(__ldg(lengths + n), 0), units);
  const long long bytes = units * s.unit;
  switch (s.width) {
    case 16: move_tile<uint4, KB>(s, par, bytes, n, seg, tile); break;
    case 8: move_tile<uint2, KB>(s, par, bytes, n, seg, tile); break;
    case 4: move_tile<unsigned, KB>(s, par, bytes, n, seg, tile); break;
    case 2: move_tile<unsigned short, KB>(s, par, bytes, n, seg, tile); break;
    default: move_tile<unsigned char, KB>(s, par, bytes, n, seg, tile); break;
  }
}

// Whether two sets of rows share a byte.  Exact where they repeat with the same strides (views of one buffer, whether
// they interleave by beam or by utterance), or lie apart within one beam stride; other ranges that interleave count as
// shared.
bool rows_clash(const RowSet& a, const RowSet& b, int N) {
  if (a.end(N) <= b.base || b.end(N) <= a.base) return false;
  if (a.inner == b.inner && a.len <= a.inner && b.len <= b.inner &&
      (N == 1 || (a.outer % a.inner == 0 && b.outer % b.inner == 0))) {
    const long long d = (long long)((a.base > b.base ? a.base - b.base : b.base - a.base) % (size_t)a.inner);
    const long long first = a.base > b.base ? b.len : a.len, second = a.base > b.base ? a.len : b.len;
    if (first <= d && d + second <= a.inner) return false;
  }
  if (N > 1 && a.outer != b.outer) return true;
  if (a.rows > 1 && b.rows > 1 && a.inner != b.inner) return true;
  const Level utts{N, N, a.outer}, beams{a.rows, b.rows, a.rows > 1 ? a.inner : b.inner};
  return larger_first(utts, beams, [&](const Level& big, const Level& small) {
    return meets(big, (long long)(b.base - a.base), (small.na - 1) * small.stride + a.len,
                 (small.nb - 1) * small.stride + b.len,
                 [&](long long d) { return meets(small, d, a.len, b.len, [](long long) { return true; }); });
  });
}

pctc_status_t check_move(const pctc_beam_state_t* st, int n, int N, int B, int K, const int32_t* lengths) {
  if (n < 0 || N <= 0 || B <= 0 || K <= 0 || (n && !st)) return PCTC_ERR_INVALID_ARG;
  if (B > SEL_MAX || K > SEL_MAX || N > 0x7fffffff / SEL_MAX) return PCTC_ERR_UNSUPPORTED;
  for (int i = 0; i < n; ++i) {
    const pctc_beam_state_t& s = st[i];
    if (!s.src || !s.dst || s.segments <= 0 || s.units < 0 || s.unit_bytes <= 0) return PCTC_ERR_INVALID_ARG;
    if (s.timed & ~1) return PCTC_ERR_INVALID_ARG;
    if (s.timed && !lengths) return PCTC_ERR_INVALID_ARG;
    const long long most = 1LL << 46;
    if (s.unit_bytes > most || s.units > most / s.unit_bytes || s.segments > 0x7fffffffLL || s.units > 0x7fffffffLL)
      return PCTC_ERR_UNSUPPORTED;
    const long long len = s.units * s.unit_bytes;
    if (s.segments > 1 && (s.segment_stride < len || s.segment_stride > most / s.segments)) return PCTC_ERR_INVALID_ARG;
    const long long row = (s.segments - 1) * s.segment_stride + len;
    if (s.src_stride_b < 0 || s.dst_stride_b < 0 || s.src_stride_n < 0 || s.dst_stride_n < 0) return PCTC_ERR_INVALID_ARG;
    if (s.src_stride_b > most || s.dst_stride_b > most || s.src_stride_n > most / N || s.dst_stride_n > most / N)
      return PCTC_ERR_UNSUPPORTED;
    // written rows are apart: beams inside utterances, or utterances inside beams
    const long long sn = N > 1 ? s.dst_stride_n : most, sb = K > 1 ? s.dst_stride_b : most;
    const bool by_utt = sb >= row && (N == 1 || sn >= (K > 1 ? (K - 1) * sb : 0) + row);
    const bool by_beam = sn >= row && (K == 1 || sb >= (N > 1 ? (N - 1) * sn : 0) + row);
    if (!by_utt && !by_beam) return PCTC_ERR_INVALID_ARG;
    if (s.src == s.dst && (K != B || (B > 1 && s.src_stride_b != s.dst_stride_b) ||
                           (N > 1 && s.src_stride_n != s.dst_stride_n)))
      return PCTC_ERR_INVALID_ARG;
  }
  return PCTC_OK;
}

// What the call writes may overlap nothing else that it takes (in place: a state's own rows, which are one set).
pctc_status_t check_overlap(const pctc_beam_state_t* st, int n, int N, int B, int K, const int32_t* parents,
                            const int32_t* lengths) {
  RowSet* r = new (std::nothrow) RowSet[2 * (size_t)n + 2];
  if (!r) return PCTC_ERR_HOST_MEMORY;
  int m = 0;
  r[m++] = RowSet{(size_t)parents, 4LL * K, 4LL * K, 4LL * K, 1, false};
  if (lengths) r[m++] = RowSet{(size_t)lengths, 4, 4, 4, 1, false};
  for (int i = 0; i < n; ++i) {
    const pctc_beam_state_t& s = st[i];
    const long long row = (s.segments - 1) * s.segment_stride + s.units * s.unit_bytes;
    if (row == 0) continue;
    r[m++] = RowSet{(size_t)s.dst, s.dst_stride_n, s.dst_stride_b, row, K, true};
    if (s.src != s.dst) r[m++] = RowSet{(size_t)s.src, s.src_stride_n, s.src_stride_b, row, B, false};
  }
  std::sort(r, r + m, [](const RowSet& a, const RowSet& b) { return a.base < b.base; });
  bool clash = false;
  for (int i = 0; i < m && !clash; ++i) {
    const size_t end = r[i].end(N);
    for (int j = i + 1; j < m && r[j].base < end && !clash; ++j)
      if (r[i].write || r[j].write) clash = rows_clash(r[i], r[j], N);
  }
  delete[] r;
  return clash ? PCTC_ERR_INVALID_ARG : PCTC_OK;
}

template <int LIM, int KB>
cudaError_t launch_move(const MoveTable<LIM>& tab, const int* parents, const int* lengths, int N, int B, int K,
                        cudaStream_t stream) {
  k_beam_move<LIM, KB><<<tab.tile0[tab.n], MOVE_THREADS, 0, stream>>>(tab, parents, lengths, N, B, K);
  return cudaGetLastError();
}

template <int LIM>
pctc_status_t move_all(const pctc_beam_state_t* st, int n, int N, int B, int K, const int* parents, const int* lengths,
                       cudaStream_t stream) {
  MoveTable<LIM> tab;
  for (int i0 = 0; i0 < n; i0 += LIM) {
    tab.n = 0;
    long long tiles = 0;
    for (int i = i0; i < n && i < i0 + LIM; ++i) {
      const pctc_beam_state_t& s = st[i];
      const long long len = s.units * s.unit_bytes;
      if (len == 0) continue;
      MoveState& m = tab.s[tab.n];
      m.src = (const char*)s.src;
      m.dst = (char*)s.dst;
      m.src_n = N > 1 ? s.src_stride_n : 0;
      m.src_b = B > 1 ? s.src_stride_b : 0;
      m.dst_n = N > 1 ? s.dst_stride_n : 0;
      m.dst_b = K > 1 ? s.dst_stride_b : 0;
      m.seg = s.segments > 1 ? s.segment_stride : 0;
      m.unit = s.timed ? s.unit_bytes : len;
      m.units = s.timed ? (int)s.units : 1;
      m.segments = (int)s.segments;
      m.timed = s.timed;
      // as wide as all addresses and lengths allow
      const size_t all = (size_t)m.src | (size_t)m.dst | (size_t)(m.src_n | m.src_b | m.dst_n | m.dst_b | m.seg | m.unit);
      m.width = 16;
      while (all & (size_t)(m.width - 1)) m.width /= 2;
      const long long per = (long long)move_rows(K) * MOVE_THREADS * m.width, t = (len + per - 1) / per;
      if (t > 0x7fffffffLL) return PCTC_ERR_UNSUPPORTED;
      m.tiles = (int)t;
      tab.tile0[tab.n++] = (int)tiles;
      if (t * N > 0x7fffffffLL / m.segments) return PCTC_ERR_UNSUPPORTED;
      tiles += t * N * m.segments;
      if (tiles > 0x7fff0000LL) return PCTC_ERR_UNSUPPORTED;
    }
    tab.tile0[tab.n] = (int)tiles;
    if (!tab.n) continue;
    const cudaError_t e = K <= 4 ? launch_move<LIM, 4>(tab, parents, lengths, N, B, K, stream)
                        : K <= 8 ? launch_move<LIM, 8>(tab, parents, lengths, N, B, K, stream)
                        : K <= 16 ? launch_move<LIM, 16>(tab, parents, lengths, N, B, K, stream)
                                  : launch_move<LIM, 32>(tab, parents, lengths, N, B, K, stream);
    if (e != cudaSuccess) return PCTC_ERR_CUDA;
  }
  return PCTC_OK;
}

}  // namespace
}  // namespace pctc

extern "C" {

pctc_status_t pctc_beam_reorder(int32_t n_states, const pctc_beam_state_t* states, int32_t N, int32_t B, int32_t K,
                                const int32_t* parents, const int32_t* lengths, void* stream_v) {
  pctc_status_t st = check_move(states, n_states, N, B, K, lengths);
  if (st != PCTC_OK) return st;
  if (!parents || ((size_t)parents & 3) || ((size_t)lengths & 3)) return PCTC_ERR_INVALID_ARG;
  st = check_overlap(states, n_states, N, B, K, parents, lengths);
  if (st != PCTC_OK) return st;
  cudaStream_t stream = (cudaStream_t)stream_v;
  return n_states <= MOVE_SMALL ? move_all<MOVE_SMALL>(states, n_states, N, B, K, parents, lengths, stream)
                                : move_all<MOVE_LARGE>(states, n_states, N, B, K, parents, lengths, stream);
}

}  // extern "C"
