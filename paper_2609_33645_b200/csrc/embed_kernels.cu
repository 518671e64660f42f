// Rows of the vocabulary matrix for tokens, and the gradient of that lookup:
//   y[i] = scale * W[t_i],           dW[v] = scale * sum over i with t_i = v of g[i]  (+ dW[v]),
// where a token outside [0, V) (the -1 of padded targets and of beams without a candidate) is a row of zeros
// and gives no gradient.  In 8 bits a row of W is s_v * q[v].
//
// The gradient is made without atomics on values: the positions are sorted by token, positions of one token in
// ascending order, and the sums run over the sorted positions, so repeated calls agree bit for bit.
//   k_sort_tokens  one CTA for each of about 148 ranges of the vocabulary reads all tokens twice (they are in L2) and
//                  lays its own out in order: no CTA needs another's result, so one launch sorts.
//   k_embed_grad   a thread sums eight columns over a window of sorted positions.  A token whose positions pass the
//                  end of a window leaves a partial sum for each window, and the last of its threads adds these up in
//                  order.  The same launch fills the rows of tokens that do not occur with zeros.
// Both directions are bound by HBM.
#include "../../include/prunedctc.h"
#include "pctc_internal.h"
#include "vec8.cuh"

#include <cmath>

namespace pctc {
namespace {

constexpr int EMBED_THREADS = 256;
constexpr int EMBED_VECS = 4;                    // groups of eight values a thread

struct EmbedArgs {
  const int* tokens;
  const void* W;
  const float* row_scales;                       // 8-bit matrix: [V], else null
  void* out;
  long long M, V, D, ld_w, ld_out;
  long long groups;                              // M * per_row
  unsigned per_row;                              // groups of eight (or single values) a row
  float scale;
};

// VEC = 8: whole groups of aligned values; VEC = 1: single values, any address and stride.
template <typename W, typename T, int VEC>
__global__ void __launch_bounds__(EMBED_THREADS) k_embed(const EmbedArgs a) {
  const long long g0 = (long long)blockIdx.x * (EMBED_THREADS * EMBED_VECS) + threadIdx.x;
  // the row of the first group by division, those of the others by what they are further on
  long long row = g0 / a.per_row;
  unsigned col = (unsigned)(g0 - row * a.per_row);
  long long rows[EMBED_VECS];
  unsigned cols[EMBED_VECS];
  int token[EMBED_VECS];
#pragma unroll
  for (int k = 0; k < EMBED_VECS; ++k) {
    rows[k] = row;
    cols[k] = col;
    token[k] = row < a.M ? a.tokens[row] : -1;
    col += EMBED_THREADS;
    if (col >= a.per_row) { row += col / a.per_row; col %= a.per_row; }
  }
  if constexpr (VEC == 8) {
    Vec8<W> v[EMBED_VECS];
    float f[EMBED_VECS];
#pragma unroll
    for (int k = 0; k < EMBED_VECS; ++k) {
      const bool there = (unsigned long long)(long long)token[k] < (unsigned long long)a.V;
      if (!there) token[k] = -1;
      if (there) v[k].load((const W*)a.W + token[k] * a.ld_w + cols[k] * 8ll);
      f[k] = there && a.row_scales ? a.row_scales[token[k]] * a.scale : a.scale;
    }
#pragma unroll
    for (int k = 0; k < EMBED_VECS; ++k) {
      if (rows[k] >= a.M) continue;
      float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      if (token[k] >= 0) {
        v[k].get(x);
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] *= f[k];
      }
      Vec8<T>::store((T*)a.out + rows[k] * a.ld_out + cols[k] * 8ll, x);
    }
  } else {
#pragma unroll
    for (int k = 0; k < EMBED_VECS; ++k) {
      if (rows[k] >= a.M) continue;
      float x = 0.f;
      if ((unsigned long long)(long long)token[k] < (unsigned long long)a.V) {
        const float f = a.row_scales ? a.row_scales[token[k]] * a.scale : a.scale;
        x = to_float(((const W*)a.W)[token[k] * a.ld_w + cols[k]]) * f;
      }
      ((T*)a.out)[rows[k] * a.ld_out + cols[k]] = from_float<T>(x);
    }
  }
}

// ---------------------------------------------------------------------------------------------
// Gradient
// ---------------------------------------------------------------------------------------------
constexpr int SORT_THREADS = 512;
constexpr int SORT_WARPS = SORT_THREADS / 32;
constexpr int SORT_BUCKETS = 148;                // ranges of the vocabulary: one CTA on every SM of a B200
constexpr int SORT_MAX_WIDTH = 2048;             // tokens of a range: a counter for each and every warp, 128 KB

struct SortArgs {
  const int* tokens;
  int M;
  long long V;
  int width;                                     // tokens of a range
  int* order;                                    // [M] positions by (token, position)
  int* key;                                      // [M] their tokens
  int* first;                                    // [V + 1] where a token's positions begin
  int* clear;                                    // counters of k_embed_grad, zeroed here
  long long n_clear;
};

__global__ void __launch_bounds__(SORT_THREADS) k_sort_tokens(const SortArgs a) {
  extern __shared__ int count[];                 // [SORT_WARPS][width], then the offsets of the warps
  __shared__ int below_sum[SORT_WARPS], scan_sum[SORT_WARPS];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const long long lo = (long long)blockIdx.x * a.width;
  const int width = (int)min((long long)a.width, a.V - lo);
  for (long long i = (long long)blockIdx.x * SORT_THREADS + threadIdx.x; i < a.n_clear; i += (long long)gridDim.x * SORT_THREADS)
    a.clear[i] = 0;
  for (int i = threadIdx.x; i < SORT_WARPS * a.width; i += SORT_THREADS) count[i] = 0;
  __syncthreads();

  // a warp takes a run of positions, so that warps, steps and lanes in order are positions in order
  const int run = (int)(((long long)a.M + SORT_WARPS * 32 - 1) / (SORT_WARPS * 32)) * 32;
  const int p0 = (int)min((long long)warp * run, (long long)a.M), p1 = (int)min((long long)p0 + run, (long long)a.M);
  int* mine = count + warp * a.width;
  int below = 0;
#pragma unroll 8
  for (int p = p0 + lane; p < p1; p += 32) {
    const int t = a.tokens[p];
    if (t < 0) continue;
    if (t < lo) ++below;
    else if (t - lo < width) atomicAdd(&mine[t - lo], 1);
  }
  below = __reduce_add_sync(0xffffffffu, below);
  if (lane == 0) below_sum[warp] = below;
  __syncthreads();

  // counts -> where each warp's first position of each token goes
  const int per = (width + SORT_THREADS - 1) / SORT_THREADS, k0 = threadIdx.x * per;
  int sum = 0;
  for (int k = k0; k < k0 + per && k < width; ++k)
    for (int w = 0; w < SORT_WARPS; ++w) sum += count[w * a.width + k];
  int scan = sum;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int up = __shfl_up_sync(0xffffffffu, scan, d);
    if (lane >= d) scan += up;
  }
  if (lane == 31) scan_sum[warp] = scan;
  __syncthreads();
  int at = scan - sum;
  for (int w = 0; w < SORT_WARPS; ++w) at += below_sum[w] + (w < warp ? scan_sum[w] : 0);
  for (int k = k0; k < k0 + per && k < width; ++k) {
    a.first[lo + k] = at;
    for (int w = 0; w < SORT_WARPS; ++w) {
      const int c = count[w * a.width + k];
      count[w * a.width + k] = at;
      at += c;
    }
  }
  if (k0 < width && k0 + per >= width && lo + width == a.V) a.first[a.V] = at;
  __syncthreads();

  for (int p = p0; p < p1; p += 32) {
    const int t = p + lane < p1 ? a.tokens[p + lane] : -1;
    const bool hit = t >= lo && t - lo < width;
    const unsigned hits = __ballot_sync(0xffffffffu, hit);
    if (hits == 0) continue;
    if (hit) {
      const unsigned equal = __match_any_sync(hits, t);
      const int rank = __popc(equal & ((1u << lane) - 1));
      const int to = mine[t - lo] + rank;
      __syncwarp(hits);
      if (rank == 0) mine[t - lo] = to + __popc(equal);
      a.order[to] = p + lane;
      a.key[to] = t;
    }
    __syncwarp();
  }
}

struct GradArgs {
  const void* g;
  void* dW;
  const int* order;
  const int* key;
  const int* first;
  float* part;                                   // [windows][2][per_row * VEC]
  int* arrived;                                  // [windows][per_row]
  long long ld_g, ld_w, V;
  long long windows;
  unsigned per_row;                              // groups of eight (or single values) a row
  int window;                                    // sorted positions a thread takes
  int accumulate;
  unsigned sum_blocks;                           // blocks that sum; the others fill rows with zeros
  float scale;
};

template <typename T, int VEC>
struct Piece {                                   // VEC consecutive values of a row
  Vec8<T> v;
  __device__ __forceinline__ void load(const T* p) { v.load_once(p); }
  __device__ __forceinline__ void add(float (&x)[8]) const {
    float y[8];
    v.get(y);
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] += y[j];
  }
};
template <typename T>
struct Piece<T, 1> {
  T v;
  __device__ __forceinline__ void load(const T* p) { v = *p; }
  __device__ __forceinline__ void add(float (&x)[1]) const { x[0] += to_float(v); }
};
template <typename T, int VEC>
__device__ __forceinline__ void write_row(T* p, const float (&sum)[VEC], float scale, bool accumulate) {
  float x[VEC];
#pragma unroll
  for (int j = 0; j < VEC; ++j) x[j] = sum[j] * scale;
  if constexpr (VEC == 8) {
    if (accumulate) {
      Vec8<T> old;
      old.load(p);
      float y[8];
      old.get(y);
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] += y[j];
    }
    Vec8<T>::store(p, x);
  } else {
    if (accumulate) x[0] += to_float(*p);
    *p = from_float<T>(x[0]);
  }
}

constexpr int GRAD_THREADS = 256;
constexpr int GRAD_ZERO_VECS = 8;
constexpr int GRAD_AHEAD = 8;                    // rows that a thread loads before it adds the first

template <typename G, typename T, int VEC>
__global__ void __launch_bounds__(GRAD_THREADS) k_embed_grad(const GradArgs a) {
  if (blockIdx.x >= a.sum_blocks) {              // rows of tokens that do not occur
    const long long total = a.V * a.per_row;
    long long g = (long long)(blockIdx.x - a.sum_blocks) * (GRAD_THREADS * GRAD_ZERO_VECS) + threadIdx.x;
    const float none[VEC] = {};
#pragma unroll
    for (int k = 0; k < GRAD_ZERO_VECS; ++k, g += GRAD_THREADS) {
      if (g >= total) break;
      const long long v = g / a.per_row;
      if (a.first[v] == a.first[v + 1])
        write_row<T, VEC>((T*)a.dW + v * a.ld_w + (g - v * a.per_row) * VEC, none, 0.f, false);
    }
    return;
  }
  const long long id = (long long)blockIdx.x * GRAD_THREADS + threadIdx.x;
  const long long w = id / a.per_row;
  const unsigned c = (unsigned)(id - w * a.per_row);
  const int n = a.first[a.V];                    // positions with a token
  const long long s0 = w * a.window;
  if (s0 >= n) return;
  const int s1 = (int)min(s0 + a.window, (long long)n);
  const G* g = (const G*)a.g + (long long)c * VEC;

  // the sum of a token's positions [begin, end) of this window: final, or a part of the token's sum
  const auto flush = [&](int v, const float (&sum)[VEC]) {
    const int from = a.first[v], to = a.first[v + 1];
    T* row = (T*)a.dW + v * a.ld_w + (long long)c * VEC;
    if (from >= s0 && to <= s1) {
      write_row<T, VEC>(row, sum, a.scale, a.accumulate);
      return;
    }
    const long long width = (long long)a.per_row * VEC, w0 = from / a.window, w1 = (to - 1) / a.window;
    float* p = a.part + (w * 2 + (from >= s0 ? 1 : 0)) * width + (long long)c * VEC;
#pragma unroll
    for (int j = 0; j < VEC; ++j) __stcg(p + j, sum[j]);
    __threadfence();
    if (atomicAdd(&a.arrived[w0 * a.per_row + c], 1) != (int)(w1 - w0)) return;
    __threadfence();
    float all[VEC] = {};
    for (long long u = w0; u <= w1; ++u) {       // in order, whoever comes last
      const float* q = a.part + (u * 2 + (u == w0 ? 1 : 0)) * width + (long long)c * VEC;
#pragma unroll
      for (int j = 0; j < VEC; ++j) all[j] += __ldcg(q + j);
    }
    write_row<T, VEC>(row, all, a.scale, a.accumulate);
  };

  float sum[VEC] = {};
  int v = a.key[s0];
  for (int s = (int)s0; s < s1; s += GRAD_AHEAD) {
    Piece<G, VEC> x[GRAD_AHEAD];
    int key[GRAD_AHEAD];
#pragma unroll
    for (int k = 0; k < GRAD_AHEAD; ++k)
      if (s + k < s1) {
        key[k] = a.key[s + k];
        x[k].load(g + a.order[s + k] * a.ld_g);
      }
#pragma unroll
    for (int k = 0; k < GRAD_AHEAD; ++k)
      if (s + k < s1) {
        if (key[k] != v) {
          flush(v, sum);
          v = key[k];
#pragma unroll
          for (int j = 0; j < VEC; ++j) sum[j] = 0.f;
        }
        x[k].add(sum);
      }
  }
  flush(v, sum);
}

// ---------------------------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------------------------
constexpr size_t EMBED_ALIGN = 256;
size_t up(size_t b) { return (b + EMBED_ALIGN - 1) / EMBED_ALIGN * EMBED_ALIGN; }

struct GradPlan {
  int window;
  long long windows;
  size_t order, key, first, part, arrived, total;
};
// The window: enough threads to fill the GPU, and no more partial sums than that takes.
GradPlan grad_plan(const pctc_embed_t* p) {
  GradPlan g;
  const double threads = (double)p->M * ((p->D + 7) / 8);
  int window = 8;
  while (window < 64 && threads / window > 148.0 * 2048) window *= 2;
  g.window = window;
  g.windows = (p->M + window - 1) / window;
  size_t o = 0;
  const auto take = [&](size_t bytes) { const size_t r = o; o += up(bytes); return r; };
  g.order = take((size_t)p->M * 4);
  g.key = take((size_t)p->M * 4);
  g.first = take(((size_t)p->V + 1) * 4);
  g.arrived = take((size_t)g.windows * p->D * 4);       // a counter a group of eight, or a value
  g.part = take((size_t)g.windows * 2 * p->D * 4);
  g.total = o;
  return g;
}

pctc_status_t check_embed(const pctc_embed_t* p) {
  if (!p || p->M < 0 || p->V < 1 || p->D < 1 || !std::isfinite(p->scale)) return PCTC_ERR_INVALID_ARG;
  if (p->ld_w < p->D || p->ld_x < p->D) return PCTC_ERR_INVALID_ARG;
  if (p->M > 0x7fffffffLL - 64 || p->V > 0x7fffffffLL - 1 || p->D > (1 << 24)) return PCTC_ERR_UNSUPPORTED;
  if (p->ld_w > MAX_ELEMENTS / p->V || p->ld_x > MAX_ELEMENTS / (p->M + 1)) return PCTC_ERR_UNSUPPORTED;
  return PCTC_OK;
}
size_t size_of(int dtype) { return dtype == PCTC_BF16 ? 2 : dtype == PCTC_FP32 ? 4 : 1; }
bool wide(const void* p, long long ld, size_t size) {   // groups of eight values can be moved as such
  return ((size_t)p & (size == 1 ? 7 : 15)) == 0 && (ld * (long long)size) % (size == 1 ? 8 : 16) == 0;
}

template <typename W, typename T>
cudaError_t embed_launch(EmbedArgs a, bool vec, cudaStream_t stream) {
  a.per_row = (unsigned)(vec ? a.D / 8 : a.D);
  a.groups = a.M * a.per_row;
  const long long blocks = (a.groups + EMBED_THREADS * EMBED_VECS - 1) / (EMBED_THREADS * EMBED_VECS);
  if (blocks > 0x7fffffffLL) return cudaErrorInvalidValue;
  if (vec) k_embed<W, T, 8><<<(unsigned)blocks, EMBED_THREADS, 0, stream>>>(a);
  else k_embed<W, T, 1><<<(unsigned)blocks, EMBED_THREADS, 0, stream>>>(a);
  return cudaGetLastError();
}
template <typename W>
cudaError_t embed_launch(const EmbedArgs& a, int out, bool vec, cudaStream_t stream) {
  return out == PCTC_BF16 ? embed_launch<W, __nv_bfloat16>(a, vec, stream) : embed_launch<W, float>(a, vec, stream);
}

template <typename G, typename T>
cudaError_t grad_launch(GradArgs a, long long D, bool vec, cudaStream_t stream) {
  a.per_row = (unsigned)(vec ? D / 8 : D);
  const long long sums = (a.windows * a.per_row + GRAD_THREADS - 1) / GRAD_THREADS;
  const long long zeros = a.accumulate ? 0 : (a.V * a.per_row + GRAD_THREADS * GRAD_ZERO_VECS - 1) / (GRAD_THREADS * GRAD_ZERO_VECS);
  if (sums + zeros > 0x7fffffffLL) return cudaErrorInvalidValue;
  a.sum_blocks = (unsigned)sums;
  if (vec) k_embed_grad<G, T, 8><<<(unsigned)(sums + zeros), GRAD_THREADS, 0, stream>>>(a);
  else k_embed_grad<G, T, 1><<<(unsigned)(sums + zeros), GRAD_THREADS, 0, stream>>>(a);
  return cudaGetLastError();
}

pctc_status_t status_of(cudaError_t e) {
  return e == cudaSuccess ? PCTC_OK : e == cudaErrorInvalidValue ? PCTC_ERR_UNSUPPORTED : PCTC_ERR_CUDA;
}

}  // namespace
}  // namespace pctc

using namespace pctc;

extern "C" {

pctc_status_t pctc_embed(const pctc_embed_t* p, const int32_t* tokens, const void* W, const float* row_scales, void* out,
                         void* stream_v) {
  const pctc_status_t st = check_embed(p);
  if (st != PCTC_OK) return st;
  if (p->dtype_w != PCTC_BF16 && p->dtype_w != PCTC_FP32 && p->dtype_w != PCTC_INT8) return PCTC_ERR_UNSUPPORTED;
  if (p->dtype_x != PCTC_BF16 && p->dtype_x != PCTC_FP32) return PCTC_ERR_UNSUPPORTED;
  if ((p->dtype_w == PCTC_INT8) != (row_scales != nullptr)) return PCTC_ERR_INVALID_ARG;
  if (p->M == 0) return PCTC_OK;
  const size_t ws = size_of(p->dtype_w), xs = size_of(p->dtype_x);
  if (!tokens || !W || !out || ((size_t)tokens & 3) || ((size_t)row_scales & 3) || ((size_t)W & (ws - 1)) || ((size_t)out & (xs - 1)))
    return PCTC_ERR_INVALID_ARG;
  const Rows to{out, p->M, p->ld_x, p->D, xs};
  if (to.overlaps(Rows{W, p->V, p->ld_w, p->D, ws}) || to.overlaps(Rows{tokens, 1, p->M, p->M, 4}) ||
      to.overlaps(Rows{row_scales, 1, p->V, p->V, 4}))
    return PCTC_ERR_INVALID_ARG;
  EmbedArgs a = {};
  a.tokens = tokens;
  a.W = W;
  a.row_scales = row_scales;
  a.out = out;
  a.M = p->M; a.V = p->V; a.D = p->D;
  a.ld_w = p->ld_w;
  a.ld_out = p->ld_x;
  a.scale = p->scale;
  const bool vec = p->D % 8 == 0 && wide(W, p->ld_w, ws) && wide(out, p->ld_x, xs);
  cudaStream_t stream = (cudaStream_t)stream_v;
  return status_of(p->dtype_w == PCTC_BF16   ? embed_launch<__nv_bfloat16>(a, p->dtype_x, vec, stream)
                   : p->dtype_w == PCTC_FP32 ? embed_launch<float>(a, p->dtype_x, vec, stream)
                                             : embed_launch<signed char>(a, p->dtype_x, vec, stream));
}

pctc_status_t pctc_embed_grad_workspace_bytes(const pctc_embed_t* p, size_t* bytes_out) {
  if (!bytes_out) return PCTC_ERR_INVALID_ARG;
  const pctc_status_t st = check_embed(p);
  if (st != PCTC_OK) return st;
  *bytes_out = grad_plan(p).total;
  return PCTC_OK;
}

pctc_status_t pctc_embed_grad(const pctc_embed_t* p, const int32_t* tokens, const void* grad, void* dW, void* workspace,
                              size_t workspace_bytes, void* stream_v) {
  const pctc_status_t st = check_embed(p);
  if (st != PCTC_OK) return st;
  for (const int32_t t : {p->dtype_w, p->dtype_x})
    if (t != PCTC_BF16 && t != PCTC_FP32) return PCTC_ERR_UNSUPPORTED;
  if (p->M == 0 && p->accumulate) return PCTC_OK;
  const size_t ws = size_of(p->dtype_w), xs = size_of(p->dtype_x);
  if (!dW || ((size_t)dW & (ws - 1)) || !workspace || ((size_t)workspace & (EMBED_ALIGN - 1))) return PCTC_ERR_INVALID_ARG;
  if (p->M > 0 && (!tokens || !grad || ((size_t)tokens & 3) || ((size_t)grad & (xs - 1)))) return PCTC_ERR_INVALID_ARG;
  const GradPlan g = grad_plan(p);
  if (workspace_bytes < g.total) return PCTC_ERR_WORKSPACE_TOO_SMALL;
  const Rows to{dW, p->V, p->ld_w, p->D, ws}, own{workspace, 1, (long long)g.total, (long long)g.total, 1},
      from{grad, p->M, p->ld_x, p->D, xs}, ids{tokens, 1, p->M, p->M, 4};
  if (to.overlaps(from) || to.overlaps(ids) || to.overlaps(own) || own.overlaps(from) || own.overlaps(ids)) return PCTC_ERR_INVALID_ARG;

  cudaStream_t stream = (cudaStream_t)stream_v;
  char* w = (char*)workspace;
  const bool vec = p->D % 8 == 0 && wide(dW, p->ld_w, ws) && wide(grad, p->ld_x, xs);
  const long long width = (p->V + SORT_BUCKETS - 1) / SORT_BUCKETS;
  SortArgs s = {};
  s.tokens = tokens;
  s.M = (int)p->M;
  s.V = p->V;
  s.width = (int)(width < SORT_MAX_WIDTH ? width : SORT_MAX_WIDTH);
  s.order = (int*)(w + g.order);
  s.key = (int*)(w + g.key);
  s.first = (int*)(w + g.first);
  s.clear = (int*)(w + g.arrived);
  s.n_clear = g.windows * (vec ? p->D / 8 : p->D);
  const int smem = SORT_WARPS * s.width * 4;
  cudaError_t e = cudaFuncSetAttribute(k_sort_tokens, cudaFuncAttributeMaxDynamicSharedMemorySize, SORT_WARPS * SORT_MAX_WIDTH * 4);
  if (e != cudaSuccess) return PCTC_ERR_CUDA;
  k_sort_tokens<<<(unsigned)((p->V + s.width - 1) / s.width), SORT_THREADS, smem, stream>>>(s);
  e = cudaGetLastError();
  if (e != cudaSuccess) return PCTC_ERR_CUDA;

  GradArgs a = {};
  a.g = grad;
  a.dW = dW;
  a.order = s.order;
  a.key = s.key;
  a.first = s.first;
  a.part = (float*)(w + g.part);
  a.arrived = s.clear;
  a.ld_g = p->ld_x;
  a.ld_w = p->ld_w;
  a.V = p->V;
  a.windows = g.windows;
  a.window = g.window;
  a.accumulate = p->accumulate;
  a.scale = p->scale;
  if (p->dtype_x == PCTC_BF16)
    e = p->dtype_w == PCTC_BF16 ? grad_launch<__nv_bfloat16, __nv_bfloat16>(a, p->D, vec, stream)
                                : grad_launch<__nv_bfloat16, float>(a, p->D, vec, stream);
  else
    e = p->dtype_w == PCTC_BF16 ? grad_launch<float, __nv_bfloat16>(a, p->D, vec, stream)
                                : grad_launch<float, float>(a, p->D, vec, stream);
  return status_of(e);
}

}  // extern "C"
