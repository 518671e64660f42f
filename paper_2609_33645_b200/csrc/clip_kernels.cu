// Global gradient norm over many tensors, and clipping:
//   S = sum over all tensors and values of g^2,   norm = sqrt(S),
//   f = min(1, max_norm / (norm + eps)),          out = round(f * g).
//
// Every value has to be read once for S before the first one may be scaled, so a call is two passes:
// k_square_sums reads everything and leaves one partial sum per CTA, k_scale adds the partials up (every
// CTA the same ones in the same order, so all agree on f) and scales.  In place with f = 1 the second
// pass ends there: the usual step of a training run reads its gradients once and writes nothing.
// Both are bound by HBM; the arithmetic is one multiply-add a value.
//
// Measured: 156M bf16 values into another buffer 140 us (three passes of 312 MB at the rate of a copy: 143; the last 64 MB
// of the first pass are still in L2 for the second); 64M bf16 values in 384 tensors, in place below the limit, 27 us
// (one pass: 20; a bare read of the same bytes: 23); 100,000 fp32 values in 7 tensors 6.3 us in one launch (two
// launches cost the host 6 us more).
#include "../../include/prunedctc.h"
#include "pctc_internal.h"

#include <cooperative_groups.h>

#include <cfloat>
#include <cmath>
#include <new>

namespace cg = cooperative_groups;

namespace pctc {
namespace {

// Work is cut into chunks of 16 KB of one tensor: 256 threads with four 16-byte loads each, in a persistent grid of
// CLIP_CTAS_PER_SM such CTAs an SM.
constexpr int CLIP_THREADS = 256;
constexpr int CLIP_VECS = 4;
constexpr int CLIP_CHUNK_BYTES = CLIP_THREADS * CLIP_VECS * 16;
constexpr int CLIP_CTAS_PER_SM = 6;              // first pass: 49 us for 312 MB (4: 53)
constexpr int CLIP_SCALE_CTAS_PER_SM = 4;        // second pass: 105 us for 312 MB in and out (6: 119)
constexpr int CLIP_KEEP_CHUNKS = 4096;           // the last 64 MB of the first pass stay in L2, the rest goes past it
constexpr int CLIP_EACH_CHUNKS = 2048;           // from so many chunks on (32 MB: 21.4 against 22.0 us; 312 MB: 150 against
                                                 // 165) the second pass takes a CTA a chunk
constexpr int CLIP_CLUSTER = 8;
constexpr int CLIP_CLUSTER_CHUNKS = 32;          // up to so many chunks one cluster does all
constexpr int CLIP_MAX_GRID = 1024;              // most partial sums of one launch

enum : unsigned char { IN_F32 = 1, OUT_F32 = 2, OUT_VEC = 4, IN_PLACE = 8 };

// The tensors of one launch travel as a kernel parameter (at most 32,764 bytes of them).
template <int LIM>
struct ClipTable {
  const void* in[LIM];
  void* out[LIM];
  long long numel[LIM];
  int chunk0[LIM + 1];                           // chunks before tensor i
  unsigned char kind[LIM];
  int n;
  int in_place;                                  // all of them
};
constexpr int CLIP_LARGE = 1024;                 // tensors of one launch; lists of up to 48, 192 and 512 take smaller tables
static_assert(sizeof(ClipTable<CLIP_LARGE>) <= 32000, "kernel parameters");

// The piece of a tensor that a chunk covers: values [start, start + count), the first `nvec` groups of 16 bytes
// read a group at a time; chunk 0 also takes the `head` values in front of the first 16-byte boundary.
struct Piece {
  const void* p;
  long long start;
  int count, nvec, head, kind, tensor;
};
__host__ __device__ __forceinline__ int head_of(const void* p, long long numel, int es) {
  const int mis = (int)((size_t)p & 15);
  const int head = mis ? (16 - mis) / es : 0;
  return head < numel ? head : (int)numel;
}

// The last tensor whose first chunk is <= c, by a whole warp: 32 probes of the table at a time.  `chunk0` is a copy in
// shared memory: a binary search of the parameter by every thread takes as many instructions as a chunk's sums (384
// tensors of 128 MB: 25.3 us against 24.5).
__device__ __forceinline__ int tensor_of(const int* chunk0, int n, int c) {
  const int lane = threadIdx.x & 31;
  int lo = 0;
  while (n > 1) {
    const int step = (n + 31) >> 5, at = lane * step;
    const unsigned m = __ballot_sync(0xffffffffu, at < n && chunk0[lo + min(at, n - 1)] <= c);
    const int k = 31 - __clz(m);                 // the first probe always holds
    lo += k * step;
    n = min(step, n - k * step);
  }
  return lo;
}
template <int LIM>
__device__ __forceinline__ void copy_chunks(int* chunk0, const ClipTable<LIM>& tab) {
  for (int i = threadIdx.x; i < tab.n; i += CLIP_THREADS) chunk0[i] = tab.chunk0[i];
  __syncthreads();
}

__device__ __forceinline__ float bf16_lo(unsigned v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float bf16_hi(unsigned v) { return __uint_as_float(v & 0xffff0000u); }

// Sum of squares of a few values.  fp32 while the sum lies where fp32 squares neither overflow nor lose
// bits to underflow (values between 1e-15 and 3e18); otherwise again in 64 bits.  The partial sums of
// a few values are then added in 64 bits, so that a sum over 1e9 values is good to 1e-7.
template <int K>
__device__ __forceinline__ double square_sum(const float (&x)[K]) {
  float s = x[0] * x[0];
#pragma unroll
  for (int i = 1; i < K; ++i) s = fmaf(x[i], x[i], s);
  if (s > 1e-30f && s < 1e37f) return (double)s;
  float big = 0.f;
#pragma unroll
  for (int i = 0; i < K; ++i) big = fmaxf(big, fabsf(x[i]));
  if (s == 0.f && big == 0.f) return 0.0;
  double d = 0.0;
#pragma unroll
  for (int i = 0; i < K; ++i) d += (double)x[i] * (double)x[i];
  return d;
}

template <typename T>
__device__ __forceinline__ float load1(const void* p, long long i);
template <>
__device__ __forceinline__ float load1<float>(const void* p, long long i) { return ((const float*)p)[i]; }
template <>
__device__ __forceinline__ float load1<__nv_bfloat16>(const void* p, long long i) {
  return __bfloat162float(((const __nv_bfloat16*)p)[i]);
}

__device__ __forceinline__ double square_sum_vec(const uint4& v, bool f32) {
  if (f32) {
    const float x[4] = {__uint_as_float(v.x), __uint_as_float(v.y), __uint_as_float(v.z), __uint_as_float(v.w)};
    return square_sum(x);
  }
  const float x[8] = {bf16_lo(v.x), bf16_hi(v.x), bf16_lo(v.y), bf16_hi(v.y),
                      bf16_lo(v.z), bf16_hi(v.z), bf16_lo(v.w), bf16_hi(v.w)};
  return square_sum(x);
}

template <int LIM>
__device__ __forceinline__ Piece piece_in(const ClipTable<LIM>& tab, int tensor, int c) {
  Piece r;
  r.tensor = tensor;
  r.p = tab.in[r.tensor];
  r.kind = tab.kind[r.tensor];
  const long long numel = tab.numel[r.tensor];
  const int local = c - tab.chunk0[r.tensor], shift = r.kind & IN_F32 ? 2 : 1;
  const int head = head_of(r.p, numel, 1 << shift);
  r.start = head + ((long long)local << (14 - shift));
  const long long left = numel - r.start;
  r.count = (int)(left < (CLIP_CHUNK_BYTES >> shift) ? left : CLIP_CHUNK_BYTES >> shift);
  r.nvec = r.count >> (4 - shift);
  r.head = local ? 0 : head;
  return r;
}
template <int LIM>
__device__ __forceinline__ Piece piece_of(const ClipTable<LIM>& tab, const int* chunk0, int c) {
  return piece_in(tab, tensor_of(chunk0, tab.n, c), c);
}
template <int LIM>
__device__ __forceinline__ Piece piece_of(const ClipTable<LIM>& tab, int c) {
  int lo = 0, hi = tab.n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (tab.chunk0[mid] <= c) lo = mid; else hi = mid - 1;
  }
  return piece_in(tab, lo, c);
}
static_assert(CLIP_CHUNK_BYTES == 1 << 14, "chunks are 16 KB");

__device__ __forceinline__ const uint4* vectors(const Piece& r) {
  return (const uint4*)((const char*)r.p + (r.start << (r.kind & IN_F32 ? 2 : 1)));
}
// keep: leave the lines in L2 for the second pass.
__device__ __forceinline__ void load_piece(uint4 (&v)[CLIP_VECS], const Piece& r, bool keep) {
  const uint4* p = vectors(r);
#pragma unroll
  for (int j = 0; j < CLIP_VECS; ++j) {
    const int i = threadIdx.x + j * CLIP_THREADS;
    v[j] = i < r.nvec ? (keep ? p[i] : __ldcs(p + i)) : make_uint4(0, 0, 0, 0);
  }
}
__device__ __forceinline__ float one_value(const Piece& r, long long i) {
  return r.kind & IN_F32 ? load1<float>(r.p, i) : load1<__nv_bfloat16>(r.p, i);
}
__device__ __forceinline__ double piece_squares(const uint4 (&v)[CLIP_VECS], const Piece& r) {
  const bool f32 = r.kind & IN_F32;
  double acc = 0.0;
#pragma unroll
  for (int j = 0; j < CLIP_VECS; ++j) acc += square_sum_vec(v[j], f32);
  const int body = r.nvec * (f32 ? 4 : 8);
  if ((int)threadIdx.x < r.head) { const float x[1] = {one_value(r, threadIdx.x)}; acc += square_sum(x); }
  if ((int)threadIdx.x < r.count - body) { const float x[1] = {one_value(r, r.start + body + threadIdx.x)}; acc += square_sum(x); }
  return acc;
}

__device__ __forceinline__ double block_sum(double v) {
  __shared__ double part[CLIP_THREADS / 32];
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
  __syncthreads();
  double s = 0.0;
#pragma unroll
  for (int w = 0; w < CLIP_THREADS / 32; ++w) s += part[w];
  return s;
}

template <int LIM>
__device__ __forceinline__ double square_sums(const ClipTable<LIM>& tab, const int* chunk0, int first, int step) {
  double acc = 0.0;
  const int total = tab.chunk0[tab.n];
  for (int c = first; c < total; c += step) {
    const Piece r = piece_of(tab, chunk0, c);
    uint4 v[CLIP_VECS];
    load_piece(v, r, c >= total - CLIP_KEEP_CHUNKS);
    acc += piece_squares(v, r);
  }
  return acc;
}

template <int LIM>
__global__ void __launch_bounds__(CLIP_THREADS, CLIP_CTAS_PER_SM) k_square_sums(const __grid_constant__ ClipTable<LIM> tab,
                                                                                double* __restrict__ partial) {
  __shared__ int chunk0[LIM];
  copy_chunks(chunk0, tab);
  const double s = block_sum(square_sums(tab, chunk0, blockIdx.x, gridDim.x));
  if (threadIdx.x == 0) partial[blockIdx.x] = s;
}

__global__ void __launch_bounds__(CLIP_THREADS) k_sum_partials(const double* __restrict__ partial, int np,
                                                               double* __restrict__ sqsum) {
  double acc = 0.0;
  for (int i = threadIdx.x; i < np; i += CLIP_THREADS) acc += partial[i];
  const double s = block_sum(acc);
  if (threadIdx.x == 0) *sqsum = s;
}

__device__ __forceinline__ void store1(void* p, long long i, float x, bool f32) {
  if (f32) ((float*)p)[i] = x; else ((__nv_bfloat16*)p)[i] = __float2bfloat16_rn(x);
}
__device__ __forceinline__ unsigned pack_bf16(float lo, float hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const unsigned*>(&h);
}

// g * f in fp32; by a factor below fp32's normal range (TINY) in 64 bits.
template <bool TINY>
__device__ __forceinline__ float scaled(float x, float f, double fd) {
  return TINY ? (float)((double)x * fd) : x * f;
}

template <bool F32, bool TINY>
__device__ __forceinline__ void scale_piece(const uint4 (&v)[CLIP_VECS], const Piece& r, void* o, float f, double fd) {
  constexpr int VE = F32 ? 4 : 8;
  const bool of32 = r.kind & OUT_F32, vec = r.kind & OUT_VEC;
#pragma unroll
  for (int j = 0; j < CLIP_VECS; ++j) {
    const int i = threadIdx.x + j * CLIP_THREADS;
    if (i >= r.nvec) continue;
    const unsigned w[4] = {v[j].x, v[j].y, v[j].z, v[j].w};
    float x[VE];
#pragma unroll
    for (int q = 0; q < VE; ++q) {
      const float g = F32 ? __uint_as_float(w[q & 3]) : q & 1 ? bf16_hi(w[q / 2]) : bf16_lo(w[q / 2]);
      x[q] = scaled<TINY>(g, f, fd);
    }
    const long long at = r.start + (long long)i * VE;
    if (vec && of32) {
      float4* d = (float4*)((float*)o + at);
#pragma unroll
      for (int q = 0; q < VE / 4; ++q) __stcs(d + q, make_float4(x[4 * q], x[4 * q + 1], x[4 * q + 2], x[4 * q + 3]));
    } else if (vec && !F32) {
      __stcs((uint4*)((__nv_bfloat16*)o + at), make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]),
                                                          pack_bf16(x[VE - 4], x[VE - 3]), pack_bf16(x[VE - 2], x[VE - 1])));
    } else {
#pragma unroll
      for (int q = 0; q < VE; ++q) store1(o, at + q, x[q], of32);
    }
  }
}
__device__ __forceinline__ void scale_one(const Piece& r, void* o, long long i, float f, double fd) {
  store1(o, i, f >= FLT_MIN ? scaled<false>(one_value(r, i), f, fd) : scaled<true>(one_value(r, i), f, fd), r.kind & OUT_F32);
}

// Scales a chunk that has been loaded.
template <int LIM>
__device__ __forceinline__ void scale_chunk(const ClipTable<LIM>& tab, const Piece& r, const uint4 (&v)[CLIP_VECS], float f,
                                            double fd) {
  void* o = tab.out[r.tensor];
  if (f >= FLT_MIN) {
    if (r.kind & IN_F32) scale_piece<true, false>(v, r, o, f, fd);
    else scale_piece<false, false>(v, r, o, f, fd);
  } else {
    if (r.kind & IN_F32) scale_piece<true, true>(v, r, o, f, fd);
    else scale_piece<false, true>(v, r, o, f, fd);
  }
  const int body = r.nvec * (r.kind & IN_F32 ? 4 : 8);
  if ((int)threadIdx.x < r.head) scale_one(r, o, threadIdx.x, f, fd);
  if ((int)threadIdx.x < r.count - body) scale_one(r, o, r.start + body + threadIdx.x, f, fd);
}

// Chunks first, first - step, ...  Backwards: those that the first pass read last are still in L2.
template <int LIM>
__device__ __forceinline__ void scale_all(const ClipTable<LIM>& tab, const int* chunk0, int first, int step, float f,
                                          double fd) {
  for (int c = first; c >= 0; c -= step) {
    const Piece r = piece_of(tab, chunk0, c);
    if (f == 1.0f && (r.kind & IN_PLACE)) continue;
    uint4 v[CLIP_VECS];
    load_piece(v, r, false);
    scale_chunk(tab, r, v, f, fd);
  }
}

// The factor, in 64 bits.  A norm that is not finite (in fp32, as the caller sees it) scales nothing: no factor
// would mend such a step.
__device__ __forceinline__ double factor_of(double norm, float max_norm, float eps) {
  const double ratio = (double)max_norm / (norm + (double)eps);
  return isfinite((float)norm) && ratio < 1.0 ? ratio : 1.0;
}

// Norm and factor from the partial sums, then the scaled values.
template <int LIM>
__global__ void __launch_bounds__(CLIP_THREADS) k_scale(const __grid_constant__ ClipTable<LIM> tab,
                                                        const double* __restrict__ partial, int np, float max_norm,
                                                        float eps, float* __restrict__ norm_out) {
  double acc = 0.0;
  for (int i = threadIdx.x; i < np; i += CLIP_THREADS) acc += partial[i];
  const double norm = sqrt(block_sum(acc));
  const double fd = factor_of(norm, max_norm, eps);
  const float f = (float)fd;
  if (norm_out && blockIdx.x == 0 && threadIdx.x == 0) *norm_out = (float)norm;
  if (f == 1.0f && tab.in_place) return;
  __shared__ int chunk0[LIM];
  copy_chunks(chunk0, tab);
  scale_all(tab, chunk0, tab.chunk0[tab.n] - 1 - (int)blockIdx.x, gridDim.x, f, fd);
}

// The same for many values that all have to be written, with one CTA a chunk: CTAs that start in order keep reads and
// writes of HBM closer together than a persistent grid, whose CTAs drift apart (99 against 111 us for 327 MB in and
// out).  The sum is a single value here, and a CTA's loads are under way while it makes the factor of it.
template <int LIM>
__global__ void __launch_bounds__(CLIP_THREADS) k_scale_each(const __grid_constant__ ClipTable<LIM> tab,
                                                             const double* __restrict__ sqsum, float max_norm, float eps,
                                                             float* __restrict__ norm_out) {
  __shared__ double factor;
  const Piece r = piece_of(tab, gridDim.x - 1 - blockIdx.x);     // searches the parameter: one chunk is all there is
  uint4 v[CLIP_VECS];
  load_piece(v, r, false);
  if (threadIdx.x == 0) {
    const double norm = sqrt(*sqsum);
    factor = factor_of(norm, max_norm, eps);
    if (norm_out && blockIdx.x == 0) *norm_out = (float)norm;
  }
  __syncthreads();
  const double fd = factor;
  const float f = (float)fd;
  if (f == 1.0f && (r.kind & IN_PLACE)) return;
  scale_chunk(tab, r, v, f, fd);
}

// Few values: all of it in one launch, by one cluster of CTAs that add their sums up in distributed shared memory.  A CTA
// keeps its chunks (at most four) in registers from the sum to the scaling, so that every value is read once.
template <int LIM>
__global__ void __cluster_dims__(CLIP_CLUSTER, 1, 1) __launch_bounds__(CLIP_THREADS)
    k_clip_small(const __grid_constant__ ClipTable<LIM> tab, float max_norm, float eps, float* __restrict__ norm_out) {
  constexpr int MOST = CLIP_CLUSTER_CHUNKS / CLIP_CLUSTER;
  __shared__ double mine;
  cg::cluster_group cluster = cg::this_cluster();
  const int total = tab.chunk0[tab.n], rank = blockIdx.x;
  Piece r[MOST];
  uint4 v[MOST][CLIP_VECS];
#pragma unroll
  for (int u = 0; u < MOST; ++u) {
    const int c = rank + u * CLIP_CLUSTER;
    if (c < total) {
      r[u] = piece_of(tab, c);
      load_piece(v[u], r[u], true);
    }
  }
  double acc = 0.0;
#pragma unroll
  for (int u = 0; u < MOST; ++u)
    if (rank + u * CLIP_CLUSTER < total) acc += piece_squares(v[u], r[u]);
  const double s = block_sum(acc);
  if (threadIdx.x == 0) mine = s;
  cluster.sync();
  double all = 0.0;
#pragma unroll
  for (int o = 0; o < CLIP_CLUSTER; ++o) all += *cluster.map_shared_rank(&mine, o);
  cluster.sync();                                 // nobody leaves before all have read
  const double norm = sqrt(all), fd = factor_of(norm, max_norm, eps);
  const float f = (float)fd;
  if (rank == 0 && threadIdx.x == 0) *norm_out = (float)norm;
#pragma unroll
  for (int u = 0; u < MOST; ++u)
    if (rank + u * CLIP_CLUSTER < total && !(f == 1.0f && (r[u].kind & IN_PLACE))) scale_chunk(tab, r[u], v[u], f, fd);
}

struct ClipList {
  int n;
  const void* const* grads;
  void* const* outs;                             // null: in place
  const int64_t* numels;
  const int32_t* dtypes;
  const int32_t* out_dtypes;                     // null: as dtypes
  const void* in(int i) const { return grads[i]; }
  void* out(int i) const { return outs ? outs[i] : const_cast<void*>(grads[i]); }
  int out_dtype(int i) const { return out_dtypes ? out_dtypes[i] : dtypes[i]; }
};

int elem_bytes(int dtype) { return dtype == PCTC_BF16 ? 2 : 4; }

// Host checks of the list.  `writes`: the call scales, so that what it writes may overlap nothing else; `own` is the
// norm, and the workspace or the sum of squares.
pctc_status_t check_list(const ClipList& l, bool writes, Span own0, Span own1) {
  if (l.n < 0) return PCTC_ERR_INVALID_ARG;
  if (l.n && (!l.grads || !l.numels || !l.dtypes)) return PCTC_ERR_INVALID_ARG;
  for (int i = 0; i < l.n; ++i) {
    if (l.numels[i] < 0) return PCTC_ERR_INVALID_ARG;
    if (l.dtypes[i] != PCTC_BF16 && l.dtypes[i] != PCTC_FP32) return PCTC_ERR_UNSUPPORTED;
    if (writes && l.out_dtype(i) != l.dtypes[i] && l.out_dtype(i) != PCTC_FP32) return PCTC_ERR_UNSUPPORTED;
    if (l.numels[i] == 0) continue;
    if (l.numels[i] > (1LL << 42)) return PCTC_ERR_UNSUPPORTED;
    if (!l.in(i) || ((size_t)l.in(i) & (elem_bytes(l.dtypes[i]) - 1))) return PCTC_ERR_INVALID_ARG;
    if (!writes) continue;
    if (!l.out(i) || ((size_t)l.out(i) & (elem_bytes(l.out_dtype(i)) - 1))) return PCTC_ERR_INVALID_ARG;
    if (l.out(i) == l.in(i) && l.out_dtype(i) != l.dtypes[i]) return PCTC_ERR_INVALID_ARG;
  }
  Span* spans = new (std::nothrow) Span[2 * (size_t)l.n + 2];
  if (!spans) return PCTC_ERR_HOST_MEMORY;
  size_t ns = 0;
  for (const Span& own : {own0, own1})
    if (own.lo < own.hi) spans[ns++] = own;
  for (int i = 0; i < l.n; ++i) {
    if (l.numels[i] == 0) continue;
    const size_t a = (size_t)l.in(i), b = (size_t)l.out(i);
    if (writes) spans[ns++] = Span{b, b + (size_t)l.numels[i] * elem_bytes(l.out_dtype(i)), true};
    if (!writes || a != b) spans[ns++] = Span{a, a + (size_t)l.numels[i] * elem_bytes(l.dtypes[i]), false};
  }
  const bool clash = spans_conflict(spans, ns);
  delete[] spans;
  return clash ? PCTC_ERR_INVALID_ARG : PCTC_OK;
}

template <int LIM>
pctc_status_t fill_table(const ClipList& l, int i0, int i1, bool writes, ClipTable<LIM>* tab) {
  tab->n = 0;
  tab->in_place = 1;
  long long chunks = 0;
  for (int i = i0; i < i1; ++i) {
    if (l.numels[i] == 0) continue;
    const int k = tab->n++;
    const int es = elem_bytes(l.dtypes[i]);
    tab->in[k] = l.in(i);
    tab->numel[k] = l.numels[i];
    tab->chunk0[k] = (int)chunks;
    unsigned char kind = l.dtypes[i] == PCTC_FP32 ? IN_F32 : 0;
    void* out = nullptr;
    if (writes) {
      out = l.out(i);
      if (out == l.in(i)) kind |= IN_PLACE; else tab->in_place = 0;
      if (l.out_dtype(i) == PCTC_FP32) kind |= OUT_F32;
      // stores are as wide as the loads where the output reaches a 16-byte boundary with the input
      const size_t head = head_of(l.in(i), l.numels[i], es);
      if ((((size_t)out + head * elem_bytes(l.out_dtype(i))) & 15) == 0) kind |= OUT_VEC;
    }
    tab->out[k] = out;
    tab->kind[k] = kind;
    const long long body = l.numels[i] - head_of(l.in(i), l.numels[i], es), per = CLIP_CHUNK_BYTES / es;
    chunks += body ? (body + per - 1) / per : 1;
    if (chunks > 0x7fff0000LL) return PCTC_ERR_UNSUPPORTED;
  }
  tab->chunk0[tab->n] = (int)chunks;
  return PCTC_OK;
}

int clip_grid(int chunks, int per_sm) {
  int dev = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
    sms = 148;
  int most = sms * per_sm;
  if (most > CLIP_MAX_GRID) most = CLIP_MAX_GRID;
  return chunks < 1 ? 1 : chunks < most ? chunks : most;
}

template <int LIM>
pctc_status_t sum_launch(const ClipTable<LIM>& tab, double* partial, int* np, cudaStream_t stream) {
  const int grid = clip_grid(tab.chunk0[tab.n], CLIP_CTAS_PER_SM);
  k_square_sums<LIM><<<grid, CLIP_THREADS, 0, stream>>>(tab, partial + *np);
  *np += grid;
  return cudaGetLastError() == cudaSuccess ? PCTC_OK : PCTC_ERR_CUDA;
}

// sums: np of them, and room for one more behind them (np == 1: the whole sum, which nothing is written to).
template <int LIM>
pctc_status_t scale_launch(const ClipTable<LIM>& tab, const double* sums, int np, float max_norm, float eps, float* norm,
                           cudaStream_t stream) {
  const int chunks = tab.chunk0[tab.n];
  if (!tab.in_place && chunks >= CLIP_EACH_CHUNKS) {
    if (np > 1) {
      k_sum_partials<<<1, CLIP_THREADS, 0, stream>>>(sums, np, const_cast<double*>(sums) + np);
      sums += np;
    }
    k_scale_each<LIM><<<chunks, CLIP_THREADS, 0, stream>>>(tab, sums, max_norm, eps, norm);
  } else {
    k_scale<LIM><<<clip_grid(chunks, CLIP_SCALE_CTAS_PER_SM), CLIP_THREADS, 0, stream>>>(tab, sums, np, max_norm, eps, norm);
  }
  return cudaGetLastError() == cudaSuccess ? PCTC_OK : PCTC_ERR_CUDA;
}

// The launches of a call: the sums of all tensors (given == null), then the scaling (max_norm > 0), LIM tensors at a
// time.  With one table for all tensors both passes share it, and few values need one launch.
template <int LIM>
pctc_status_t clip_launches(const ClipList& l, const double* given, double* partial, double* sqsum, float max_norm, float eps,
                            float* norm, cudaStream_t stream) {
  ClipTable<LIM> tab;
  const bool scaling = max_norm > 0.f, one = l.n <= LIM;
  int np = 0;
  for (int i0 = 0; !given && (i0 == 0 || i0 < l.n); i0 += LIM) {
    pctc_status_t st = fill_table<LIM>(l, i0, one ? l.n : l.n < i0 + LIM ? l.n : i0 + LIM, scaling, &tab);
    if (st != PCTC_OK) return st;
    if (one && scaling && tab.chunk0[tab.n] <= CLIP_CLUSTER_CHUNKS) {
      k_clip_small<LIM><<<CLIP_CLUSTER, CLIP_THREADS, 0, stream>>>(tab, max_norm, eps, norm);
      return cudaGetLastError() == cudaSuccess ? PCTC_OK : PCTC_ERR_CUDA;
    }
    st = sum_launch(tab, partial, &np, stream);
    if (st != PCTC_OK) return st;
  }
  if (!scaling) {
    k_sum_partials<<<1, CLIP_THREADS, 0, stream>>>(partial, np, sqsum);
    return cudaGetLastError() == cudaSuccess ? PCTC_OK : PCTC_ERR_CUDA;
  }
  for (int i0 = 0; i0 == 0 || i0 < l.n; i0 += LIM) {
    if (given || !one) {
      const pctc_status_t st = fill_table<LIM>(l, i0, l.n < i0 + LIM ? l.n : i0 + LIM, true, &tab);
      if (st != PCTC_OK) return st;
    }
    const pctc_status_t st = scale_launch(tab, given ? given : partial, given ? 1 : np, max_norm, eps, i0 == 0 ? norm : nullptr, stream);
    if (st != PCTC_OK) return st;
  }
  return PCTC_OK;
}

pctc_status_t clip_call(const ClipList& l, const double* given, double* partial, double* sqsum, float max_norm, float eps,
                        float* norm, void* stream_v) {
  cudaStream_t stream = (cudaStream_t)stream_v;
  // a launch copies its whole table, so the smallest that holds the list
  return l.n <= 48    ? clip_launches<48>(l, given, partial, sqsum, max_norm, eps, norm, stream)
         : l.n <= 192 ? clip_launches<192>(l, given, partial, sqsum, max_norm, eps, norm, stream)
         : l.n <= 512 ? clip_launches<512>(l, given, partial, sqsum, max_norm, eps, norm, stream)
                      : clip_launches<CLIP_LARGE>(l, given, partial, sqsum, max_norm, eps, norm, stream);
}

bool bad_limits(float max_norm, float eps) {
  return !(max_norm > 0.f) || !(eps >= 0.f) || std::isinf(eps);
}
Span span(const void* p, size_t bytes, bool write) { return Span{(size_t)p, p ? (size_t)p + bytes : 0, write}; }
size_t partial_count(int n) { return 32 + (size_t)CLIP_MAX_GRID * (n <= CLIP_LARGE ? 1 : ((size_t)n + CLIP_LARGE - 1) / CLIP_LARGE); }

}  // namespace
}  // namespace pctc

using namespace pctc;

extern "C" {

pctc_status_t pctc_clip_workspace_bytes(int32_t n, size_t* bytes_out) {
  if (!bytes_out || n < 0) return PCTC_ERR_INVALID_ARG;
  *bytes_out = partial_count(n) * sizeof(double);
  return PCTC_OK;
}

pctc_status_t pctc_grad_sqsum(int32_t n, const void* const* grads, const int64_t* numels, const int32_t* dtypes,
                              double* sqsum, void* workspace, size_t workspace_bytes, void* stream_v) {
  const ClipList l{n, grads, nullptr, numels, dtypes, nullptr};
  const size_t need = partial_count(n) * sizeof(double);
  pctc_status_t st = check_list(l, false, span(sqsum, 8, true), span(workspace, need, true));
  if (st != PCTC_OK) return st;
  if (!sqsum || ((size_t)sqsum & 7) || !workspace || ((size_t)workspace & 255)) return PCTC_ERR_INVALID_ARG;
  if (workspace_bytes < need) return PCTC_ERR_WORKSPACE_TOO_SMALL;
  return clip_call(l, nullptr, (double*)workspace, sqsum, 0.f, 0.f, nullptr, stream_v);
}

pctc_status_t pctc_grad_scale(int32_t n, const void* const* grads, void* const* outs, const int64_t* numels,
                              const int32_t* dtypes, const int32_t* out_dtypes, const double* sqsum, float max_norm,
                              float eps, float* norm, void* stream_v) {
  const ClipList l{n, grads, outs, numels, dtypes, out_dtypes};
  pctc_status_t st = check_list(l, true, span(norm, 4, true), span(sqsum, 8, false));
  if (st != PCTC_OK) return st;
  if (!sqsum || ((size_t)sqsum & 7) || ((size_t)norm & 3) || bad_limits(max_norm, eps)) return PCTC_ERR_INVALID_ARG;
  return clip_call(l, sqsum, nullptr, nullptr, max_norm, eps, norm, stream_v);
}

pctc_status_t pctc_clip_grad_norm(int32_t n, const void* const* grads, void* const* outs, const int64_t* numels,
                                  const int32_t* dtypes, const int32_t* out_dtypes, float max_norm, float eps,
                                  float* norm, void* workspace, size_t workspace_bytes, void* stream_v) {
  const ClipList l{n, grads, outs, numels, dtypes, out_dtypes};
  const size_t need = partial_count(n) * sizeof(double);
  pctc_status_t st = check_list(l, true, span(norm, 4, true), span(workspace, need, true));
  if (st != PCTC_OK) return st;
  if (!norm || ((size_t)norm & 3) || !workspace || ((size_t)workspace & 255) || bad_limits(max_norm, eps)) return PCTC_ERR_INVALID_ARG;
  if (workspace_bytes < need) return PCTC_ERR_WORKSPACE_TOO_SMALL;
  return clip_call(l, nullptr, (double*)workspace, nullptr, max_norm, eps, norm, stream_v);
}

}  // extern "C"
