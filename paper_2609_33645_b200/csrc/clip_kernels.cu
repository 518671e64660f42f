// Global gradient norm over many tensors, and clipping:
//   S = sum over all tensors and values of g^2,   norm = sqrt(S),
//   f = min(1, max_norm / (norm + eps)),          out = round(f * g).
//
// Every value has to be read once for S before the first one may be scaled, so a call is two passes:
// k_square_sums reads everything and leaves one partial sum per CTA, k_scale adds the partials up (every
// CTA the same ones in the same order, so all agree on f) and scales.  In place with f = 1 the second
// pass ends there: the usual step of a training run reads its gradients once and writes nothing.
// Both are bound by HBM; the arithmetic is one multiply-add a value.
#include "../../include/prunedctc.h"
#include "pctc_internal.h"

#include <cmath>
#include <new>

namespace pctc {
namespace {

// Work is cut into chunks of 8,192 values of one tensor: 256 threads with four (bf16) or eight (fp32)
// 16-byte loads in flight each, eight such CTAs an SM.
constexpr int CLIP_THREADS = 256;
constexpr int CLIP_CHUNK = 8192;
constexpr int CLIP_CTAS_PER_SM = 8;
constexpr int CLIP_MAX_GRID = 2048;              // most partial sums of one launch

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
};
constexpr int CLIP_SMALL = 48, CLIP_LARGE = 1024;
static_assert(sizeof(ClipTable<CLIP_LARGE>) <= 32000, "kernel parameters");

// The piece of a tensor that a chunk covers: values [lo, hi), of which [start, start + nvec * VE) can be
// read 16 bytes at a time; chunk 0 also takes the `head` values in front of the first 16-byte boundary.
struct Piece {
  long long start, hi;
  int head;
};
__device__ __forceinline__ Piece piece_of(const void* p, long long numel, int es, int c) {
  Piece r;
  const int mis = (int)((size_t)p & 15);
  const long long head = mis ? (16 - mis) / es : 0;
  r.head = (int)(head < numel ? head : numel);
  r.start = r.head + (long long)c * CLIP_CHUNK;
  r.hi = r.start + CLIP_CHUNK < numel ? r.start + CLIP_CHUNK : numel;
  if (c) r.head = 0;
  return r;
}

template <int LIM>
__device__ __forceinline__ int tensor_of(const ClipTable<LIM>& tab, int c) {
  int lo = 0, hi = tab.n - 1;                    // the last tensor whose first chunk is <= c
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (tab.chunk0[mid] <= c) lo = mid; else hi = mid - 1;
  }
  return lo;
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

template <typename T>
__device__ __forceinline__ double chunk_squares(const void* p, long long numel, int c) {
  constexpr int VE = 16 / (int)sizeof(T), NV = CLIP_CHUNK / (VE * CLIP_THREADS);
  const Piece r = piece_of(p, numel, (int)sizeof(T), c);
  const int tid = threadIdx.x;
  const uint4* body = (const uint4*)((const T*)p + r.start);
  const int left = (int)(r.hi - r.start);        // may be <= 0 when the head is all there is
  const int nvec = left > 0 ? left / VE : 0;
  uint4 v[NV];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int i = tid + j * CLIP_THREADS;
    v[j] = i < nvec ? body[i] : make_uint4(0, 0, 0, 0);
  }
  double acc = 0.0;
#pragma unroll
  for (int j = 0; j < NV; ++j) acc += square_sum_vec(v[j], sizeof(T) == 4);
  const int tail = left > 0 ? left - nvec * VE : 0;
  if (tid < r.head) { const float x[1] = {load1<T>(p, tid)}; acc += square_sum(x); }
  if (tid < tail) { const float x[1] = {load1<T>(p, r.start + nvec * VE + tid)}; acc += square_sum(x); }
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
__global__ void __launch_bounds__(CLIP_THREADS) k_square_sums(const __grid_constant__ ClipTable<LIM> tab,
                                                              double* __restrict__ partial) {
  double acc = 0.0;
  const int total = tab.chunk0[tab.n];
  for (int c = blockIdx.x; c < total; c += gridDim.x) {
    const int i = tensor_of(tab, c);
    acc += (tab.kind[i] & IN_F32) ? chunk_squares<float>(tab.in[i], tab.numel[i], c - tab.chunk0[i])
                                  : chunk_squares<__nv_bfloat16>(tab.in[i], tab.numel[i], c - tab.chunk0[i]);
  }
  const double s = block_sum(acc);
  if (threadIdx.x == 0) partial[blockIdx.x] = s;
}

__global__ void __launch_bounds__(CLIP_THREADS) k_sum_partials(const double* __restrict__ partial, int np,
                                                               double* __restrict__ sqsum) {
  double acc = 0.0;
  for (int i = threadIdx.x; i < np; i += CLIP_THREADS) acc += partial[i];
  const double s = block_sum(acc);
  if (threadIdx.x == 0) *sqsum = s;
}

template <typename T>
__device__ __forceinline__ void store1(void* p, long long i, float x, bool f32) {
  if (f32) ((float*)p)[i] = x; else ((__nv_bfloat16*)p)[i] = __float2bfloat16_rn(x);
}
__device__ __forceinline__ unsigned pack_bf16(float lo, float hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const unsigned*>(&h);
}

// g * f in fp32; by a factor below fp32's normal range in 64 bits.
__device__ __forceinline__ float scaled(float x, float f, double fd) {
  return f >= 1.1754944e-38f ? x * f : (float)((double)x * fd);
}

template <typename T>
__device__ __forceinline__ void chunk_scale(const void* p, void* o, long long numel, int c, int kind, float f,
                                            double fd) {
  constexpr int VE = 16 / (int)sizeof(T), NV = CLIP_CHUNK / (VE * CLIP_THREADS);
  const Piece r = piece_of(p, numel, (int)sizeof(T), c);
  const int tid = threadIdx.x;
  const bool of32 = kind & OUT_F32, vec = kind & OUT_VEC;
  const uint4* body = (const uint4*)((const T*)p + r.start);
  const int left = (int)(r.hi - r.start);
  const int nvec = left > 0 ? left / VE : 0;
  uint4 v[NV];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int i = tid + j * CLIP_THREADS;
    if (i < nvec) v[j] = body[i];
  }
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int i = tid + j * CLIP_THREADS;
    if (i >= nvec) continue;
    float x[VE];
    if (sizeof(T) == 4) {
      x[0] = __uint_as_float(v[j].x); x[1] = __uint_as_float(v[j].y);
      x[2] = __uint_as_float(v[j].z); x[3] = __uint_as_float(v[j].w);
    } else {
      const unsigned w[4] = {v[j].x, v[j].y, v[j].z, v[j].w};
#pragma unroll
      for (int q = 0; q < VE / 2; ++q) { x[2 * q] = bf16_lo(w[q & 3]); x[2 * q + 1] = bf16_hi(w[q & 3]); }
    }
#pragma unroll
    for (int q = 0; q < VE; ++q) x[q] = scaled(x[q], f, fd);
    const long long at = r.start + (long long)i * VE;
    if (vec && of32) {
      float4* d = (float4*)((float*)o + at);
#pragma unroll
      for (int q = 0; q < VE / 4; ++q) d[q] = make_float4(x[4 * q], x[4 * q + 1], x[4 * q + 2], x[4 * q + 3]);
    } else if (vec && sizeof(T) == 2) {
      *(uint4*)((__nv_bfloat16*)o + at) = make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]),
                                                     pack_bf16(x[VE - 4], x[VE - 3]), pack_bf16(x[VE - 2], x[VE - 1]));
    } else {
#pragma unroll
      for (int q = 0; q < VE; ++q) store1<T>(o, at + q, x[q], of32);
    }
  }
  const int tail = left > 0 ? left - nvec * VE : 0;
  if (tid < r.head) store1<T>(o, tid, scaled(load1<T>(p, tid), f, fd), of32);
  if (tid < tail) {
    const long long at = r.start + nvec * VE + tid;
    store1<T>(o, at, scaled(load1<T>(p, at), f, fd), of32);
  }
}

// norm and factor from the partial sums, then the scaled values.  The chunks are walked from the last to
// the first: the ones that the first pass read last are still in L2.
template <int LIM>
__global__ void __launch_bounds__(CLIP_THREADS) k_scale(const __grid_constant__ ClipTable<LIM> tab,
                                                        const double* __restrict__ partial, int np, float max_norm,
                                                        float eps, float* __restrict__ norm_out) {
  double acc = 0.0;
  for (int i = threadIdx.x; i < np; i += CLIP_THREADS) acc += partial[i];
  const double norm = sqrt(block_sum(acc));
  // a norm that is not finite (in fp32, as the caller sees it) scales nothing: no factor would mend such a step
  const double ratio = (double)max_norm / (norm + (double)eps);
  const double fd = (isfinite((float)norm) && ratio < 1.0) ? ratio : 1.0;
  const float f = (float)fd;
  if (norm_out && blockIdx.x == 0 && threadIdx.x == 0) *norm_out = (float)norm;
  const int total = tab.chunk0[tab.n];
  for (int c = total - 1 - (int)blockIdx.x; c >= 0; c -= gridDim.x) {
    const int i = tensor_of(tab, c);
    const int kind = tab.kind[i];
    if (f == 1.0f && (kind & IN_PLACE)) continue;
    if (kind & IN_F32) chunk_scale<float>(tab.in[i], tab.out[i], tab.numel[i], c - tab.chunk0[i], kind, f, fd);
    else chunk_scale<__nv_bfloat16>(tab.in[i], tab.out[i], tab.numel[i], c - tab.chunk0[i], kind, f, fd);
  }
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

// Host checks of the list.  `writes`: the call scales, so that what it writes may overlap nothing else.
pctc_status_t check_list(const ClipList& l, bool writes) {
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
  if (!writes || l.n == 0) return PCTC_OK;
  Span* spans = new (std::nothrow) Span[2 * (size_t)l.n];
  if (!spans) return PCTC_ERR_HOST_MEMORY;
  size_t ns = 0;
  for (int i = 0; i < l.n; ++i) {
    if (l.numels[i] == 0) continue;
    const size_t a = (size_t)l.in(i), b = (size_t)l.out(i);
    spans[ns++] = Span{b, b + (size_t)l.numels[i] * elem_bytes(l.out_dtype(i)), true};
    if (a != b) spans[ns++] = Span{a, a + (size_t)l.numels[i] * elem_bytes(l.dtypes[i]), false};
  }
  const bool clash = spans_conflict(spans, ns);
  delete[] spans;
  return clash ? PCTC_ERR_INVALID_ARG : PCTC_OK;
}

template <int LIM>
pctc_status_t fill_table(const ClipList& l, int i0, int i1, bool writes, ClipTable<LIM>* tab) {
  tab->n = 0;
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
      if (out == l.in(i)) kind |= IN_PLACE;
      if (l.out_dtype(i) == PCTC_FP32) kind |= OUT_F32;
      // stores are as wide as the loads where the output reaches a 16-byte boundary with the input
      const size_t head = (((16 - ((size_t)l.in(i) & 15)) & 15) / es);
      if ((((size_t)out + head * elem_bytes(l.out_dtype(i))) & 15) == 0) kind |= OUT_VEC;
    }
    tab->out[k] = out;
    tab->kind[k] = kind;
    const size_t mis = (size_t)l.in(i) & 15;
    const long long head = mis ? (long long)((16 - mis) / es) : 0;
    const long long body = l.numels[i] > head ? l.numels[i] - head : 0;
    chunks += body ? (body + CLIP_CHUNK - 1) / CLIP_CHUNK : 1;
    if (chunks > 0x7fff0000LL) return PCTC_ERR_UNSUPPORTED;
  }
  tab->chunk0[tab->n] = (int)chunks;
  return PCTC_OK;
}

int clip_grid(int chunks) {
  int dev = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
    sms = 148;
  int most = sms * CLIP_CTAS_PER_SM;
  if (most > CLIP_MAX_GRID) most = CLIP_MAX_GRID;
  return chunks < 1 ? 1 : chunks < most ? chunks : most;
}

template <int LIM>
pctc_status_t square_sums(const ClipList& l, double* partial, int* np, cudaStream_t stream) {
  ClipTable<LIM> tab;
  *np = 0;
  for (int i0 = 0; i0 == 0 || i0 < l.n; i0 += LIM) {
    const pctc_status_t st = fill_table<LIM>(l, i0, l.n < i0 + LIM ? l.n : i0 + LIM, false, &tab);
    if (st != PCTC_OK) return st;
    const int grid = clip_grid(tab.chunk0[tab.n]);
    k_square_sums<LIM><<<grid, CLIP_THREADS, 0, stream>>>(tab, partial + *np);
    if (cudaGetLastError() != cudaSuccess) return PCTC_ERR_CUDA;
    *np += grid;
  }
  return PCTC_OK;
}

template <int LIM>
pctc_status_t scale(const ClipList& l, const double* partial, int np, float max_norm, float eps, float* norm,
                    cudaStream_t stream) {
  ClipTable<LIM> tab;
  for (int i0 = 0; i0 == 0 || i0 < l.n; i0 += LIM) {
    const pctc_status_t st = fill_table<LIM>(l, i0, l.n < i0 + LIM ? l.n : i0 + LIM, true, &tab);
    if (st != PCTC_OK) return st;
    k_scale<LIM><<<clip_grid(tab.chunk0[tab.n]), CLIP_THREADS, 0, stream>>>(tab, partial, np, max_norm, eps,
                                                                           i0 == 0 ? norm : nullptr);
    if (cudaGetLastError() != cudaSuccess) return PCTC_ERR_CUDA;
  }
  return PCTC_OK;
}

bool bad_limits(float max_norm, float eps) {
  return !(max_norm > 0.f) || !(eps >= 0.f) || std::isinf(eps);
}
size_t partial_count(int n) { return (size_t)CLIP_MAX_GRID * (n <= CLIP_LARGE ? 1 : ((size_t)n + CLIP_LARGE - 1) / CLIP_LARGE); }

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
  pctc_status_t st = check_list(l, false);
  if (st != PCTC_OK) return st;
  if (!sqsum || ((size_t)sqsum & 7) || !workspace || ((size_t)workspace & 255)) return PCTC_ERR_INVALID_ARG;
  if (workspace_bytes < partial_count(n) * sizeof(double)) return PCTC_ERR_WORKSPACE_TOO_SMALL;
  cudaStream_t stream = (cudaStream_t)stream_v;
  double* partial = (double*)workspace;
  int np = 0;
  st = n <= CLIP_SMALL ? square_sums<CLIP_SMALL>(l, partial, &np, stream) : square_sums<CLIP_LARGE>(l, partial, &np, stream);
  if (st != PCTC_OK) return st;
  k_sum_partials<<<1, CLIP_THREADS, 0, stream>>>(partial, np, sqsum);
  return cudaGetLastError() == cudaSuccess ? PCTC_OK : PCTC_ERR_CUDA;
}

pctc_status_t pctc_grad_scale(int32_t n, const void* const* grads, void* const* outs, const int64_t* numels,
                              const int32_t* dtypes, const int32_t* out_dtypes, const double* sqsum, float max_norm,
                              float eps, float* norm, void* stream_v) {
  const ClipList l{n, grads, outs, numels, dtypes, out_dtypes};
  pctc_status_t st = check_list(l, true);
  if (st != PCTC_OK) return st;
  if (!sqsum || ((size_t)sqsum & 7) || bad_limits(max_norm, eps)) return PCTC_ERR_INVALID_ARG;
  cudaStream_t stream = (cudaStream_t)stream_v;
  return n <= CLIP_SMALL ? scale<CLIP_SMALL>(l, sqsum, 1, max_norm, eps, norm, stream)
                         : scale<CLIP_LARGE>(l, sqsum, 1, max_norm, eps, norm, stream);
}

pctc_status_t pctc_clip_grad_norm(int32_t n, const void* const* grads, void* const* outs, const int64_t* numels,
                                  const int32_t* dtypes, const int32_t* out_dtypes, float max_norm, float eps,
                                  float* norm, void* workspace, size_t workspace_bytes, void* stream_v) {
  const ClipList l{n, grads, outs, numels, dtypes, out_dtypes};
  pctc_status_t st = check_list(l, true);
  if (st != PCTC_OK) return st;
  if (!norm || !workspace || ((size_t)workspace & 255) || bad_limits(max_norm, eps)) return PCTC_ERR_INVALID_ARG;
  if (workspace_bytes < partial_count(n) * sizeof(double)) return PCTC_ERR_WORKSPACE_TOO_SMALL;
  cudaStream_t stream = (cudaStream_t)stream_v;
  double* partial = (double*)workspace;
  int np = 0;
  st = n <= CLIP_SMALL ? square_sums<CLIP_SMALL>(l, partial, &np, stream) : square_sums<CLIP_LARGE>(l, partial, &np, stream);
  if (st != PCTC_OK) return st;
  return n <= CLIP_SMALL ? scale<CLIP_SMALL>(l, partial, np, max_norm, eps, norm, stream)
                         : scale<CLIP_LARGE>(l, partial, np, max_norm, eps, norm, stream);
}

}  // extern "C"
