// Dropout from a counter-based generator, forward and backward:
//   y = u < limit ? 0 : x * 65536 / (65536 - limit)   (+ residual),    limit = round(65536 p),
// with u a 16-bit word that is a function of the value's index, the seed and the offset alone, so that no mask is
// stored: the backward pass is the same call on the gradient.  The words are those of Philox-4x32 with ten rounds
// (Salmon, Moraes, Dror, Shaw: "Parallel random numbers: as easy as 1, 2, 3", 2011): block b = index / 8 as counter, one
// 16-bit half for each of its eight values.  Halves instead of whole words: a block of ten rounds is some 75
// instructions, and with four values a block a bf16 call would be bound by them and not by HBM.  With eight it is bound by HBM
// and what stays in L2 of the results (64,000 x 1,024 bf16 with a residual: 393 MB in 56.4 us, of which some 360 cross HBM), a
// small one by the launch.
#include "../../include/prunedctc.h"
#include "pctc_internal.h"
#include "vec8.cuh"

#include <cmath>

namespace pctc {
namespace {

constexpr int DROP_THREADS = 256;

struct DropArgs {
  const void* x;
  const void* residual;                          // null: none
  void* out;
  const long long* step;                         // null, or a word that is added to the offset
  long long rows, cols;                          // a contiguous array is one row
  long long ld_x, ld_res, ld_out;
  long long groups, groups_per_row;              // groups of eight values
  unsigned long long seed, offset;
  unsigned limit;
  float scale;
};

__device__ __forceinline__ void philox_round(unsigned (&c)[4], unsigned k0, unsigned k1) {
  const unsigned long long a = (unsigned long long)c[0] * 0xD2511F53u, b = (unsigned long long)c[2] * 0xCD9E8D57u;
  const unsigned c1 = c[1], c3 = c[3];
  c[0] = (unsigned)(b >> 32) ^ c1 ^ k0;
  c[1] = (unsigned)b;
  c[2] = (unsigned)(a >> 32) ^ c3 ^ k1;
  c[3] = (unsigned)a;
}
__device__ __forceinline__ void philox(unsigned (&c)[4], unsigned long long block, unsigned long long offset,
                                       unsigned long long seed) {
  c[0] = (unsigned)block;
  c[1] = (unsigned)(block >> 32);
  c[2] = (unsigned)offset;
  c[3] = (unsigned)(offset >> 32);
  unsigned k0 = (unsigned)seed, k1 = (unsigned)(seed >> 32);
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    philox_round(c, k0, k1);
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
}
// Value j of a block: the low half of word j / 2 where j is even, else the high half.
__device__ __forceinline__ unsigned half_of(const unsigned (&c)[4], int j) {
  return (j & 1) ? c[j >> 1] >> 16 : c[j >> 1] & 0xffffu;
}

// What is dropped is zero whatever it was, infinities and NaN too.  32 bits until the one rounding at the end.
__device__ __forceinline__ float drop_one(float x, unsigned u, unsigned limit, float scale) {
  return u < limit ? 0.f : x * scale;
}

// Groups that lie in one row, 16-byte aligned in every array.  One a thread: two or four, loaded ahead, were slower at every size
// (64,000 x 1,024 bf16 with a residual: 56.3, 56.8 and 57.5 us; 4,800 x 1,024: 5.6, 6.0 and 6.5).
template <typename T, bool RES, bool ROWS>
__global__ void __launch_bounds__(DROP_THREADS) k_dropout_vec(const DropArgs a) {
  const unsigned long long offset = a.offset + (a.step ? (unsigned long long)*a.step : 0ull);
  const long long g = (long long)blockIdx.x * DROP_THREADS + threadIdx.x;
  if (g >= a.groups) return;
  const long long row = ROWS ? g / a.groups_per_row : 0, col = (g - row * a.groups_per_row) * 8;
  Vec8<T> x, r;
  x.load((const T*)a.x + row * a.ld_x + col);
  if (RES) r.load((const T*)a.residual + row * a.ld_res + col);
  unsigned c[4];
  philox(c, (unsigned long long)g, offset, a.seed);
  float v[8], add[8];
  x.get(v);
  if (RES) r.get(add);
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    v[j] = drop_one(v[j], half_of(c, j), a.limit, a.scale);
    if (RES) v[j] += add[j];
  }
  Vec8<T>::store((T*)a.out + row * a.ld_out + col, v);
}

// Any strides and addresses; also what is left behind the last whole group (from group `first` on).
template <typename T, bool RES>
__global__ void __launch_bounds__(DROP_THREADS) k_dropout_any(const DropArgs a, long long first) {
  const unsigned long long offset = a.offset + (a.step ? (unsigned long long)*a.step : 0ull);
  const long long n = a.rows * a.cols;
  const long long b = first + (long long)blockIdx.x * DROP_THREADS + threadIdx.x;
  if (b * 8 >= n) return;
  unsigned c[4];
  philox(c, (unsigned long long)b, offset, a.seed);
  long long row = b * 8 / a.cols, col = b * 8 - row * a.cols;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    if (b * 8 + j >= n) break;
    float v = drop_one(to_float(((const T*)a.x)[row * a.ld_x + col]), half_of(c, j), a.limit, a.scale);
    if (RES) v += to_float(((const T*)a.residual)[row * a.ld_res + col]);
    ((T*)a.out)[row * a.ld_out + col] = from_float<T>(v);
    if (++col == a.cols) { col = 0; ++row; }
  }
}

template <typename T, bool RES>
cudaError_t dropout_launch(DropArgs a, bool aligned, cudaStream_t stream) {
  const long long n = a.rows * a.cols;
  long long done = 0;                            // groups taken by the wide form
  if (aligned && (a.rows == 1 || a.cols % 8 == 0)) {
    a.groups_per_row = a.cols / 8;
    a.groups = a.rows * a.groups_per_row;
    const long long blocks = (a.groups + DROP_THREADS - 1) / DROP_THREADS;
    if (blocks > 0x7fffffffLL) return cudaErrorInvalidValue;
    if (blocks > 0) {
      if (a.rows == 1) k_dropout_vec<T, RES, false><<<(unsigned)blocks, DROP_THREADS, 0, stream>>>(a);
      else k_dropout_vec<T, RES, true><<<(unsigned)blocks, DROP_THREADS, 0, stream>>>(a);
      const cudaError_t e = cudaGetLastError();
      if (e != cudaSuccess) return e;
    }
    done = a.groups;
  }
  if (done * 8 >= n) return cudaSuccess;
  const long long blocks = ((n + 7) / 8 - done + DROP_THREADS - 1) / DROP_THREADS;
  if (blocks > 0x7fffffffLL) return cudaErrorInvalidValue;
  k_dropout_any<T, RES><<<(unsigned)blocks, DROP_THREADS, 0, stream>>>(a, done);
  return cudaGetLastError();
}

}  // namespace
}  // namespace pctc

using namespace pctc;

extern "C" pctc_status_t pctc_dropout(const pctc_dropout_t* p, const void* x, const void* residual, const int64_t* step,
                                      void* out, void* stream_v) {
  if (!p || p->rows < 0 || p->cols < 0 || !(p->p >= 0.0 && p->p <= 1.0)) return PCTC_ERR_INVALID_ARG;
  if (p->dtype != PCTC_BF16 && p->dtype != PCTC_FP32) return PCTC_ERR_UNSUPPORTED;
  if (p->rows == 0 || p->cols == 0) return PCTC_OK;
  if (!x || !out || p->ld_x < p->cols || p->ld_out < p->cols || (residual && p->ld_res < p->cols)) return PCTC_ERR_INVALID_ARG;
  const size_t es = p->dtype == PCTC_BF16 ? 2 : 4;
  if (((size_t)x | (size_t)out | (size_t)residual) & (es - 1) || ((size_t)step & 7)) return PCTC_ERR_INVALID_ARG;
  if (p->rows > MAX_ELEMENTS / p->cols) return PCTC_ERR_UNSUPPORTED;
  for (const int64_t ld : {p->ld_x, p->ld_out, residual ? p->ld_res : p->cols})
    if (ld > MAX_ELEMENTS / p->rows) return PCTC_ERR_UNSUPPORTED;
  // in place: the same rows, each value read by the thread that writes it; no other overlap
  const Rows to{out, p->rows, p->ld_out, p->cols, es}, from{x, p->rows, p->ld_x, p->cols, es},
      res{residual, p->rows, p->ld_res, p->cols, es}, counter{step, 1, 1, 1, 8};
  if ((!to.same(from) && to.overlaps(from)) || (!to.same(res) && to.overlaps(res)) || to.overlaps(counter))
    return PCTC_ERR_INVALID_ARG;

  DropArgs a = {};
  a.x = x;
  a.residual = residual;
  a.out = out;
  a.step = (const long long*)step;
  a.rows = p->rows;
  a.cols = p->cols;
  a.ld_x = p->ld_x;
  a.ld_out = p->ld_out;
  a.ld_res = residual ? p->ld_res : p->cols;
  if (p->rows == 1 || (a.ld_x == a.cols && a.ld_out == a.cols && a.ld_res == a.cols)) {
    a.cols *= a.rows;
    a.rows = 1;
    a.ld_x = a.ld_out = a.ld_res = a.cols;
  }
  a.seed = p->seed;
  a.offset = p->offset;
  const double limit = std::floor(p->p * 65536.0 + 0.5);
  a.limit = p->p < 1.0 && limit > 65535.0 ? 65535u : (unsigned)limit;
  a.scale = a.limit < 65536u ? 65536.f / (float)(65536u - a.limit) : 0.f;
  const bool aligned = (((size_t)x | (size_t)out | (size_t)residual) & 15) == 0 &&
                       (a.rows == 1 || ((a.ld_x | a.ld_out | a.ld_res) & (16 / (int64_t)es - 1)) == 0);
  cudaStream_t stream = (cudaStream_t)stream_v;
  cudaError_t e;
  if (p->dtype == PCTC_BF16)
    e = residual ? dropout_launch<__nv_bfloat16, true>(a, aligned, stream) : dropout_launch<__nv_bfloat16, false>(a, aligned, stream);
  else
    e = residual ? dropout_launch<float, true>(a, aligned, stream) : dropout_launch<float, false>(a, aligned, stream);
  return e == cudaSuccess ? PCTC_OK : e == cudaErrorInvalidValue ? PCTC_ERR_UNSUPPORTED : PCTC_ERR_CUDA;
}
