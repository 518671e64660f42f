// The head in 8-bit integers:  C[i,j] = T(float(sum_k qa[i,k] qb[j,k]) * sa[i] * sb[j] + bias[j]),  with rows quantized as
//   s = max|x| / 127,   q = round(x * (127 / max|x|)).
// Sums are whole numbers of 32 bits (exact for k < 2^17); nothing is rounded before the scales.
//
// k_i8_gemm is a persistent tcgen05 kernel (kind::i8) in three forms; roles, ring and bounded waits are those of the bf16
// kernel in umma_gemm.cu.
//   very few tokens (up to 8,192 values, of rows that are read in eights): as below, and every CTA quantizes the tokens itself,
//     into the operand's place in shared memory, while its first ring of the head is on its way: one launch.
//   few tokens (up to 128), CTAS = 1: the rows of the accumulators are channels (rows of the head), the columns tokens, tiles
//     128 x 16 .. 128 x 128: the head streams once through a deep ring, and 32 lanes of a warp hold 32 neighbouring
//     channels of a token, which is the order of C.  Bound by HBM (4 x 151,936 x 1,024: 31 us, 5.1 TB/s).
//   many tokens, CTAS = 2: 256 tokens x 256 channels a CTA pair (cta_group::2), the rows are tokens, and results leave
//     through shared memory and TMA stores as in the bf16 kernel (with channels as rows a result took 10 instructions and
//     more: 512 x 151,936 x 512 113 us against 56).  Bound by the tensor pipe (2,048 x 151,936 x 4,096: 870 to 1,000 us under
//     the power cap, 2.6 to 2.9 POP/s), or by the results where sums are short.  (72 and 128 tokens in pairs, 151,936 x 1,024: 38 and
//     39 us against 32 and 35 as few.)
#include "../../include/prunedctc.h"
#include "i8_gemm.h"
#include "pctc_internal.h"
#include "umma_ptx.cuh"
#include "vec8.cuh"

#include <cmath>

namespace pctc {
namespace {

// ---------------------------------------------------------------------------------------------
// Quantization, a row at a time
// ---------------------------------------------------------------------------------------------
constexpr int QUANT_THREADS = 256;
constexpr float QUANT_TINY = 7.888609052210118e-31f;   // 2^-100: below it 127 / max would leave the range of fp32

struct QuantArgs {
  const void* x;
  signed char* q;
  float* scales;
  int* clear;                                    // null, or a status word to zero for the kernel behind
  long long rows, cols, ld_x, ld_q;
};

// The largest magnitude as bits: NaN counts as the largest of all.
__device__ __forceinline__ unsigned magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// 127 / max and max / 127; a row with a value that is not finite becomes NaN, one without values above 2^-100 zero.
__device__ __forceinline__ float row_factor(unsigned top, float& scale) {
  const float m = __uint_as_float(top);
  if (top >= 0x7f800000u) {
    scale = __uint_as_float(0x7fc00000u);
    return 0.f;
  }
  if (m < QUANT_TINY) {
    scale = 0.f;
    return 0.f;
  }
  scale = __fdiv_rn(m, 127.f);
  return __fdiv_rn(127.f, m);
}
__device__ __forceinline__ int quantize_one(float x, float f) {
  if (f == 0.f) return 0;
  return max(-127, min(127, __float2int_rn(x * f)));
}

// The kernel behind this one reports to the status word when one of its waits has run out, 3,000 cycles (test build) or two seconds
// after it has started: long after this.  (Zeroing it ahead of launch_next() costs a call of 37 tokens 0.6 of 12.6 us.)
__device__ __forceinline__ void launch_next_and_clear(int* status) {
  launch_next();
  if (status && blockIdx.x == 0 && threadIdx.x == 0) *status = 0;
}

// GROUP threads hold a row: NV pieces of N values each, loaded once.
template <typename T, int N, int GROUP, int NV>
__global__ void __launch_bounds__(QUANT_THREADS) k_quantize(const QuantArgs a) {
  __shared__ unsigned tops[QUANT_THREADS / 32];
  launch_next_and_clear(a.clear);
  const long long row = (long long)blockIdx.x * (QUANT_THREADS / GROUP) + threadIdx.x / GROUP;
  const int at = threadIdx.x % GROUP, per_row = row < a.rows ? (int)(a.cols / N) : 0;
  VecN<T, N> v[NV];
  unsigned top = 0;
#pragma unroll
  for (int k = 0; k < NV; ++k)
    if (at + k * GROUP < per_row) v[k].load((const T*)a.x + row * a.ld_x + (at + k * GROUP) * N);
#pragma unroll
  for (int k = 0; k < NV; ++k)
    if (at + k * GROUP < per_row)
#pragma unroll
      for (int j = 0; j < N; ++j) top = max(top, magnitude(v[k].value(j)));
  top = __reduce_max_sync(0xffffffffu, top);
  if (GROUP > 32) {
    if ((threadIdx.x & 31) == 0) tops[threadIdx.x >> 5] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < QUANT_THREADS / 32; ++w) top = max(top, tops[w]);
  }
  if (per_row == 0) return;
  float scale;
  const float f = row_factor(top, scale);
  if (at == 0) a.scales[row] = scale;
#pragma unroll
  for (int k = 0; k < NV; ++k)
    if (at + k * GROUP < per_row) {
      unsigned w[2] = {0u, 0u};
#pragma unroll
      for (int j = 0; j < N; ++j) w[j >> 2] |= ((unsigned)quantize_one(v[k].value(j), f) & 0xffu) << (8 * (j & 3));
      signed char* to = a.q + row * a.ld_q + (at + k * GROUP) * N;
      if constexpr (N == 8) *reinterpret_cast<uint2*>(to) = make_uint2(w[0], w[1]);
      else if constexpr (N == 4) *reinterpret_cast<unsigned*>(to) = w[0];
      else if constexpr (N == 2) *reinterpret_cast<unsigned short*>(to) = (unsigned short)w[0];
      else *to = (signed char)w[0];
    }
}

// Rows of any length, stride and address, read twice.
template <typename T>
__global__ void __launch_bounds__(QUANT_THREADS) k_quantize_any(const QuantArgs a) {
  __shared__ unsigned tops[QUANT_THREADS / 32];
  launch_next_and_clear(a.clear);
  const long long row = blockIdx.x;
  const T* x = (const T*)a.x + row * a.ld_x;
  unsigned top = 0;
  for (long long c = threadIdx.x; c < a.cols; c += QUANT_THREADS) top = max(top, magnitude(to_float(x[c])));
  top = __reduce_max_sync(0xffffffffu, top);
  if ((threadIdx.x & 31) == 0) tops[threadIdx.x >> 5] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < QUANT_THREADS / 32; ++w) top = max(top, tops[w]);
  float scale;
  const float f = row_factor(top, scale);
  if (threadIdx.x == 0) a.scales[row] = scale;
  for (long long c = threadIdx.x; c < a.cols; c += QUANT_THREADS)
    a.q[row * a.ld_q + c] = (signed char)quantize_one(to_float(x[c]), f);
}

template <typename T, int N, int GROUP, int NV>
void quantize_rows(const QuantArgs& a, cudaStream_t stream) {
  constexpr int per = QUANT_THREADS / GROUP;
  k_quantize<T, N, GROUP, NV><<<(unsigned)((a.rows + per - 1) / per), QUANT_THREADS, 0, stream>>>(a);
}
// A warp a row up to 128 pieces, a block up to 2,048; of few rows a block from 33 pieces on (128 x 1,024 bf16: 2.8 -> 2.0 us; 592:
// 2.9 -> 2.4, 2,048: 3.4 -> 5.1).
constexpr long long QUANT_FEW = 148 * 4;
template <typename T, int N>
void quantize_pieces(const QuantArgs& a, cudaStream_t stream) {
  const long long v = a.cols / N;
  if (v <= 32) quantize_rows<T, N, 32, 1>(a, stream);
  else if (v <= 64 && a.rows > QUANT_FEW) quantize_rows<T, N, 32, 2>(a, stream);
  else if (v <= 128 && a.rows > QUANT_FEW) quantize_rows<T, N, 32, 4>(a, stream);
  else if (v <= 256) quantize_rows<T, N, 256, 1>(a, stream);
  else if (v <= 512) quantize_rows<T, N, 256, 2>(a, stream);
  else if (v <= 1024) quantize_rows<T, N, 256, 4>(a, stream);
  else if (v <= 2048 && N <= 4) quantize_rows<T, N, 256, 8>(a, stream);
  else k_quantize_any<T><<<(unsigned)a.rows, QUANT_THREADS, 0, stream>>>(a);
}
template <typename T>
cudaError_t quantize_launch(const QuantArgs& a, cudaStream_t stream) {
  const auto fits = [&](int n) {
    const size_t bytes = n * sizeof(T) < 16 ? n * sizeof(T) : 16;
    return a.cols % n == 0 && (size_t)a.x % bytes == 0 && a.ld_x * sizeof(T) % bytes == 0 && (size_t)a.q % n == 0 && a.ld_q % n == 0;
  };
  if (fits(8)) quantize_pieces<T, 8>(a, stream);
  else if (fits(4)) quantize_pieces<T, 4>(a, stream);
  else if (fits(2)) quantize_pieces<T, 2>(a, stream);
  else quantize_pieces<T, 1>(a, stream);
  return cudaGetLastError();
}

// ---------------------------------------------------------------------------------------------
// Product
// ---------------------------------------------------------------------------------------------
constexpr int I8_ROWS = 128;                     // channels of a CTA's tile
constexpr int I8_BK = 128;                       // bytes of k a stage: one 128-byte swizzled row
constexpr int I8_W_STAGE = I8_ROWS * I8_BK;
constexpr int I8_EPI_WARPS = 8;
constexpr int I8_THREADS = 64 + 32 * I8_EPI_WARPS;
constexpr int I8_MAX_STAGES = 12;
constexpr int I8_TMEM_COLS = 512;
constexpr int I8_OWN_VALUES = 8192;              // up to so many values of tokens are quantized by the product itself
                                                 // (4 x 151,936 x 1,024: 33.2 -> 31.5 us; 16 x 1,024 values: 32.8 -> 35.2),
constexpr int I8_OWN_SINGLE = 1024;              // or so many that are read one by one (50,001 x 516, 1 and 4 tokens: 12.4 and 14.8 us
                                                 // against 13.0 and 13.2 with a launch ahead)

struct I8Args {
  int n, m, k;                                   // channels, tokens, contraction
  int rows;                                      // CTAS = 1: channels of a tile, up to 128
  int cols;                                      // columns of a tile: tokens (CTAS = 1) or channels (CTAS = 2)
  int stages;
  int band;                                      // CTAS = 2: token tiles that are walked together (their rows stay in L2)
  const float* a_scale;                          // [m]
  const float* b_scale;                          // [n]
  const void* bias;                              // [n] or null
  int bias_bf16;
  void* C;
  long long ldc;
  int aligned;                                   // CTAS = 1: two neighbouring bf16 channels can be stored as one word;
                                                 // CTAS = 2: rows of C can be stored by TMA
  int behind;                                    // the launch before this one makes the tokens (and nothing else that is read here)
  const void* x;                                 // tokens that are quantized here [m, k] (then there is no a_scale)
  long long ld_x;
  int wide_x;                                    // ... whose rows can be read in groups of eight
  int* status;
};

// Shared memory behind the ring: CTAS = 1: the tokens' scales; CTAS = 2: the scales and biases of every epilogue warp's channels,
// and its results on their way out: two boxes of 32 rows x 64 bytes (64-byte swizzle) for TMA, or, where rows of C are not
// 16-byte aligned, 32 rows of 256 bytes each as far from a 16-byte boundary as they will be in C (a stage of the ring less).
constexpr int I8_BOX = 2048, I8_WARP_COLS = 128, I8_ROW_BYTES = 256, I8_ROW_PITCH = I8_ROW_BYTES + 16;
constexpr int i8_ring(int ctas, bool aligned) { return ctas == 2 ? (aligned ? 5 : 4) * 2 * I8_ROWS * I8_BK : 216 * 1024; }
constexpr int i8_out(bool aligned) { return aligned ? 2 * I8_BOX : 32 * I8_ROW_PITCH; }
constexpr int i8_extra(int ctas, bool aligned) { return ctas == 2 ? I8_EPI_WARPS * (i8_out(aligned) + I8_WARP_COLS * 8) : I8_ROWS * 4; }
struct I8Tail {
  unsigned long long full[I8_MAX_STAGES];
  unsigned long long empty[I8_MAX_STAGES];
  unsigned long long tmem_full[2];
  unsigned long long tmem_empty[2];
  unsigned long long done;
  unsigned tmem_base;
  int abort;
  unsigned tops[I8_ROWS];                        // tokens quantized here: the largest magnitude of each
};
constexpr int i8_smem(int ctas) {
  const int more = i8_ring(ctas, true) + i8_extra(ctas, true), less = i8_ring(ctas, false) + i8_extra(ctas, false);
  return 1024 + (more > less ? more : less) + (int)sizeof(I8Tail);
}
static_assert(i8_smem(1) <= 227 * 1024 && i8_smem(2) <= 227 * 1024, "shared memory budget");

__device__ __forceinline__ void tc_mma_i8_pair(unsigned tmem_d, unsigned long long adesc, unsigned long long bdesc,
                                               unsigned idesc, unsigned accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::i8 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(tmem_d), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void tc_mma_i8(unsigned tmem_d, unsigned long long adesc, unsigned long long bdesc,
                                          unsigned idesc, unsigned accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(tmem_d), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}
// Descriptor of a 128-byte-swizzled tile with k contiguous: rows of 128 bytes, groups of eight rows 1024 bytes apart.
__device__ __forceinline__ unsigned long long i8_smem_desc(unsigned addr) {
  return (unsigned long long)((addr & 0x3FFFFu) >> 4) | (1ull << 16) | ((unsigned long long)(1024 >> 4) << 32) | (1ull << 46) |
         (2ull << 61);
}

// Unit u -> first channel and first token of its tile.  With pairs the token tiles run fastest inside a band, so that the
// head's rows are read once a band while the band's token rows stay in L2.
template <int CTAS>
__device__ __forceinline__ void i8_tile(const I8Args& a, int u, int n_tiles, int m_tiles, int& channel, int& token) {
  if (CTAS == 1) {
    channel = u * a.rows;
    token = 0;
    return;
  }
  const int b = u / (a.band * n_tiles), r = u - b * a.band * n_tiles, rows = min(a.band, m_tiles - b * a.band), nt = r / rows;
  channel = nt * a.cols;
  token = (b * a.band + (r - nt * rows)) * (2 * I8_ROWS);
}

// The tokens in 8 bits as the tensor core reads them (blocks of 128 k, rows of 128 bytes with the 128-byte swizzle), and
// their scales.  A thread takes groups of eight values, whatever row they are in; they are loaded before anything else of the
// kernel, since behind the first loads of the head they would wait for microseconds.  Rows and k past the last are left as
// they are: their products are not looked at, or zero.
template <typename X>
struct OwnTokens {
  static constexpr int MOST = (I8_OWN_VALUES / 8 + I8_THREADS - 1) / I8_THREADS;
  Vec8<X> v[MOST];

  __device__ __forceinline__ void load(const I8Args& a) {
    if (!a.wide_x) return;
    const unsigned per = a.k / 8, groups = per * a.m;
#pragma unroll
    for (int i = 0; i < MOST; ++i) {
      const unsigned g = threadIdx.x + i * I8_THREADS, row = g / per;
      if (g < groups) v[i].load((const X*)a.x + row * a.ld_x + (g - row * per) * 8);
    }
  }
  // tops: zeros [m]; all threads of the block
  __device__ __forceinline__ void store(const I8Args& a, unsigned char* tokens, unsigned* tops, float* scales) const {
    const unsigned per = a.wide_x ? a.k / 8 : a.k, groups = per * a.m;
    const auto place = [&](unsigned row, unsigned c) {
      return tokens + (c >> 7) * a.cols * I8_BK + row * I8_BK + (((c >> 4 & 7) ^ (row & 7)) << 4) + (c & 15);
    };
    if (a.wide_x) {
#pragma unroll
      for (int i = 0; i < MOST; ++i) {
        const unsigned g = threadIdx.x + i * I8_THREADS;
        if (g >= groups) continue;
        float x[8];
        v[i].get(x);
        unsigned top = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) top = max(top, magnitude(x[j]));
        atomicMax(&tops[g / per], top);
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < MOST; ++i) {
        const unsigned g = threadIdx.x + i * I8_THREADS, row = g / per;
        if (g >= groups) continue;
        float x[8], scale;
        v[i].get(x);
        const float f = row_factor(tops[row], scale);
        unsigned w[2] = {0u, 0u};
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j >> 2] |= ((unsigned)quantize_one(x[j], f) & 0xffu) << (8 * (j & 3));
        *reinterpret_cast<uint2*>(place(row, (g - row * per) * 8)) = make_uint2(w[0], w[1]);
        if (g == row * per) scales[row] = scale;
      }
    } else {
#pragma unroll 4
      for (unsigned g = threadIdx.x; g < groups; g += I8_THREADS) {
        const unsigned row = g / per;
        atomicMax(&tops[row], magnitude(to_float(((const X*)a.x)[row * a.ld_x + (g - row * per)])));
      }
      __syncthreads();
#pragma unroll 4
      for (unsigned g = threadIdx.x; g < groups; g += I8_THREADS) {
        const unsigned row = g / per, c = g - row * per;
        float scale;
        const float f = row_factor(tops[row], scale);
        *place(row, c) = (unsigned char)quantize_one(to_float(((const X*)a.x)[row * a.ld_x + c]), f);
        if (c == 0) scales[row] = scale;
      }
    }
  }
};
struct NoTokens {};

// 32 rows of 256 bytes from `stage` to `to` (rows `pitch` bytes apart, `rows` of them there): whole 16-byte pieces by half a
// warp a row, then the pieces at both ends, a row a lane.
__device__ __forceinline__ void store_rows(const unsigned char* stage, unsigned char* to, long long pitch, int rows, int lane) {
  const unsigned c = lane & 15;
  unsigned char* row = to + (lane >> 4) * pitch;
#pragma unroll 8
  for (int i = 0; i < 16; ++i, row += 2 * pitch) {
    const unsigned a = (unsigned)(size_t)row & 15u;
    const int r = 2 * i + (lane >> 4);
    if (r < rows && (c > 0 || a == 0))
      *reinterpret_cast<uint4*>(row - a + c * 16) = *reinterpret_cast<const uint4*>(stage + r * I8_ROW_PITCH + c * 16);
  }
  if (lane < rows) {
    row = to + lane * pitch;
    const unsigned a = (unsigned)(size_t)row & 15u;
    const unsigned char* from = stage + lane * I8_ROW_PITCH;
    row -= a;
    unsigned x = a;
    if (x & 2) { *reinterpret_cast<unsigned short*>(row + x) = *reinterpret_cast<const unsigned short*>(from + x); x += 2; }
    if (x & 4) { *reinterpret_cast<unsigned*>(row + x) = *reinterpret_cast<const unsigned*>(from + x); x += 4; }
    if (x & 8) *reinterpret_cast<uint2*>(row + x) = *reinterpret_cast<const uint2*>(from + x);
    x = I8_ROW_BYTES;
    if (a & 8) { *reinterpret_cast<uint2*>(row + x) = *reinterpret_cast<const uint2*>(from + x); x += 8; }
    if (a & 4) { *reinterpret_cast<unsigned*>(row + x) = *reinterpret_cast<const unsigned*>(from + x); x += 4; }
    if (a & 2) *reinterpret_cast<unsigned short*>(row + x) = *reinterpret_cast<const unsigned short*>(from + x);
  }
}

template <typename T, int CTAS, typename X>
__global__ void __launch_bounds__(I8_THREADS, 1)
k_i8_gemm(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmX, const __grid_constant__ CUtensorMap tmC,
          const I8Args a) {
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem = (unsigned char*)(((size_t)smem_raw + 1023) & ~(size_t)1023);
  constexpr bool OWN = !std::is_void<X>::value;  // this kernel quantizes the tokens (CTAS = 1); they lie in front of the ring
  const bool boxes_out = CTAS == 1 || a.aligned;
  unsigned char* extra = smem + (boxes_out ? i8_ring(CTAS, true) : i8_ring(CTAS, false));
  I8Tail* st = (I8Tail*)(extra + (boxes_out ? i8_extra(CTAS, true) : i8_extra(CTAS, false)));
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = CTAS == 2 ? (int)cluster_ctarank() : 0;
  const int group = blockIdx.x / CTAS, ngroups = gridDim.x / CTAS;
  // a stage of this CTA: 128 rows of the accumulators' rows (of which the loads fill a.rows), then its part of their columns
  const int x_stage = OWN ? 0 : a.cols / CTAS * I8_BK, stage_bytes = I8_W_STAGE + x_stage;
  const int load_bytes = (CTAS == 1 ? a.rows : I8_ROWS) * I8_BK + x_stage;
  const int w_offset = CTAS == 1 ? 0 : I8_W_STAGE, x_offset = CTAS == 1 ? I8_W_STAGE : 0;
  const int w_rows = CTAS == 1 ? 0 : rank * (a.cols / CTAS), x_rows = CTAS == 1 ? 0 : rank * I8_ROWS;   // this CTA's part of a tile
  const int n_tiles = CTAS == 1 ? (a.n + a.rows - 1) / a.rows : (a.n + a.cols - 1) / a.cols;
  const int m_tiles = CTAS == 1 ? 1 : (a.m + 2 * I8_ROWS - 1) / (2 * I8_ROWS);
  const int units = n_tiles * m_tiles, k_blocks = (a.k + I8_BK - 1) / I8_BK;
  unsigned char* tokens = smem;
  typename std::conditional<OWN, OwnTokens<X>, NoTokens>::type own;
  if constexpr (OWN) {
    smem += k_blocks * a.cols * I8_BK;
    own.load(a);
    if (threadIdx.x < I8_ROWS) {
      ((float*)extra)[threadIdx.x] = 0.f;        // the scales,
      st->tops[threadIdx.x] = 0;                 // and the largest magnitudes
    }
  }

  if (threadIdx.x == 0) {
    for (int s = 0; s < a.stages; ++s) { mbar_init(&st->full[s], 1); mbar_init(&st->empty[s], 1); }
    for (int s = 0; s < 2; ++s) { mbar_init(&st->tmem_full[s], 1); mbar_init(&st->tmem_empty[s], I8_EPI_WARPS * CTAS); }
    mbar_init(&st->done, 1);
    st->abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 1) {
    if (CTAS == 2) {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&st->tmem_base)),
                   "r"(I8_TMEM_COLS)
                   : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&st->tmem_base)),
                   "r"(I8_TMEM_COLS)
                   : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
  }
  tc_fence_before();
  __syncthreads();
  if (CTAS == 2) cluster_sync_all();     // the peer's barriers exist before anything signals them
  tc_fence_after();
  const unsigned tmem_base = st->tmem_base;
  volatile int* abort_flag = &st->abort;

  // the head does not depend on the tokens: what the first ring takes of it is under way before these are there
  int early = 0;
  if (OWN || a.behind) {
    const int mine = group < units ? (units - 1 - group) / ngroups + 1 : 0;      // tiles of this CTA (pair)
    early = (long long)mine * k_blocks < a.stages ? mine * k_blocks : a.stages;
    if (warp == 0 && lane == 0) {
      for (int j = 0, u = group, kb = 0; j < early; ++j) {
        int channel, token;
        i8_tile<CTAS>(a, u, n_tiles, m_tiles, channel, token);
        if (rank == 0) mbar_expect_tx(&st->full[j], CTAS * load_bytes);
        unsigned char* dst = smem + (size_t)j * stage_bytes + w_offset;
        if (CTAS == 2) tma_load_2d_pair(dst, &tmW, kb * I8_BK, channel + w_rows, &st->full[j]);
        else tma_load_2d(dst, &tmW, kb * I8_BK, channel + w_rows, &st->full[j]);
        if (++kb == k_blocks) { kb = 0; u += ngroups; }
      }
    }
    __syncwarp();
  }
  if constexpr (OWN) {
    // Blocks are started together and nobody gives up a wait within two seconds (PCTC_WAIT_LIMIT_CYCLES), so that this comes before
    // whatever another block reports; this one waits for nothing before it.
    if (blockIdx.x == 0 && threadIdx.x == 0 && a.status) *a.status = 0;
    own.store(a, tokens, st->tops, (float*)extra);
    fence_async_smem();                  // the tensor core reads what was stored here
    __syncthreads();
  }

  if (warp == 0) {
    // ===================== TMA producer =====================
    if (lane == 0) {
      unsigned g = 0;
      int s = 0;
      unsigned ph = 0;
      bool ok = true;
      const auto load = [&](unsigned char* dst, const CUtensorMap* map, int k, int row, unsigned long long* bar) {
        if (CTAS == 2) tma_load_2d_pair(dst, map, k, row, bar); else tma_load_2d(dst, map, k, row, bar);
      };
      const auto load_w = [&](int stage, int kb, int channel) {
        load(smem + (size_t)stage * stage_bytes + w_offset, &tmW, kb * I8_BK, channel + w_rows, &st->full[stage]);
      };
      int channel, token;
      if (a.behind) wait_for_previous();
      for (int u = group; u < units && ok; u += ngroups) {
        i8_tile<CTAS>(a, u, n_tiles, m_tiles, channel, token);
        for (int kb = 0; kb < k_blocks; ++kb, ++g) {
          if ((int)g >= early) {
            if (!mbar_wait(&st->empty[s], ph ^ 1u, abort_flag, a.status, 1)) { ok = false; break; }
            if (rank == 0) mbar_expect_tx(&st->full[s], CTAS * load_bytes);   // the leader's barrier counts both CTAs
            load_w(s, kb, channel);
          }
          if (!OWN) load(smem + (size_t)s * stage_bytes + x_offset, &tmX, kb * I8_BK, token + x_rows, &st->full[s]);
          if (++s == a.stages) { s = 0; ph ^= 1u; }
        }
      }
      // every copy issued has landed before the CTA may exit (the leader's barriers count the peer's bytes too)
      if (rank == 0) {
        const unsigned n = (unsigned)a.stages;
        for (unsigned j = (g > n ? g - n : 0); j < g; ++j) mbar_wait_drain(&st->full[j % n], (j / n) & 1u);
      }
    }
  } else if (warp == 1) {
    // ===================== MMA issuer (in the pair's leader) =====================
    if (lane == 0 && rank == 0) {
      // accumulators of 32-bit integers, both operands signed 8-bit, k contiguous
      const unsigned idesc = (2u << 4) | (1u << 7) | (1u << 10) | ((unsigned)(a.cols >> 3) << 17) |
                             ((unsigned)((I8_ROWS * CTAS) >> 4) << 24);
      const auto commit = [&](unsigned long long* bar) { if (CTAS == 2) tc_commit_pair(bar); else tc_commit(bar); };
      unsigned it = 0, ph = 0;
      int s = 0;
      bool ok = true;
      for (int u = group; u < units && ok; u += ngroups, ++it) {
        const unsigned acc = it & 1u, aph = (it >> 1) & 1u;
        if (!mbar_wait(&st->tmem_empty[acc], aph ^ 1u, abort_flag, a.status, 2)) { ok = false; break; }
        tc_fence_after();
        const unsigned d_tmem = tmem_base + acc * 256;
        for (int kb = 0; kb < k_blocks; ++kb) {
          if (!mbar_wait(&st->full[s], ph, abort_flag, a.status, 3)) { ok = false; break; }
          tc_fence_after();
          const unsigned at = smem_u32(smem + (size_t)s * stage_bytes);
          const unsigned long long rdesc = i8_smem_desc(at);
          const unsigned long long cdesc = i8_smem_desc(OWN ? smem_u32(tokens) + kb * a.cols * I8_BK : at + I8_W_STAGE);
#pragma unroll
          for (int kk = 0; kk < I8_BK / 32; ++kk) {               // 32 k an instruction: 32 bytes further on
            const unsigned more = (kb != 0 || kk != 0) ? 1u : 0u;
            if (CTAS == 2) tc_mma_i8_pair(d_tmem, rdesc + kk * 2, cdesc + kk * 2, idesc, more);
            else tc_mma_i8(d_tmem, rdesc + kk * 2, cdesc + kk * 2, idesc, more);
          }
          commit(&st->empty[s]);
          if (++s == a.stages) { s = 0; ph ^= 1u; }
        }
        if (ok) commit(&st->tmem_full[acc]);
      }
      if (CTAS == 2) tc_commit_pair_local(&st->done); else tc_commit(&st->done);
      mbar_wait_drain(&st->done, 0);
    }
  } else {
    // ===================== epilogue warps: two for each quarter of the lanes =====================
    const int ew = warp - 2, q = warp & 3;
    T* C = (T*)a.C;
    unsigned it = 0, boxes = 0;
    bool ok = true;
    const auto bias_of = [&](int j) {
      return !a.bias ? 0.f : a.bias_bf16 ? __bfloat162float(((const __nv_bfloat16*)a.bias)[j]) : ((const float*)a.bias)[j];
    };
    const auto sums_ready = [&](unsigned acc, unsigned aph) {
      int got = 0;
      if (lane == 0) got = mbar_wait(&st->tmem_full[acc], aph, abort_flag, a.status, 4) ? 1 : 0;
      got = __shfl_sync(0xffffffffu, got, 0);
      if (got) tc_fence_after();
      return got != 0;
    };
    const auto sums_read = [&](unsigned acc) {
      tc_fence_before();
      __syncwarp();
      if (lane == 0) { if (CTAS == 2) mbar_arrive_leader(&st->tmem_empty[acc]); else mbar_arrive(&st->tmem_empty[acc]); }
    };
    if (a.behind) wait_for_previous();
    if constexpr (CTAS == 1) {
      // a lane is a channel; the columns are all tokens there are, in groups of 32 that the two warps take in turn
      float* sa = (float*)extra;
      if (!OWN) {
        for (int i = lane; i < I8_ROWS; i += 32) sa[i] = i < a.m ? a.a_scale[i] : 0.f;   // the same by every warp
        __syncwarp();
      }
      // what a tile needs beside its sums is loaded a tile ahead
      const auto channel_of = [&](int u) { return q * 32 + lane < a.rows ? u * a.rows + q * 32 + lane : a.n; };
      float next_sb = 0.f, next_bias = 0.f;
      const auto prefetch = [&](int u) {
        const int j = channel_of(u);
        next_sb = j < a.n ? a.b_scale[j] : 0.f;
        next_bias = j < a.n ? bias_of(j) : 0.f;
      };
      if (group < units) prefetch(group);
      for (int u = group; u < units && ok; u += ngroups, ++it) {
        const int j = channel_of(u);
        const bool row_ok = j < a.n;
        const float sb = next_sb, bias = next_bias;
        if (u + ngroups < units) prefetch(u + ngroups);
        const unsigned acc = it & 1u;
        if (!sums_ready(acc, (it >> 1) & 1u)) { ok = false; break; }
        for (int i0 = (ew >> 2) * 32; i0 < a.m; i0 += 64) {
          float v[32];
          tmem_ld32(tmem_base + ((unsigned)(q * 32) << 16) + acc * 256 + i0, v);
          T* to = C + (long long)i0 * a.ldc + j;
          // lanes 2l and 2l + 1 hold neighbouring channels: of bf16 the even one stores both of token c, the odd one of token c + 1
          const bool odd = lane & 1, pairs = sizeof(T) == 2 && a.aligned && __all_sync(0xffffffffu, !row_ok || (j | 1) < a.n);
          const unsigned pick = odd ? 0x3276u : 0x5410u;
#pragma unroll
          for (int b = 0; b < 32; b += 8) {
            const int cnt = min(8, a.m - i0 - b);                 // tokens of this eighth
            if (cnt <= 0) break;
#pragma unroll
            for (int c = b; c < b + 8; c += 4) {
              const float4 f = *reinterpret_cast<const float4*>(sa + i0 + c);
              v[c] = fmaf((float)__float_as_int(v[c]), f.x * sb, bias);
              v[c + 1] = fmaf((float)__float_as_int(v[c + 1]), f.y * sb, bias);
              v[c + 2] = fmaf((float)__float_as_int(v[c + 2]), f.z * sb, bias);
              v[c + 3] = fmaf((float)__float_as_int(v[c + 3]), f.w * sb, bias);
            }
            T* at = to + (long long)b * a.ldc;
            if constexpr (sizeof(T) == 2) {
              if (pairs) {
                at += odd ? a.ldc - 1 : 0;
#pragma unroll
                for (int c = 0; c < 8; c += 2, at += 2 * a.ldc) {
                  const __nv_bfloat162 p = __floats2bfloat162_rn(v[b + c], v[b + c + 1]);
                  const unsigned mine = *reinterpret_cast<const unsigned*>(&p);
                  const unsigned w = __byte_perm(mine, __shfl_xor_sync(0xffffffffu, mine, 1), pick);
                  if (row_ok && c + (odd ? 1 : 0) < cnt) *reinterpret_cast<unsigned*>(at) = w;
                }
                continue;
              }
            }
            if (row_ok)
#pragma unroll
              for (int c = 0; c < 8; ++c, at += a.ldc)
                if (c < cnt) *at = from_float<T>(v[b + c]);
          }
        }
        sums_read(acc);
      }
    } else {
      // a lane is a token; a warp takes 128 channels, 32 at a time
      unsigned char* stage = extra + ew * i8_out(true);
      float* sb = (float*)(extra + I8_EPI_WARPS * i8_out(true)) + ew * (2 * I8_WARP_COLS);
      if (!a.aligned) {
        stage = extra + ew * i8_out(false);
        sb = (float*)(extra + I8_EPI_WARPS * i8_out(false)) + ew * (2 * I8_WARP_COLS);
      }
      float* bias = sb + I8_WARP_COLS;
      const unsigned swizzle = (unsigned)((lane >> 1) & 3);       // 64-byte swizzle of a row of a box
      // what a tile needs beside its sums is loaded a tile ahead
      int next_row0 = 0, next_j0 = 0;
      float next_sa = 0.f, next_sb[I8_WARP_COLS / 32], next_bias[I8_WARP_COLS / 32];
      const auto prefetch = [&](int u) {
        int channel, token;
        i8_tile<2>(a, u, n_tiles, m_tiles, channel, token);
        next_row0 = token + rank * I8_ROWS + q * 32;
        next_j0 = channel + (ew >> 2) * I8_WARP_COLS;
        next_sa = next_row0 + lane < a.m ? a.a_scale[next_row0 + lane] : 0.f;
#pragma unroll
        for (int c = 0; c < I8_WARP_COLS / 32; ++c) {
          const int j = next_j0 + c * 32 + lane;
          next_sb[c] = j < a.n ? a.b_scale[j] : 0.f;
          next_bias[c] = a.bias && j < a.n ? bias_of(j) : 0.f;
        }
      };
      if (group < units) prefetch(group);
      for (int u = group; u < units && ok; u += ngroups, ++it) {
        const int row0 = next_row0, j0 = next_j0, rows = min(32, a.m - row0);
        const float sa = next_sa;
        __syncwarp();
#pragma unroll
        for (int c = 0; c < I8_WARP_COLS / 32; ++c) {
          sb[c * 32 + lane] = next_sb[c];
          bias[c * 32 + lane] = next_bias[c];
        }
        __syncwarp();
        const unsigned acc = it & 1u;
        if (!sums_ready(acc, (it >> 1) & 1u)) { ok = false; break; }
        const unsigned taddr = tmem_base + ((unsigned)(q * 32) << 16) + acc * 256 + (ew >> 2) * I8_WARP_COLS;
        unsigned r[2][32];
        tmem_issue32(taddr, r[0]);
        if (u + ngroups < units) prefetch(u + ngroups);
        const bool whole = j0 + I8_WARP_COLS <= a.n;
        unsigned carry = 0;                                       // the last two bf16 values of the group before
        const unsigned shift = (unsigned)(size_t)(C + (long long)(row0 + lane) * a.ldc + j0) & 15u;   // how far this lane's row is from 16 bytes
#pragma unroll
        for (int g = 0; g < I8_WARP_COLS / 32; ++g) {
          const int c0 = g * 32;
          tmem_wait32(r[g & 1]);
          if (g + 1 < I8_WARP_COLS / 32) tmem_issue32(taddr + c0 + 32, r[(g + 1) & 1]);
          if (j0 + c0 >= a.n) continue;
          float v[32];
#pragma unroll
          for (int c = 0; c < 32; c += 4) {
            const float4 f = *reinterpret_cast<const float4*>(sb + c0 + c), b = *reinterpret_cast<const float4*>(bias + c0 + c);
            v[c] = fmaf((float)(int)r[g & 1][c], sa * f.x, b.x);
            v[c + 1] = fmaf((float)(int)r[g & 1][c + 1], sa * f.y, b.y);
            v[c + 2] = fmaf((float)(int)r[g & 1][c + 2], sa * f.z, b.z);
            v[c + 3] = fmaf((float)(int)r[g & 1][c + 3], sa * f.w, b.w);
          }
          if (a.aligned) {
            // 32 bf16 channels a box, or 16 fp32 ones; one box fills while the other is read out
#pragma unroll
            for (int b = 0; b < (int)sizeof(T) / 2; ++b) {
              if (j0 + c0 + b * 16 >= a.n) break;
              if (lane == 0) bulk_wait_read1();
              __syncwarp();
              unsigned char* box = stage + (boxes++ & 1u) * I8_BOX;
              unsigned char* row = box + lane * 64;
#pragma unroll
              for (int p = 0; p < 4; ++p) {
                uint4 w;
                if constexpr (sizeof(T) == 4) {
                  const float* x = v + b * 16 + p * 4;
                  w = make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
                } else {
                  const float x[8] = {v[p * 8], v[p * 8 + 1], v[p * 8 + 2], v[p * 8 + 3], v[p * 8 + 4], v[p * 8 + 5], v[p * 8 + 6], v[p * 8 + 7]};
                  w = Vec8<__nv_bfloat16>::pack(x);
                }
                *reinterpret_cast<uint4*>(row + (((unsigned)p ^ swizzle) << 4)) = w;
              }
              fence_async_smem();
              __syncwarp();
              if (lane == 0) {
                tma_store_2d(&tmC, box, j0 + c0 + b * 16, row0);  // rows and channels past the extents are clipped
                bulk_commit();
              }
            }
          } else if (whole) {
            // rows of 256 bytes are gathered, each as far from a 16-byte boundary as it will be in C
            constexpr int PER = 32 * (int)sizeof(T) / 4;           // words of a group
            constexpr int GROUPS = I8_ROW_BYTES / (32 * (int)sizeof(T));
            unsigned* to = reinterpret_cast<unsigned*>(stage + lane * I8_ROW_PITCH) + (shift >> 2) + (g % GROUPS) * PER;
            if (g % GROUPS == 0) __syncwarp();
            if constexpr (sizeof(T) == 4) {
#pragma unroll
              for (int c = 0; c < 32; ++c) to[c] = __float_as_uint(v[c]);
            } else {
              const unsigned pick = (shift & 2) ? 0x5432u : 0x7654u;   // half a word further on: the value before and this one
#pragma unroll
              for (int c = 0; c < 32; c += 2) {
                const __nv_bfloat162 p = __floats2bfloat162_rn(v[c], v[c + 1]);
                const unsigned w = *reinterpret_cast<const unsigned*>(&p);
                to[c / 2] = __byte_perm(carry, w, pick);
                carry = w;
              }
              if (g % GROUPS == GROUPS - 1 && (shift & 2)) to[PER] = carry >> 16;
            }
            if (g % GROUPS == GROUPS - 1) {
              __syncwarp();
              store_rows(stage, (unsigned char*)(C + (long long)row0 * a.ldc + j0 + c0 + 32) - I8_ROW_BYTES, a.ldc * (long long)sizeof(T), rows, lane);
            }
          } else {
            // the last channels: turned in shared memory, so that a row's 32 are stored by 32 lanes
            float* turn = (float*)stage;
            __syncwarp();
#pragma unroll
            for (int c = 0; c < 32; ++c) turn[lane * 32 + (c ^ lane)] = v[c];
            __syncwarp();
            const int j = j0 + c0 + lane;
            if (j < a.n) {
              T* to = C + (long long)row0 * a.ldc + j;
#pragma unroll 8
              for (int i = 0; i < rows; ++i, to += a.ldc) *to = from_float<T>(turn[i * 32 + (lane ^ i)]);
            }
          }
        }
        sums_read(acc);
      }
      if (lane == 0) bulk_wait0();                                // this warp's stores have completed
    }
  }

  tc_fence_before();
  __syncthreads();
  if (*abort_flag) {                     // a copy that the peer may still have in flight lands meanwhile (see umma_gemm.cu)
    const long long t0 = clock64();
    while (clock64() - t0 < ABORT_LINGER_CYCLES) { }
    __syncthreads();
  }
  if (CTAS == 2) cluster_sync_all();     // no CTA of a pair leaves while the other may still signal it
  if (warp == 1) {
    tc_fence_after();
    if (CTAS == 2)
      asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(I8_TMEM_COLS) : "memory");
    else
      asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(I8_TMEM_COLS) : "memory");
  }
}

// ---------------------------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------------------------
bool i8_map_out(CUtensorMap* map, void* C, long long n, long long m, long long ldc, bool bf16) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  cuuint64_t dims[2] = {(cuuint64_t)n, (cuuint64_t)m};
  cuuint64_t strides[1] = {(cuuint64_t)(ldc * (bf16 ? 2 : 4))};
  cuuint32_t box[2] = {bf16 ? 32u : 16u, 32};
  cuuint32_t estr[2] = {1, 1};
  return fn(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 2, C, dims, strides, box, estr,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_NONE,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
bool i8_map(CUtensorMap* map, const void* base, long long k, long long rows, long long ld, unsigned box_rows) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  cuuint64_t dims[2] = {(cuuint64_t)k, (cuuint64_t)rows};
  cuuint64_t strides[1] = {(cuuint64_t)ld};
  cuuint32_t box[2] = {I8_BK, box_rows};
  cuuint32_t estr[2] = {1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(base), dims, strides, box, estr,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename T, int CTAS, typename X>
cudaError_t i8_launch(const CUtensorMap& tmW, const CUtensorMap& tmX, const CUtensorMap& tmC, const I8Args& a, int units, cudaStream_t stream) {
  static std::atomic<int> groups_on[MAX_DEVICES];       // CTA groups that can be resident at once; 0: not configured there yet
  auto kern = k_i8_gemm<T, CTAS, X>;
  const int dev = current_device();
  int most = groups_on[dev].load(std::memory_order_acquire);
  if (most == 0) {
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, i8_smem(CTAS));
    if (e != cudaSuccess) return e;
  }
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = CTAS;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.blockDim = dim3(I8_THREADS);
  cfg.dynamicSmemBytes = i8_smem(CTAS);
  cfg.stream = stream;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  if (most == 0) {
    cfg.gridDim = dim3((unsigned)(sm_count() / CTAS * CTAS));
    int n = 0;
    if (cudaOccupancyMaxActiveClusters(&n, kern, &cfg) != cudaSuccess || n <= 0) n = sm_count() / CTAS;
    most = n;
    groups_on[dev].store(n, std::memory_order_release);
  }
  cfg.gridDim = dim3((unsigned)((units < most ? units : most) * CTAS));
  cfg.numAttrs = a.behind ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kern, tmW, tmX, tmC, a);
}

// Whether the rows of the tokens can be read in aligned groups of eight.
bool in_eights(const void* x, long long ld_x, bool bf16, int k) {
  return k % 8 == 0 && ((size_t)x & 15) == 0 && ld_x * (bf16 ? 2 : 4) % 16 == 0;
}

constexpr long long I8_BAND_BYTES = 32LL << 20;         // token rows of a band: a quarter of the L2

}  // namespace

cudaError_t i8_gemm(const signed char* A, long long lda, const float* a_scale, const signed char* B, long long ldb,
                    const float* b_scale, const void* bias, bool bias_bf16, int m, int n, int k, void* C, long long ldc,
                    bool out_bf16, int* status, bool behind, cudaStream_t stream, const void* x, long long ld_x, bool x_bf16) {
  if (m <= 0 || n <= 0) return cudaSuccess;
  if (x && !i8_own_tokens(x, ld_x, x_bf16, m, k)) return cudaErrorInvalidValue;
  // up to 128 tokens: tiles as wide as the tokens, so that the head is read once and the ring is deep
  const bool pair = m > I8_ROWS;
  I8Args a = {};
  a.n = n; a.m = m; a.k = k;
  // (a TMA store clips a row at 16 bytes, not at its last value)
  const int es = out_bf16 ? 2 : 4;
  a.aligned = pair ? ((size_t)C & 15) == 0 && ldc * es % 16 == 0 && (long long)n * es % 16 == 0 : ((size_t)C & 3) == 0 && ldc % 2 == 0;
  a.cols = pair ? 256 : (m + 15) / 16 * 16;
  const int blocks = (k + I8_BK - 1) / I8_BK, stage = I8_W_STAGE + (x ? 0 : a.cols / (pair ? 2 : 1) * I8_BK);
  const int fit = (i8_ring(pair ? 2 : 1, a.aligned) - (x ? blocks * a.cols * I8_BK : 0)) / stage;
  a.stages = fit < I8_MAX_STAGES ? fit : I8_MAX_STAGES;
  // few tokens and long rows: tiles of equal height that fill whole rounds of the SMs (4 x 151,936 x 4,096: 143 -> 105 us; a
  // multiple of 4 keeps pairs of channels together); with short rows the results count, and tiles of 128 keep them aligned
  // (1 x 38,998 x 320: 8.8 us against 10.2)
  const long long sms = sm_count(), rounds = ((long long)n + sms * I8_ROWS - 1) / (sms * I8_ROWS);
  a.rows = pair || k < 2048 || n < sms * I8_ROWS ? I8_ROWS : (int)((n + rounds * sms - 1) / (rounds * sms) + 3) / 4 * 4;
  const long long n_tiles = pair ? ((long long)n + 255) / 256 : ((long long)n + a.rows - 1) / a.rows, m_tiles = pair ? ((long long)m + 255) / 256 : 1;
  if (n_tiles * m_tiles > 0x7fffffffLL - (1 << 20)) return cudaErrorInvalidValue;
  long long band = I8_BAND_BYTES / (256LL * k);
  band = band < 1 ? 1 : band > m_tiles ? m_tiles : band;
  if (band * n_tiles > 0x7fffffffLL) band = 1;
  a.band = (int)band;
  a.a_scale = a_scale;
  a.b_scale = b_scale;
  a.bias = bias;
  a.bias_bf16 = bias_bf16 ? 1 : 0;
  a.C = C;
  a.ldc = ldc;
  a.status = status;
  a.behind = behind ? 1 : 0;
  a.x = x;
  a.ld_x = ld_x;
  a.wide_x = in_eights(x, ld_x, x_bf16, k);
  alignas(64) CUtensorMap tmW, tmX = {}, tmC = {};
  if (!i8_map(&tmW, B, k, n, ldb, (unsigned)a.rows)) return cudaErrorInvalidValue;
  if (!x && !i8_map(&tmX, A, k, m, lda, pair ? I8_ROWS : (unsigned)a.cols)) return cudaErrorInvalidValue;
  if (pair && a.aligned && !i8_map_out(&tmC, C, n, m, ldc, out_bf16)) return cudaErrorInvalidValue;
  const int units = (int)(n_tiles * m_tiles);
  const auto launch = [&](auto out) {
    using T = decltype(out);
    if (pair) return i8_launch<T, 2, void>(tmW, tmX, tmC, a, units, stream);
    if (!x) return i8_launch<T, 1, void>(tmW, tmX, tmC, a, units, stream);
    return x_bf16 ? i8_launch<T, 1, __nv_bfloat16>(tmW, tmX, tmC, a, units, stream) : i8_launch<T, 1, float>(tmW, tmX, tmC, a, units, stream);
  };
  return out_bf16 ? launch(__nv_bfloat16()) : launch(float());
}

// Whether the product quantizes so many tokens itself: they are columns of one tile, and fit beside a ring of 100 KB and more.
bool i8_own_tokens(const void* x, long long ld_x, bool bf16, int m, int k) {
  return m <= I8_ROWS && (long long)m * k <= (in_eights(x, ld_x, bf16, k) ? I8_OWN_VALUES : I8_OWN_SINGLE) &&
         (long long)(m + 15) / 16 * 16 * ((k + 127) / 128 * 128) <= 98304;
}

cudaError_t i8_quantize(const void* x, bool bf16, long long rows, long long cols, long long ld_x, signed char* q, long long ld_q,
                        float* scales, int* clear, cudaStream_t stream) {
  if (rows <= 0) return cudaSuccess;
  const QuantArgs a{x, q, scales, clear, rows, cols, ld_x, ld_q};
  return bf16 ? quantize_launch<__nv_bfloat16>(a, stream) : quantize_launch<float>(a, stream);
}

namespace {

size_t up(size_t b) { return (b + 255) / 256 * 256; }
struct I8Plan {
  size_t q, scales, total;
  long long ld;
};
I8Plan i8_plan(const pctc_i8_t* p) {
  I8Plan w;
  w.ld = ((long long)p->k + 127) / 128 * 128;    // (a row that is loaded from 128-byte boundaries on comes in whole lines)
  w.q = 256;                                     // the status word comes first
  w.scales = w.q + up((size_t)p->m * w.ld);
  w.total = w.scales + up((size_t)p->m * 4);
  return w;
}

pctc_status_t check_i8(const pctc_i8_t* p) {
  if (!p || p->m < 0 || p->n < 1 || p->k < 1) return PCTC_ERR_INVALID_ARG;
  if (p->k > PCTC_I8_MAX_K || p->m > 0x7fffffff - 256 || p->n > 0x7fffffff - 256) return PCTC_ERR_UNSUPPORTED;
  if (p->out_dtype != PCTC_BF16 && p->out_dtype != PCTC_FP32) return PCTC_ERR_UNSUPPORTED;
  if (p->ldc < p->n) return PCTC_ERR_INVALID_ARG;
  if (p->ldc > MAX_ELEMENTS / (p->m + 1)) return PCTC_ERR_UNSUPPORTED;
  return PCTC_OK;
}
// The 8-bit operand [rows, k] of pitch ld.
bool bad_operand(const void* q, long long ld, const float* scales, int k) {
  return !q || ((size_t)q & 15) || ld < k || ld % 16 || ld >= (1LL << 40) || !scales || ((size_t)scales & 3);
}

}  // namespace
}  // namespace pctc

using namespace pctc;

extern "C" {

pctc_status_t pctc_i8_quantize(int64_t rows, int64_t cols, int32_t dtype, const void* x, int64_t ld_x, int8_t* q, int64_t ld_q,
                               float* scales, void* stream_v) {
  if (rows < 0 || cols < 1 || ld_x < cols || ld_q < cols) return PCTC_ERR_INVALID_ARG;
  if (dtype != PCTC_BF16 && dtype != PCTC_FP32) return PCTC_ERR_UNSUPPORTED;
  if (rows > 0x7fffffffLL || ld_x > MAX_ELEMENTS / (rows + 1) || ld_q > MAX_ELEMENTS / (rows + 1)) return PCTC_ERR_UNSUPPORTED;
  if (rows == 0) return PCTC_OK;
  const size_t es = dtype == PCTC_BF16 ? 2 : 4;
  if (!x || ((size_t)x & (es - 1)) || !q || !scales || ((size_t)scales & 3)) return PCTC_ERR_INVALID_ARG;
  const Rows from{x, rows, ld_x, cols, es}, to{q, rows, ld_q, cols, 1}, s{scales, 1, rows, rows, 4};
  if (to.overlaps(from) || s.overlaps(from) || s.overlaps(to)) return PCTC_ERR_INVALID_ARG;
  return i8_quantize(x, dtype == PCTC_BF16, rows, cols, ld_x, (signed char*)q, ld_q, scales, nullptr, (cudaStream_t)stream_v) ==
                 cudaSuccess
             ? PCTC_OK
             : PCTC_ERR_CUDA;
}

pctc_status_t pctc_i8_matmul(const pctc_i8_t* p, const int8_t* A, const float* a_scales, const int8_t* B, const float* b_scales,
                             const void* bias, void* C, int32_t* device_status, void* stream_v) {
  const pctc_status_t st = check_i8(p);
  if (st != PCTC_OK) return st;
  if (bias && p->bias_dtype != PCTC_BF16 && p->bias_dtype != PCTC_FP32) return PCTC_ERR_UNSUPPORTED;
  if (p->m == 0) return PCTC_OK;
  const size_t es = p->out_dtype == PCTC_BF16 ? 2 : 4, bs = p->bias_dtype == PCTC_BF16 ? 2 : 4;
  if (bad_operand(A, p->lda, a_scales, p->k) || bad_operand(B, p->ldb, b_scales, p->k)) return PCTC_ERR_INVALID_ARG;
  if (!C || ((size_t)C & (es - 1)) || ((size_t)bias & (bs - 1)) || ((size_t)device_status & 3)) return PCTC_ERR_INVALID_ARG;
  const Rows to{C, p->m, p->ldc, p->n, es}, word{device_status, 1, 1, 1, 4};
  const Rows in[] = {{A, p->m, p->lda, p->k, 1}, {B, p->n, p->ldb, p->k, 1}, {a_scales, 1, p->m, p->m, 4},
                     {b_scales, 1, p->n, p->n, 4}, {bias, 1, p->n, p->n, bs}};
  if (to.overlaps(word)) return PCTC_ERR_INVALID_ARG;
  for (const Rows& r : in)
    if (to.overlaps(r) || word.overlaps(r)) return PCTC_ERR_INVALID_ARG;
  if (!umma_available()) return PCTC_ERR_CUDA;
  const cudaError_t e = i8_gemm((const signed char*)A, p->lda, a_scales, (const signed char*)B, p->ldb, b_scales, bias,
                                p->bias_dtype == PCTC_BF16, p->m, p->n, p->k, C, p->ldc, p->out_dtype == PCTC_BF16, device_status, false,
                                (cudaStream_t)stream_v, nullptr, 0, false);
  return e == cudaSuccess ? PCTC_OK : e == cudaErrorInvalidValue ? PCTC_ERR_UNSUPPORTED : PCTC_ERR_CUDA;
}

pctc_status_t pctc_i8_logits_workspace_bytes(const pctc_i8_t* p, size_t* bytes_out) {
  if (!bytes_out) return PCTC_ERR_INVALID_ARG;
  const pctc_status_t st = check_i8(p);
  if (st != PCTC_OK) return st;
  *bytes_out = i8_plan(p).total;
  return PCTC_OK;
}

pctc_status_t pctc_i8_logits(const pctc_i8_t* p, const void* x, int32_t x_dtype, const int8_t* B, const float* b_scales,
                             const void* bias, void* C, void* workspace, size_t workspace_bytes, void* stream_v) {
  const pctc_status_t st = check_i8(p);
  if (st != PCTC_OK) return st;
  if (x_dtype != PCTC_BF16 && x_dtype != PCTC_FP32) return PCTC_ERR_UNSUPPORTED;
  if (bias && p->bias_dtype != PCTC_BF16 && p->bias_dtype != PCTC_FP32) return PCTC_ERR_UNSUPPORTED;
  if (p->m == 0) return PCTC_OK;
  const size_t xs = x_dtype == PCTC_BF16 ? 2 : 4, es = p->out_dtype == PCTC_BF16 ? 2 : 4, bs = p->bias_dtype == PCTC_BF16 ? 2 : 4;
  if (!x || ((size_t)x & (xs - 1)) || p->lda < p->k || bad_operand(B, p->ldb, b_scales, p->k)) return PCTC_ERR_INVALID_ARG;
  if (p->lda > MAX_ELEMENTS / p->m) return PCTC_ERR_UNSUPPORTED;
  if (!C || ((size_t)C & (es - 1)) || ((size_t)bias & (bs - 1)) || !workspace || ((size_t)workspace & 255)) return PCTC_ERR_INVALID_ARG;
  const I8Plan w = i8_plan(p);
  if (workspace_bytes < w.total) return PCTC_ERR_WORKSPACE_TOO_SMALL;
  const Rows to{C, p->m, p->ldc, p->n, es}, own{workspace, 1, (long long)w.total, (long long)w.total, 1};
  const Rows in[] = {{x, p->m, p->lda, p->k, xs}, {B, p->n, p->ldb, p->k, 1}, {b_scales, 1, p->n, p->n, 4}, {bias, 1, p->n, p->n, bs}};
  if (to.overlaps(own)) return PCTC_ERR_INVALID_ARG;
  for (const Rows& r : in)
    if (to.overlaps(r) || own.overlaps(r)) return PCTC_ERR_INVALID_ARG;
  if (!umma_available()) return PCTC_ERR_CUDA;
  char* ws = (char*)workspace;
  signed char* q = (signed char*)(ws + w.q);
  float* scales = (float*)(ws + w.scales);
  cudaStream_t stream = (cudaStream_t)stream_v;
  const bool fused = i8_own_tokens(x, p->lda, x_dtype == PCTC_BF16, p->m, p->k);
  if (!fused && i8_quantize(x, x_dtype == PCTC_BF16, p->m, p->k, p->lda, q, w.ld, scales, (int*)ws, stream) != cudaSuccess) return PCTC_ERR_CUDA;
  const cudaError_t e = i8_gemm(q, w.ld, scales, (const signed char*)B, p->ldb, b_scales, bias, p->bias_dtype == PCTC_BF16, p->m, p->n,
                                p->k, C, p->ldc, p->out_dtype == PCTC_BF16, (int*)ws, !fused, stream, fused ? x : nullptr, p->lda,
                                x_dtype == PCTC_BF16);
  return e == cudaSuccess ? PCTC_OK : e == cudaErrorInvalidValue ? PCTC_ERR_UNSUPPORTED : PCTC_ERR_CUDA;
}

}  // extern "C"
