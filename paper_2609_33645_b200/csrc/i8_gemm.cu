// The head in 8-bit integers:  C[i,j] = T(float(sum_k qa[i,k] qb[j,k]) * sa[i] * sb[j] + bias[j]),  with rows quantized as
//   s = max|x| / 127,   q = round(x * (127 / max|x|)).
// Sums are whole numbers of 32 bits (exact for k < 2^17); nothing is rounded before the scales.
//
// k_i8_gemm is a persistent tcgen05 kernel (kind::i8).  The rows of its accumulators are the channels j (the head's rows) and
// the columns the tokens i: with few tokens the head streams through a deep ring as the wide operand of 128 x 16 ..
// 128 x 128 tiles, and 32 lanes of a warp hold 32 neighbouring channels of a token, which is the order of C.  Many tokens
// take 256 x 256 tiles of CTA pairs (cta_group::2).  Roles, rings and bounded waits are those of the bf16 kernel in umma_gemm.cu.
//   few tokens: bound by HBM, the head's bytes once;   many: by the tensor pipe.
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

// GROUP threads hold a row: NV groups of eight values each.
template <typename T, int GROUP, int NV>
__global__ void __launch_bounds__(QUANT_THREADS) k_quantize(const QuantArgs a) {
  __shared__ unsigned tops[QUANT_THREADS / 32];
  if (a.clear && blockIdx.x == 0 && threadIdx.x == 0) *a.clear = 0;
  const long long row = (long long)blockIdx.x * (QUANT_THREADS / GROUP) + threadIdx.x / GROUP;
  const int at = threadIdx.x % GROUP, per_row = (int)(a.cols / 8);
  const bool there = row < a.rows;
  Vec8<T> v[NV];
  unsigned top = 0;
#pragma unroll
  for (int k = 0; k < NV; ++k)
    if (there && at + k * GROUP < per_row) v[k].load((const T*)a.x + row * a.ld_x + (at + k * GROUP) * 8);
#pragma unroll
  for (int k = 0; k < NV; ++k)
    if (there && at + k * GROUP < per_row) {
      float x[8];
      v[k].get(x);
#pragma unroll
      for (int j = 0; j < 8; ++j) top = max(top, magnitude(x[j]));
    }
  top = __reduce_max_sync(0xffffffffu, top);
  if (GROUP > 32) {
    if ((threadIdx.x & 31) == 0) tops[threadIdx.x >> 5] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < QUANT_THREADS / 32; ++w) top = max(top, tops[w]);
  }
  if (!there) return;
  float scale;
  const float f = row_factor(top, scale);
  if (at == 0) a.scales[row] = scale;
#pragma unroll
  for (int k = 0; k < NV; ++k)
    if (at + k * GROUP < per_row) {
      float x[8];
      v[k].get(x);
      unsigned w[2] = {0u, 0u};
#pragma unroll
      for (int j = 0; j < 8; ++j) w[j >> 2] |= ((unsigned)quantize_one(x[j], f) & 0xffu) << (8 * (j & 3));
      *reinterpret_cast<uint2*>(a.q + row * a.ld_q + (at + k * GROUP) * 8) = make_uint2(w[0], w[1]);
    }
}

// Rows of any length, stride and address, read twice.
template <typename T>
__global__ void __launch_bounds__(QUANT_THREADS) k_quantize_any(const QuantArgs a) {
  __shared__ unsigned tops[QUANT_THREADS / 32];
  if (a.clear && blockIdx.x == 0 && threadIdx.x == 0) *a.clear = 0;
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

template <typename T, int GROUP, int NV>
void quantize_rows(const QuantArgs& a, cudaStream_t stream) {
  constexpr int per = QUANT_THREADS / GROUP;
  k_quantize<T, GROUP, NV><<<(unsigned)((a.rows + per - 1) / per), QUANT_THREADS, 0, stream>>>(a);
}
template <typename T>
cudaError_t quantize_launch(const QuantArgs& a, cudaStream_t stream) {
  const bool vec = a.cols % 8 == 0 && ((size_t)a.x & 15) == 0 && (a.ld_x * (long long)sizeof(T)) % 16 == 0 &&
                   ((size_t)a.q & 7) == 0 && a.ld_q % 8 == 0;
  const long long v = a.cols / 8;
  if (!vec || v > 256 * 4) k_quantize_any<T><<<(unsigned)a.rows, QUANT_THREADS, 0, stream>>>(a);
  else if (v <= 32) quantize_rows<T, 32, 1>(a, stream);
  else if (v <= 64) quantize_rows<T, 32, 2>(a, stream);
  else if (v <= 128) quantize_rows<T, 32, 4>(a, stream);
  else if (v <= 256) quantize_rows<T, 256, 1>(a, stream);
  else if (v <= 512) quantize_rows<T, 256, 2>(a, stream);
  else quantize_rows<T, 256, 4>(a, stream);
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
constexpr int I8_RING = 216 * 1024;              // shared memory for the ring
constexpr int I8_TMEM_COLS = 512;

struct I8Args {
  int n, m, k;                                   // channels, tokens, contraction
  int cols;                                      // tokens of a tile
  int stages;
  int band;                                      // token tiles that are walked together (their rows stay in L2)
  const float* a_scale;                          // [m]
  const float* b_scale;                          // [n]
  const void* bias;                              // [n] or null
  int bias_bf16;
  void* C;
  long long ldc;
  int pairs;                                     // two neighbouring bf16 channels can be stored as one word
  int* status;
};

struct I8Tail {
  unsigned long long full[I8_MAX_STAGES];
  unsigned long long empty[I8_MAX_STAGES];
  unsigned long long tmem_full[2];
  unsigned long long tmem_empty[2];
  unsigned long long done;
  unsigned tmem_base;
  int abort;
  float scale[I8_EPI_WARPS][32];                 // token scales of the columns that a warp works on
};
constexpr int I8_SMEM = 1024 + I8_RING + (int)((sizeof(I8Tail) + 255) / 256 * 256);
static_assert(I8_SMEM <= 227 * 1024, "shared memory budget");

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

// Tile u: token tiles run fastest inside a band, so that the head's rows are read once a band while the band's token
// rows stay in L2.
__device__ __forceinline__ void i8_tile(int u, int n_tiles, int m_tiles, int band, int& nt, int& mt) {
  const int b = u / (band * n_tiles), r = u - b * band * n_tiles, rows = min(band, m_tiles - b * band);
  nt = r / rows;
  mt = b * band + (r - nt * rows);
}

template <typename T, int CTAS>
__global__ void __launch_bounds__(I8_THREADS, 1)
k_i8_gemm(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmX, const I8Args a) {
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem = (unsigned char*)(((size_t)smem_raw + 1023) & ~(size_t)1023);
  I8Tail* st = (I8Tail*)(smem + I8_RING);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = CTAS == 2 ? (int)cluster_ctarank() : 0;
  const int group = blockIdx.x / CTAS, ngroups = gridDim.x / CTAS;
  const int x_stage = a.cols / CTAS * I8_BK, stage_bytes = I8_W_STAGE + x_stage;   // this CTA's part of a stage
  const int n_tiles = (a.n + I8_ROWS * CTAS - 1) / (I8_ROWS * CTAS), m_tiles = (a.m + a.cols - 1) / a.cols;
  const int units = n_tiles * m_tiles, k_blocks = (a.k + I8_BK - 1) / I8_BK;

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

  if (warp == 0) {
    // ===================== TMA producer =====================
    if (lane == 0) {
      unsigned g = 0;
      int s = 0;
      unsigned ph = 0;
      bool ok = true;
      for (int u = group; u < units && ok; u += ngroups) {
        int nt, mt;
        i8_tile(u, n_tiles, m_tiles, a.band, nt, mt);
        const int row_w = nt * (I8_ROWS * CTAS) + rank * I8_ROWS, row_x = mt * a.cols + rank * (a.cols / CTAS);
        for (int kb = 0; kb < k_blocks; ++kb, ++g) {
          if (!mbar_wait(&st->empty[s], ph ^ 1u, abort_flag, a.status, 1)) { ok = false; break; }
          if (rank == 0) mbar_expect_tx(&st->full[s], CTAS * stage_bytes);   // the leader's barrier counts both CTAs
          unsigned char* dst = smem + (size_t)s * stage_bytes;
          if (CTAS == 2) {
            tma_load_2d_pair(dst, &tmW, kb * I8_BK, row_w, &st->full[s]);
            tma_load_2d_pair(dst + I8_W_STAGE, &tmX, kb * I8_BK, row_x, &st->full[s]);
          } else {
            tma_load_2d(dst, &tmW, kb * I8_BK, row_w, &st->full[s]);
            tma_load_2d(dst + I8_W_STAGE, &tmX, kb * I8_BK, row_x, &st->full[s]);
          }
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
          const unsigned long long wdesc = i8_smem_desc(at), xdesc = i8_smem_desc(at + I8_W_STAGE);
#pragma unroll
          for (int kk = 0; kk < I8_BK / 32; ++kk) {               // 32 k an instruction: 32 bytes further on
            const unsigned more = (kb != 0 || kk != 0) ? 1u : 0u;
            if (CTAS == 2) tc_mma_i8_pair(d_tmem, wdesc + kk * 2, xdesc + kk * 2, idesc, more);
            else tc_mma_i8(d_tmem, wdesc + kk * 2, xdesc + kk * 2, idesc, more);
          }
          if (CTAS == 2) tc_commit_pair(&st->empty[s]); else tc_commit(&st->empty[s]);
          if (++s == a.stages) { s = 0; ph ^= 1u; }
        }
        if (ok) { if (CTAS == 2) tc_commit_pair(&st->tmem_full[acc]); else tc_commit(&st->tmem_full[acc]); }
      }
      if (CTAS == 2) tc_commit_pair_local(&st->done); else tc_commit(&st->done);
      mbar_wait_drain(&st->done, 0);
    }
  } else {
    // ===================== epilogue warps: two for each quarter of the lanes =====================
    const int ew = warp - 2, q = warp & 3;
    const int groups = (a.cols + 31) / 32;                        // groups of 32 tokens; the two warps take turns
    float* sa = st->scale[ew];
    T* C = (T*)a.C;
    unsigned it = 0;
    bool ok = true;
    for (int u = group; u < units && ok; u += ngroups, ++it) {
      int nt, mt;
      i8_tile(u, n_tiles, m_tiles, a.band, nt, mt);
      const int j = nt * (I8_ROWS * CTAS) + rank * I8_ROWS + q * 32 + lane;          // this lane's channel
      const bool row_ok = j < a.n;
      const float sb = row_ok ? a.b_scale[j] : 0.f;
      float bias = 0.f;
      if (a.bias && row_ok) bias = a.bias_bf16 ? __bfloat162float(((const __nv_bfloat16*)a.bias)[j]) : ((const float*)a.bias)[j];
      const unsigned acc = it & 1u, aph = (it >> 1) & 1u;
      int got = 0;
      if (lane == 0) got = mbar_wait(&st->tmem_full[acc], aph, abort_flag, a.status, 4) ? 1 : 0;
      got = __shfl_sync(0xffffffffu, got, 0);
      if (!got) { ok = false; break; }
      tc_fence_after();
      const unsigned taddr = tmem_base + ((unsigned)(q * 32) << 16) + acc * 256;
      for (int cg = ew >> 2; cg < groups; cg += 2) {
        const int i0 = mt * a.cols + cg * 32;
        const int cnt = min(min(32, a.cols - cg * 32), a.m - i0);                     // tokens of this group
        if (cnt <= 0) break;
        __syncwarp();
        sa[lane] = lane < cnt ? a.a_scale[i0 + lane] : 0.f;
        float v[32];
        tmem_ld32(taddr + cg * 32, v);
        __syncwarp();
#pragma unroll
        for (int c = 0; c < 32; c += 4) {
          const float4 f = *reinterpret_cast<const float4*>(sa + c);
          v[c] = fmaf((float)__float_as_int(v[c]), f.x * sb, bias);
          v[c + 1] = fmaf((float)__float_as_int(v[c + 1]), f.y * sb, bias);
          v[c + 2] = fmaf((float)__float_as_int(v[c + 2]), f.z * sb, bias);
          v[c + 3] = fmaf((float)__float_as_int(v[c + 3]), f.w * sb, bias);
        }
        if constexpr (sizeof(T) == 4) {
          if (row_ok) {
            T* to = C + (long long)i0 * a.ldc + j;
#pragma unroll
            for (int c = 0; c < 32; ++c)
              if (c < cnt) to[c * a.ldc] = v[c];
          }
        } else {
          // lanes 2l and 2l + 1 hold neighbouring channels: the even one stores both of token c, the odd one of token c + 1
          const bool odd = lane & 1, both = (j | 1) < a.n && a.pairs;
          T* to = C + (long long)(i0 + (odd ? 1 : 0)) * a.ldc + (j & ~1);
#pragma unroll
          for (int c = 0; c < 32; c += 2) {
            const __nv_bfloat162 p = __floats2bfloat162_rn(v[c], v[c + 1]);
            const unsigned mine = *reinterpret_cast<const unsigned*>(&p);
            const unsigned other = __shfl_xor_sync(0xffffffffu, mine, 1);
            if (both) {
              const unsigned w = odd ? __byte_perm(other, mine, 0x7632) : __byte_perm(mine, other, 0x5410);
              if (c + (odd ? 1 : 0) < cnt) *reinterpret_cast<unsigned*>(to + c * a.ldc) = w;
            } else if (row_ok) {
              T* one = C + (long long)(i0 + c) * a.ldc + j;
              if (c < cnt) one[0] = p.x;
              if (c + 1 < cnt) one[a.ldc] = p.y;
            }
          }
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) { if (CTAS == 2) mbar_arrive_leader(&st->tmem_empty[acc]); else mbar_arrive(&st->tmem_empty[acc]); }
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

template <typename T, int CTAS>
cudaError_t i8_launch(const CUtensorMap& tmW, const CUtensorMap& tmX, const I8Args& a, int units, cudaStream_t stream) {
  static std::atomic<int> groups_on[MAX_DEVICES];       // CTA groups that can be resident at once; 0: not configured there yet
  auto kern = k_i8_gemm<T, CTAS>;
  const int dev = current_device();
  int most = groups_on[dev].load(std::memory_order_acquire);
  if (most == 0) {
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, I8_SMEM);
    if (e != cudaSuccess) return e;
  }
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = CTAS;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.blockDim = dim3(I8_THREADS);
  cfg.dynamicSmemBytes = I8_SMEM;
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
  return cudaLaunchKernelEx(&cfg, kern, tmW, tmX, a);
}

constexpr long long I8_BAND_BYTES = 32LL << 20;         // token rows of a band: a quarter of the L2

}  // namespace

cudaError_t i8_gemm(const signed char* A, long long lda, const float* a_scale, const signed char* B, long long ldb,
                    const float* b_scale, const void* bias, bool bias_bf16, int m, int n, int k, void* C, long long ldc,
                    bool out_bf16, int* status, cudaStream_t stream) {
  if (m <= 0 || n <= 0) return cudaSuccess;
  // up to 128 tokens: tiles as wide as the tokens, so that the head is read once and the ring is deep
  const bool pair = m > 128;
  I8Args a = {};
  a.n = n; a.m = m; a.k = k;
  a.cols = pair ? 256 : (m + 15) / 16 * 16;
  const int stage = I8_W_STAGE + a.cols / (pair ? 2 : 1) * I8_BK;
  a.stages = I8_RING / stage < I8_MAX_STAGES ? I8_RING / stage : I8_MAX_STAGES;
  const int rows = I8_ROWS * (pair ? 2 : 1);
  const long long n_tiles = ((long long)n + rows - 1) / rows, m_tiles = ((long long)m + a.cols - 1) / a.cols;
  if (n_tiles * m_tiles > 0x7fffffffLL - (1 << 20)) return cudaErrorInvalidValue;
  long long band = I8_BAND_BYTES / ((long long)a.cols * k);
  band = band < 1 ? 1 : band > m_tiles ? m_tiles : band;
  if (band * n_tiles > 0x7fffffffLL) band = 1;
  a.band = (int)band;
  a.a_scale = a_scale;
  a.b_scale = b_scale;
  a.bias = bias;
  a.bias_bf16 = bias_bf16 ? 1 : 0;
  a.C = C;
  a.ldc = ldc;
  a.pairs = ((size_t)C & 3) == 0 && ldc % 2 == 0;
  a.status = status;
  alignas(64) CUtensorMap tmW, tmX;
  if (!i8_map(&tmW, B, k, n, ldb, I8_ROWS) || !i8_map(&tmX, A, k, m, lda, (unsigned)(a.cols / (pair ? 2 : 1))))
    return cudaErrorInvalidValue;
  const int units = (int)(n_tiles * m_tiles);
  if (pair)
    return out_bf16 ? i8_launch<__nv_bfloat16, 2>(tmW, tmX, a, units, stream) : i8_launch<float, 2>(tmW, tmX, a, units, stream);
  return out_bf16 ? i8_launch<__nv_bfloat16, 1>(tmW, tmX, a, units, stream) : i8_launch<float, 1>(tmW, tmX, a, units, stream);
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
  w.ld = ((long long)p->k + 15) / 16 * 16;
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
                                p->bias_dtype == PCTC_BF16, p->m, p->n, p->k, C, p->ldc, p->out_dtype == PCTC_BF16, device_status,
                                (cudaStream_t)stream_v);
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
  if (i8_quantize(x, x_dtype == PCTC_BF16, p->m, p->k, p->lda, q, w.ld, scales, (int*)ws, stream) != cudaSuccess) return PCTC_ERR_CUDA;
  const cudaError_t e = i8_gemm(q, w.ld, scales, (const signed char*)B, p->ldb, b_scales, bias, p->bias_dtype == PCTC_BF16, p->m, p->n,
                                p->k, C, p->ldc, p->out_dtype == PCTC_BF16, (int*)ws, stream);
  return e == cudaSuccess ? PCTC_OK : e == cudaErrorInvalidValue ? PCTC_ERR_UNSUPPORTED : PCTC_ERR_CUDA;
}

}  // extern "C"
