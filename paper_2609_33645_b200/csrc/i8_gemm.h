// The head in 8-bit integers, as the recognition path calls it (host-side launch wrappers).
#pragma once

#include <cuda_runtime.h>

namespace pctc {

// C[i,j] = sum_k A[i,k] B[j,k] * a_scale[i] * b_scale[j] + bias[j]; A [m, k] and B [n, k] 16-byte aligned, pitches multiples
// of 16.  status: device word that receives a non-zero code if a bounded wait gives up, or null.  behind: the call directly
// before this one on the stream is the i8_quantize that makes A and a_scale; this one's launch is then set up meanwhile.
// x: states that the product quantizes itself (i8_own_tokens; A and a_scale are then not looked at, *status is zeroed), or null.
cudaError_t i8_gemm(const signed char* A, long long lda, const float* a_scale, const signed char* B, long long ldb,
                    const float* b_scale, const void* bias, bool bias_bf16, int m, int n, int k, void* C, long long ldc,
                    bool out_bf16, int* status, bool behind, cudaStream_t stream, const void* x = nullptr,
                    long long ld_x = 0, bool x_bf16 = false);
bool i8_own_tokens(const void* x, long long ld_x, bool bf16, int m, int k);

// q[r,:] = round(x[r,:] * 127 / max|x[r]|), scales[r] = max|x[r]| / 127; zeroes *clear (null: nothing).
cudaError_t i8_quantize(const void* x, bool bf16, long long rows, long long cols, long long ld_x, signed char* q, long long ld_q,
                        float* scales, int* clear, cudaStream_t stream);

}  // namespace pctc
