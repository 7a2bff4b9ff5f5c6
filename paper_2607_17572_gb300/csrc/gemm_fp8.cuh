// Products of 8-bit operands with a scale for each group of 128 along K (host-side interface).
#pragma once

#include "common.cuh"

namespace jagg {

// C[m, n] (+)= sum_g sa[g, m] sb[g, n] sum_{k in g} A[m, k] B[n, k] (+ bias[n]).  An operand is K-major
// (rows of K) or MN-major (rows of M or N, `mn`); its scales are a vector per group (`ld` floats
// apart) or one value per 128 x 128 block: value (r / 128, g) at scale[r / 128 * row_step + g * ld].
struct Fp8Operand {
  const uint8_t* q = nullptr;
  int64_t ldq = 0;
  const float* scale = nullptr;
  int64_t ld = 0;        // floats between groups along K
  int64_t row_step = 0;  // blocks: floats between blocks of rows; unused for vectors
  bool mn = false, block = false;
};
struct GemmFp8Args {
  int64_t M = 0, N = 0, K = 0;
  Fp8Operand a, b;
  void* C = nullptr;
  int64_t ldc = 0;
  int c_dtype = JAGG_DTYPE_F32;
  const void* bias = nullptr;
  int bias_dtype = JAGG_DTYPE_F32;
  bool accumulate = false;
};

int gemm_fp8(const GemmFp8Args& g, cudaStream_t s);

}  // namespace jagg
