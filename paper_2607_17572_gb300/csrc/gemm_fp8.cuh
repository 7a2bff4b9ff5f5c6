// Products of 8-bit operands with a scale for each group of 128 along K (interface of the two
// kernels, and the device code that they share).
#pragma once

#include "fp8.cuh"
#include "ptx.cuh"
#include "tmap.cuh"

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

// How a product is computed: by CTA pairs in tiles of `pair` columns (gemm_fp8_pair.cu; 0: not), or by
// one CTA per tile or a cluster of `splits` that splits K (gemm_fp8.cu), the accumulator's columns being
// 128 of B, or with `swap` `nt` rows of A.
struct Fp8Plan {
  int pair, nt, splits;
  bool swap;
};
int gemm_fp8(const GemmFp8Args& g, cudaStream_t s);
int gemm_fp8_as(const GemmFp8Args& g, const Fp8Plan& p, cudaStream_t s);
int gemm_fp8_pair(const GemmFp8Args& g, int bn, cudaStream_t s);

// Tensor map of a K-major operand (boxes of `box_rows` rows x 128 codes) or an MN-major one (128 rows of K x
// 128 codes).
int fp8_operand_map(CUtensorMap* m, const Fp8Operand& o, int64_t rows, int64_t K, int box_rows);
// Tensor map of an operand's vector scales [groups of K, rows]: boxes of `box_rows` values of each of
// `box_groups` groups.
int fp8_scale_map(CUtensorMap* m, const Fp8Operand& o, int64_t rows, int64_t K, int box_rows, int box_groups);

namespace fp8 {

constexpr int SCALE_KB = 8;  // k-blocks whose vector scales arrive in one load

__device__ __forceinline__ void named_sync(int id, int threads) {
  asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory");
}
__device__ __forceinline__ void named_arrive(int id, int threads) {
  asm volatile("bar.arrive %0, %1;" ::"r"(id), "r"(threads) : "memory");
}

// acc[j] += s d[j] (q[j]) over CW columns of an accumulator, from tensor-memory address `t`: the inner
// sum of one group times its two scales.  s: the row's scale (times the columns' where they share one);
// q: address of the columns' scales in shared memory when QVEC.
//
// One f32 instruction per element: the paired form takes half as many, and as many moves again to
// form its register pairs from the loaded words.
template <int CW, bool QVEC, int STEP>
__device__ __forceinline__ void scaled_add(float (&acc)[CW], uint32_t t, float s, uint32_t q) {
#pragma unroll
  for (int c = 0; c < CW; c += STEP) {
    uint32_t r[STEP];
    if constexpr (STEP == 8)
      ptx::tmem_ld_32x32b_x8(t + c, r);
    else if constexpr (STEP == 16)
      ptx::tmem_ld_32x32b_x16(t + c, r);
    else
      ptx::tmem_ld_32x32b_x32(t + c, r);
    ptx::tmem_ld_wait();
#pragma unroll
    for (int j = 0; j < STEP; j += 4) {
      float4 f = make_float4(s, s, s, s);
      if constexpr (QVEC) {
        f = ptx::ld_shared_v4(q + (c + j) * 4);
        f.x *= s; f.y *= s; f.z *= s; f.w *= s;
      }
      acc[c + j] = fmaf(__uint_as_float(r[j]), f.x, acc[c + j]);
      acc[c + j + 1] = fmaf(__uint_as_float(r[j + 1]), f.y, acc[c + j + 1]);
      acc[c + j + 2] = fmaf(__uint_as_float(r[j + 2]), f.z, acc[c + j + 2]);
      acc[c + j + 3] = fmaf(__uint_as_float(r[j + 3]), f.w, acc[c + j + 3]);
    }
  }
}

}  // namespace fp8
}  // namespace jagg
