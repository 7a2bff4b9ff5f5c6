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

// Named barriers between the warp that watches the accumulators, which arrives, and the epilogue warps of some
// columns, which wait.  A kernel with n accumulators goes round n + 2 sets of them: when the watcher
// has seen accumulator k - 1 complete, all have passed barrier k - n - 1, so that neither its arrival at
// barrier k nor the next meets a phase of the same set that is still open.  When the wait for accumulator
// k runs out it arrives all the same, and from barrier k + 1 on it waits at the barriers too, which
// keeps them all in step; no warp waits for anything else any more, so that all come to the end.  (Instead,
// letting the epilogue warps read at every k-block whether to go on cost 10 %, a vote of the watcher
// before it arrives 3 %, sets shared by two slices 4 %.)
__device__ __forceinline__ void named_sync(int id, int threads) {
  asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory");
}
__device__ __forceinline__ void named_arrive(int id, int threads) {
  asm volatile("bar.arrive %0, %1;" ::"r"(id), "r"(threads) : "memory");
}

// (x, y) += (a, b) f, as one paired instruction.
__device__ __forceinline__ void add2(float& x, float& y, uint32_t a, uint32_t b, float2 f) {
  asm volatile(
      "{\n\t.reg .b64 d, c, q;\n\t"
      "mov.b64 d, {%2, %3};\n\tmov.b64 q, {%4, %5};\n\tmov.b64 c, {%0, %1};\n\t"
      "fma.rn.f32x2 c, d, q, c;\n\tmov.b64 {%0, %1}, c;\n\t}"
      : "+f"(x), "+f"(y)
      : "r"(a), "r"(b), "f"(f.x), "f"(f.y));
}

// acc[j] += s d[j] (q[j]) over CW columns of an accumulator, from tensor-memory address `t`: the inner
// sum of one group times its two scales.  s: the row's scale (times the columns' where they share one);
// q: address of the columns' scales in shared memory when QVEC.
//
// `read()` is called by the warp once all of its columns have been read, before the last are added: the
// accumulator goes back to the tensor core that much earlier.
template <int CW, bool QVEC, int STEP, class Read>
__device__ __forceinline__ void scaled_add(float (&acc)[CW], uint32_t t, float s, uint32_t q, Read read) {
#pragma unroll
  for (int c = 0; c < CW; c += STEP) {
    uint32_t r[STEP];
    if constexpr (STEP == 16)
      ptx::tmem_ld_32x32b_x16(t + c, r);
    else
      ptx::tmem_ld_32x32b_x32(t + c, r);
    ptx::tmem_ld_wait();
    if (c + STEP >= CW) {
      ptx::tc_fence_before();
      __syncwarp();
      read();
    }
#pragma unroll
    for (int j = 0; j < STEP; j += 4) {
      float2 f = make_float2(s, s), g = f;
      if constexpr (QVEC) {
        const float4 v = ptx::ld_shared_v4(q + (c + j) * 4);
        f = ptx::mul2(make_float2(v.x, v.y), f);
        g = ptx::mul2(make_float2(v.z, v.w), g);
      }
      add2(acc[c + j], acc[c + j + 1], r[j], r[j + 1], f);
      add2(acc[c + j + 2], acc[c + j + 3], r[j + 2], r[j + 3], g);
    }
  }
}

}  // namespace fp8
}  // namespace jagg
