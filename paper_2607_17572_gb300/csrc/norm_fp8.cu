// RMS norm with the residual's addition and an 8-bit output, its backward pass, and the
// quantisation of a matrix in groups of 128 (include/jagg.h, "8-bit operands").
//
// All three are bound by device memory: each input is read once, held in registers, and each output
// written once.  A thread owns runs of eight consecutive elements (16 bytes of bf16), so 16
// neighbouring lanes hold one group of 128 columns and its largest magnitude is four shuffles.
#include "fp8.cuh"

namespace jagg {
namespace {

using namespace fp8;

constexpr int64_t NORM_MAX_D = 32768;

__device__ __forceinline__ float half_warp_amax(float a) {
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) a = amax(a, __shfl_xor_sync(0xffffffffu, a, o));
  return a;
}

struct NormParams {
  const void* x;
  int64_t ldx;
  const void* residual;
  int64_t ldh;
  const void* weight;
  int w_f32;
  int64_t rows;
  int d;
  float eps;
  void* h_out;
  uint8_t* q;
  int64_t ldq;
  float* scale;
  int64_t lds;
  float* rstd;
};

// The value that h_dtype keeps of v.
template <typename H>
__device__ __forceinline__ float kept(float v) {
  if constexpr (sizeof(H) == 2) return __bfloat162float(__float2bfloat16_rn(v));
  return v;
}

// A row for blockDim.x threads (whole warps), blockDim.y rows to a CTA, C runs of eight elements per
// thread.
template <typename X, typename H, int C>
__global__ void __launch_bounds__(1024) rms_norm_fp8_kernel(const NormParams p) {
  __shared__ float part[32];
  pdl_wait();
  const int64_t row = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
  const bool live = row < p.rows;
  const int warps = blockDim.x >> 5, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  float v[C][8];
  float ss = 0.f;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int col = (c * (int)blockDim.x + (int)threadIdx.x) * 8;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[c][i] = 0.f;
    if (live && col < p.d) {
      load8(static_cast<const X*>(p.x) + row * p.ldx + col, v[c]);
      if (p.residual) {
        float r[8];
        load8(static_cast<const H*>(p.residual) + row * p.ldh + col, r);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[c][i] += r[i];
      }
    }
  }
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int col = (c * (int)blockDim.x + (int)threadIdx.x) * 8;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      v[c][i] = kept<H>(v[c][i]);
      ss = fmaf(v[c][i], v[c][i], ss);
    }
    if (p.h_out && live && col < p.d) store8(static_cast<H*>(p.h_out) + row * p.ldh + col, v[c]);
  }
  ss = warp_sum(ss);
  if (warps > 1) {
    if (lane == 0) part[threadIdx.y * warps + warp] = ss;
    __syncthreads();
    ss = 0.f;
    for (int w = 0; w < warps; ++w) ss += part[threadIdx.y * warps + w];
  }
  const float rstd = 1.f / sqrtf(ss / (float)p.d + p.eps);
  if (p.rstd && live && threadIdx.x == 0) p.rstd[row] = rstd;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int col = (c * (int)blockDim.x + (int)threadIdx.x) * 8;
    const bool in = live && col < p.d;
    float w[8], a = 0.f;
    if (p.weight && in) {
      load8_any(p.weight, p.w_f32, col, w);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i] = 1.f;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      v[c][i] = v[c][i] * rstd * w[i];
      a = amax(a, v[c][i]);
    }
    a = half_warp_amax(in ? a : 0.f);
    const float s = scale_of(a);
    if (in) {
      *reinterpret_cast<uint2*>(p.q + row * p.ldq + col) = pack8(v[c], 1.f / s);
      if ((lane & 15) == 0) p.scale[(int64_t)(col / GROUP) * p.lds + row] = s;
    }
  }
}

// Rows of any width and alignment, element by element: a CTA of eight warps per row, and in it a warp
// takes whole groups of 128 columns (its lanes four columns each, 32 apart): group warp, warp + 8, ..
// G of them are held in registers; a longer row is read again (from the L2) for the second pass.  Codes leave a
// byte at a time: 10000 x 1001 takes 26 to 27 us, against 10 (bf16) to 19 (f32) of the bytes.
constexpr int ANY_WARPS = 8;
template <typename X, typename H, int G>
__global__ void __launch_bounds__(32 * ANY_WARPS) rms_norm_fp8_any_kernel(const NormParams p) {
  __shared__ float part[ANY_WARPS];
  pdl_wait();
  const int64_t row = blockIdx.x;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const X* x = static_cast<const X*>(p.x) + row * p.ldx;
  const H* r = p.residual ? static_cast<const H*>(p.residual) + row * p.ldh : nullptr;
  H* h = p.h_out ? static_cast<H*>(p.h_out) + row * p.ldh : nullptr;
  auto column = [&](int g, int i) { return (warp + g * ANY_WARPS) * GROUP + lane + 32 * i; };
  const int groups = (p.d + GROUP * ANY_WARPS - 1) / (GROUP * ANY_WARPS);  // of a warp
  float v[G][4], ss = 0.f;
#pragma unroll
  for (int g = 0; g < G; ++g)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int c = column(g, i);
      v[g][i] = c < p.d ? ld(x + c) + (r ? ld(r + c) : 0.f) : 0.f;
    }
#pragma unroll
  for (int g = 0; g < G; ++g)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int c = column(g, i);
      v[g][i] = kept<H>(v[g][i]);
      if (h && c < p.d) st(h + c, v[g][i]);
      ss = fmaf(v[g][i], v[g][i], ss);
    }
  for (int g = G; g < groups; ++g)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int c = column(g, i);
      if (c >= p.d) continue;
      const float f = kept<H>(ld(x + c) + (r ? ld(r + c) : 0.f));
      if (h) st(h + c, f);
      ss = fmaf(f, f, ss);
    }
  ss = warp_sum(ss);
  if (lane == 0) part[warp] = ss;
  __syncthreads();
  ss = 0.f;
  for (int w = 0; w < ANY_WARPS; ++w) ss += part[w];
  const float rstd = 1.f / sqrtf(ss / (float)p.d + p.eps);
  if (p.rstd && threadIdx.x == 0) p.rstd[row] = rstd;
  auto put = [&](int g, float (&f)[4]) {
    float a = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int c = column(g, i);
      f[i] = c < p.d ? f[i] * rstd * (p.weight ? load_any(p.weight, p.w_f32, c) : 1.f) : 0.f;
      a = amax(a, f[i]);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) a = amax(a, __shfl_xor_sync(0xffffffffu, a, o));
    const float s = scale_of(a), inv = 1.f / s;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int c = column(g, i);
      if (c < p.d) p.q[row * p.ldq + c] = (uint8_t)pack2(f[i] * inv, 0.f);
    }
    const int grp = warp + g * ANY_WARPS;
    if (lane == 0 && grp * GROUP < p.d) p.scale[(int64_t)grp * p.lds + row] = s;
  };
#pragma unroll
  for (int g = 0; g < G; ++g) put(g, v[g]);
  for (int g = G; g < groups; ++g) {  // a thread reads what it wrote itself, or forms it again
    float f[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int c = column(g, i);
      f[i] = c >= p.d ? 0.f : h ? ld(h + c) : kept<H>(ld(x + c) + (r ? ld(r + c) : 0.f));
    }
    put(g, f);
  }
}

template <typename X, typename H>
int launch_norm(const NormParams& p, bool vec, cudaStream_t s) {
  if (!vec) {
    const dim3 grid((unsigned)p.rows);
    const int groups = ceil_div(p.d, GROUP * ANY_WARPS);
    if (groups == 1)
      JAGG_CUDA_TRY(launch(rms_norm_fp8_any_kernel<X, H, 1>, grid, 32 * ANY_WARPS, 0, s, p));
    else if (groups <= 4)
      JAGG_CUDA_TRY(launch(rms_norm_fp8_any_kernel<X, H, 4>, grid, 32 * ANY_WARPS, 0, s, p));
    else
      JAGG_CUDA_TRY(launch(rms_norm_fp8_any_kernel<X, H, 8>, grid, 32 * ANY_WARPS, 0, s, p));
    JAGG_LAUNCHED();
    return JAGG_OK;
  }
  const int chunks = ceil_div(p.d, 256);  // runs of eight for a warp
  // up to four runs per thread: more rows' loads in flight than with longer runs
  const int warps = ceil_div(chunks, 4), per = ceil_div(chunks, warps);
  const int rows = warps >= 4 ? 1 : 4 / warps;
  const dim3 block(32 * warps, rows), grid((unsigned)((p.rows + rows - 1) / rows));
  switch (per) {
    case 1: JAGG_CUDA_TRY(launch(rms_norm_fp8_kernel<X, H, 1>, grid, block, 0, s, p)); break;
    case 2: JAGG_CUDA_TRY(launch(rms_norm_fp8_kernel<X, H, 2>, grid, block, 0, s, p)); break;
    case 3: JAGG_CUDA_TRY(launch(rms_norm_fp8_kernel<X, H, 3>, grid, block, 0, s, p)); break;
    default: JAGG_CUDA_TRY(launch(rms_norm_fp8_kernel<X, H, 4>, grid, block, 0, s, p)); break;
  }
  JAGG_LAUNCHED();
  return JAGG_OK;
}

// ------------------------------------------------------------------ backward
struct NormBwdParams {
  const void* dy;
  int64_t lddy;
  const void* h;
  int64_t ldh;
  const void* weight;
  int w_f32;
  const float* rstd;
  const void* dh;
  void* dx;
  int64_t ldg;
  int64_t rows;
  int d;
  float* part;  // [gridDim.x][d] sums of dy xhat, or null
};

// Eight consecutive elements as they lie in memory, on their way through registers.
template <typename T>
struct Raw8 {
  uint4 w[sizeof(T) / 2];
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) w[i] = reinterpret_cast<const uint4*>(p)[i];
  }
  __device__ __forceinline__ void values(float (&v)[8]) const {
    const uint32_t u[8] = {w[0].x, w[0].y, w[0].z, w[0].w, w[sizeof(T) / 2 - 1].x, w[sizeof(T) / 2 - 1].y,
                           w[sizeof(T) / 2 - 1].z, w[sizeof(T) / 2 - 1].w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (sizeof(T) == 2) {
        v[2 * i] = __uint_as_float(u[i] << 16);
        v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
      } else {
        v[2 * i] = __uint_as_float(u[2 * i]);
        v[2 * i + 1] = __uint_as_float(u[2 * i + 1]);
      }
    }
  }
};
template <typename Y, typename H, int C>
struct BwdRow {  // a thread's part of one row: dy, h and dh of C runs of eight columns
  Raw8<Y> y[C];
  Raw8<H> h[C], g[C];
  float rstd;
  __device__ __forceinline__ void load(const NormBwdParams& p, int64_t row) {
    rstd = p.rstd[row];
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int col = (c * (int)blockDim.x + (int)threadIdx.x) * 8;
      if (col < p.d) {
        y[c].load(static_cast<const Y*>(p.dy) + row * p.lddy + col);
        h[c].load(static_cast<const H*>(p.h) + row * p.ldh + col);
        if (p.dh) g[c].load(static_cast<const H*>(p.dh) + row * p.ldg + col);
      }
    }
  }
};

// A CTA holds blockDim.y row slots of blockDim.x threads (whole warps, C runs of eight columns per
// thread) and walks the rows in strides; a thread's columns stay the same, so their weight and their
// sums over rows live in registers.  The next row of a slot is on its way while the last one is
// reduced and written.
template <typename Y, typename H, int C>
__global__ void __launch_bounds__(C == 1 ? 640 : 512, 1) rms_norm_bwd_kernel(const NormBwdParams p) {
  __shared__ float part[2][20];
  extern __shared__ float cols[];  // [blockDim.y][d] when a CTA has several slots
  pdl_wait();
  const int warps = blockDim.x >> 5, warp = threadIdx.x >> 5, lane = threadIdx.x & 31, slot = threadIdx.y;
  const float per_d = 1.f / (float)p.d;
  float w[C][8], dw[C][8];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int col = (c * (int)blockDim.x + (int)threadIdx.x) * 8;
#pragma unroll
    for (int i = 0; i < 8; ++i) w[c][i] = 1.f, dw[c][i] = 0.f;
    if (p.weight && col < p.d) load8_any(p.weight, p.w_f32, col, w[c]);
  }
  const int64_t step = (int64_t)gridDim.x * blockDim.y;
  int64_t row = (int64_t)blockIdx.x * blockDim.y + slot;
  BwdRow<Y, H, C> next;
  if (row < p.rows) next.load(p, row);
  int turn = 0;
  for (; row < p.rows; row += step) {
    const BwdRow<Y, H, C> r = next;
    if (row + step < p.rows) next.load(p, row + step);
    float g[C][8], xh[C][8], sum = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if ((c * (int)blockDim.x + (int)threadIdx.x) * 8 < p.d) {
        r.y[c].values(g[c]);
        r.h[c].values(xh[c]);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          xh[c][i] *= r.rstd;
          dw[c][i] = fmaf(g[c][i], xh[c][i], dw[c][i]);
          g[c][i] *= w[c][i];
          sum = fmaf(g[c][i], xh[c][i], sum);
        }
      }
    }
    sum = warp_sum(sum);
    if (warps > 1) {  // the slot's warps meet; a slot's barrier is its own
      float* at = &part[turn][slot * warps];
      if (lane == 0) at[warp] = sum;
      asm volatile("bar.sync %0, %1;" ::"r"(1 + slot), "r"((int)blockDim.x) : "memory");
      sum = warp_sum(lane < warps ? at[lane] : 0.f);
      turn ^= 1;
    }
    const float mean = sum * per_d;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int col = (c * (int)blockDim.x + (int)threadIdx.x) * 8;
      if (col < p.d) {
        float o[8];
        if (p.dh) {
          r.g[c].values(o);
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) o[i] = 0.f;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = fmaf(r.rstd, fmaf(-mean, xh[c][i], g[c][i]), o[i]);
        store8(static_cast<H*>(p.dx) + row * p.ldg + col, o);
      }
    }
  }
  if (!p.part) return;
  float* out = p.part + (int64_t)blockIdx.x * p.d;
  if (blockDim.y > 1) out = cols + (int64_t)slot * p.d;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int col = (c * (int)blockDim.x + (int)threadIdx.x) * 8;
    if (col < p.d) store8(out + col, dw[c]);
  }
  if (blockDim.y > 1) {
    __syncthreads();
    const int t = threadIdx.y * blockDim.x + threadIdx.x, n = blockDim.x * blockDim.y;
    for (int c = t; c < p.d; c += n) {
      float s = 0.f;
      for (int r = 0; r < (int)blockDim.y; ++r) s += cols[(int64_t)r * p.d + c];
      p.part[(int64_t)blockIdx.x * p.d + c] = s;
    }
  }
}

// Rows of any width and alignment, element by element: a CTA of T threads takes a row at a time, a
// thread the columns t, t + T, ..; E of them and their sums over rows are held in registers, the rest
// of a longer row is read again for the second pass and summed in shared memory.  Loads of one element
// and no row ahead: 10000 x 1001 (bf16 dy, f32 h) takes 33 us against 21 of its bytes, 3000 x 5001 in bf16 (one CTA of
// 512 threads per SM) 128 against 18, 4000 x 12288 (bf16 dy, f32 h) 343 against 101.
template <typename Y, typename H, int E, int T>
__global__ void __launch_bounds__(T) rms_norm_bwd_any_kernel(const NormBwdParams p) {
  __shared__ float part[2][T / 32];
  extern __shared__ float cols[];  // sums of the columns from T E on
  pdl_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, t = threadIdx.x;
  float w[E], dw[E];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const int c = t + T * e;
    w[e] = c < p.d && p.weight ? load_any(p.weight, p.w_f32, c) : 1.f;
    dw[e] = 0.f;
  }
  if (p.part)
    for (int c = t + T * E; c < p.d; c += T) cols[c - T * E] = 0.f;  // a thread's columns are its own throughout
  int turn = 0;
  for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
    const Y* dy = static_cast<const Y*>(p.dy) + row * p.lddy;
    const H* h = static_cast<const H*>(p.h) + row * p.ldh;
    const H* dh = p.dh ? static_cast<const H*>(p.dh) + row * p.ldg : nullptr;
    H* dx = static_cast<H*>(p.dx) + row * p.ldg;
    const float rstd = p.rstd[row];
    float g[E], xh[E], o[E], sum = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int c = t + T * e;
      const bool in = c < p.d;
      g[e] = in ? ld(dy + c) : 0.f;
      xh[e] = in ? ld(h + c) : 0.f;
      o[e] = in && dh ? ld(dh + c) : 0.f;
    }
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (t + T * e < p.d) {  // (a column past the row takes no part, whatever rstd is)
        xh[e] *= rstd;
        dw[e] = fmaf(g[e], xh[e], dw[e]);
        g[e] *= w[e];
        sum = fmaf(g[e], xh[e], sum);
      }
    for (int c = t + T * E; c < p.d; c += T) {
      const float y = ld(dy + c), x = ld(h + c) * rstd;
      if (p.part) cols[c - T * E] = fmaf(y, x, cols[c - T * E]);
      sum = fmaf(y * (p.weight ? load_any(p.weight, p.w_f32, c) : 1.f), x, sum);
    }
    sum = warp_sum(sum);
    if (lane == 0) part[turn][warp] = sum;
    __syncthreads();
    sum = 0.f;
    for (int k = 0; k < T / 32; ++k) sum += part[turn][k];
    turn ^= 1;
    const float mean = sum / (float)p.d;
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (t + T * e < p.d) st(dx + t + T * e, fmaf(rstd, g[e] - xh[e] * mean, o[e]));
    for (int c = t + T * E; c < p.d; c += T) {
      const float y = ld(dy + c) * (p.weight ? load_any(p.weight, p.w_f32, c) : 1.f), x = ld(h + c) * rstd;
      st(dx + c, fmaf(rstd, y - x * mean, dh ? ld(dh + c) : 0.f));
    }
  }
  if (!p.part) return;
  float* out = p.part + (int64_t)blockIdx.x * p.d;
#pragma unroll
  for (int e = 0; e < E; ++e)
    if (t + T * e < p.d) out[t + T * e] = dw[e];
  for (int c = t + T * E; c < p.d; c += T) out[c] = cols[c - T * E];
}

// dweight (+)= the column sums of part [n, d], in order: 32 columns x 32 row lanes per CTA, so that a
// column's 152 rows (a CTA per SM) are five loads in flight per thread.
__global__ void __launch_bounds__(1024) dweight_kernel(const float* part, int n, int d, float* dweight, int accumulate) {
  __shared__ float red[32][33];
  pdl_wait();
  const int lane = threadIdx.x & 31, r0 = threadIdx.x >> 5;
  const int c = blockIdx.x * 32 + lane;
  float s = 0.f;
  if (c < d) {
#pragma unroll 8
    for (int r = r0; r < n; r += 32) s += part[(int64_t)r * d + c];
  }
  red[r0][lane] = s;
  __syncthreads();
  s = warp_sum(red[lane][r0]);  // warp r0 joins column r0
  const int out = blockIdx.x * 32 + r0;
  if (lane == 0 && out < d) dweight[out] = accumulate ? dweight[out] + s : s;
}

// Row slots of `warps` warps each: CTAs of about 16 warps, one per SM, as many CTAs as there are rows
// where rows are few.
constexpr int WALK_WARPS = 20;  // of a row, with 96 registers per thread
struct Slots {
  int slots, ctas;
};
Slots row_slots(int64_t rows, int warps) {
  const int most = warps >= 16 ? 1 : 16 / warps < 15 ? 16 / warps : 15;  // a named barrier each
  const int sms = sm_count();
  const int64_t each = (rows + sms - 1) / sms;
  Slots s;
  s.slots = (int)(each < most ? each : most);
  const int64_t ctas = (rows + s.slots - 1) / s.slots;
  s.ctas = (int)(ctas < sms ? ctas : sms);
  return s;
}

// 16 warps of two runs per thread, which spill up to 316 bytes a thread with both types f32, 152 with bf16 dy and
// an f32 h (9217 x 6144 in f32 takes 270 us against 133 of its bytes, 4000 x 7168 mixed 97 against 59); wider rows, aligned
// or not, go element by element.
constexpr int64_t BWD_VEC_MAX_D = 8192;
constexpr int BWD_MAX_CTAS = 608;        // rows of partial sums in the workspace at most (four CTAs per SM)

template <typename Y, typename H>
int launch_norm_bwd(const NormBwdParams& p, bool vec, float* dweight, int accumulate, cudaStream_t s) {
  int ctas;
  if (!vec) {
    ctas = (int)(p.rows < BWD_MAX_CTAS ? p.rows : BWD_MAX_CTAS);
    auto any = [&](auto kernel, OncePerDevice& once, int threads, int each) -> int {
      const int held = threads * each;
      JAGG_CUDA_TRY(allow_smem(once, kernel, (int)NORM_MAX_D * 4));
      JAGG_CUDA_TRY(launch(kernel, ctas, threads, p.part && p.d > held ? (size_t)(p.d - held) * 4 : 0, s, p));
      return JAGG_OK;
    };
    static OncePerDevice once[4];
    if (p.d <= 1024)
      JAGG_TRY(any(rms_norm_bwd_any_kernel<Y, H, 4, 256>, once[0], 256, 4));
    else if (p.d <= 2048)
      JAGG_TRY(any(rms_norm_bwd_any_kernel<Y, H, 4, 512>, once[1], 512, 4));
    else if (p.d <= 4096)
      JAGG_TRY(any(rms_norm_bwd_any_kernel<Y, H, 8, 512>, once[2], 512, 8));
    else
      JAGG_TRY(any(rms_norm_bwd_any_kernel<Y, H, 16, 512>, once[3], 512, 16));
  } else {
    const int chunks = ceil_div(p.d, 256);
    // A run per thread up to 20 warps, else two.  Two also for many bf16 rows where that keeps 14 warps
    // or more busy: half the warps meet for a row (18432 x 4096: 122 us -> 111, 5000 x 1536 19.5 -> 16.9; but
    // 9217 x 5120, 10 warps, 71 -> 90, and 300 x 4096 5.9 -> 6.4).
    const int half = ceil_div(chunks, 2);
    const bool two = chunks > WALK_WARPS ||
                     (sizeof(Y) + sizeof(H) == 4 && chunks % 2 == 0 && half <= 8 && 16 / half * half >= 14 &&
                      p.rows >= 16 * (int64_t)sm_count());
    const int per = two ? 2 : 1, warps = two ? half : chunks;
    const Slots sl = row_slots(p.rows, warps);
    const int slots = sl.slots;
    ctas = sl.ctas < BWD_MAX_CTAS ? sl.ctas : BWD_MAX_CTAS;
    const dim3 block(32 * warps, slots);
    const size_t smem = slots > 1 && p.part ? (size_t)slots * p.d * 4 : 0;
    if (per == 2)
      JAGG_CUDA_TRY(launch(rms_norm_bwd_kernel<Y, H, 2>, ctas, block, smem, s, p));
    else
      JAGG_CUDA_TRY(launch(rms_norm_bwd_kernel<Y, H, 1>, ctas, block, smem, s, p));
  }
  JAGG_LAUNCHED();
  if (p.part) {
    JAGG_CUDA_TRY(launch(dweight_kernel, ceil_div(p.d, 32), 1024, 0, s, (const float*)p.part, ctas, p.d, dweight,
                         accumulate));
    JAGG_LAUNCHED();
  }
  return JAGG_OK;
}

// ------------------------------------------------------------------ quantisation
struct QuantParams {
  const void* x;
  int64_t ldx;
  int64_t rows, cols;
  const float* row_mul;
  const void* col_mul;
  int col_f32;
  jagg_fp8_out row, col, block;
};

// Eight elements of a tile held between the passes over it: as f32, or as they were read (half the
// registers for bf16, so that twice as many CTAs are resident: 4608 x 4096 in bf16, row and column
// groups, 25.2 -> 16.5 us).
template <typename T>
struct Kept8 {
  float v[8];
  __device__ __forceinline__ float at(int i) const { return v[i]; }
  __device__ __forceinline__ void set(int i, float x) { v[i] = x; }
  __device__ __forceinline__ void forget() {}
};
template <>
struct Kept8<bf16> {
  uint32_t w[4];
  __device__ __forceinline__ float at(int i) const {
    return __uint_as_float(i & 1 ? w[i >> 1] & 0xffff0000u : w[i >> 1] << 16);
  }
  // The compiler forgets what it has unpacked (it would keep both forms in registers).
  __device__ __forceinline__ void forget() {
    asm volatile("" : "+r"(w[0]), "+r"(w[1]), "+r"(w[2]), "+r"(w[3]));
  }
  __device__ __forceinline__ void set(int i, float x) {
    const uint32_t b = __bfloat16_as_ushort(__float2bfloat16_rn(x));  // exact: x is a bf16 value
    w[i >> 1] = i & 1 ? (w[i >> 1] & 0xffffu) | (b << 16) : (w[i >> 1] & 0xffff0000u) | b;
  }
};

// A 128 x 128 tile per CTA of 256 threads: thread (c, r) = (t & 15, t >> 4) holds columns 8 c .. + 7
// (element by element, without VEC: c, c + 16, ..) of the rows r, r + 16, .., r + 112, so a row group is one
// half warp's and a column group is 16 threads' eight rows each, joined in shared memory.  K: what a thread
// keeps its elements as (bf16 only where no multipliers change them).
//
// Measured, in bf16 / f32: 4608 x 4096 in column groups 11.4 / 16.7 us, with both multipliers 26.8 / 21.0 (f32 kept: two
// CTAs per SM instead of four); 10000 x 1001 in row and column groups 23.4 / 19.0, against 5.9 / 8.9 of the bytes, with
// single-byte stores and 36 bytes a thread spilt in bf16.
template <typename X, typename K, bool VEC>
__global__ void __launch_bounds__(256, sizeof(K) == 2 ? (VEC ? 4 : 3) : 2) quantize_kernel(const QuantParams p) {
  __shared__ float peak[16][GROUP];
  __shared__ float whole[8];
  pdl_wait();
  const int c = threadIdx.x & 15, r = threadIdx.x >> 4;
  constexpr int STEP = VEC ? 1 : 16;  // between a thread's columns: element by element, 16 lanes take neighbours
  const int at0 = VEC ? 8 * c : c;    // the thread's first column in the tile
  const int64_t row0 = (int64_t)blockIdx.y * GROUP, col0 = (int64_t)blockIdx.x * GROUP + at0;
  const int64_t left = p.cols - col0;
  const int live = left <= 0 ? 0 : left >= 8 * STEP ? 8 : (int)((left + STEP - 1) / STEP);  // columns of this thread
  Kept8<K> v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int64_t row = row0 + r + 16 * i;
    const X* x = static_cast<const X*>(p.x) + row * p.ldx + col0;
    if constexpr (VEC && sizeof(X) == 2 && sizeof(K) == 2) {
      uint4 w = make_uint4(0, 0, 0, 0);
      if (row < p.rows && live) w = *reinterpret_cast<const uint4*>(x);
      v[i].w[0] = w.x; v[i].w[1] = w.y; v[i].w[2] = w.z; v[i].w[3] = w.w;
    } else {
      float f[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) f[j] = 0.f;
      if (row < p.rows) {
        if (VEC) {
          if (live) load8(x, f);
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (j < live) f[j] = ld(x + j * STEP);
        }
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i].set(j, f[j]);
    }
  }
  if constexpr (sizeof(K) == 4) {
    if (p.row_mul) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int64_t row = row0 + r + 16 * i;
        const float m = row < p.rows ? p.row_mul[row] : 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (row < p.rows && j < live) v[i].v[j] *= m;
      }
    }
    if (p.col_mul) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (j >= live) continue;
        const float m = load_any(p.col_mul, p.col_f32, col0 + j * STEP);
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (row0 + r + 16 * i < p.rows) v[i].v[j] *= m;
      }
    }
  }
  auto put = [&](uint8_t* q, int64_t ldq, int64_t row, const float (&o)[8], float inv) {
    const uint2 w = pack8(o, inv);
    uint8_t* at = q + row * ldq + col0;
    if (VEC) {
      *reinterpret_cast<uint2*>(at) = w;
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (j < live) at[j * STEP] = (uint8_t)((j < 4 ? w.x : w.y) >> (8 * (j & 3)));
    }
  };
  if (p.row.q) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int64_t row = row0 + r + 16 * i;
      float o[8], a = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        o[j] = v[i].at(j);
        a = amax(a, o[j]);
      }
      v[i].forget();
      const float s = scale_of(half_warp_amax(a));
      if (row < p.rows && live) {
        put(p.row.q, p.row.ldq, row, o, 1.f / s);
        if (c == 0) p.row.scale[(int64_t)blockIdx.x * p.row.lds + row] = s;
      }
    }
  }
  if (p.col.q) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float a = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) a = amax(a, v[i].at(j));
      peak[r][at0 + j * STEP] = a;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i].forget();
    __syncthreads();
    if (threadIdx.x < GROUP) {
      float a = 0.f;
#pragma unroll
      for (int k = 0; k < 16; ++k) a = amax(a, peak[k][threadIdx.x]);
      const float s = scale_of(a);
      const int64_t col = (int64_t)blockIdx.x * GROUP + threadIdx.x;
      if (col < p.cols) p.col.scale[(int64_t)blockIdx.y * p.col.lds + col] = s;
      peak[0][threadIdx.x] = 1.f / s;  // row 0 of this column has been read by this thread alone
    }
    __syncthreads();
    float inv[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) inv[j] = peak[0][at0 + j * STEP];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int64_t row = row0 + r + 16 * i;
      if (row < p.rows && live) {
        float o[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) o[j] = v[i].at(j) * inv[j];
        put(p.col.q, p.col.ldq, row, o, 1.f);
      }
      v[i].forget();
    }
  }
  if (p.block.q) {
    float a = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) a = amax(a, v[i].at(j));
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i].forget();
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) a = amax(a, __shfl_xor_sync(0xffffffffu, a, o));
    if ((threadIdx.x & 31) == 0) whole[threadIdx.x >> 5] = a;
    __syncthreads();
    a = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) a = amax(a, whole[k]);
    const float s = scale_of(a), inv = 1.f / s;
    if (threadIdx.x == 0) p.block.scale[(int64_t)blockIdx.y * p.block.lds + blockIdx.x] = s;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int64_t row = row0 + r + 16 * i;
      if (row < p.rows && live) {
        float o[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) o[j] = v[i].at(j);
        put(p.block.q, p.block.ldq, row, o, inv);
      }
    }
  }
}

template <typename X, typename K>
int launch_quant(const QuantParams& p, bool vec, dim3 grid, cudaStream_t s) {
  if (vec)
    JAGG_CUDA_TRY(launch(quantize_kernel<X, K, true>, grid, 256, 0, s, p));
  else
    JAGG_CUDA_TRY(launch(quantize_kernel<X, K, false>, grid, 256, 0, s, p));
  JAGG_LAUNCHED();
  return JAGG_OK;
}

// `step`: what the pitch of the scales is a multiple of (1: blocks, which need no alignment either).
int check_out(const char* who, const char* form, const jagg_fp8_out* o, int64_t cols, int64_t lds, int step) {
  JAGG_CHECK_ARG(o->scale, "%s: %s codes without scales", who, form);
  JAGG_CHECK_ARG(aligned(o->q, 16) && o->ldq % 16 == 0 && o->ldq >= cols,
                 "%s: %s codes need a 16-byte aligned base and a row pitch that is a multiple of 16 and >= %lld (got %lld)",
                 who, form, (long long)cols, (long long)o->ldq);
  JAGG_CHECK_ARG(aligned(o->scale, 4 * step) && o->lds % step == 0 && o->lds >= lds,
                 "%s: %s scales need a %d-byte aligned base and a pitch that is a multiple of %d and >= %lld (got %lld)", who,
                 form, 4 * step, step, (long long)lds, (long long)o->lds);
  return JAGG_OK;
}

}  // namespace
}  // namespace jagg

using namespace jagg;

extern "C" int jagg_rms_norm_fp8(const void* x, int x_dtype, int64_t ldx, const void* residual, int h_dtype,
                                 int64_t ldh, const void* weight, int w_dtype, int64_t rows, int64_t d, float eps,
                                 void* h_out, uint8_t* q, int64_t ldq, float* scale, int64_t lds, float* rstd,
                                 cudaStream_t stream) {
  const char* who = "jagg_rms_norm_fp8";
  JAGG_CHECK_ARG(is_dtype(x_dtype) && is_dtype(h_dtype) && is_dtype(w_dtype), "%s: bad dtype", who);
  JAGG_CHECK_ARG(rows >= 0 && rows <= INT32_MAX, "%s: rows=%lld outside [0, 2^31)", who, (long long)rows);
  JAGG_CHECK_ARG(d >= 1, "%s: d=%lld must be positive", who, (long long)d);
  if (d > NORM_MAX_D) {
    set_last_error("%s: d=%lld, rows of at most %lld elements are implemented", who, (long long)d, (long long)NORM_MAX_D);
    return JAGG_ERR_UNSUPPORTED;
  }
  if (rows == 0) return JAGG_OK;
  JAGG_CHECK_ARG(x && q && scale, "%s: null pointer", who);
  JAGG_CHECK_ARG(ldx >= d && (ldh >= d || (!residual && !h_out)), "%s: a row pitch is below d=%lld", who, (long long)d);
  const int xs = size_of(x_dtype), hs = size_of(h_dtype), ws = size_of(w_dtype);
  JAGG_CHECK_ARG(aligned(x, xs) && aligned(residual, hs) && aligned(h_out, hs) && aligned(weight, ws) && aligned(rstd, 4),
                 "%s: a pointer is not aligned to its elements", who);
  JAGG_CHECK_ARG(eps >= 0.f, "%s: eps must not be negative", who);
  const jagg_fp8_out o{q, ldq, scale, lds};
  JAGG_TRY(check_out(who, "row", &o, d, rows, 4));
  const NormParams p{x, ldx, residual, ldh, weight, w_dtype == JAGG_DTYPE_F32, rows, (int)d, eps, h_out, q, ldq,
                     scale, lds, rstd};
  const bool vec = d % 8 == 0 && aligned(x, 16) && ldx * xs % 16 == 0 && aligned(weight, 16) &&
                   ((!residual && !h_out) || (aligned(residual, 16) && aligned(h_out, 16) && ldh * hs % 16 == 0));
  const bool xf = x_dtype == JAGG_DTYPE_F32, hf = h_dtype == JAGG_DTYPE_F32;
  const int tok = prof_start(stream);
  if (xf)
    JAGG_TRY((hf ? launch_norm<float, float>(p, vec, stream) : launch_norm<float, bf16>(p, vec, stream)));
  else
    JAGG_TRY((hf ? launch_norm<bf16, float>(p, vec, stream) : launch_norm<bf16, bf16>(p, vec, stream)));
  prof_stop(tok, stream, PROF_NORM_FP8, 0.0, (double)rows * d * (xs + (residual ? hs : 0) + (h_out ? hs : 0) + 1));
  return JAGG_OK;
}

extern "C" int64_t jagg_rms_norm_bwd_workspace_bytes(int64_t rows, int64_t d) {
  if (rows <= 0 || d <= 0) return 0;
  return (rows < BWD_MAX_CTAS ? rows : BWD_MAX_CTAS) * d * 4;
}

extern "C" int jagg_rms_norm_bwd(const void* dy, int dy_dtype, int64_t lddy, const void* h, int h_dtype, int64_t ldh,
                                 const void* weight, int w_dtype, const float* rstd, const void* dh, void* dx,
                                 int64_t ldg, int64_t rows, int64_t d, float* dweight, int accumulate, void* ws,
                                 size_t ws_bytes, cudaStream_t stream) {
  const char* who = "jagg_rms_norm_bwd";
  JAGG_CHECK_ARG(is_dtype(dy_dtype) && is_dtype(h_dtype) && is_dtype(w_dtype), "%s: bad dtype", who);
  JAGG_CHECK_ARG(rows >= 0 && rows <= INT32_MAX, "%s: rows=%lld outside [0, 2^31)", who, (long long)rows);
  JAGG_CHECK_ARG(d >= 1, "%s: d=%lld must be positive", who, (long long)d);
  if (d > NORM_MAX_D) {
    set_last_error("%s: d=%lld, rows of at most %lld elements are implemented", who, (long long)d, (long long)NORM_MAX_D);
    return JAGG_ERR_UNSUPPORTED;
  }
  JAGG_CHECK_ARG(aligned(dweight, 4), "%s: dweight is not aligned to its elements", who);
  if (rows == 0) {
    if (dweight && !accumulate) JAGG_CUDA_TRY(cudaMemsetAsync(dweight, 0, d * 4, stream));
    return JAGG_OK;
  }
  JAGG_CHECK_ARG(dy && h && rstd && dx, "%s: null pointer", who);
  JAGG_CHECK_ARG(lddy >= d && ldh >= d && ldg >= d, "%s: a row pitch is below d=%lld", who, (long long)d);
  const int ys = size_of(dy_dtype), hs = size_of(h_dtype), wb = size_of(w_dtype);
  JAGG_CHECK_ARG(aligned(dy, ys) && aligned(h, hs) && aligned(dh, hs) && aligned(dx, hs) && aligned(weight, wb) &&
                     aligned(rstd, 4),
                 "%s: a pointer is not aligned to its elements", who);
  if (dweight) {
    const int64_t need = jagg_rms_norm_bwd_workspace_bytes(rows, d);
    if (!ws || (int64_t)ws_bytes < need) {
      set_last_error("%s: workspace %zu < %lld bytes", who, ws ? ws_bytes : (size_t)0, (long long)need);
      return JAGG_ERR_WORKSPACE;
    }
    JAGG_CHECK_ARG(aligned(ws, 16), "%s: workspace not 16-byte aligned", who);
  }
  const NormBwdParams p{dy, lddy, h, ldh, weight, w_dtype == JAGG_DTYPE_F32, rstd, dh, dx, ldg, rows, (int)d,
                        dweight ? static_cast<float*>(ws) : nullptr};
  const bool vec = d % 8 == 0 && d <= BWD_VEC_MAX_D && aligned(dy, 16) && lddy * ys % 16 == 0 && aligned(h, 16) && ldh * hs % 16 == 0 &&
                   aligned(dh, 16) && aligned(dx, 16) && ldg * hs % 16 == 0 && aligned(weight, 16);
  const bool yf = dy_dtype == JAGG_DTYPE_F32, hf = h_dtype == JAGG_DTYPE_F32;
  const int tok = prof_start(stream);
  if (yf)
    JAGG_TRY((hf ? launch_norm_bwd<float, float>(p, vec, dweight, accumulate, stream)
                 : launch_norm_bwd<float, bf16>(p, vec, dweight, accumulate, stream)));
  else
    JAGG_TRY((hf ? launch_norm_bwd<bf16, float>(p, vec, dweight, accumulate, stream)
                 : launch_norm_bwd<bf16, bf16>(p, vec, dweight, accumulate, stream)));
  prof_stop(tok, stream, PROF_NORM_BWD, 0.0, (double)rows * d * (ys + (dh ? 3 : 2) * hs));
  return JAGG_OK;
}

extern "C" int jagg_quantize_fp8(const void* x, int x_dtype, int64_t ldx, int64_t rows, int64_t cols,
                                 const float* row_mul, const void* col_mul, int col_mul_dtype,
                                 const jagg_fp8_out* by_row, const jagg_fp8_out* by_col, const jagg_fp8_out* by_block,
                                 cudaStream_t stream) {
  const char* who = "jagg_quantize_fp8";
  JAGG_CHECK_ARG(is_dtype(x_dtype) && is_dtype(col_mul_dtype), "%s: bad dtype", who);
  JAGG_CHECK_ARG(rows >= 0 && rows <= 65535ll * GROUP, "%s: rows=%lld outside [0, %lld]", who, (long long)rows,
                 65535ll * GROUP);
  JAGG_CHECK_ARG(cols >= 0 && cols <= INT32_MAX, "%s: cols=%lld outside [0, 2^31)", who, (long long)cols);
  QuantParams p{x, ldx, rows, cols, row_mul, col_mul, col_mul_dtype == JAGG_DTYPE_F32, {}, {}, {}};
  const int64_t gr = (rows + GROUP - 1) / GROUP, gc = (cols + GROUP - 1) / GROUP;
  if (by_row && by_row->q) p.row = *by_row;
  if (by_col && by_col->q) p.col = *by_col;
  if (by_block && by_block->q) p.block = *by_block;
  JAGG_CHECK_ARG(p.row.q || p.col.q || p.block.q || rows == 0 || cols == 0, "%s: no form asked for", who);
  if (rows == 0 || cols == 0) return JAGG_OK;
  if (p.row.q) JAGG_TRY(check_out(who, "row", &p.row, cols, rows, 4));
  if (p.col.q) JAGG_TRY(check_out(who, "column", &p.col, cols, cols, 4));
  if (p.block.q) JAGG_TRY(check_out(who, "block", &p.block, cols, gc, 1));
  JAGG_CHECK_ARG(x && ldx >= cols, "%s: null input or row pitch below cols=%lld", who, (long long)cols);
  const int xs = size_of(x_dtype);
  JAGG_CHECK_ARG(aligned(x, xs) && aligned(row_mul, 4) && aligned(col_mul, size_of(col_mul_dtype)),
                 "%s: a pointer is not aligned to its elements", who);
  const bool vec = cols % 8 == 0 && aligned(x, 16) && ldx * xs % 16 == 0;
  const dim3 grid((unsigned)gc, (unsigned)gr);
  const int tok = prof_start(stream);
  if (x_dtype == JAGG_DTYPE_F32)
    JAGG_TRY((launch_quant<float, float>(p, vec, grid, stream)));
  else if (row_mul || col_mul)
    JAGG_TRY((launch_quant<bf16, float>(p, vec, grid, stream)));
  else
    JAGG_TRY((launch_quant<bf16, bf16>(p, vec, grid, stream)));
  prof_stop(tok, stream, PROF_QUANT_FP8, 0.0,
            (double)rows * cols * (xs + (p.row.q != nullptr) + (p.col.q != nullptr) + (p.block.q != nullptr)));
  return JAGG_OK;
}
