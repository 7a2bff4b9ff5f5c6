// Products of 8-bit operands with a scale for each group of 128 along K (include/jagg.h,
// jagg_gemm_fp8): the kernel of one CTA per tile, the choice of kernel, and the entry point.
//
//   C[m, n] = sum_g sa[g, m] sb[g, n] sum_{k in g} A[m, k] B[n, k]
//
// The inner sums run on the tensor cores (tcgen05.mma.kind::f8f6f4, f32 accumulators in tensor
// memory); a k-block is one group, so each accumulator is one inner sum.  The epilogue warps read it
// back, multiply by the two scales and add to f32 registers while the tensor core works on the next
// groups in the other accumulators.
//
// One CTA holds a tile of 128 rows of one operand ("P", the rows of the accumulator) and up to 128
// of the other ("Q", its columns).  With few rows of A the weight is P and the tokens are Q, so that the
// tensor core's 128 rows are all in use and a token tile is as narrow as 16.  A cluster of up to 8
// CTAs splits K: each sums its k-blocks, the partial tiles meet in shared memory and every CTA
// joins and stores its part of the tile, in the order of the ranks (no atomics, no workspace).
//
// Vector scales arrive by TMA beside the operands, eight k-blocks at a time; block scales are read 32
// k-blocks at a time, one per lane.
//
// Roles: warp 0 TMA producer, warp 1 MMA issuer, warp 2 watches the accumulators' barriers for the
// epilogue warps (which would slow each other down by polling), warps 4 and up the epilogue
// (tensor-memory lanes 32 (warp % 4) .. + 31, 64 or fewer columns); all warps join and store.
#include <cmath>

#include "../../include/jagg_testing.h"
#include "gemm_fp8.cuh"

namespace jagg {

int unit_status_gemm_fp8(unsigned* v, int clear) { return read_unit_status(v, clear); }

namespace {

using fp8::GROUP;
using fp8::SCALE_KB;

constexpr int F_ROWS = 128;                  // P rows of a tile
constexpr int F_TILE = F_ROWS * GROUP;       // bytes of a whole operand tile of a k-block
constexpr int F_ACCS = 4;                    // accumulators in tensor memory
constexpr int F_BARS = F_ACCS + 2;           // sets of named barriers (fp8::named_arrive)
constexpr int F_MAX_STAGES = 10;
constexpr int F_MAX_SPLITS = 8;              // portable cluster size
constexpr int F_SMEM = 200 * 1024;

template <int NT, bool Q_MN>
struct FCfg {
  // MN-major Q rows arrive in whole 128-byte rows (the width of the swizzle), whatever part is used
  static constexpr int Q_BYTES = Q_MN ? F_TILE : NT * GROUP;
  static constexpr int STAGE = F_TILE + Q_BYTES;
  static constexpr int FIT = F_SMEM / STAGE;
  static constexpr int STAGES = FIT < F_MAX_STAGES ? FIT : F_MAX_STAGES;
  static constexpr int SMEM = STAGES * STAGE + 1024;
  static constexpr int COLS = F_ACCS * NT < 32 ? 32 : F_ACCS * NT;  // tensor-memory columns
  static constexpr int CW = NT < 64 ? NT : NT / 2;                  // columns of an epilogue warp
  static constexpr int EW = 4 * (NT / CW);                          // epilogue warps
  static constexpr int THREADS = 128 + 32 * EW;
};

struct FParams {
  int P, Q;                // rows of the two operands
  int tiles_p, k_blocks, splits;
  const float* block;      // block scales of P or Q: value (r / 128, g) at r / 128 * block_step + g * block_ld
  int64_t block_ld, block_step;
  int p_block, p_mn;
  void* C;
  int64_t ldc;
  int c_f32, accumulate, c_vec;
  const void* bias;
  int bias_f32;
};
struct FMaps {
  CUtensorMap p, q, ps, qs;  // operands, their vector scales
};

// SWAP: P is B and Q is A (the tile is C's transpose).  QVEC: Q has a scale per row, else per block.
template <int NT, bool Q_MN, bool SWAP, bool QVEC>
__global__ void __launch_bounds__(FCfg<NT, Q_MN>::THREADS, 1)
    gemm_fp8_kernel(const __grid_constant__ FMaps maps, const FParams p) {
  using Cfg = FCfg<NT, Q_MN>;
  constexpr int CW = Cfg::CW;
  extern __shared__ uint8_t smem_f8[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_f8) + 1023) & ~uintptr_t(1023));
  __shared__ uint64_t full[F_MAX_STAGES], empty[F_MAX_STAGES], tfull[F_ACCS], tempty[F_ACCS], drainbar;
  __shared__ uint64_t sfull[2], sempty[2];
  __shared__ uint32_t tmem_slot;
  __shared__ volatile int abort_flag;
  __shared__ __align__(128) float pscale[2][SCALE_KB][F_ROWS], qscale[2][SCALE_KB][NT];

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = p.splits > 1 ? (int)ptx::cluster_ctarank() : 0;
  const int tile = blockIdx.x / p.splits;
  const int p0 = (tile % p.tiles_p) * F_ROWS, q0 = (tile / p.tiles_p) * NT;
  const int kb0 = (int)((long long)p.k_blocks * rank / p.splits);
  const int kb1 = (int)((long long)p.k_blocks * (rank + 1) / p.splits);

  if (threadIdx.x == 0) {
    abort_flag = 0;
    for (int s = 0; s < Cfg::STAGES; ++s) {
      ptx::mbar_init(&full[s], 1);
      ptx::mbar_init(&empty[s], 1);
    }
    for (int a = 0; a < F_ACCS; ++a) {
      ptx::mbar_init(&tfull[a], 1);
      ptx::mbar_init(&tempty[a], Cfg::EW);
    }
    for (int i = 0; i < 2; ++i) {
      ptx::mbar_init(&sfull[i], 1);
      ptx::mbar_init(&sempty[i], Cfg::EW);
    }
    ptx::mbar_init(&drainbar, 1);
    ptx::fence_mbar_init();
    if (p.k_blocks > 0) {
      ptx::prefetch_tmap(&maps.p);
      ptx::prefetch_tmap(&maps.q);
      if (!p.p_block) ptx::prefetch_tmap(&maps.ps);
      if (QVEC) ptx::prefetch_tmap(&maps.qs);
    }
  }
  if (warp == 1) {
    ptx::tmem_alloc(&tmem_slot, Cfg::COLS);
    ptx::tmem_relinquish();
  }
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  const uint32_t tmem = tmem_slot;
  pdl_wait();

  float acc[CW];
#pragma unroll
  for (int j = 0; j < CW; ++j) acc[j] = 0.f;

  if (warp == 0) {
    if (ptx::elect_one()) {
      // ---------------- TMA producer
      int stage = 0;
      uint32_t phase = 0, issued = 0, issued_parity = 0;
      uint32_t slots = 0;  // of scales asked for so far
      for (int kb = kb0; kb < kb1; ++kb) {
        if (!ptx::mbar_wait(&empty[stage], phase ^ 1)) { abort_flag = 1; break; }
        uint8_t* sP = smem + stage * Cfg::STAGE;
        ptx::mbar_arrive_expect_tx(&full[stage], Cfg::STAGE);
        if (p.p_mn)
          ptx::tma_load_2d(sP, &maps.p, &full[stage], p0, kb * GROUP);
        else
          ptx::tma_load_2d(sP, &maps.p, &full[stage], kb * GROUP, p0);
        if (Q_MN)
          ptx::tma_load_2d(sP + F_TILE, &maps.q, &full[stage], q0, kb * GROUP);
        else
          ptx::tma_load_2d(sP + F_TILE, &maps.q, &full[stage], kb * GROUP, q0);
        issued |= 1u << stage;
        issued_parity = (issued_parity & ~(1u << stage)) | (phase << stage);
        if ((kb - kb0) % SCALE_KB == 0) {
          const uint32_t slot = slots & 1;
          if (!ptx::mbar_wait(&sempty[slot], ((slots >> 1) & 1) ^ 1)) { abort_flag = 1; break; }
          ptx::mbar_arrive_expect_tx(&sfull[slot], SCALE_KB * 4 * ((p.p_block ? 0 : F_ROWS) + (QVEC ? NT : 0)));
          if (!p.p_block) ptx::tma_load_2d(pscale[slot], &maps.ps, &sfull[slot], p0, kb);
          if (QVEC) ptx::tma_load_2d(qscale[slot], &maps.qs, &sfull[slot], q0, kb);
          ++slots;
        }
        if (++stage == Cfg::STAGES) { stage = 0; phase ^= 1; }
      }
      // every load has landed before shared memory is used again
      for (int s = 0; s < Cfg::STAGES; ++s)
        if (issued & (1u << s)) ptx::mbar_wait(&full[s], (issued_parity >> s) & 1u);
      for (uint32_t n = slots > 2 ? slots - 2 : 0; n < slots; ++n) ptx::mbar_wait(&sfull[n & 1], (n >> 1) & 1);
    }
  } else if (warp == 1) {
    if (ptx::elect_one()) {
      // ---------------- MMA issuer: one accumulator per k-block
      const uint32_t idesc = ptx::idesc_e4m3(F_ROWS, NT, p.p_mn != 0, Q_MN);
      // 32 elements of K: 32 bytes inside the swizzled K-major row, or four 1024-byte atoms of
      // eight MN-major rows
      const uint64_t p_step = p.p_mn ? 256 : 2, q_step = Q_MN ? 256 : 2;
      int stage = 0, a = 0;
      uint32_t phase = 0, a_phase = 0;
      bool ok = true;
      for (int kb = kb0; kb < kb1; ++kb) {
        if (!ptx::mbar_wait(&tempty[a], a_phase ^ 1) || !ptx::mbar_wait(&full[stage], phase)) { ok = false; break; }
        ptx::tc_fence_after();
        const uint32_t sP = ptx::smem_u32(smem + stage * Cfg::STAGE);
        const uint64_t pd = ptx::sdesc_sw128(sP, p.p_mn ? F_TILE : 16, 1024);
        const uint64_t qd = ptx::sdesc_sw128(sP + F_TILE, Q_MN ? F_TILE : 16, 1024);
#pragma unroll
        for (int k = 0; k < GROUP / 32; ++k)
          ptx::umma_f8(tmem + a * NT, pd + k * p_step, qd + k * q_step, idesc, k > 0 ? 1u : 0u);
        ptx::umma_commit(&empty[stage]);
        ptx::umma_commit(&tfull[a]);
        if (++stage == Cfg::STAGES) { stage = 0; phase ^= 1; }
        if (++a == F_ACCS) { a = 0; a_phase ^= 1; }
      }
      if (!ok) abort_flag = 1;
      if (abort_flag) {  // products may still be running
        ptx::umma_commit(&drainbar);
        ptx::mbar_wait(&drainbar, 0);
      }
    }
  } else if (warp == 2) {
    // ---------------- watcher
    int a = 0, bar = 0;
    uint32_t a_phase = 0;
    bool ok = true;
    for (int kb = kb0; kb < kb1; ++kb) {
      const int id = 1 + bar * (Cfg::EW / 4);
      if (ok) {
        ok = ptx::mbar_wait(&tfull[a], a_phase);
        if (!ok) abort_flag = 1;
        __syncwarp();
#pragma unroll
        for (int sl = 0; sl < Cfg::EW / 4; ++sl) fp8::named_arrive(id + sl, 160);
        ok = __all_sync(0xffffffffu, ok);
      } else {
        for (int sl = 0; sl < Cfg::EW / 4; ++sl) fp8::named_sync(id + sl, 160);
      }
      if (++a == F_ACCS) { a = 0; a_phase ^= 1; }
      if (++bar == F_BARS) bar = 0;
    }
  } else if (warp >= 4) {
    // ---------------- epilogue: thread = P row, CW columns of Q
    const int q4 = warp & 3, sl = (warp - 4) >> 2, c0 = sl * CW;
    const uint32_t t0 = tmem + ((uint32_t)(q4 * 32) << 16) + c0;
    // block scales of 32 k-blocks, one per lane, and of the 32 after them
    const bool block = p.p_block || !QVEC;
    const float* bs = p.block + (int64_t)((p.p_block ? p0 : q0) / GROUP) * p.block_step;
    auto block_at = [&](int kb) { return block && kb < kb1 ? bs[(int64_t)kb * p.block_ld] : 1.f; };
    float bcur = block_at(kb0 + lane), bnext = block_at(kb0 + 32 + lane);
    int a = 0, bar = 0;
    uint32_t slots = 0, ps = 0, qs = 0;  // addresses of this k-block's scales: of the row, of the columns
    bool alive = true;
    for (int kb = kb0; kb < kb1; ++kb) {
      const int at = (kb - kb0) & 31;
      if (at == 0 && kb > kb0) {
        bcur = bnext;
        bnext = block_at(kb + 32 + lane);
      }
      if (at % SCALE_KB == 0) {
        if (alive) alive = ptx::mbar_wait(&sfull[slots & 1], (slots >> 1) & 1);
        if (!alive) abort_flag = 1;
        __syncwarp();
        ps = ptx::smem_u32(&pscale[slots & 1][0][q4 * 32 + lane]);
        qs = ptx::smem_u32(&qscale[slots & 1][0][c0]);
      }
      float s = __shfl_sync(0xffffffffu, bcur, at);
      if (!p.p_block) s *= ptx::ld_shared(ps);
      fp8::named_sync(1 + bar * (Cfg::EW / 4) + sl, 160);  // the watcher has seen the accumulator complete
      ptx::tc_fence_after();
      fp8::scaled_add<CW, QVEC, (CW < 32 ? 16 : 32)>(acc, t0 + a * NT, s, qs, [&] {
        if (lane == 0) ptx::mbar_arrive(&tempty[a]);
      });
      if (++a == F_ACCS) a = 0;
      if (++bar == F_BARS) bar = 0;
      ps += F_ROWS * 4;
      qs += NT * 4;
      if (at % SCALE_KB == SCALE_KB - 1) {
        __syncwarp();  // every lane has used its scales
        if (lane == 0) ptx::mbar_arrive(&sempty[slots & 1]);
        ++slots;
      }
    }
  }
  ptx::tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    ptx::tc_fence_after();
    ptx::tmem_dealloc(tmem, Cfg::COLS);
  }
  // ---------------- join the splits and store; the operand ring is free (every load has been
  // consumed by products that have completed)
  constexpr int PITCH = SWAP ? F_ROWS : NT + 4;  // SWAP: [NT][128]; else [128][NT + 4]
  static_assert((SWAP ? NT * PITCH : F_ROWS * PITCH) * 4 <= Cfg::STAGES * Cfg::STAGE, "the partial tile fits the ring");
  float* tilebuf = reinterpret_cast<float*>(smem);
  if (warp >= 4) {
    const int c0 = ((warp - 4) >> 2) * CW, row = (warp & 3) * 32 + lane;
#pragma unroll
    for (int j = 0; j < CW; j += 4) {
      if constexpr (SWAP) {
        float* at = tilebuf + (c0 + j) * PITCH + row;
        at[0] = acc[j]; at[PITCH] = acc[j + 1]; at[2 * PITCH] = acc[j + 2]; at[3 * PITCH] = acc[j + 3];
      } else {
        *reinterpret_cast<float4*>(tilebuf + row * PITCH + c0 + j) = make_float4(acc[j], acc[j + 1], acc[j + 2], acc[j + 3]);
      }
    }
  }
  if (p.splits > 1)
    ptx::cluster_sync();
  else
    __syncthreads();
  const uint32_t base = ptx::smem_u32(tilebuf);
  uint32_t peer[F_MAX_SPLITS];
#pragma unroll
  for (int c = 0; c < F_MAX_SPLITS; ++c)
    peer[c] = p.splits > 1 ? ptx::mapa(base, c < p.splits ? c : 0) : base;
  auto finish = [&](float v, int m, int n) {
    if (p.bias) v += fp8::load_any(p.bias, p.bias_f32, n);
    const int64_t at = (int64_t)m * p.ldc + n;
    if (p.c_f32) {
      float* c = static_cast<float*>(p.C) + at;
      *c = p.accumulate ? *c + v : v;
    } else {
      static_cast<bf16*>(p.C)[at] = __float2bfloat16_rn(v);
    }
  };
  if constexpr (SWAP) {
    // columns (tokens) NT rank / splits ..: a warp's lanes store neighbouring n
    const int j0 = NT * rank / p.splits, j1 = NT * (rank + 1) / p.splits;
    const int n = p0 + (threadIdx.x & 127);
    for (int j = j0 + (threadIdx.x >> 7); j < j1; j += Cfg::THREADS / 128) {
      const int m = q0 + j;
      if (m >= p.Q) break;
      const uint32_t off = (uint32_t)(j * PITCH + (threadIdx.x & 127)) * 4;
      float v = 0.f;
#pragma unroll
      for (int c = 0; c < F_MAX_SPLITS; ++c)
        if (c < p.splits) v += ptx::ld_cluster(peer[c] + off);
      if (n < p.P) finish(v, m, n);
    }
  } else {
    // rows 128 rank / splits ..: a warp's lanes store neighbouring runs of four columns
    const int r0 = F_ROWS * rank / p.splits, r1 = F_ROWS * (rank + 1) / p.splits;
    constexpr int RUNS = NT / 4;
    for (int e = r0 * RUNS + threadIdx.x; e < r1 * RUNS; e += Cfg::THREADS) {
      const int r = e / RUNS, c4 = (e % RUNS) * 4;
      const int m = p0 + r, n = q0 + c4;
      if (m >= p.P || n >= p.Q) continue;
      const uint32_t off = (uint32_t)(r * PITCH + c4) * 4;
      float v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < F_MAX_SPLITS; ++c)
        if (c < p.splits) {
          const float4 f = ptx::ld_cluster_v4(peer[c] + off);
          v[0] += f.x; v[1] += f.y; v[2] += f.z; v[3] += f.w;
        }
      if (p.c_vec && n + 4 <= p.Q) {
        if (p.bias) {
#pragma unroll
          for (int i = 0; i < 4; ++i) v[i] += fp8::load_any(p.bias, p.bias_f32, n + i);
        }
        const int64_t at = (int64_t)m * p.ldc + n;
        if (p.c_f32) {
          float4* c = reinterpret_cast<float4*>(static_cast<float*>(p.C) + at);
          if (p.accumulate) {
            const float4 o = *c;
            v[0] += o.x; v[1] += o.y; v[2] += o.z; v[3] += o.w;
          }
          *c = make_float4(v[0], v[1], v[2], v[3]);
        } else {
          __nv_bfloat162 lo = __floats2bfloat162_rn(v[0], v[1]), hi = __floats2bfloat162_rn(v[2], v[3]);
          *reinterpret_cast<uint2*>(static_cast<bf16*>(p.C) + at) =
              make_uint2(*reinterpret_cast<uint32_t*>(&lo), *reinterpret_cast<uint32_t*>(&hi));
        }
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (n + i < p.Q) finish(v[i], m, n + i);
      }
    }
  }
  if (p.splits > 1) ptx::cluster_sync();  // no CTA leaves while another may read its tile
}

// ------------------------------------------------------------------ host side
template <int NT, bool Q_MN, bool SWAP, bool QVEC>
int launch_f8(const GemmFp8Args& g, int splits, cudaStream_t s) {
  using Cfg = FCfg<NT, Q_MN>;
  const Fp8Operand &po = SWAP ? g.b : g.a, &qo = SWAP ? g.a : g.b;
  FParams p{};
  p.P = (int)(SWAP ? g.N : g.M);
  p.Q = (int)(SWAP ? g.M : g.N);
  p.tiles_p = ceil_div(p.P, F_ROWS);
  p.k_blocks = ceil_div(g.K, GROUP);
  p.splits = splits;
  const Fp8Operand& bo = po.block ? po : qo;
  p.block = bo.scale; p.block_ld = bo.ld; p.block_step = bo.row_step;
  p.p_block = po.block; p.p_mn = po.mn;
  p.C = g.C; p.ldc = g.ldc;
  p.c_f32 = g.c_dtype == JAGG_DTYPE_F32;
  p.accumulate = g.accumulate;
  p.c_vec = p.c_f32 ? fp8::aligned(g.C, 16) && g.ldc % 4 == 0 : fp8::aligned(g.C, 8) && g.ldc % 4 == 0;
  p.bias = g.bias;
  p.bias_f32 = g.bias_dtype == JAGG_DTYPE_F32;
  FMaps maps{};
  if (g.K > 0) {
    JAGG_TRY(fp8_operand_map(&maps.p, po, p.P, g.K, F_ROWS));
    JAGG_TRY(fp8_operand_map(&maps.q, qo, p.Q, g.K, NT));
    if (!po.block) JAGG_TRY(fp8_scale_map(&maps.ps, po, p.P, g.K, F_ROWS, SCALE_KB));
    if (QVEC) JAGG_TRY(fp8_scale_map(&maps.qs, qo, p.Q, g.K, NT, SCALE_KB));
  }
  auto kernel = gemm_fp8_kernel<NT, Q_MN, SWAP, QVEC>;
  static OncePerDevice once;
  JAGG_CUDA_TRY(allow_smem(once, kernel, Cfg::SMEM));
  cudaLaunchAttribute attr[2] = {};
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = splits;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)(p.tiles_p * ceil_div(p.Q, NT) * splits));
  cfg.blockDim = Cfg::THREADS;
  cfg.dynamicSmemBytes = Cfg::SMEM;
  cfg.stream = s;
  cfg.attrs = attr;
  cfg.numAttrs = splits > 1 ? 2 : 1;
  JAGG_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, maps, p));
  JAGG_LAUNCHED();
  return JAGG_OK;
}

// Microseconds that a k-block takes, by kernel and tile, and what a tile and a launch take besides,
// fitted to products of 1 to 8192 rows with 512 to 8192 along K: 4864 x 4096 x 4096 takes 66 us in pair tiles
// of 256 columns, 93 in tiles of 128 and 115 in single CTAs, 512 x 4096 x 4096 17.7, 14.6 and 15.0,
// 128 x 4096 x 4096 split four ways 9.0, against 14.0 for either unsplit.  B's vector scales cost a
// multiplication per element more than block scales.
constexpr double US_LAUNCH = 2.0, US_TILE_ONE = 2.5, US_TILE_PAIR = 2.2, US_JOIN = 0.5;
double us_one(int nt, bool qvec) { return nt == 16 ? 0.165 : nt == 32 ? 0.28 : nt == 64 ? 0.42 : qvec ? 0.5 : 0.35; }
double us_pair(int bn, bool qvec) { return bn == 256 ? (qvec ? 0.67 : 0.44) : qvec ? 0.48 : 0.31; }

// CTAs that run at one time in clusters of n: a cluster has to fit into the SMs of one GPC, so that up
// to an eighth of the machine stays idle (18 tiles split 8 ways, 144 CTAs, take two turns: 15.6 us,
// against 6.9 split 4 ways).  Asked once per size and device; all instances take an SM each.
int ask_cluster_ctas(int n, int* ctas) {
  auto kernel = gemm_fp8_kernel<128, false, false, false>;
  using Cfg = FCfg<128, false>;
  static OncePerDevice once;
  JAGG_CUDA_TRY(allow_smem(once, kernel, Cfg::SMEM));
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = n;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(n * sm_count());
  cfg.blockDim = Cfg::THREADS;
  cfg.dynamicSmemBytes = Cfg::SMEM;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  int clusters = 0;
  JAGG_CUDA_TRY(cudaOccupancyMaxActiveClusters(&clusters, kernel, &cfg));
  *ctas = clusters > 0 ? clusters * n : n;
  return JAGG_OK;
}
int cluster_ctas(int dev, int n, int* ctas) {
  static NumberPerDevice known[F_MAX_SPLITS + 1];
  return known[n].get(dev, ctas, [&](int* found) { return ask_cluster_ctas(n, found); });
}

int plan_of(const GemmFp8Args& g, Fp8Plan* plan) {
  const int kb = ceil_div(g.K, GROUP), sms = sm_count();
  int room[F_MAX_SPLITS + 1] = {0, sms};
  int dev = 0;
  JAGG_CUDA_TRY(cudaGetDevice(&dev));
  for (int s = 2; s <= F_MAX_SPLITS; ++s) JAGG_TRY(cluster_ctas(dev, s, &room[s]));
  Fp8Plan& best = *plan;
  double least = 0.0;
  auto offer = [&](const Fp8Plan& p, double us) {
    if (least == 0.0 || us < least) {
      least = us;
      best = p;
    }
  };
  auto tiles = [](int64_t rows, int64_t cols, int tr, int tc) {
    return (double)((rows + tr - 1) / tr) * (double)((cols + tc - 1) / tc);
  };
  auto one = [&](bool swap, int nt) {
    const double t = swap ? tiles(g.N, g.M, F_ROWS, nt) : tiles(g.M, g.N, F_ROWS, nt);
    const bool qvec = swap || !g.b.block;
    for (int s = 1; s <= F_MAX_SPLITS && (s == 1 || s <= kb); ++s)
      offer({0, nt, s, swap}, US_LAUNCH + ceil(t * s / room[s]) * (ceil_div(kb, s) * us_one(nt, qvec) + US_TILE_ONE) +
                                  (s > 1 ? US_JOIN : 0.0));
  };
  one(false, 128);
  // few rows of A: as many columns of an accumulator as there are tokens (an MN-major A arrives in
  // whole 128-byte rows, so there is nothing to gain)
  if (!g.a.mn && g.M <= 64) one(true, g.M <= 16 ? 16 : g.M <= 32 ? 32 : 64);
  if (g.K > 0)
    for (int bn : {256, 128})
      offer({bn, 0, 1, false}, US_LAUNCH + ceil(tiles(g.M, g.N, 256, bn) / (sms / 2)) *
                                               (kb * us_pair(bn, !g.b.block) + US_TILE_PAIR));
  return JAGG_OK;
}

int run_plan(const GemmFp8Args& g, const Fp8Plan& p, cudaStream_t s) {
  if (p.pair) return gemm_fp8_pair(g, p.pair, s);
  if (p.swap) {
    if (p.nt == 16) return launch_f8<16, false, true, true>(g, p.splits, s);
    if (p.nt == 32) return launch_f8<32, false, true, true>(g, p.splits, s);
    return launch_f8<64, false, true, true>(g, p.splits, s);
  }
  if (g.b.mn)
    return g.b.block ? launch_f8<128, true, false, false>(g, p.splits, s)
                     : launch_f8<128, true, false, true>(g, p.splits, s);
  return g.b.block ? launch_f8<128, false, false, false>(g, p.splits, s)
                   : launch_f8<128, false, false, true>(g, p.splits, s);
}

}  // namespace

int fp8_operand_map(CUtensorMap* m, const Fp8Operand& o, int64_t rows, int64_t K, int box_rows) {
  const uint64_t dims[2] = {(uint64_t)(o.mn ? rows : K), (uint64_t)(o.mn ? K : rows)};
  const uint64_t strides[1] = {(uint64_t)o.ldq};
  const uint32_t box[2] = {128u, (uint32_t)(o.mn ? GROUP : box_rows)};
  return encode_tmap_as(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, o.q, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B);
}

int fp8_scale_map(CUtensorMap* m, const Fp8Operand& o, int64_t rows, int64_t K, int box_rows, int box_groups) {
  const uint64_t dims[2] = {(uint64_t)rows, (uint64_t)((K + GROUP - 1) / GROUP)};
  const uint64_t strides[1] = {(uint64_t)o.ld * 4};
  const uint32_t box[2] = {(uint32_t)box_rows, (uint32_t)box_groups};
  return encode_tmap(m, true, 2, o.scale, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_NONE);
}

int gemm_fp8(const GemmFp8Args& g, cudaStream_t s) {
  Fp8Plan p;
  JAGG_TRY(plan_of(g, &p));
  return gemm_fp8_as(g, p, s);
}

int gemm_fp8_as(const GemmFp8Args& g, const Fp8Plan& p, cudaStream_t s) {
  const int tok = prof_start(s);
  JAGG_TRY(run_plan(g, p, s));
  prof_stop(tok, s, PROF_GEMM_FP8, 2.0 * g.M * g.N * g.K,
            (double)g.M * g.K + (double)g.N * g.K + (double)g.M * g.N * (g.c_dtype == JAGG_DTYPE_F32 ? 4 : 2), (int)g.M,
            (int)g.N, (int)g.K);
  return JAGG_OK;
}

}  // namespace jagg

using namespace jagg;

// The product that a descriptor asks for; *empty: there is nothing to compute.
static int fp8_args(const char* who, const jagg_gemm_fp8_desc* d, GemmFp8Args* args, bool* empty) {
  *empty = false;
  JAGG_CHECK_ARG(d, "%s: null descriptor", who);
  JAGG_CHECK_ARG(d->M >= 0 && d->N >= 0 && d->K >= 0 && d->M < INT32_MAX - 256 && d->N < INT32_MAX - 256 &&
                     d->K < INT32_MAX - 256,
                 "%s: M=%lld N=%lld K=%lld outside [0, 2^31 - 257)", who, (long long)d->M, (long long)d->N,
                 (long long)d->K);
  if ((d->M + 127) / 128 * ((d->N + 127) / 128) > INT32_MAX / F_MAX_SPLITS) {
    set_last_error("%s: an output of %lld x %lld is not implemented", who, (long long)d->M, (long long)d->N);
    return JAGG_ERR_UNSUPPORTED;
  }
  JAGG_CHECK_ARG(fp8::is_dtype(d->c_dtype) && fp8::is_dtype(d->bias_dtype), "%s: bad dtype", who);
  JAGG_CHECK_ARG(!d->accumulate || d->c_dtype == JAGG_DTYPE_F32, "%s: accumulation needs an f32 output", who);
  *empty = d->M == 0 || d->N == 0;
  if (*empty) return JAGG_OK;
  JAGG_CHECK_ARG(d->C && d->ldc >= d->N && fp8::aligned(d->C, fp8::size_of(d->c_dtype)),
                 "%s: output null, misaligned, or with a row pitch below N=%lld", who, (long long)d->N);
  JAGG_CHECK_ARG(fp8::aligned(d->bias, fp8::size_of(d->bias_dtype)), "%s: bias is not aligned to its elements", who);
  const int64_t kg = (d->K + GROUP - 1) / GROUP, ng = (d->N + GROUP - 1) / GROUP;
  if (d->K > 0) {
    const int64_t a_cols = d->a_trans ? d->M : d->K, b_cols = d->b_trans ? d->N : d->K;
    JAGG_CHECK_ARG(d->A && fp8::aligned(d->A, 16) && d->lda % 16 == 0 && d->lda >= a_cols,
                   "%s: A needs a 16-byte aligned base and a row pitch that is a multiple of 16 and >= %lld (got %lld)", who,
                   (long long)a_cols, (long long)d->lda);
    JAGG_CHECK_ARG(d->B && fp8::aligned(d->B, 16) && d->ldb % 16 == 0 && d->ldb >= b_cols,
                   "%s: B needs a 16-byte aligned base and a row pitch that is a multiple of 16 and >= %lld (got %lld)", who,
                   (long long)b_cols, (long long)d->ldb);
    JAGG_CHECK_ARG(d->a_scale && fp8::aligned(d->a_scale, 16) && d->lda_scale % 4 == 0 && d->lda_scale >= d->M,
                   "%s: A's scales need a 16-byte aligned base and a pitch that is a multiple of 4 and >= M=%lld (got %lld)",
                   who, (long long)d->M, (long long)d->lda_scale);
    const int64_t b_need = !d->b_block ? d->N : d->b_trans ? ng : kg;
    JAGG_CHECK_ARG(d->b_scale && fp8::aligned(d->b_scale, d->b_block ? 4 : 16) &&
                       (d->b_block || d->ldb_scale % 4 == 0) && d->ldb_scale >= b_need,
                   "%s: B's scales null, misaligned, or with a pitch that does not fit: >= %lld%s (got %lld)", who,
                   (long long)b_need, d->b_block ? "" : " and a multiple of 4", (long long)d->ldb_scale);
  }
  GemmFp8Args& g = *args;
  g.M = d->M; g.N = d->N; g.K = d->K;
  g.a.q = d->A; g.a.ldq = d->lda; g.a.scale = d->a_scale; g.a.ld = d->lda_scale; g.a.mn = d->a_trans != 0;
  g.b.q = d->B; g.b.ldq = d->ldb; g.b.scale = d->b_scale; g.b.mn = d->b_trans != 0; g.b.block = d->b_block != 0;
  // blocks stored [N, K]: a row of blocks per 128 of N; stored [K, N]: per 128 of K
  g.b.ld = !g.b.block || g.b.mn ? d->ldb_scale : 1;
  g.b.row_step = g.b.block ? (g.b.mn ? 1 : d->ldb_scale) : 0;
  g.C = d->C; g.ldc = d->ldc; g.c_dtype = d->c_dtype;
  g.bias = d->bias; g.bias_dtype = d->bias_dtype;
  g.accumulate = d->accumulate != 0;
  return JAGG_OK;
}

extern "C" int jagg_gemm_fp8(const jagg_gemm_fp8_desc* desc, cudaStream_t stream) {
  GemmFp8Args g;
  bool empty;
  JAGG_TRY(fp8_args("jagg_gemm_fp8", desc, &g, &empty));
  return empty ? JAGG_OK : gemm_fp8(g, stream);
}

extern "C" int jagg_test_gemm_fp8(const jagg_gemm_fp8_desc* desc, int pair, int nt, int splits, int swap,
                                  cudaStream_t stream) {
  const char* who = "jagg_test_gemm_fp8";
  GemmFp8Args g;
  bool empty;
  JAGG_TRY(fp8_args(who, desc, &g, &empty));
  const int kb = ceil_div(g.K, GROUP);
  JAGG_CHECK_ARG(!empty && kb > 0, "%s: an empty product", who);
  if (pair) {
    JAGG_CHECK_ARG(pair == 128 || pair == 256, "%s: pair tiles of %d columns", who, pair);
  } else {
    JAGG_CHECK_ARG(splits >= 1 && splits <= F_MAX_SPLITS && splits <= kb, "%s: %d splits of %d k-blocks", who, splits, kb);
    JAGG_CHECK_ARG(swap ? (nt == 16 || nt == 32 || nt == 64) && !g.a.mn : nt == 128, "%s: tiles of %d columns", who, nt);
  }
  return gemm_fp8_as(g, {pair, nt, splits, swap != 0}, stream);
}
