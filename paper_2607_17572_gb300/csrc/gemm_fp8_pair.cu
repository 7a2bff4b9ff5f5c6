// Products of 8-bit operands in tiles of 256 rows x up to 256 columns on CTA pairs
// (tcgen05.mma.cta_group::2, kind::f8f6f4).
//
// As in gemm_fp8.cu a k-block is one group of 128 along K and an accumulator one inner sum; the
// epilogue adds it, scaled, to f32 registers.  Two CTAs (the two SMs of a TPC) own one tile: each
// stages its 128 rows of A and its half of the columns of B, the leader issues the products of
// both, and each CTA's tensor memory holds its 128 rows of the accumulator.
//
// Per k-block of a tile of 256 columns an SM's tensor core works 512 clocks.  Meanwhile its epilogue
// has to read 128 x 256 f32 from tensor memory and to add them, 256 clocks of f32 arithmetic, and hand the
// accumulator back: two accumulators of 256 columns fill tensor memory, so while one is added the other
// is all that the tensor core has to work on.  Each of 16 epilogue warps therefore owns 64 columns of 32
// rows, and hands its accumulator back as soon as the last of them are in registers, before they are
// added.
//
// Measured on 18432 x 12288 x 4096 with block scales: 772 us on the GPU (777 to 805 a call), 2400 TFLOP/s, at 1365 W and
// 1890 MHz (the power limit; 7 % less in the first 50 ms).  That is 46 turns of 32 k-blocks of about 980 clocks, and
// the tensor pipe is 51 to 61 % active: the epilogue's step, not the tensor core, sets the pace.  It issues
// about 530 instructions per scheduler and k-block (54 % of the slots), of which the paired additions and
// the loads of four warps are some 150; what the others are has not been counted.  With vector scales on both
// sides, 4096 x 12288 x 8192: 456 us, 1810 TFLOP/s: a load and a multiplication per pair of columns more.
//
// Roles per CTA: warp 0 TMA producer (operands and vector scales), warp 1 MMA issuer (leader only), warp
// 2 watches the accumulators' barriers for the epilogue warps (16 warps that poll slow down those
// that work), warps 4-19 the epilogue: thread = output row, 64 columns; results through a swizzled
// shared-memory box into TMA stores (f32 reduce-adds when accumulating: one addition per element), or
// copied from there where C's alignment does not allow those.
#include "gemm_fp8.cuh"

namespace jagg {

int unit_status_gemm_fp8_pair(unsigned* v, int clear) { return read_unit_status(v, clear); }

namespace {

using fp8::GROUP;
using fp8::SCALE_KB;

constexpr int W_ROWS = 256, W_MAX_N = 256;
constexpr int W_ACCS = 2;             // accumulators in tensor memory
constexpr int W_SLICES = 4;           // slices of columns
constexpr int W_BARS = W_ACCS + 2;    // sets of named barriers (fp8::named_arrive), one of each per slice: all 16
static_assert(W_BARS % W_ACCS == 0 && (W_BARS & (W_BARS - 1)) == 0, "a set tells its accumulator");
constexpr int W_EW = 16, W_CW = 64;
constexpr int W_THREADS = 128 + 32 * W_EW;
constexpr int W_HALF = 128 * GROUP;   // bytes of a CTA's half of an operand tile
constexpr int W_MAX_STAGES = 6;
constexpr int W_GROUP = 19;           // row tiles walked together (gemm_pair.cu)

template <bool QVEC>
struct WCfg {
  static constexpr int STAGES = QVEC ? 5 : 6;
  static constexpr int STEP = 16;  // columns of a load (32 would spill)
  static constexpr int BOX = QVEC ? 2048 : 1024;  // an epilogue warp's staging box: 32 rows of 64 or 32 bytes
  static constexpr int ROW = BOX / 32;
  static constexpr int SLOT = SCALE_KB * (128 + (QVEC ? W_MAX_N : 0));  // floats: [kb][rows of A], [kb][columns of B]
  static constexpr int SMEM = STAGES * 2 * W_HALF + W_EW * BOX + 2 * SLOT * 4 + 1024;
};
static_assert(WCfg<false>::SMEM <= 232448 - 1024 && WCfg<true>::SMEM <= 232448 - 1024, "shared memory");

struct WParams {
  int M, N, bn, tiles_m, tiles_n, k_blocks;
  const float* bs;         // block scales of B
  int64_t bs_ld, bs_step;
  int a_mn, b_mn;
  void* C;
  int64_t ldc;
  int c_f32, accumulate, c_tma;
  const void* bias;
  int bias_f32;
};
struct WMaps {
  CUtensorMap a, b, c, as, bs;
};

__device__ __forceinline__ void w_decode(const WParams& p, int t, int& tm, int& tn) {
  const int per_group = W_GROUP * p.tiles_n;
  const int grp = t / per_group, in = t - grp * per_group;
  const int gm = min(W_GROUP, p.tiles_m - grp * W_GROUP);
  tm = grp * W_GROUP + in % gm;
  tn = in / gm;
}

// A box into rows of C that a TMA store cannot write (it writes whole 16-byte pieces): neighbouring lanes
// take neighbouring elements of a row.  Element by element from the accumulators a row per lane, 300 x 700
// x 900 in bf16 took 40 us.
template <int ROW>
__device__ __forceinline__ void copy_out(const WParams& p, const uint8_t* box, int lane, int m0, int x) {
  constexpr int PIECES = ROW / 16;
  const int size = p.c_f32 ? 4 : 2, row_elements = ROW / size, rows = 32 / row_elements;
  const int e = lane % row_elements;
#pragma unroll 1
  for (int r = lane / row_elements; r < 32; r += rows) {
    const int swz = PIECES == 4 ? (r >> 1) & 3 : (r >> 2) & 1;
    const uint8_t* from = box + r * ROW + (((e * size >> 4) ^ swz) << 4) + (e * size & 15);
    if (m0 + r >= p.M || x + e >= p.N) continue;
    const int64_t at = (int64_t)(m0 + r) * p.ldc + x + e;
    if (p.c_f32) {
      float* c = static_cast<float*>(p.C) + at;
      const float v = *reinterpret_cast<const float*>(from);
      *c = p.accumulate ? *c + v : v;
    } else {
      static_cast<bf16*>(p.C)[at] = *reinterpret_cast<const bf16*>(from);
    }
  }
  __syncwarp();  // the box has been read
}

template <bool QVEC>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(W_THREADS, 1)
    gemm_fp8_pair_kernel(const __grid_constant__ WMaps maps, const __grid_constant__ WParams p) {
  using Cfg = WCfg<QVEC>;
  constexpr int STAGES = Cfg::STAGES, STAGE = 2 * W_HALF;
  extern __shared__ uint8_t smem_w8[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_w8) + 1023) & ~uintptr_t(1023));
  float* scales = reinterpret_cast<float*>(smem + STAGES * STAGE);  // two slots
  uint8_t* boxes = reinterpret_cast<uint8_t*>(scales + 2 * Cfg::SLOT);
  __shared__ uint64_t full[W_MAX_STAGES];   // leader's: a stage landed in both CTAs
  __shared__ uint64_t empty[W_MAX_STAGES];  // per CTA: the products reading the stage are done
  __shared__ uint64_t tfull[W_ACCS];        // per CTA: an accumulator is complete
  __shared__ uint64_t tempty[W_ACCS];       // leader's: both CTAs' epilogue warps have read it
  __shared__ uint64_t sfull[2], sempty[2];  // per CTA: a slot of scales landed, has been used
  __shared__ uint64_t drainbar, never;
  __shared__ uint32_t tmem_slot;
  __shared__ volatile int abort_flag, last_tile;

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = ptx::cluster_ctarank();

  if (threadIdx.x == 0) {
    abort_flag = 0;
    last_tile = -1;
    for (int s = 0; s < STAGES; ++s) {
      ptx::mbar_init(&full[s], 1);
      ptx::mbar_init(&empty[s], 1);
    }
    for (int a = 0; a < W_ACCS; ++a) {
      ptx::mbar_init(&tfull[a], 1);
      ptx::mbar_init(&tempty[a], 2 * 4 * (p.bn / W_CW));
    }
    for (int i = 0; i < 2; ++i) {
      ptx::mbar_init(&sfull[i], 1);
      ptx::mbar_init(&sempty[i], 4 * (p.bn / W_CW));
    }
    ptx::mbar_init(&drainbar, 1);
    ptx::mbar_init(&never, 1);
    ptx::fence_mbar_init();
    ptx::prefetch_tmap(&maps.a);
    ptx::prefetch_tmap(&maps.b);
    ptx::prefetch_tmap(&maps.as);
    if (QVEC) ptx::prefetch_tmap(&maps.bs);
    if (p.c_tma) ptx::prefetch_tmap(&maps.c);
  }
  if (warp == 1) {
    ptx::tmem_alloc_pair(&tmem_slot, 512);
    ptx::tmem_relinquish_pair();
  }
  ptx::tc_fence_before();
  __syncthreads();
  ptx::cluster_sync();  // the peer's barriers are initialised
  ptx::tc_fence_after();
  const uint32_t tmem = tmem_slot;
  pdl_wait();

  const int total = p.tiles_m * p.tiles_n, npairs = gridDim.x >> 1;
  const int half_n = p.bn >> 1, slices = p.bn / W_CW;

  if (warp == 0) {
    if (ptx::elect_one()) {
      // ---------------- TMA producer: this CTA's halves of A and B, and the scales of its accumulator
      int stage = 0;
      uint32_t phase = 0, issued = 0, issued_parity = 0;
      uint32_t slots = 0;  // of scales asked for so far
      // MN-major B arrives in whole 128-byte rows (of which half_n are used)
      const uint32_t stage_bytes = 2u * (W_HALF + (p.b_mn ? W_HALF : half_n * GROUP));
      for (int t = blockIdx.x >> 1; t < total && !abort_flag; t += npairs) {
        int tm, tn;
        w_decode(p, t, tm, tn);
        const int ma = tm * W_ROWS + (int)rank * 128, nb = tn * p.bn + (int)rank * half_n;
        for (int kb = 0; kb < p.k_blocks; ++kb) {
          if (!ptx::mbar_wait(&empty[stage], phase ^ 1)) { abort_flag = 1; break; }
          uint8_t* sA = smem + stage * STAGE;
          if (rank == 0) ptx::mbar_arrive_expect_tx(&full[stage], stage_bytes);
          const uint32_t bar = ptx::mapa(ptx::smem_u32(&full[stage]), 0);
          if (p.a_mn)
            ptx::tma_load_2d_pair(sA, &maps.a, bar, ma, kb * GROUP);
          else
            ptx::tma_load_2d_pair(sA, &maps.a, bar, kb * GROUP, ma);
          if (p.b_mn)
            ptx::tma_load_2d_pair(sA + W_HALF, &maps.b, bar, nb, kb * GROUP);
          else
            ptx::tma_load_2d_pair(sA + W_HALF, &maps.b, bar, kb * GROUP, nb);
          issued |= 1u << stage;
          issued_parity = (issued_parity & ~(1u << stage)) | (phase << stage);
          if (kb % SCALE_KB == 0) {
            const uint32_t slot = slots & 1;
            if (!ptx::mbar_wait(&sempty[slot], ((slots >> 1) & 1) ^ 1)) { abort_flag = 1; break; }
            float* sc = scales + slot * Cfg::SLOT;
            ptx::mbar_arrive_expect_tx(&sfull[slot], Cfg::SLOT * 4);
            ptx::tma_load_2d(sc, &maps.as, &sfull[slot], ma, kb);
            if (QVEC) ptx::tma_load_2d(sc + SCALE_KB * 128, &maps.bs, &sfull[slot], tn * p.bn, kb);
            ++slots;
          }
          if (++stage == STAGES) { stage = 0; phase ^= 1; }
        }
      }
      // No load outlives the block: the leader waits for the last phase of every stage.  The peer's loads
      // complete on the leader's barriers; after a give-up it waits for the length of one bounded wait.
      for (uint32_t n = slots > 2 ? slots - 2 : 0; n < slots; ++n) ptx::mbar_wait(&sfull[n & 1], (n >> 1) & 1);
      if (rank == 0) {
        for (int s = 0; s < STAGES; ++s)
          if (issued & (1u << s)) ptx::mbar_wait(&full[s], (issued_parity >> s) & 1u);
      } else if (abort_flag && issued) {
        ptx::mbar_wait(&never, 0);
      }
    }
  } else if (warp == 1) {
    if (rank == 0 && ptx::elect_one()) {
      // ---------------- MMA issuer for both CTAs: one accumulator per k-block
      const uint32_t idesc = ptx::idesc_e4m3(W_ROWS, p.bn, p.a_mn != 0, p.b_mn != 0);
      const uint64_t a_step = p.a_mn ? 256 : 2, b_step = p.b_mn ? 256 : 2;
      const uint32_t s0 = ptx::smem_u32(smem);
      uint64_t ad = ptx::sdesc_sw128(s0, p.a_mn ? W_HALF : 16, 1024);
      uint64_t bd = ptx::sdesc_sw128(s0 + W_HALF, p.b_mn ? W_HALF : 16, 1024);
      const uint64_t ad0 = ad, bd0 = bd;
      int stage = 0, acc = 0;
      uint32_t phase = 0, acc_phase = 0;
      for (int t = blockIdx.x >> 1; t < total && !abort_flag; t += npairs) {
        for (int kb = 0; kb < p.k_blocks; ++kb) {
          if (!ptx::mbar_wait(&full[stage], phase) || !ptx::mbar_wait(&tempty[acc], acc_phase ^ 1)) {
            abort_flag = 1;
            break;
          }
          ptx::tc_fence_after();
#pragma unroll
          for (int k = 0; k < GROUP / 32; ++k)
            ptx::umma_f8_pair(tmem + acc * W_MAX_N, ad + k * a_step, bd + k * b_step, idesc, k > 0 ? 1u : 0u);
          ptx::umma_commit_pair(&tfull[acc]);
          ptx::umma_commit_pair(&empty[stage]);
          if (++acc == W_ACCS) { acc = 0; acc_phase ^= 1; }
          ad += STAGE / 16;
          bd += STAGE / 16;
          if (++stage == STAGES) { stage = 0; phase ^= 1; ad = ad0; bd = bd0; }
        }
      }
      if (abort_flag) {  // products may still be running: drain them before tensor memory is freed
        ptx::umma_commit_local(&drainbar);
        ptx::mbar_wait(&drainbar, 0);
      }
    }
  } else if (warp == 2) {
    // ---------------- watcher: waits for accumulators and lets the epilogue warps go, which would
    // slow the others down by polling
    uint32_t bar = 0;
    uint32_t a_phase = 0;
    bool ok = true, left = false;
    for (int t = blockIdx.x >> 1; t < total && !left; t += npairs) {
      for (int kb = 0; kb < p.k_blocks; ++kb) {
        const int id = bar * W_SLICES;
        if (ok) {
          ok = ptx::mbar_wait(&tfull[bar % W_ACCS], a_phase);
          if (!ok) abort_flag = 1;
          __syncwarp();
          fp8::named_arrive(id, 160);
          fp8::named_arrive(id + 1, 160);
          if (slices == W_SLICES) {
            fp8::named_arrive(id + 2, 160);
            fp8::named_arrive(id + 3, 160);
          }
          ok = __all_sync(0xffffffffu, ok);
        } else {
          if (kb == p.k_blocks - 1) {
            last_tile = t;
            left = true;
          }
          for (int sl = 0; sl < slices; ++sl) fp8::named_sync(id + sl, 160);
        }
        bar = (bar + 1) % W_BARS;
        if (bar % W_ACCS == 0) a_phase ^= 1;
      }
    }
  } else if (warp >= 4 && (warp - 4) / 4 < slices) {
    // ---------------- epilogue: tensor-memory lanes 32 q .. + 31, columns c0 .. c0 + 63
    const int q = warp & 3, ew = warp - 4, sl = ew >> 2, c0 = sl * W_CW;
    uint8_t* box = boxes + ew * Cfg::BOX;
    const uint32_t t0 = tmem + ((uint32_t)(q * 32) << 16) + c0;
    const uint32_t te = ptx::mapa(ptx::smem_u32(&tempty[0]), 0);
    // block scales: of 32 k-blocks, one per lane, and of the 32 after them (or the next tile's first)
    auto block_at = [&](int t, int kb) {
      if (QVEC || t >= total || kb >= p.k_blocks) return 1.f;
      int tm, tn;
      w_decode(p, t, tm, tn);
      const int n = min(tn * p.bn + c0, p.N - 1);
      return p.bs[(int64_t)(n / GROUP) * p.bs_step + (int64_t)kb * p.bs_ld];
    };
    const uint32_t row4 = (q * 32 + lane) * 4, sbase = ptx::smem_u32(scales) + row4;
    uint32_t bar = 0;
    uint32_t slots = 0;
    float bcur = 1.f, bnext = block_at(blockIdx.x >> 1, lane);
    bool alive = true;
    for (int t = blockIdx.x >> 1; t < total; t += npairs) {
      float acc[W_CW];
#pragma unroll
      for (int j = 0; j < W_CW; ++j) acc[j] = 0.f;
      uint32_t sc = 0, qc = 0;  // addresses of this k-block's scales: of the row, of the columns
#pragma unroll 1
      for (int kb = 0; kb < p.k_blocks; ++kb) {
        if (kb % SCALE_KB == 0) {
          if (!QVEC && kb % 32 == 0) {
            bcur = bnext;
            bnext = kb + 32 < p.k_blocks ? block_at(t, kb + 32 + lane) : block_at(t + npairs, lane);
          }
          if (alive) alive = ptx::mbar_wait(&sfull[slots & 1], (slots >> 1) & 1);
          if (!alive) abort_flag = 1;
          __syncwarp();
          sc = sbase + (slots & 1) * Cfg::SLOT * 4;
          qc = sc + SCALE_KB * 128 * 4 + c0 * 4 - row4;
        }
        float s = ptx::ld_shared(sc);
        if (!QVEC) s *= __shfl_sync(0xffffffffu, bcur, kb & 31);
        const int a = bar % W_ACCS;
        fp8::named_sync(bar * W_SLICES + sl, 160);  // the watcher has seen the accumulator complete
        ptx::tc_fence_after();
        fp8::scaled_add<W_CW, QVEC, Cfg::STEP>(acc, t0 + a * W_MAX_N, s, qc, [&] {
          if (lane == 0) ptx::mbar_arrive_peer(te + a * 8);
        });
        bar = (bar + 1) % W_BARS;
        sc += 128 * 4;
        qc += W_MAX_N * 4;
        if (kb % SCALE_KB == SCALE_KB - 1 || kb == p.k_blocks - 1) {
          __syncwarp();  // every lane has used its scales
          if (lane == 0) ptx::mbar_arrive(&sempty[slots & 1]);
          ++slots;
        }
      }
      if (last_tile == t) break;
      if (__any_sync(0xffffffffu, abort_flag)) continue;  // dropped; all warps leave together, after last_tile
      int tm, tn;
      w_decode(p, t, tm, tn);
      const int m0 = tm * W_ROWS + (int)rank * 128 + q * 32, n0 = tn * p.bn + c0;
      if (m0 >= p.M || n0 >= p.N) continue;
      // eight columns of this lane's row, with their bias
      auto take = [&](int c, float (&v)[8]) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = acc[c + i];
        if (p.bias) {
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (n0 + c + i < p.N) v[i] += fp8::load_any(p.bias, p.bias_f32, n0 + c + i);
        }
      };
      // ROW bytes of this lane's row at a time: 16-byte pieces swizzled as the tensor map says
      constexpr int PIECES = Cfg::ROW / 16;
      const int swz = PIECES == 4 ? (lane >> 1) & 3 : (lane >> 2) & 1;
      const int per = p.c_f32 ? 4 : 8;  // elements of a piece
#pragma unroll
      for (int c = 0; c < W_CW; c += 8) {  // one bf16 piece, or two of f32
        const int at = c / per % PIECES;
        if (at == 0) {
          if (n0 + c >= p.N) break;
          if (lane == 0) ptx::bulk_wait_read<0>();  // the last store has read the box
          __syncwarp();
        }
        float v[8];
        take(c, v);
        uint8_t* mine = box + lane * Cfg::ROW;
        if (p.c_f32) {
          *reinterpret_cast<float4*>(mine + ((at ^ swz) << 4)) = make_float4(v[0], v[1], v[2], v[3]);
          *reinterpret_cast<float4*>(mine + (((at + 1) ^ swz) << 4)) = make_float4(v[4], v[5], v[6], v[7]);
        } else {
          fp8::store8(reinterpret_cast<bf16*>(mine + ((at ^ swz) << 4)), v);
        }
        if (at + 8 / per == PIECES) {
          const int x = n0 + c + 8 - PIECES * per;
          if (p.c_tma) {
            ptx::fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) {
              if (p.accumulate)
                ptx::tma_reduce_add_2d(&maps.c, box, x, m0);
              else
                ptx::tma_store_2d(&maps.c, box, x, m0);
              ptx::bulk_commit();
            }
          } else {
            __syncwarp();
            copy_out<Cfg::ROW>(p, box, lane, m0, x);
          }
        }
      }
    }
    pdl_trigger();  // only the stores in flight are left
    if (lane == 0) ptx::bulk_wait<0>();
    __syncwarp();
  }
  ptx::tc_fence_before();
  __syncwarp();  // (no __syncthreads: its barrier may be in use by other warps)
  ptx::cluster_sync();  // neither CTA's shared or tensor memory is in use by the other any more
  if (warp == 1) {
    ptx::tc_fence_after();
    ptx::tmem_dealloc_pair(tmem, 512);
  }
}

template <bool QVEC>
int launch_w8(const GemmFp8Args& g, int bn, cudaStream_t s) {
  using Cfg = WCfg<QVEC>;
  WParams p{};
  p.M = (int)g.M; p.N = (int)g.N; p.bn = bn;
  p.tiles_m = ceil_div(g.M, W_ROWS);
  p.tiles_n = ceil_div(g.N, bn);
  p.k_blocks = ceil_div(g.K, GROUP);
  p.bs = g.b.scale; p.bs_ld = g.b.ld; p.bs_step = g.b.row_step;
  p.a_mn = g.a.mn; p.b_mn = g.b.mn;
  p.C = g.C; p.ldc = g.ldc;
  p.c_f32 = g.c_dtype == JAGG_DTYPE_F32;
  p.accumulate = g.accumulate;
  // a TMA store writes whole 16-byte pieces, also of the last one of a row
  p.c_tma = fp8::aligned(g.C, 16) && g.ldc * fp8::size_of(g.c_dtype) % 16 == 0 && g.N * fp8::size_of(g.c_dtype) % 16 == 0;
  p.bias = g.bias;
  p.bias_f32 = g.bias_dtype == JAGG_DTYPE_F32;
  WMaps maps;
  JAGG_TRY(fp8_operand_map(&maps.a, g.a, g.M, g.K, 128));
  JAGG_TRY(fp8_operand_map(&maps.b, g.b, g.N, g.K, bn / 2));
  JAGG_TRY(fp8_scale_map(&maps.as, g.a, g.M, g.K, 128, SCALE_KB));
  maps.c = maps.bs = maps.as;  // unused ones
  if (QVEC) JAGG_TRY(fp8_scale_map(&maps.bs, g.b, g.N, g.K, W_MAX_N, SCALE_KB));
  if (p.c_tma) {
    const uint64_t dims[2] = {(uint64_t)g.N, (uint64_t)g.M};
    const uint64_t strides[1] = {(uint64_t)g.ldc * fp8::size_of(g.c_dtype)};
    const uint32_t box[2] = {(uint32_t)(Cfg::ROW / fp8::size_of(g.c_dtype)), 32u};
    JAGG_TRY(encode_tmap(&maps.c, p.c_f32, 2, g.C, dims, strides, box,
                         Cfg::ROW == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_32B));
  }
  auto kernel = gemm_fp8_pair_kernel<QVEC>;
  static OncePerDevice once;
  JAGG_CUDA_TRY(allow_smem(once, kernel, Cfg::SMEM));
  const int64_t tiles = (int64_t)p.tiles_m * p.tiles_n;
  const int np = sm_count() / 2;
  JAGG_CUDA_TRY(launch(kernel, 2 * (int)(tiles < np ? tiles : np), W_THREADS, Cfg::SMEM, s, maps, p));
  JAGG_LAUNCHED();
  return JAGG_OK;
}

}  // namespace

int gemm_fp8_pair(const GemmFp8Args& g, int bn, cudaStream_t s) {
  return g.b.block ? launch_w8<false>(g, bn, s) : launch_w8<true>(g, bn, s);
}

}  // namespace jagg
