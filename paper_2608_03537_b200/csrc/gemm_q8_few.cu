// The 8-bit integer product for few rows: Y = act(sa sb (A . B^T) + bias) + R.
//
// What bounds it: the weights' bytes, and for small layers the latency of one pass.  As in the bf16 form for few rows the product is turned
// round: the weights are the UMMA's 128-row operand, the rows its N operand (MT = 16 .. 128), so a CTA computes 128 channels of MT rows
// and the tensor core's work follows the rows that exist.  A cluster of `split` CTAs shares a tile's contraction.  Their int32
// accumulators go to shared memory as [row][channel]; behind a cluster barrier each CTA adds its slice of the rows from all of them through
// distributed shared memory and finishes it, a warp per row and 4 channels per lane.  Integer sums are exact, so the split changes no bit
// of the result.
#include <algorithm>
#include <cstdio>
#include <type_traits>

#include "q8_common.cuh"
#include "q8_params.h"

namespace comfuse {
namespace {

template <int MT>
struct FewCfg {
  static constexpr int kEpiWarps = 8;
  static constexpr int kThreads = 32 * (2 + kEpiWarps);
  static constexpr int W_BYTES = 128 * 128;  // weights of one K block: 128 channels x 128 bytes
  static constexpr int X_BYTES = MT * 128;
  static constexpr int STAGE_BYTES = W_BYTES + X_BYTES;
  static constexpr int MISC_BYTES = 256 + 1024;
  // The ring takes all of an SM: its depth is worth more than a second CTA beside it, which would even out the SMs' shares (40 x 4096 x 4096 with
  // 9 stages 7.7 us, with 4 stages and two CTAs an SM 8.8; 64 x 4096 x 16384 15.6 / 18.5; 40 x 16384 x 4096 14.9 / 15.6).
  static constexpr int NSTAGES = (232448 - MISC_BYTES) / STAGE_BYTES > 10 ? 10 : (232448 - MISC_BYTES) / STAGE_BYTES;
  static constexpr int ASK = 8;  // 128 KB of weights
  static constexpr int OFF_BAR = NSTAGES * STAGE_BYTES;
  static constexpr int SMEM_BYTES = OFF_BAR + MISC_BYTES;
  static constexpr int ROW_BYTES = 128 * 4;  // one row of the tile's accumulators
  static constexpr int TMEM_COLS = MT <= 32 ? 32 : MT;
  static_assert(MT * ROW_BYTES <= NSTAGES * STAGE_BYTES, "the accumulators are staged in the idle ring");
  static_assert((2 * NSTAGES + 1) * 8 + 16 <= 256, "barrier room");
  static_assert(SMEM_BYTES <= 232448 && SMEM_BYTES > 116 * 1024, "one CTA per SM (tensor-memory allocation never waits)");
};

template <int DT, int MT>
__global__ void __launch_bounds__(FewCfg<MT>::kThreads, 1) gemm_q8_few_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmX,
                                                                          const GemmQ8Params p) {
  using Cfg = FewCfg<MT>;
  constexpr int NSTAGES = Cfg::NSTAGES;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw_addr = smem_u32(smem_raw);
  const uint32_t smem_base = (raw_addr + 1023u) & ~1023u;
  uint8_t* smem = smem_raw + (smem_base - raw_addr);
  const uint32_t bar_base = smem_base + Cfg::OFF_BAR;
  auto bar_full = [&](int s) { return bar_base + 8u * s; };
  auto bar_empty = [&](int s) { return bar_base + 8u * (NSTAGES + s); };
  const uint32_t bar_acc = bar_base + 8u * (2 * NSTAGES);  // accumulators complete
  uint32_t* s_tmem_base = reinterpret_cast<uint32_t*>(smem + Cfg::OFF_BAR + (2 * NSTAGES + 1) * 8);
  volatile int* s_abort = reinterpret_cast<volatile int*>(s_tmem_base + 1);
  volatile int* s_issued = s_abort + 1;  // K blocks whose loads are issued (fewer than all where the producer's wait expires)

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = static_cast<int>(blockIdx.x % p.split);  // share of the contraction, and slice of the rows in the epilogue
  const int tile = static_cast<int>(blockIdx.x / p.split);
  const int nt = tile % p.ntiles, grp = (tile / p.ntiles) % p.mtiles, b = tile / (p.ntiles * p.mtiles);
  const int n0 = nt * 128, m0 = grp * MT;
  const int rows = p.M - m0 < MT ? p.M - m0 : MT;
  const int KB = (p.K + 127) >> 7;
  const int kb0 = static_cast<int>(static_cast<long long>(KB) * rank / p.split), kb1 = static_cast<int>(static_cast<long long>(KB) * (rank + 1) / p.split);
  const WaitCtx w{s_abort, p.status, p.timeout_ns};
  griddep_launch_dependents();  // the next kernel's set-up may overlap this kernel (it waits before touching memory)

  if (threadIdx.x == 0) {
    for (int s = 0; s < NSTAGES; ++s) {
      mbar_init(bar_full(s), 1);
      mbar_init(bar_empty(s), 1);
    }
    mbar_init(bar_acc, 1);
    *s_abort = 0;
    *s_issued = kb1 - kb0;
    fence_mbar_init();
    prefetch_tensormap(&tmW);
    prefetch_tensormap(&tmX);
  }
  // The weights are asked of the L2 while the previous kernel may still run (a prefetch returns nothing, so it may stand in front of the wait
  // whoever writes them: writes meet in the L2 too): 128 KB a CTA, by one group of rows.  us with weights from memory, without / with: 8 x 4096 x 4096
  // 7.0 / 6.8, 40 x 16384 x 4096 14.9 / 14.7, 64 x 1024 x 4096 6.3 / 6.0; 128 rows 10.7 / 10.9, so not there.
  if (MT <= 64 && warp == 2 && grp == 0 && elect_one()) {
#pragma unroll 1
    for (int kb = kb0; kb < kb1 && kb < kb0 + Cfg::ASK; ++kb) tma_prefetch_l2_3d(&tmW, kb * 128, n0, b);
  }
  if (warp == 1) {
    tmem_alloc(smem_u32(s_tmem_base), Cfg::TMEM_COLS);
    tmem_relinquish_alloc_permit();
  }
  tcgen05_fence_before_sync();
  __syncthreads();
  tcgen05_fence_after_sync();
  const uint32_t tmem_base = *s_tmem_base;
  griddep_wait();

  // Epilogue: a warp finishes every 8th row of the CTA's slice, a lane 4 channels of it.  RB rows advance together: what they need from
  // global memory is asked for at once, for the first RB while the products still run.
  constexpr int RB = 4;
  const int rs = (rows + p.split - 1) / p.split;  // rows per slice
  const int row1 = (rank + 1) * rs < rows ? (rank + 1) * rs : rows;
  int row = rank * rs + warp - 2;
  const int col = n0 + 4 * lane;
  const bool whole = col + 4 <= p.N;
  const float* scale_a = p.scale_a + static_cast<long long>(b) * p.M + m0;
  const char* res = static_cast<const char*>(p.residual) + (b * p.batch_stride_r + m0 * p.ldr + col) * Elem<DT>::kBytes;
  char* out = static_cast<char*>(p.Y) + (b * p.batch_stride_y + m0 * p.ldy + col) * Elem<DT>::kBytes;
  float sa[RB], sb[4], bias[4];
  uint32_t rw[RB][Elem<DT>::kBytes];
  auto fetch = [&]() {
#pragma unroll
    for (int k = 0; k < RB; ++k) {
      const int r = row + k * Cfg::kEpiWarps;
      if (r < row1) {
        sa[k] = scale_a[r];
        if (p.residual) {
          const char* from = res + r * p.ldr * Elem<DT>::kBytes;
          if (whole) {
            if constexpr (Elem<DT>::kBytes == 4) ld_16(from, rw[k]);
            else ld_8(from, rw[k]);
          } else {
            float e[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) e[i] = col + i < p.N ? Elem<DT>::get(from, i) : 0.f;
            Elem<DT>::pack(e, rw[k]);
          }
        }
      }
    }
  };

  if (warp == 0) {
    // ------------------------------------------------------------------------------------------ TMA producer
    if (elect_one()) {
      int stage = 0;
      uint32_t phase = 0;
      for (int kb = kb0; kb < kb1; ++kb) {
        if (!mbar_wait<false>(bar_empty(stage), phase ^ 1u, w)) {  // passes on a fresh barrier
          *s_issued = kb - kb0;
          break;
        }
        const uint32_t sw = smem_base + stage * Cfg::STAGE_BYTES;
        mbar_arrive_expect_tx(bar_full(stage), Cfg::STAGE_BYTES);
        tma_load_3d(sw, &tmW, bar_full(stage), kb * 128, n0, b);
        tma_load_3d(sw + Cfg::W_BYTES, &tmX, bar_full(stage), kb * 128, m0, b);
        if (++stage == NSTAGES) { stage = 0; phase ^= 1u; }
      }
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------------------------------------ UMMA issuer
    if (elect_one()) {
      int stage = 0;
      uint32_t phase = 0;
      constexpr uint32_t idesc = make_idesc_i8(128, MT);
      for (int kb = kb0; kb < kb1; ++kb) {
        if (!mbar_wait<false>(bar_full(stage), phase, w)) break;
        tcgen05_fence_after_sync();
        const uint32_t sw = smem_base + stage * Cfg::STAGE_BYTES;
        const uint64_t wdesc = make_smem_desc_sw128(sw, 16, 1024), xdesc = make_smem_desc_sw128(sw + Cfg::W_BYTES, 16, 1024);
#pragma unroll
        for (int k = 0; k < 4; ++k)  // 32 bytes of the contraction an instruction
          umma_i8_ss(tmem_base, wdesc + static_cast<uint64_t>(2 * k), xdesc + static_cast<uint64_t>(2 * k), idesc, (kb != kb0 || k != 0) ? 1u : 0u);
        umma_commit(bar_empty(stage));
        if (++stage == NSTAGES) { stage = 0; phase ^= 1u; }
      }
      umma_commit(bar_acc);
      mbar_drain(bar_acc, 0, w);  // nothing may still be writing tensor memory when it is freed
    }
  } else {
    const int q = warp & 3, half = (warp - 2) >> 2;  // TMEM lane quarter; which half of the rows this warp moves to shared memory
    constexpr int MOVE = MT / 2, STEP = MOVE < 16 ? 8 : 16;
    fetch();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      sb[i] = col + i < p.N ? p.scale_b[static_cast<long long>(b) * p.N + col + i] : 0.f;
      bias[i] = p.bias && col + i < p.N ? Elem<DT>::get(p.bias, col + i) : 0.f;
    }
    mbar_wait<false>(bar_acc, 0, w);
    __syncwarp();
    tcgen05_fence_after_sync();
    // accumulators -> [row][channel] in the ring, which nothing uses any more (every load has landed and has been multiplied)
    const uint32_t dst = smem_base + static_cast<uint32_t>((q * 32 + lane) * 4);
#pragma unroll 2
    for (int i = half * MOVE; i < (half + 1) * MOVE && i < rows; i += STEP) {
      uint32_t v[STEP];
      const uint32_t taddr = tmem_base + (static_cast<uint32_t>(q * 32) << 16) + i;
      if constexpr (STEP == 16) {
        tmem_ld_issue_16(taddr, v);
        tmem_ld_wait_16(v);
      } else {
        tmem_ld_issue_8(taddr, v);
        tmem_ld_wait_8(v);
      }
#pragma unroll
      for (int k = 0; k < STEP; ++k)
        if (i + k < rows) asm volatile("st.shared.b32 [%0], %1;" ::"r"(dst + (i + k) * Cfg::ROW_BYTES), "r"(v[k]) : "memory");
    }
  }
  __syncwarp();
  if (p.split > 1) cluster_sync_all();  // everyone's shares are in place
  else __syncthreads();

  if (warp >= 2) {
    while (row < row1) {
      int acc[RB][4] = {};
      for (int s = 0; s < p.split; ++s) {
        const uint32_t src = smem_base + static_cast<uint32_t>(row * Cfg::ROW_BYTES + lane * 16);
        const uint32_t at = p.split > 1 ? map_to_cta(src, static_cast<uint32_t>(s)) : src;
#pragma unroll
        for (int k = 0; k < RB; ++k) {
          if (row + k * Cfg::kEpiWarps >= row1) continue;
          int o[4];
          asm volatile("ld.shared::cluster.v4.s32 {%0, %1, %2, %3}, [%4];"
                       : "=r"(o[0]), "=r"(o[1]), "=r"(o[2]), "=r"(o[3])
                       : "r"(at + static_cast<uint32_t>(k * Cfg::kEpiWarps * Cfg::ROW_BYTES))
                       : "memory");
#pragma unroll
          for (int i = 0; i < 4; ++i) acc[k][i] += o[i];
        }
      }
#pragma unroll
      for (int k = 0; k < RB; ++k) {
        const int r = row + k * Cfg::kEpiWarps;
        if (r >= row1) break;
        float z[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) z[i] = fmaf(static_cast<float>(acc[k][i]) * sb[i], sa[k], bias[i]);
        activate(z, p.activation);
        char* to = out + r * p.ldy * Elem<DT>::kBytes;
        if (p.residual) {
#pragma unroll
          for (int i = 0; i < 4; ++i) z[i] += Elem<DT>::of(rw[k], i);
        }
        if (whole) {
          uint32_t ow[Elem<DT>::kBytes];
          Elem<DT>::pack(z, ow);
          if (COMFUSE_IN_BOUNDS(m0 + r < p.M && col + 3 < p.N && b < p.batch, p.status)) {
            if constexpr (Elem<DT>::kBytes == 4) st_16(to, ow);
            else st_8(to, ow);
          }
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (col + i < p.N && COMFUSE_IN_BOUNDS(m0 + r < p.M && b < p.batch, p.status)) Elem<DT>::put(to, i, z[i]);
        }
      }
      row += RB * Cfg::kEpiWarps;
      fetch();
    }
  }

  // -------------------------------------------------------------------------------------------- teardown
  tcgen05_fence_before_sync();
  __syncwarp();
  if (p.split > 1) cluster_sync_all();  // no CTA leaves while another still reads its shared memory
  else __syncthreads();
  if (warp == 1) {
    tcgen05_fence_after_sync();
    tmem_release<false>(tmem_base, Cfg::TMEM_COLS);
  }
  if (warp == 0 && lane == 0 && *s_abort) {  // a wait expired: loads may still be on their way into this CTA's shared memory
    const int issued = *s_issued;
    for (int u = issued > NSTAGES ? issued - NSTAGES : 0; u < issued; ++u) mbar_drain(bar_full(u % NSTAGES), (u / NSTAGES) & 1u, w);
  }
}

template <int DT, int MT>
cudaError_t launch_instance(const CUtensorMap& tmW, const CUtensorMap& tmX, const GemmQ8Params& p, cudaStream_t stream) {
  using Cfg = FewCfg<MT>;
  auto kern = gemm_q8_few_kernel<DT, MT>;
  const DeviceInfo* dev = current_device_info();
  if (!dev) return cudaErrorInvalidDevice;
  constexpr int kMaxDev = 64;
  static std::atomic<bool> ready[kMaxDev];  // set (released) once the kernel's attributes are in place on that device
  const int di = dev->device < kMaxDev ? dev->device : kMaxDev - 1;
  if (!ready[di].load(std::memory_order_acquire)) {
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg::SMEM_BYTES);
    if (e != cudaSuccess) return e;
    ready[di].store(true, std::memory_order_release);
  }
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[2];
  cfg.gridDim = dim3(static_cast<unsigned>(p.tiles * p.split), 1, 1);
  cfg.blockDim = dim3(Cfg::kThreads, 1, 1);
  cfg.dynamicSmemBytes = Cfg::SMEM_BYTES;
  cfg.stream = stream;
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = static_cast<unsigned>(p.split);
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;  // set-up may overlap the previous kernel's tail
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = programmatic_launch_enabled() ? 2 : 1;
  count_launch();
  return cudaLaunchKernelEx(&cfg, kern, tmW, tmX, p);
}

template <int DT>
cudaError_t launch_rows(int rows, const CUtensorMap& tmW, const CUtensorMap& tmX, const GemmQ8Params& p, cudaStream_t stream) {
  switch (rows) {
    case 16: return launch_instance<DT, 16>(tmW, tmX, p, stream);
    case 32: return launch_instance<DT, 32>(tmW, tmX, p, stream);
    case 64: return launch_instance<DT, 64>(tmW, tmX, p, stream);
    default: return launch_instance<DT, 128>(tmW, tmX, p, stream);
  }
}

}  // namespace

GemmQ8FewPlan gemm_q8_few_plan(int batch, int M, int N, int K, bool long_epilogue, const DeviceInfo& dev) {
  // Both this form's cut and the choice between it and the tile kernel by estimates of their times in us, fitted to 4238 cuts of 368 calls (20 .. 400
  // rows, 128 .. 16384 channels, 128 .. 16384 codes a row; the cut that they choose is 1 % above the fastest cut of this form on average, 11 % at worst).
  // Between the forms, against fixed groups of rows: 956 calls 13 % faster in the geometric mean, some slower (47 x 3593 x 3268 fp32 8.0 -> 9.1 us, 938 x 530 x
  // 4655 14.1 -> 15.5, 82 x 13169 x 112 7.7 -> 8.3).
  //   * A CTA does one tile and the next one's set-up starts behind it, so a round of tiles costs its whole latency: set-up, the rows' epilogue, the K
  //     blocks, and, where shares meet, the cluster's barriers.  Groups of 16 rows read the weights again for each group, out of the L2; small weights
  //     are cheaper to read often than their epilogue is to do in one CTA: us with 16 / 64 rows a CTA, 64 x 1024 x 128 3.0 / 4.7, 64 x 1024 x 1024 4.0 / 5.0.
  //   * Shares keep 4 K blocks each, and more clusters than fit at once are another round (16 of 8 CTAs do not fit: 256 x 1024 x 8192 17.4 as
  //     those, 8.7 as 32 of 4).
  //   * The tile kernel is persistent: many short tiles are cheaper there (96 x 40 x 1024 x 64 15.4 us, 26.6 here; 64 x 4096 x 8192 17.4, 10.1 here).
  GemmQ8FewPlan c;
  const int KB = (K + 127) / 128;
  const long long ntiles = static_cast<long long>(batch) * ((N + 127) / 128);
  static ResidentClusters resident;  // (every instance has an SM to itself)
  double best = 1e30;
  for (const int rows : {16, 32, 64, 128}) {
    if (rows > 16 && M <= rows / 2) break;
    const long long tiles = ntiles * ((M + rows - 1ll) / rows);
    for (const int split : {1, 2, 3, 4, 6, 8}) {
      if (split > 1 && (split * 4 > KB || tiles * split > dev.sm_count)) break;
      int at_once = dev.sm_count;
      if (split > 1)
        at_once = std::max(1, resident.of(reinterpret_cast<const void*>(gemm_q8_few_kernel<COMFUSE_DTYPE_BF16, 64>), FewCfg<64>::kThreads, FewCfg<64>::SMEM_BYTES, split, dev));
      const double rounds = static_cast<double>((tiles + at_once - 1) / at_once);
      double us = rounds * (2.3 + (long_epilogue ? 0.06 : 0.032) * std::min(M, rows) + 0.144 * ((KB + split - 1) / split)) + 1.6e-8 * tiles * (128. + rows) * K;
      if (split > 1) us += 1.2 * rounds + 0.6 * static_cast<double>(tiles * split) / dev.sm_count;
      if (us < best && tiles * split <= 0x7FFFFFFF) {  // (a grid is counted in 32 bits)
        best = us;
        c.rows = rows;
        c.split = split;
      }
    }
  }
  const bool narrow = gemm_q8_pair_columns(batch, M, N, dev) == 128;
  const long long there = static_cast<long long>(batch) * ((M + 255ll) / 256) * (narrow ? (N + 127) / 128 : (N + 255) / 256), pairs = dev.sm_count / 2;
  const double round = narrow ? std::max(0.26 * KB, 1.55) : std::max(0.35 * KB + 0.65, long_epilogue ? 3.9 : 2.0);
  const double around = narrow ? (long_epilogue ? 4.3 : 2.8) : 3.5;
  if (best >= around + round * static_cast<double>((there + pairs - 1) / pairs)) c.rows = 0;
  return c;
}

cudaError_t launch_gemm_q8_few(int dtype, const GemmQ8FewPlan& plan, const CUtensorMap& tmW, const CUtensorMap& tmX, GemmQ8Params p, cudaStream_t stream) {
  p.split = plan.split;
  p.mtiles = (p.M + plan.rows - 1) / plan.rows;
  p.ntiles = (p.N + 127) / 128;
  p.tiles = static_cast<long long>(p.batch) * p.mtiles * p.ntiles;
  if (verbose_enabled())
    std::fprintf(stderr, "comfuse: gemm_q8 dtype=%d: few rows, rows=%d shares=%d long_epilogue=%d\n", dtype, plan.rows, plan.split,
                 p.residual || (p.activation != 0 && p.activation != COMFUSE_OP_RELU));
  switch (dtype) {
    case COMFUSE_DTYPE_BF16: return launch_rows<COMFUSE_DTYPE_BF16>(plan.rows, tmW, tmX, p, stream);
    case COMFUSE_DTYPE_F16: return launch_rows<COMFUSE_DTYPE_F16>(plan.rows, tmW, tmX, p, stream);
    default: return launch_rows<COMFUSE_DTYPE_F32>(plan.rows, tmW, tmX, p, stream);
  }
}

}  // namespace comfuse
