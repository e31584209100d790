// The 8-bit integer product for many rows: Y = act(sa sb (A . B^T) + bias) + R, on CTA pairs.
//
// What bounds it: the tensor cores (int8 at twice the bf16 rate), and behind short contractions the bytes of Y.  As in the bf16 tile
// kernel two CTAs multiply a 256 x BN tile (cta_group::2): each holds its own 128 rows of A and half of B's BN (256, or 128 where that fills
// more SMs).  Clusters of two are persistent and walk the tiles in bands of 8 row blocks, so that the tiles in flight share their
// operands in the L2.  Two accumulators alternate: a tile's epilogue runs under the next one's products.
//
// Epilogue: thread = one row of the tile, 32 columns (16 with sixteen warps in fp32) at a time, a warp half or a quarter of the columns.  The
// channel's scale and bias come from shared memory (broadcast), the row's scale is a register.  Results leave as boxes of 32 rows x 128 bytes
// staged in shared memory and stored by TMA; the residual comes in the same way, into the box that its sum leaves from.  A TMA store writes whole 16-byte units (measured: up to
// seven bf16 behind the last column), so Y's map ends at the last whole unit and the columns behind it are stored one by one.
#include <algorithm>
#include <cstdio>
#include <type_traits>

#include "q8_common.cuh"
#include "q8_params.h"

namespace comfuse {
namespace {

template <int DT, int BN, int STAGES, int BOXES, int EPW>
struct PairQ8Cfg {
  static constexpr int NSTAGES = STAGES;
  static constexpr int kEpiWarps = 4 * EPW;  // EPW for each quarter of the accumulator's lanes
  static constexpr int kThreads = 32 * (2 + kEpiWarps);
  static constexpr int A_BYTES = 128 * 128;              // 128 rows of A x 128 bytes
  static constexpr int STAGE_BYTES = A_BYTES + BN / 2 * 128;
  static constexpr int BOX_BYTES = 32 * 128;
  static constexpr int OFF_BOX = NSTAGES * STAGE_BYTES;  // BOXES staging boxes a warp
  static constexpr int COLS = BN / EPW;                  // of a tile, for one epilogue warp
  static constexpr int VEC_BYTES = COLS * (4 + Elem<DT>::kBytes);  // their scales and biases, each warp's own
  static constexpr int OFF_VEC = OFF_BOX + kEpiWarps * BOXES * BOX_BYTES;
  static constexpr int OFF_BAR = OFF_VEC + kEpiWarps * VEC_BYTES;
  static constexpr int NUM_BARS = 2 * NSTAGES + 5 + kEpiWarps * BOXES;
  static constexpr int OFF_MISC = OFF_BAR + NUM_BARS * 8;
  static constexpr int SMEM_BYTES = OFF_MISC + 16 + 1024;
  static_assert(STAGE_BYTES % 1024 == 0, "swizzled tiles start on 1024-byte boundaries");
  static_assert(SMEM_BYTES <= 232448 && SMEM_BYTES > 116 * 1024, "one CTA per SM");
};

template <int DT, int BN, int STAGES, int BOXES, int EPW>
__global__ void __launch_bounds__(PairQ8Cfg<DT, BN, STAGES, BOXES, EPW>::kThreads, 1)
gemm_q8_pair_kernel(const __grid_constant__ GemmQ8PairMaps maps, const GemmQ8Params p) {
  using Cfg = PairQ8Cfg<DT, BN, STAGES, BOXES, EPW>;
  constexpr int NSTAGES = Cfg::NSTAGES;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw_addr = smem_u32(smem_raw);
  const uint32_t smem_base = (raw_addr + 1023u) & ~1023u;
  uint8_t* smem = smem_raw + (smem_base - raw_addr);
  const uint32_t bar_base = smem_base + Cfg::OFF_BAR;
  auto bar_full = [&](int s) { return bar_base + 8u * s; };                     // both CTAs' halves of a K block landed (even CTA)
  auto bar_empty = [&](int s) { return bar_base + 8u * (NSTAGES + s); };        // stage may be overwritten
  auto bar_tfull = [&](int a) { return bar_base + 8u * (2 * NSTAGES + a); };    // accumulator complete
  auto bar_tempty = [&](int a) { return bar_base + 8u * (2 * NSTAGES + 2 + a); };  // accumulator read by both CTAs' epilogue warps (even CTA)
  const uint32_t bar_drain = bar_base + 8u * (2 * NSTAGES + 4);
  auto bar_res = [&](int e, uint32_t k) { return bar_drain + 8u + 8u * (e * BOXES + k); };  // residual box k of epilogue warp e landed
  uint32_t* s_tmem_base = reinterpret_cast<uint32_t*>(smem + Cfg::OFF_MISC);
  volatile int* s_abort = reinterpret_cast<volatile int*>(s_tmem_base + 1);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();  // which half of the pair
  const uint32_t cluster_id = blockIdx.x >> 1, clusters = gridDim.x >> 1, tiles = static_cast<uint32_t>(p.tiles);  // (the host keeps them below 2^31)
  const int KB = (p.K + 127) >> 7;
  const WaitCtx w{s_abort, p.status, p.timeout_ns};
  griddep_launch_dependents();  // the next kernel's set-up may overlap this kernel (it waits before touching memory)

  if (threadIdx.x == 0) {
    for (int s = 0; s < NSTAGES; ++s) {
      mbar_init(bar_full(s), 2);   // one arrive.expect_tx from each CTA of the pair
      mbar_init(bar_empty(s), 1);  // one commit from the issuing CTA
    }
    for (int a = 0; a < 2; ++a) {
      mbar_init(bar_tfull(a), 1);
      mbar_init(bar_tempty(a), 2 * Cfg::kEpiWarps);
    }
    mbar_init(bar_drain, 1);
    for (int e = 0; e < Cfg::kEpiWarps; ++e)
      for (uint32_t k = 0; k < BOXES; ++k) mbar_init(bar_res(e, k), 1);
    *s_abort = 0;
    fence_mbar_init();
    prefetch_tensormap(&maps.A);
    prefetch_tensormap(&maps.B);
    prefetch_tensormap(&maps.Y);
    if (p.residual) prefetch_tensormap(&maps.R);
  }
  if (warp == 1) {
    tmem_alloc_pair(smem_u32(s_tmem_base), 2 * BN);
    tmem_relinquish_alloc_permit_pair();
  }
  tcgen05_fence_before_sync();
  __syncthreads();
  tcgen05_fence_after_sync();
  cluster_sync_after_init();  // both CTAs' barriers exist before either signals them
  const uint32_t tmem_base = *s_tmem_base;
  griddep_wait();

  // tile -> batch, first row and column: bands of 8 row blocks, in a band column by column
  auto decode = [&](uint32_t tile, int& b, int& m0, int& n0) {
    const uint32_t per = static_cast<uint32_t>(p.mtiles) * static_cast<uint32_t>(p.ntiles), bt = tile / per, t = tile - bt * per;
    const uint32_t size = 8u * static_cast<uint32_t>(p.ntiles), band = t / size, in_band = t - band * size, first = band * 8;
    const uint32_t high = p.mtiles - first < 8 ? p.mtiles - first : 8, column = in_band / high;
    b = static_cast<int>(bt);
    n0 = static_cast<int>(column) * BN;
    m0 = static_cast<int>(first + in_band - column * high) * 256;
  };

  if (warp == 0) {
    // ------------------------------------------------------------------------------------------ TMA producer
    if (elect_one()) {
      int stage = 0;
      uint32_t phase = 0;
      bool ok = true;
      for (uint32_t tile = cluster_id; tile < tiles && ok; tile += clusters) {
        int b, m0, n0;
        decode(tile, b, m0, n0);
        for (int kb = 0; kb < KB; ++kb) {
          if (!mbar_wait<false>(bar_empty(stage), phase ^ 1u, w)) { ok = false; break; }  // passes on a fresh barrier
          const uint32_t sa = smem_base + stage * Cfg::STAGE_BYTES, full = map_to_cta(bar_full(stage), 0);
          mbar_arrive_expect_tx_cluster(full, Cfg::STAGE_BYTES);
          tma_load_3d_pair(sa, &maps.A, full, kb * 128, m0 + static_cast<int>(rank) * 128, b);
          tma_load_3d_pair(sa + Cfg::A_BYTES, &maps.B, full, kb * 128, n0 + static_cast<int>(rank) * (BN / 2), b);
          if (++stage == NSTAGES) { stage = 0; phase ^= 1u; }
        }
      }
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------------------------------------ UMMA issuer (even CTA)
    if (rank == 0 && elect_one()) {
      int stage = 0;
      uint32_t phase = 0, n = 0;
      bool ok = true;
      constexpr uint32_t idesc = make_idesc_i8(256, BN);
      for (uint32_t tile = cluster_id; tile < tiles && ok; tile += clusters, ++n) {
        const uint32_t slot = n & 1u;
        if (!mbar_wait<false>(bar_tempty(slot), ((n >> 1) & 1u) ^ 1u, w)) break;
        tcgen05_fence_after_sync();
        for (int kb = 0; kb < KB; ++kb) {
          if (!mbar_wait<false>(bar_full(stage), phase, w)) { ok = false; break; }
          tcgen05_fence_after_sync();
          const uint32_t sa = smem_base + stage * Cfg::STAGE_BYTES;
          const uint64_t adesc = make_smem_desc_sw128(sa, 16, 1024), bdesc = make_smem_desc_sw128(sa + Cfg::A_BYTES, 16, 1024);
#pragma unroll
          for (int k = 0; k < 4; ++k)  // 32 bytes of the contraction an instruction
            umma_i8_ss_pair(tmem_base + slot * BN, adesc + static_cast<uint64_t>(2 * k), bdesc + static_cast<uint64_t>(2 * k), idesc, (kb | k) != 0 ? 1u : 0u);
          umma_commit_pair_both(bar_empty(stage));  // the stage is free in both CTAs once these have read it
          if (++stage == NSTAGES) { stage = 0; phase ^= 1u; }
        }
        if (ok) umma_commit_pair_both(bar_tfull(slot));
      }
      umma_commit_pair(bar_drain);  // nothing may still be writing either CTA's tensor memory when it is freed
      mbar_drain(bar_drain, 0, w);
    }
  } else {
    // ------------------------------------------------------------------------------------------ epilogue warps
    const int e = warp - 2, q = warp & 3, part = e >> 2;  // TMEM lane quarter: rows 32q ..; which part of the columns
    // columns at a time (sixteen warps in fp32: what their registers hold; 16 bits with 16 columns 8192 x 4096 x 64 19.2 us, with 32 18.2)
    constexpr int S = EPW == 4 && Elem<DT>::kBytes == 4 ? 16 : 32;
    constexpr int E = 128 / Elem<DT>::kBytes;               // columns of a box
    const uint32_t lane_addr = tmem_base + (static_cast<uint32_t>(q * 32) << 16) + part * Cfg::COLS;
    const uint32_t tempty = map_to_cta(bar_tempty(0), 0);
    const uint32_t box0 = smem_base + Cfg::OFF_BOX + e * BOXES * Cfg::BOX_BYTES;
    using Word = typename Elem<DT>::Word;
    const int whole = gemm_q8_stored_columns(DT, p.N);  // by TMA
    uint32_t n = 0, count = 0;  // tiles, and boxes of this warp
    // What a tile needs from global memory is asked for under the tile before: scales and biases of the warp's channels, the row's scale.  Every warp
    // keeps its own copy, so that the warps need not meet between tiles and one's arithmetic runs beside another's stores (with one copy
    // for all and a barrier a tile: 96 x 504 x 504 x 64 fp32 23.3 us for 22.2, 8192 x 4096 x 512 with GELU 36.5 for 33.1).
    constexpr int C = Cfg::COLS / 32;  // channels a lane fetches
    float* s_scale = reinterpret_cast<float*>(smem + Cfg::OFF_VEC + e * Cfg::VEC_BYTES);
    Word* s_bias = reinterpret_cast<Word*>(s_scale + Cfg::COLS);
    int b = 0, m0 = 0, n0 = 0;
    float sa = 0.f;
    float scale[C];
    Word bias[C];
    auto fetch = [&](uint32_t tile) {
      if (tile >= tiles) return;
      decode(tile, b, m0, n0);
      const int row = m0 + static_cast<int>(rank) * 128 + q * 32 + lane;
      sa = row < p.M ? p.scale_a[static_cast<long long>(b) * p.M + row] : 0.f;
#pragma unroll
      for (int i = 0; i < C; ++i) {
        const int c = n0 + part * Cfg::COLS + 32 * i + lane;
        scale[i] = c < p.N ? p.scale_b[static_cast<long long>(b) * p.N + c] : 0.f;
        bias[i] = p.bias && c < p.N ? static_cast<const Word*>(p.bias)[c] : static_cast<Word>(0);
      }
    };
    fetch(cluster_id);
    for (uint32_t tile = cluster_id; tile < tiles; tile += clusters, ++n) {
      const uint32_t slot = n & 1u;
      __syncwarp();  // (the tile before is read)
#pragma unroll
      for (int i = 0; i < C; ++i) {
        s_scale[32 * i + lane] = scale[i];
        s_bias[32 * i + lane] = bias[i];
      }
      const int tb = b, row0 = m0 + static_cast<int>(rank) * 128 + q * 32, col0 = n0 + part * Cfg::COLS;
      const float tsa = sa;
      fetch(tile + clusters);
      const int left = row0 < p.M && col0 < p.N ? (p.N - col0 + E - 1) / E : 0;
      const int boxes = left < Cfg::COLS / E ? left : Cfg::COLS / E;  // that hold anything of Y
      // box k of this tile: once its staging box has been read out by the store before last, ask for the residual
      auto ask = [&](int k) {
        if (lane == 0 && p.residual && k < boxes) {
          if (k == 0 || BOXES == 1) tma_store_wait_read<BOXES - 1>();
          else tma_store_wait_read<BOXES - 2 < 0 ? 0 : BOXES - 2>();
          const uint32_t sel = (count + k) % BOXES;
          mbar_arrive_expect_tx(bar_res(e, sel), Cfg::BOX_BYTES);
          tma_load_3d(box0 + sel * Cfg::BOX_BYTES, &maps.R, bar_res(e, sel), col0 + k * E, row0, tb);
        }
      };
      ask(0);
      const bool ok = mbar_wait<false>(bar_tfull(slot), (n >> 1) & 1u, w);
      __syncwarp();
      tcgen05_fence_after_sync();
      auto release = [&]() {  // the accumulator is read: it may be overwritten once everyone is here
        tcgen05_fence_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster_noflush(tempty + 8u * slot);
      };
      if (boxes == 0) release();
#pragma unroll 1
      for (int k = 0; k < boxes; ++k) {
        const uint32_t sel = (count + k) % BOXES, row_addr = box0 + sel * Cfg::BOX_BYTES + lane * 128;
        if (BOXES > 1) ask(k + 1);
        else if (k > 0) ask(k);
#pragma unroll
        for (int h = 0; h < E / S; ++h) {
          const int local = k * E + h * S;  // of the warp's columns
          uint32_t v[S];
#pragma unroll
          for (int j = 0; j < S; j += 16) tmem_ld_issue_16(lane_addr + slot * BN + k * E + h * S + j, v + j);
#pragma unroll
          for (int j = 0; j < S; j += 16) tmem_ld_wait_16(v + j);
          if (k == boxes - 1 && h == E / S - 1) release();
          float z[S];
#pragma unroll
          for (int j = 0; j < S; j += 4) {
            const float4 sv = *reinterpret_cast<const float4*>(s_scale + local + j);
            uint32_t bw[Elem<DT>::kBytes];
            if constexpr (Elem<DT>::kBytes == 4) {
              const uint4 bv = *reinterpret_cast<const uint4*>(s_bias + local + j);
              bw[0] = bv.x; bw[1] = bv.y; bw[2] = bv.z; bw[3] = bv.w;
            } else {
              const uint2 bv = *reinterpret_cast<const uint2*>(s_bias + local + j);
              bw[0] = bv.x; bw[1] = bv.y;
            }
            const float f[4] = {sv.x, sv.y, sv.z, sv.w};
#pragma unroll
            for (int u = 0; u < 4; ++u) z[j + u] = fmaf(static_cast<float>(static_cast<int>(v[j + u])) * f[u], tsa, Elem<DT>::of(bw, u));
          }
          activate(z, p.activation);
          if (h == 0) {  // the staging box is this warp's again
            if (p.residual) {
              mbar_wait<false>(bar_res(e, sel), ((count + k) / BOXES) & 1u, w);
            } else if (lane == 0) {
              tma_store_wait_read<BOXES - 1>();
            }
            __syncwarp();
          }
          constexpr int kChunks = S * Elem<DT>::kBytes / 16;
          uint32_t at[kChunks];
#pragma unroll
          for (int c = 0; c < kChunks; ++c) at[c] = row_addr + (((h * kChunks + c) ^ (lane & 7)) << 4);
          if (p.residual) {
#pragma unroll
            for (int c = 0; c < kChunks; ++c) {
              uint32_t r[4];
              asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at[c]) : "memory");
              constexpr int kEach = 16 / Elem<DT>::kBytes;
#pragma unroll
              for (int i = 0; i < kEach; ++i) z[c * kEach + i] += Elem<DT>::of(r, i);
            }
          }
          const int col = col0 + k * E + h * S;
          if (col + S > whole && ok && row0 + lane < p.M) {
            void* out = static_cast<char*>(p.Y) + (tb * p.batch_stride_y + static_cast<long long>(row0 + lane) * p.ldy) * Elem<DT>::kBytes;
#pragma unroll
            for (int i = 0; i < S; ++i)
              if (col + i >= whole && col + i < p.N && COMFUSE_IN_BOUNDS(row0 + lane < p.M && tb < p.batch, p.status)) Elem<DT>::put(out, col + i, z[i]);
          }
          __syncwarp();
          uint32_t ow[4 * kChunks];
          Elem<DT>::pack(z, ow);
#pragma unroll
          for (int c = 0; c < kChunks; ++c)
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at[c]), "r"(ow[4 * c]), "r"(ow[4 * c + 1]), "r"(ow[4 * c + 2]), "r"(ow[4 * c + 3]) : "memory");
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) {
          const int col = col0 + k * E;
          if (ok && col < whole && COMFUSE_IN_BOUNDS(col < p.N && row0 < p.M && tb < p.batch, p.status)) tma_store_3d(&maps.Y, box0 + sel * Cfg::BOX_BYTES, col, row0, tb);
          tma_store_commit();
        }
      }
      count += static_cast<uint32_t>(boxes);
    }
    if (lane == 0) tma_store_wait_read<0>();  // the staging boxes outlive the last stores' reads (the stores themselves complete at the kernel's end)
    __syncwarp();
  }

  // -------------------------------------------------------------------------------------------- teardown
  tcgen05_fence_before_sync();
  __syncthreads();
  cluster_sync_all();  // no peer may still signal this CTA's barriers, write its shared memory or its TMEM
  if (warp == 1) {
    __syncwarp();
    tcgen05_fence_after_sync();
    tmem_release<true>(tmem_base, 2 * BN);
    if (lane == 0) linger_behind_expired_wait(w);
  }
}

template <int DT, int BN, int STAGES, int BOXES, int EPW>
cudaError_t launch_instance(const GemmQ8PairMaps& maps, const GemmQ8Params& p, const DeviceInfo& dev, cudaStream_t stream) {
  using Cfg = PairQ8Cfg<DT, BN, STAGES, BOXES, EPW>;
  auto kern = gemm_q8_pair_kernel<DT, BN, STAGES, BOXES, EPW>;
  static ResidentClusters resident;  // (sets the kernel's attributes on the device the first time it is asked)
  const int fit = resident.of(reinterpret_cast<const void*>(kern), Cfg::kThreads, Cfg::SMEM_BYTES, 2, dev);
  if (fit < 1) return cudaErrorLaunchOutOfResources;
  if (verbose_enabled())
    std::fprintf(stderr, "comfuse: gemm_q8 dtype=%d: pairs, columns=%d stages=%d boxes=%d epilogue_warps=%d, %lld tiles on %d pairs\n", DT, BN, STAGES, BOXES,
                 Cfg::kEpiWarps, p.tiles, fit);
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[2];
  cfg.gridDim = dim3(static_cast<unsigned>(2 * std::min<long long>(p.tiles, fit)), 1, 1);
  cfg.blockDim = dim3(Cfg::kThreads, 1, 1);
  cfg.dynamicSmemBytes = Cfg::SMEM_BYTES;
  cfg.stream = stream;
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 2;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;  // set-up may overlap the previous kernel's tail
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = programmatic_launch_enabled() ? 2 : 1;
  count_launch();
  return cudaLaunchKernelEx(&cfg, kern, maps, p);
}

// Columns of a tile, stages of the ring, staging boxes an epilogue warp, epilogue warps a lane quarter.  Behind a long contraction the ring's
// depth is what counts, behind a short one the epilogue: more warps, which overlap each other's steps, or more boxes.  us, 8192 x 4096 bf16, 5
// stages / 4 with two boxes / 4 with sixteen warps: K = 4096 86 / 94 / 98, K = 1024 - / 31 / 32, K = 768 - / 25.8 / 26.4, K = 512 25.0 / 23.5 / 20.7, with a
// residual K = 768 - / 35.0 / 33.7, K = 512 - / 32.2 / 30.1, with GELU K = 512 42.0 / 40.6 / 31.6, K = 1536 47.0 / 48.9 / 41.9, K = 2048 52.8 / 57.8 / 54.0.
// fp32 (252 calls, K = 32 .. 256, 16 .. 148 MB of Y, each with one Y rewritten and with several in turn): sixteen warps while the call's bytes stay in the
// L2, 120 MB of its 126 (96 x 504 x 504 x 64 22.5 / 20.1, 112 x 504 x 504 25.5 / 23.5, 8192 x 2824 22.4 / 19.8; beyond, HBM takes their smaller pieces more slowly: 128 x 504 x 504
// 26.2 / 26.8, 8192 x 4096 26.4 / 27.7, 148 x 512 x 512 30.5 / 32.4), where rows are whole 32-byte sectors (8192 x 1001 12.0 / 13.0, 96 x 500 x 500 24.8 / 28.1, a leading
// dimension of 2052 for 2048 20.4 / 22.3), and in more than one round of tiles (2560 x 1792 7.3 / 7.7, 2560 x 2048 9.6 / 9.2); not with a residual (8192 x 4096 50.6 / 55.3).  Where the rule says
// sixteen they are 5.6 % faster in the geometric mean, at worst 8 % slower.  (A sixth stage,
// in the room of a box: between 3 % faster and 7 % slower from call to call under the power limit.)
template <int DT>
cudaError_t launch_columns(int columns, const GemmQ8PairMaps& maps, const GemmQ8Params& p, const DeviceInfo& dev, cudaStream_t stream) {
  if (columns == 128) return launch_instance<DT, 128, 6, 2, 2>(maps, p, dev, stream);
  const bool long_epilogue = p.activation != 0 && p.activation != COMFUSE_OP_RELU;
  const long long bytes = p.batch * (static_cast<long long>(p.M) * p.N * Elem<DT>::kBytes + (static_cast<long long>(p.M) + p.N) * p.K);
  const bool sectors = (((p.N | p.ldy | p.batch_stride_y) * Elem<DT>::kBytes | reinterpret_cast<uintptr_t>(p.Y)) & 31) == 0;
  const bool f32_sixteen = p.K <= 256 && !p.residual && sectors && p.tiles > dev.sm_count / 2 && bytes <= 120ll << 20;
  if (long_epilogue ? p.K <= 1536 : DT != COMFUSE_DTYPE_F32 ? p.K <= 768 : f32_sixteen) return launch_instance<DT, 256, 4, 1, 4>(maps, p, dev, stream);
  if (p.K <= 1024) return launch_instance<DT, 256, 4, 2, 2>(maps, p, dev, stream);
  return launch_instance<DT, 256, 5, 1, 2>(maps, p, dev, stream);
}

}  // namespace

int gemm_q8_pair_columns(int batch, int M, int N, const DeviceInfo& dev) {
  // Narrow tiles where they still run in one round: 512 x 4096 x 4096 13.0 us with tiles of 128 columns, 17.5 with 256, but 768 rows, two rounds, 18.7 / 17.0.
  const long long tiles = static_cast<long long>(batch) * ((M + 255ll) / 256) * ((N + 255) / 256);
  return 2 * tiles <= dev.sm_count / 2 || N <= 128 ? 128 : 256;
}

cudaError_t launch_gemm_q8_pair(int dtype, int columns, const GemmQ8PairMaps& maps, GemmQ8Params p, const DeviceInfo& dev, cudaStream_t stream) {
  p.mtiles = (p.M + 255) / 256;
  p.ntiles = (p.N + columns - 1) / columns;
  p.tiles = static_cast<long long>(p.batch) * p.mtiles * p.ntiles;
  switch (dtype) {
    case COMFUSE_DTYPE_BF16: return launch_columns<COMFUSE_DTYPE_BF16>(columns, maps, p, dev, stream);
    case COMFUSE_DTYPE_F16: return launch_columns<COMFUSE_DTYPE_F16>(columns, maps, p, dev, stream);
    default: return launch_columns<COMFUSE_DTYPE_F32>(columns, maps, p, dev, stream);
  }
}

}  // namespace comfuse
