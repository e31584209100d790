// The 8-bit integer product for many rows: Y = act(sa sb (A . B^T) + bias) + R, on CTA pairs.
//
// What bounds it: the tensor cores (int8 at twice the bf16 rate), and behind short contractions the bytes of Y.  As in the bf16 tile
// kernel two CTAs multiply a 256 x 256 tile (cta_group::2): each holds its own 128 rows of A and half of B's 256, 32 KB a K block of 128 bytes,
// which the tensor cores take 512 clocks for.  Clusters of two are persistent and walk the tiles in bands of 8 row blocks, so that the
// tiles in flight share their operands in the L2.  Two accumulators of 256 columns alternate: a tile's epilogue runs under the
// next one's products.
//
// Epilogue: thread = one row of the tile, 32 columns at a time, a warp 128 of the 256.  The channel's scale and bias come from shared
// memory (broadcast), the row's scale is a register.  Rows leave straight from registers, 32 bytes a store: every store fills its
// sectors, so there is nothing that staging through shared memory would save, and the room goes to a sixth stage of the ring.
#include <algorithm>
#include <type_traits>

#include "q8_common.cuh"
#include "q8_params.h"

namespace comfuse {
namespace {

struct PairQ8Cfg {
  static constexpr int NSTAGES = 6;
  static constexpr int kEpiWarps = 8;
  static constexpr int kThreads = 32 * (2 + kEpiWarps);
  static constexpr int HALF_BYTES = 128 * 128;           // 128 rows of A, or of B, x 128 bytes
  static constexpr int STAGE_BYTES = 2 * HALF_BYTES;
  static constexpr int OFF_VEC = NSTAGES * STAGE_BYTES;  // [2][256] (scale, bias) of the tile's channels
  static constexpr int OFF_BAR = OFF_VEC + 2 * 256 * 8;
  static constexpr int SMEM_BYTES = OFF_BAR + 256 + 1024;
  static_assert((2 * NSTAGES + 5) * 8 + 16 <= 256, "barrier room");
  static_assert(SMEM_BYTES <= 232448 && SMEM_BYTES > 116 * 1024, "one CTA per SM");
};

template <int DT>
__global__ void __launch_bounds__(PairQ8Cfg::kThreads, 1) gemm_q8_pair_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB,
                                                                             const GemmQ8Params p) {
  using Cfg = PairQ8Cfg;
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
  uint32_t* s_tmem_base = reinterpret_cast<uint32_t*>(smem + Cfg::OFF_BAR + (2 * NSTAGES + 5) * 8);
  volatile int* s_abort = reinterpret_cast<volatile int*>(s_tmem_base + 1);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();  // which half of the pair
  const long long cluster_id = blockIdx.x >> 1, clusters = gridDim.x >> 1;
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
    *s_abort = 0;
    fence_mbar_init();
    prefetch_tensormap(&tmA);
    prefetch_tensormap(&tmB);
  }
  if (warp == 1) {
    tmem_alloc_pair(smem_u32(s_tmem_base), 512);
    tmem_relinquish_alloc_permit_pair();
  }
  tcgen05_fence_before_sync();
  __syncthreads();
  tcgen05_fence_after_sync();
  cluster_sync_after_init();  // both CTAs' barriers exist before either signals them
  const uint32_t tmem_base = *s_tmem_base;
  griddep_wait();

  // tile -> batch, first row and column: bands of 8 row blocks, in a band column by column
  auto decode = [&](long long tile, int& b, int& m0, int& n0) {
    const long long per = static_cast<long long>(p.mtiles) * p.ntiles;
    b = static_cast<int>(tile / per);
    const long long t = tile - b * per;
    const long long band = t / (8ll * p.ntiles);
    const int in_band = static_cast<int>(t - band * 8 * p.ntiles), first = static_cast<int>(band * 8);
    const int high = p.mtiles - first < 8 ? p.mtiles - first : 8;
    n0 = (in_band / high) * 256;
    m0 = (first + in_band % high) * 256;
  };

  if (warp == 0) {
    // ------------------------------------------------------------------------------------------ TMA producer
    if (elect_one()) {
      int stage = 0;
      uint32_t phase = 0;
      bool ok = true;
      for (long long tile = cluster_id; tile < p.tiles && ok; tile += clusters) {
        int b, m0, n0;
        decode(tile, b, m0, n0);
        for (int kb = 0; kb < KB; ++kb) {
          if (!mbar_wait<false>(bar_empty(stage), phase ^ 1u, w)) { ok = false; break; }  // passes on a fresh barrier
          const uint32_t sa = smem_base + stage * Cfg::STAGE_BYTES, full = map_to_cta(bar_full(stage), 0);
          mbar_arrive_expect_tx_cluster(full, Cfg::STAGE_BYTES);
          tma_load_3d_pair(sa, &tmA, full, kb * 128, m0 + static_cast<int>(rank) * 128, b);
          tma_load_3d_pair(sa + Cfg::HALF_BYTES, &tmB, full, kb * 128, n0 + static_cast<int>(rank) * 128, b);
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
      constexpr uint32_t idesc = make_idesc_i8(256, 256);
      for (long long tile = cluster_id; tile < p.tiles && ok; tile += clusters, ++n) {
        const uint32_t slot = n & 1u;
        if (!mbar_wait<false>(bar_tempty(slot), ((n >> 1) & 1u) ^ 1u, w)) break;
        tcgen05_fence_after_sync();
        for (int kb = 0; kb < KB; ++kb) {
          if (!mbar_wait<false>(bar_full(stage), phase, w)) { ok = false; break; }
          tcgen05_fence_after_sync();
          const uint32_t sa = smem_base + stage * Cfg::STAGE_BYTES;
          const uint64_t adesc = make_smem_desc_sw128(sa, 16, 1024), bdesc = make_smem_desc_sw128(sa + Cfg::HALF_BYTES, 16, 1024);
#pragma unroll
          for (int k = 0; k < 4; ++k)  // 32 bytes of the contraction an instruction
            umma_i8_ss_pair(tmem_base + slot * 256, adesc + static_cast<uint64_t>(2 * k), bdesc + static_cast<uint64_t>(2 * k), idesc, (kb | k) != 0 ? 1u : 0u);
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
    const int q = warp & 3, half = (warp - 2) >> 2;  // TMEM lane quarter: rows 32q ..; which 128 columns
    const uint32_t lane_addr = tmem_base + (static_cast<uint32_t>(q * 32) << 16) + half * 128;
    const uint32_t tempty = map_to_cta(bar_tempty(0), 0);
    float2* s_vec = reinterpret_cast<float2*>(smem + Cfg::OFF_VEC);
    constexpr int kWords = 8 * Elem<DT>::kBytes;  // 32 elements
    uint32_t n = 0;
    for (long long tile = cluster_id; tile < p.tiles; tile += clusters, ++n) {
      int b, m0, n0;
      decode(tile, b, m0, n0);
      const uint32_t slot = n & 1u;
      {
        const int i = static_cast<int>(threadIdx.x) - 64, c = n0 + i;  // 256 threads, 256 channels
        float2 v = make_float2(0.f, 0.f);
        if (c < p.N) {
          v.x = __ldg(p.scale_b + static_cast<long long>(b) * p.N + c);
          if (p.bias) v.y = Elem<DT>::get(p.bias, c);
        }
        s_vec[slot * 256 + i] = v;  // (the barrier below keeps the warps within one tile of each other)
      }
      named_barrier_sync(1, 32 * Cfg::kEpiWarps);
      const long long row = m0 + static_cast<int>(rank) * 128 + q * 32 + lane;
      const bool live = row < p.M;
      const float sa = live ? __ldg(p.scale_a + static_cast<long long>(b) * p.M + row) : 0.f;
      const char* res = static_cast<const char*>(p.residual) + (b * p.batch_stride_r + row * p.ldr) * Elem<DT>::kBytes;
      char* out = static_cast<char*>(p.Y) + (b * p.batch_stride_y + row * p.ldy) * Elem<DT>::kBytes;
      const bool ok = mbar_wait<false>(bar_tfull(slot), (n >> 1) & 1u, w);
      __syncwarp();
      tcgen05_fence_after_sync();
#pragma unroll 1
      for (int c = 0; c < 4; ++c) {
        const int local = half * 128 + c * 32, col = n0 + local;
        const bool whole = col + 32 <= p.N;
        uint32_t rw[kWords];
        if (p.residual && live && whole) {
#pragma unroll
          for (int i = 0; i < kWords; i += 8) {
            const char* at = res + static_cast<long long>(col) * Elem<DT>::kBytes + i * 4;
            if (p.wide) {
              ld_32(at, rw + i);
            } else {
              ld_16(at, rw + i);
              ld_16(at + 16, rw + i + 4);
            }
          }
        }
        uint32_t v[32];
        tmem_ld_32cols(lane_addr + slot * 256 + c * 32, v);
        if (c == 3) {  // the last of this warp's columns is read: the accumulator may be overwritten once everyone is here
          tcgen05_fence_before_sync();
          __syncwarp();
          if (lane == 0) mbar_arrive_cluster_noflush(tempty + 8u * slot);
        }
        float z[32];
#pragma unroll
        for (int i = 0; i < 32; i += 2) {
          const float4 sv = *reinterpret_cast<const float4*>(s_vec + slot * 256 + local + i);
          z[i] = fmaf(static_cast<float>(static_cast<int>(v[i])) * sv.x, sa, sv.y);
          z[i + 1] = fmaf(static_cast<float>(static_cast<int>(v[i + 1])) * sv.z, sa, sv.w);
        }
        activate(z, p.activation);
        if (!live || !ok) continue;
        if (whole) {
          if (p.residual) {
#pragma unroll
            for (int i = 0; i < 32; ++i) z[i] += Elem<DT>::of(rw, i);
          }
          uint32_t ow[kWords];
          Elem<DT>::pack(z, ow);
          if (COMFUSE_IN_BOUNDS(row < p.M && col + 31 < p.N && b < p.batch, p.status)) {
#pragma unroll
            for (int i = 0; i < kWords; i += 8) {
              char* at = out + static_cast<long long>(col) * Elem<DT>::kBytes + i * 4;
              if (p.wide) {
                st_32(at, ow + i);
              } else {
                st_16(at, ow + i);
                st_16(at + 16, ow + i + 4);
              }
            }
          }
        } else {
#pragma unroll
          for (int i = 0; i < 32; ++i)
            if (col + i < p.N) Elem<DT>::put(out, col + i, p.residual ? z[i] + Elem<DT>::get(res, col + i) : z[i]);
        }
      }
    }
  }

  // -------------------------------------------------------------------------------------------- teardown
  tcgen05_fence_before_sync();
  __syncthreads();
  cluster_sync_all();  // no peer may still signal this CTA's barriers, write its shared memory or its TMEM
  if (warp == 1) {
    __syncwarp();
    tcgen05_fence_after_sync();
    tmem_release<true>(tmem_base, 512);
    if (lane == 0) linger_behind_expired_wait(w);
  }
}

template <int DT>
cudaError_t launch_instance(const CUtensorMap& tmA, const CUtensorMap& tmB, const GemmQ8Params& p, const DeviceInfo& dev, cudaStream_t stream) {
  using Cfg = PairQ8Cfg;
  auto kern = gemm_q8_pair_kernel<DT>;
  static ResidentClusters resident;  // (sets the kernel's attributes on the device the first time it is asked)
  const int fit = resident.of(reinterpret_cast<const void*>(kern), Cfg::kThreads, Cfg::SMEM_BYTES, 2, dev);
  if (fit < 1) return cudaErrorLaunchOutOfResources;
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
  return cudaLaunchKernelEx(&cfg, kern, tmA, tmB, p);
}

}  // namespace

cudaError_t launch_gemm_q8_pair(int dtype, const CUtensorMap& tmA, const CUtensorMap& tmB, GemmQ8Params p, const DeviceInfo& dev, cudaStream_t stream) {
  p.mtiles = (p.M + 255) / 256;
  p.ntiles = (p.N + 255) / 256;
  p.tiles = static_cast<long long>(p.batch) * p.mtiles * p.ntiles;
  switch (dtype) {
    case COMFUSE_DTYPE_BF16: return launch_instance<COMFUSE_DTYPE_BF16>(tmA, tmB, p, dev, stream);
    case COMFUSE_DTYPE_F16: return launch_instance<COMFUSE_DTYPE_F16>(tmA, tmB, p, dev, stream);
    default: return launch_instance<COMFUSE_DTYPE_F32>(tmA, tmB, p, dev, stream);
  }
}

}  // namespace comfuse
