// Rows to int8 with a scale each, alone or behind a residual addition and an RMSNorm.
//
//   h = x + r,  y = h * rstd * gamma,  rstd = rsqrt(mean(h^2) + eps),  s = max|y| / 127,  q = rint(y / s)
//
// rstd is one number for the row, so y / s = 127 * (h gamma) / max|h gamma|: the codes do not depend on the norm, only the scale does,
// and one pass over the row collects sum(h^2) and max|h gamma| together.  The row stays in registers between that pass and the
// codes, so every tensor crosses HBM once; that traffic is all that bounds it.
//
//   * Rows of up to 1024 elements: a warp per row.  Longer ones: a CTA, or a cluster of them that exchange their (sum, maximum) through
//     distributed shared memory -- for rows that one CTA's registers do not hold, and for few rows, which would leave SMs idle.
//   * A thread owns chunks of 8 elements: 16-byte accesses of 16-bit types, 8 bytes of codes; chunk j of a row belongs to thread j mod T.
//   * The maximum is taken over the bit patterns of |h gamma| as unsigned integers, where infinities and NaNs lie above every number: one
//     warp reduction instruction finds the maximum and whether the row is finite.
#include <type_traits>

#include "q8_common.cuh"
#include "q8_params.h"

namespace comfuse {
namespace {

constexpr int kMaxThreads = 512;

// 8 elements from a row's column c on, as packed words; elements from N on read as zeros
template <int DT>
__device__ __forceinline__ void load_chunk(const char* row, int c, int N, uint32_t* w) {
  constexpr int kWords = 2 * Elem<DT>::kBytes;
  if (c + 8 <= N) {
    ld_16(row + static_cast<long long>(c) * Elem<DT>::kBytes, w);
    if constexpr (kWords == 8) ld_16(row + static_cast<long long>(c) * 4 + 16, w + 4);
  } else {
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = c + i < N ? Elem<DT>::get(row, c + i) : 0.f;
    Elem<DT>::pack(v, w);  // (widened and narrowed again: the same bits)
  }
}
template <int DT>
__device__ __forceinline__ void store_chunk(char* row, int c, int N, const float (&v)[8]) {
  if (c + 8 <= N) {
    uint32_t w[2 * Elem<DT>::kBytes];
    Elem<DT>::pack(v, w);
    st_16(row + static_cast<long long>(c) * Elem<DT>::kBytes, w);
    if constexpr (Elem<DT>::kBytes == 4) st_16(row + static_cast<long long>(c) * 4 + 16, w + 4);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c + i < N) Elem<DT>::put(row, c + i, v[i]);
  }
}

// CH chunks per thread; WARP: a warp per row, else a CTA or cluster per row
template <int DT, bool NORM, int CH, bool WARP>
__global__ void __launch_bounds__(kMaxThreads) quantize_rows_kernel(const QuantizeRowsParams p) {
  __shared__ float2 s_part[16], s_peer[8];
  griddep_launch_dependents();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int threads = WARP ? 32 : static_cast<int>(blockDim.x);
  const int tid = WARP ? lane : static_cast<int>(threadIdx.x);
  const int split = WARP ? 1 : p.split;
  const int rank = split > 1 ? static_cast<int>(blockIdx.x % split) : 0;  // = the rank in the cluster
  const long long row = WARP ? static_cast<long long>(blockIdx.x) * (blockDim.x >> 5) + warp : blockIdx.x / split;
  if (split > 1) asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory");  // this CTA runs: peers may write its shared memory
  griddep_wait();
  if (WARP && row >= p.rows) return;

  constexpr int kWords = 2 * Elem<DT>::kBytes;
  const int chunks = (p.N + 7) >> 3, per = (chunks + split - 1) / split;
  const int first = rank * per, last = first + per < chunks ? first + per : chunks;
  const char* xrow = static_cast<const char*>(p.x) + row * p.ldx * Elem<DT>::kBytes;
  const char* rrow = static_cast<const char*>(p.residual) + row * p.ldr * Elem<DT>::kBytes;
  uint32_t x[CH][kWords], r[NORM ? CH : 1][kWords], g[NORM ? CH : 1][kWords];
#pragma unroll
  for (int j = 0; j < CH; ++j) {
    const int c = first + tid + j * threads;
    if (c < last) {
      load_chunk<DT>(xrow, 8 * c, p.N, x[j]);
      if (NORM && p.residual) load_chunk<DT>(rrow, 8 * c, p.N, r[j]);
      if (NORM && p.gamma) load_chunk<DT>(static_cast<const char*>(p.gamma), 8 * c, p.N, g[j]);
    }
  }
  float y[CH][8];  // h * gamma
  float sum = 0.f, high = 0.f;  // of the squares: chunks of up to 2^100, and larger ones in units of 2^192
  uint32_t top = 0u;
#pragma unroll
  for (int j = 0; j < CH; ++j) {
    const int c = first + tid + j * threads;
    if (c < last) {
#pragma unroll
      for (int i = 0; i < 8; ++i) y[j][i] = Elem<DT>::of(x[j], i);
      if constexpr (NORM) {
        if (p.residual) {
#pragma unroll
          for (int i = 0; i < 8; ++i) y[j][i] += Elem<DT>::of(r[j], i);
        }
        if (p.h) store_chunk<DT>(static_cast<char*>(p.h) + row * p.ldh * Elem<DT>::kBytes, 8 * c, p.N, y[j]);
        float part = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) part = fmaf(y[j][i], y[j][i], part);
        if (part <= 0x1p100f) {
          sum += part;
        } else {  // (rare; a chunk with a NaN comes here too, which `top` will show)
          part = 0.f;
#pragma unroll
          for (int i = 0; i < 8; ++i) part = fmaf(y[j][i] * 0x1p-96f, y[j][i] * 0x1p-96f, part);
          high += part;
        }
        if (p.gamma) {
#pragma unroll
          for (int i = 0; i < 8; ++i) y[j][i] *= Elem<DT>::of(g[j], i);
        }
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint32_t b = __float_as_uint(y[j][i]) & 0x7FFFFFFFu;
        top = b > top ? b : top;
      }
    }
  }
  top = __reduce_max_sync(0xFFFFFFFFu, top);
  if (NORM) {
    if (__any_sync(0xFFFFFFFFu, high > 0.f)) sum = -fmaf(sum * 0x1p-96f, 0x1p-96f, high);  // in the large unit, which the sign tells
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
  }
  if constexpr (!WARP) {
    // the warps' partials, then the CTAs', each added in the same order by everyone
    auto merge = [&](const float2* part, int n) {
      sum = high = 0.f;
      top = 0u;
      for (int i = 0; i < n; ++i) {
        if (NORM) {
          sum += fmaxf(part[i].x, 0.f);
          high += fmaxf(-part[i].x, 0.f);
        }
        const uint32_t b = __float_as_uint(part[i].y);
        top = b > top ? b : top;
      }
      if (NORM && high > 0.f) sum = -fmaf(sum * 0x1p-96f, 0x1p-96f, high);
    };
    if (lane == 0) s_part[warp] = make_float2(sum, __uint_as_float(top));
    __syncthreads();
    merge(s_part, threads >> 5);
    if (split > 1) {
      asm volatile("barrier.cluster.wait.acquire;" ::: "memory");  // every CTA of the cluster runs
      if (tid < split) st_cluster_f32x2(map_to_cta(smem_u32(&s_peer[rank]), static_cast<uint32_t>(tid)), sum, __uint_as_float(top));
      cluster_sync_all();  // (behind it nobody writes into another CTA any more)
      merge(s_peer, split);
    }
  }
  // A row that is not finite: scale NaN.  A maximum so small that 127 / max leaves fp32 is first multiplied by 2^100, exactly.
  float amax = __uint_as_float(top);
  const bool finite = top < 0x7F800000u;
  const float lift = amax < 0x1p-100f ? 0x1p100f : 1.f;
  const float inv = finite && amax > 0.f ? 127.f / (amax * lift) : 0.f;
  if (NORM) {
    const float mean = fabsf(sum) / static_cast<float>(p.N);
    amax = sum < 0.f ? amax * 0x1p-96f * rsqrtf(mean) : amax * rsqrtf(mean + p.eps);  // (eps is nothing beside 2^100 / N)
  }
  const float scale = finite ? amax / 127.f : __int_as_float(0x7FFFFFFF);
  if (tid == 0 && rank == 0) p.scale[row] = scale;

  constexpr float kRound = 12582912.f;  // 1.5 * 2^23: behind its addition the low byte is the rounded number in two's complement
  int8_t* qrow = p.q + row * p.ldq;
  char* vrow = reinterpret_cast<char*>(p.values + row * p.ldv);
#pragma unroll
  for (int j = 0; j < CH; ++j) {
    const int c = first + tid + j * threads;
    if (c < last) {
      uint32_t b[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float v = fmaf(finite ? y[j][i] * lift : 0.f, inv, kRound);  // (one rounding, of the exact product: to the nearest whole number)
        b[i] = __float_as_uint(v);
        y[j][i] = (v - kRound) * scale;
      }
      if (8 * c + 8 <= p.N) {
        uint32_t w[2];
#pragma unroll
        for (int k = 0; k < 2; ++k)
          w[k] = __byte_perm(__byte_perm(b[4 * k], b[4 * k + 1], 0x0040), __byte_perm(b[4 * k + 2], b[4 * k + 3], 0x0040), 0x5410);
        st_8(qrow + 8 * c, w);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (8 * c + i < p.N) qrow[8 * c + i] = static_cast<int8_t>(b[i] & 0xFFu);
      }
      if (p.values) store_chunk<COMFUSE_DTYPE_BF16>(vrow, 8 * c, p.N, y[j]);
    }
  }
}

template <int DT, bool NORM, int CH, bool WARP>
cudaError_t launch_instance(const QuantizeRowsParams& p, unsigned grid, unsigned threads, cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[2];
  cfg.gridDim = dim3(grid, 1, 1);
  cfg.blockDim = dim3(threads, 1, 1);
  cfg.stream = stream;
  int n = 0;
  if (programmatic_launch_enabled()) {
    attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[n++].val.programmaticStreamSerializationAllowed = 1;
  }
  if (p.split > 1) {
    attr[n].id = cudaLaunchAttributeClusterDimension;
    attr[n].val.clusterDim.x = static_cast<unsigned>(p.split);
    attr[n].val.clusterDim.y = 1;
    attr[n++].val.clusterDim.z = 1;
  }
  cfg.attrs = attr;
  cfg.numAttrs = n;
  count_launch();
  return cudaLaunchKernelEx(&cfg, quantize_rows_kernel<DT, NORM, CH, WARP>, p);
}

template <int DT, bool NORM>
cudaError_t launch_form(QuantizeRowsParams p, const DeviceInfo& dev, cudaStream_t stream) {
  const int chunks = (p.N + 7) / 8;
  p.split = 1;
  if (chunks <= 128) {
    constexpr int kWarps = 4;
    const unsigned grid = (static_cast<unsigned>(p.rows) + kWarps - 1) / kWarps;
    if (chunks <= 32) return launch_instance<DT, NORM, 1, true>(p, grid, 32 * kWarps, stream);
    if (chunks <= 64) return launch_instance<DT, NORM, 2, true>(p, grid, 32 * kWarps, stream);
    return launch_instance<DT, NORM, 4, true>(p, grid, 32 * kWarps, stream);
  }
  while (chunks > p.split * kMaxThreads * 4) p.split *= 2;
  while (p.split < 8 && static_cast<long long>(p.rows) * p.split * 2 <= dev.sm_count && chunks >= p.split * 512) p.split *= 2;
  const int per = (chunks + p.split - 1) / p.split;
  const int ch = per > 2 * kMaxThreads ? 4 : (per > 256 || p.rows >= 2 * dev.sm_count) ? 2 : 1;
  const unsigned threads = static_cast<unsigned>(((per + ch - 1) / ch + 31) / 32 * 32), grid = static_cast<unsigned>(p.rows) * static_cast<unsigned>(p.split);
  if (ch == 1) return launch_instance<DT, NORM, 1, false>(p, grid, threads, stream);
  if (ch == 2) return launch_instance<DT, NORM, 2, false>(p, grid, threads, stream);
  return launch_instance<DT, NORM, 4, false>(p, grid, threads, stream);
}

}  // namespace

cudaError_t launch_quantize_rows(int dtype, bool norm, QuantizeRowsParams p, const DeviceInfo& dev, cudaStream_t stream) {
  switch (dtype) {
    case COMFUSE_DTYPE_BF16: return norm ? launch_form<COMFUSE_DTYPE_BF16, true>(p, dev, stream) : launch_form<COMFUSE_DTYPE_BF16, false>(p, dev, stream);
    case COMFUSE_DTYPE_F16: return norm ? launch_form<COMFUSE_DTYPE_F16, true>(p, dev, stream) : launch_form<COMFUSE_DTYPE_F16, false>(p, dev, stream);
    default: return norm ? launch_form<COMFUSE_DTYPE_F32, true>(p, dev, stream) : launch_form<COMFUSE_DTYPE_F32, false>(p, dev, stream);
  }
}

}  // namespace comfuse
