// The 8-bit integer product for a handful of rows (a decoding step of a few sequences): Y = act(sa sb (A . B^T) + bias) + R.
//
// What bounds it: the weights' bytes and the latency of one pass.  The tensor memory, barriers and descriptors of the other forms are
// latency that so few products do not repay; here a warp asks for its weights with its first instructions and multiplies them in registers.
//
//   * A warp multiplies 16 channels by 8 rows (or 16) with the warp-wide integer instruction (16 x 8 x 32).  Which 32 bytes of the
//     contraction an instruction takes is free as long as both operands take the same ones, so a lane loads 16 consecutive bytes of its
//     channel and of its row and feeds two instructions with them: 64 bytes of 8 channels a load.  (Four-byte dot products on
//     the ordinary pipe instead: 4096 x 4096 for 1 / 4 / 8 rows 3.9 / 6.9 / 17.7 us.)
//   * `split` warps of a CTA share the contraction of their channels, 128 bytes in turn, so that small layers fill the SMs.  Up to four steps
//     of weights are asked for at once: 8 KB a warp.
//   * The shares meet in shared memory; the sums are exact in any order.
#include <cstdio>
#include <type_traits>

#include "q8_common.cuh"
#include "q8_params.h"

namespace comfuse {
namespace {

constexpr int kWarps = 8, kChannels = 16;

__device__ __forceinline__ uint4 load_codes(const int8_t* row, int k) { return *reinterpret_cast<const uint4*>(row + k); }
// 16 bytes of a row from byte k on; bytes from K on are zeros and not read
__device__ __forceinline__ uint4 load_codes(const int8_t* row, int k, int K) {
  if (k + 16 <= K) return load_codes(row, k);
  uint32_t w[4] = {0u, 0u, 0u, 0u};
  if (k < K) {
    const int words = (K - k) >> 2, bytes = (K - k) & 3;
    uint32_t last = 0u;  // the word that is there in part
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      if (i < words) w[i] = *reinterpret_cast<const uint32_t*>(row + k + 4 * i);
      if (i < bytes) last |= static_cast<uint32_t>(static_cast<uint8_t>(row[k + 4 * words + i])) << (8 * i);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = i == words ? last : w[i];
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
// D += A . B: 16 channels x 32 bytes by 8 rows x 32 bytes.  Lane 4 g + t holds channels g and g + 8, row g, and of the result rows 2t, 2t + 1.
__device__ __forceinline__ void mma_16x8(int (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+r"(d[0]), "+r"(d[1]), "+r"(d[2]), "+r"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// NT groups of 8 rows
template <int DT, int NT>
__global__ void __launch_bounds__(32 * kWarps, 2) gemm_q8_tokens_kernel(const GemmQ8TokensParams t, const GemmQ8Params p) {
  constexpr int ROWS = 8 * NT;
  __shared__ int s_part[kWarps * ROWS * kChannels];  // [share][row][channel of the CTA]
  griddep_launch_dependents();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int share = warp % p.split, group = warp / p.split;
  const int channels = kWarps / p.split * kChannels;  // of the CTA
  const int b = static_cast<int>(blockIdx.y), n0 = static_cast<int>(blockIdx.x) * channels, n = n0 + group * kChannels + (lane >> 2);
  const int8_t* A = t.A + b * t.batch_stride_a;
  const int8_t* B = t.B + b * t.batch_stride_b;
  // (a channel or row past the end repeats the last one; nothing of it is stored)
  const int8_t* w0 = B + (n < p.N ? n : p.N - 1) * t.ldb;
  const int8_t* w1 = B + (n + 8 < p.N ? n + 8 : p.N - 1) * t.ldb;
  const int8_t* x[NT];
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    const int m = 8 * i + (lane >> 2);
    x[i] = A + (m < p.M ? m : p.M - 1) * t.lda;
  }
  // The first round of weights is asked of the L2 while the previous kernel may still run (a prefetch returns nothing, so it may stand in front of
  // the wait whoever writes them): 16 channels x 4 steps of one line, two lines a lane.
  {
    const int k = share * 128 + (lane & 3) * p.split * 128;
    if (k < p.K) {
      asm volatile("prefetch.global.L2 [%0];" ::"l"(w0 + k));
      asm volatile("prefetch.global.L2 [%0];" ::"l"(w1 + k));
    }
  }
  griddep_wait();

  int acc[NT][4] = {};
  const int stride = p.split * 128;
  int k = share * 128;  // (the whole warp takes the same steps)
  const int at = (lane & 3) * 16;
  auto multiply = [&](int i, const uint4& wa, const uint4& wb, const uint4& a) {
    mma_16x8(acc[i], wa.x, wb.x, wa.y, wb.y, a.x, a.y);
    mma_16x8(acc[i], wa.z, wb.z, wa.w, wb.w, a.z, a.w);
  };
  auto rounds = [&](auto steps) {
    constexpr int S = decltype(steps)::value;
#pragma unroll 1
    for (; k + (S - 1) * stride + 128 <= p.K; k += S * stride) {
      uint4 v[S][2][2];
#pragma unroll
      for (int u = 0; u < S; ++u)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          v[u][j][0] = load_codes(w0, k + at + u * stride + 64 * j);
          v[u][j][1] = load_codes(w1, k + at + u * stride + 64 * j);
        }
#pragma unroll
      for (int u = 0; u < S; ++u)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int i = 0; i < NT; ++i) multiply(i, v[u][j][0], v[u][j][1], load_codes(x[i], k + at + u * stride + 64 * j));
    }
  };
  // Four steps under way at once, then two, then one (with fours and the step below alone: 16 rows 2048 x 2048 5.3 us for 3.9, 1024 x 1024 2.7 for 2.3).
  rounds(std::integral_constant<int, 4>{});
  rounds(std::integral_constant<int, 2>{});
  rounds(std::integral_constant<int, 1>{});
  if (k < p.K) {  // the step that is there in part
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const uint4 wa = load_codes(w0, k + at + 64 * j, p.K), wb = load_codes(w1, k + at + 64 * j, p.K);
#pragma unroll
      for (int i = 0; i < NT; ++i) multiply(i, wa, wb, load_codes(x[i], k + at + 64 * j, p.K));
    }
  }
#pragma unroll
  for (int i = 0; i < NT; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      s_part[(share * ROWS + 8 * i + 2 * (lane & 3) + (j & 1)) * channels + group * kChannels + (lane >> 2) + 8 * (j >> 1)] = acc[i][j];
  __syncthreads();
  for (int i = static_cast<int>(threadIdx.x); i < channels * p.M; i += 32 * kWarps) {
    const int m = i / channels, c = i - m * channels, col = n0 + c;
    if (col < p.N) {
      int s = 0;
      for (int j = 0; j < p.split; ++j) s += s_part[(j * ROWS + m) * channels + c];
      const float sb = p.scale_b[static_cast<long long>(b) * p.N + col], sa = p.scale_a[static_cast<long long>(b) * p.M + m];
      float z[1] = {fmaf(static_cast<float>(s) * sb, sa, p.bias ? Elem<DT>::get(p.bias, col) : 0.f)};
      activate(z, p.activation);
      if (p.residual) z[0] += Elem<DT>::get(p.residual, b * p.batch_stride_r + m * p.ldr + col);
      if (COMFUSE_IN_BOUNDS(m < p.M && b < p.batch, p.status)) Elem<DT>::put(p.Y, b * p.batch_stride_y + m * p.ldy + col, z[0]);
    }
  }
}

template <int DT, int NT>
cudaError_t launch_instance(const GemmQ8TokensParams& t, const GemmQ8Params& p, cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[1];
  const int channels = kWarps / p.split * kChannels;
  cfg.gridDim = dim3(static_cast<unsigned>((p.N + channels - 1) / channels), static_cast<unsigned>(p.batch), 1);
  cfg.blockDim = dim3(32 * kWarps, 1, 1);
  cfg.stream = stream;
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;  // set-up may overlap the previous kernel's tail
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = programmatic_launch_enabled() ? 1 : 0;
  count_launch();
  return cudaLaunchKernelEx(&cfg, gemm_q8_tokens_kernel<DT, NT>, t, p);
}

template <int DT>
cudaError_t launch_rows(const GemmQ8TokensParams& t, const GemmQ8Params& p, cudaStream_t stream) {
  if (p.M <= 8) return launch_instance<DT, 1>(t, p, stream);
  return launch_instance<DT, 2>(t, p, stream);
}

}  // namespace

bool gemm_q8_tokens_fits(int batch, int M, int N, int K, const DeviceInfo& dev) {
  if (M > kGemmQ8Tokens || batch > 65535) return false;
  // Where the weights are many enough that their stream is all that counts, the other form's deeper ring is ahead, up to one round of its
  // 128-channel tiles.  us, this form / that one: 1 row 4096 x 4096 5.5 / 6.7, 16384 x 4096 13.2 / 12.5, 65536 x 4096 43.6 / 48.9; 8 rows 6.0 / 6.8,
  // 14.6 / 12.8, 49.9 / 50.2; 16 rows 1024 x 1024 2.3 / 3.8, 4096 x 4096 6.3 / 6.9, 16384 x 4096 17.6 / 13.1; batches 32 x 16 x 1024 x 256 7.3 / 7.9, 96 x 16 x 504 x 64
  // 12.4 / 9.6, 96 x 16 x 1024 x 256 19.8 / 16.5.
  const long long codes = static_cast<long long>(batch) * N * K, tiles = static_cast<long long>(batch) * ((N + 127) / 128);
  return M <= 8 ? codes <= 3ll << 24 || tiles > dev.sm_count : codes <= 1ll << 25 && tiles <= 2ll * dev.sm_count;
}

cudaError_t launch_gemm_q8_tokens(int dtype, const GemmQ8TokensParams& t, GemmQ8Params p, const DeviceInfo& dev, cudaStream_t stream) {
  // Shares: up to the 16 warps that an SM holds, while each has a step.  us with 1 / 2 / 4 / 8 shares (8 rows): 4096 x 4096 12.9 / 9.8 / 7.0 / 5.9,
  // 16384 x 4096 18.2 / 14.0 / 14.7 / 15.9, 1024 x 1024 5.1 / 3.3 / 2.9 / 2.4; a few CTAs more than fit at once cost a second round (1 row 5120 x 1024 with
  // 4 / 8 shares 3.4 / 4.8, 20 batches of 1024 x 256 with 1 / 2 3.3 / 4.9).
  const long long groups = static_cast<long long>(p.batch) * ((p.N + kChannels - 1) / kChannels);
  p.split = 1;
  while (p.split < kWarps && groups * p.split * 2 <= 16ll * dev.sm_count && p.K > p.split * 128) p.split *= 2;
  if (verbose_enabled()) std::fprintf(stderr, "comfuse: gemm_q8 dtype=%d: a handful of rows, rows=%d shares=%d\n", dtype, p.M <= 8 ? 8 : 16, p.split);
  switch (dtype) {
    case COMFUSE_DTYPE_BF16: return launch_rows<COMFUSE_DTYPE_BF16>(t, p, stream);
    case COMFUSE_DTYPE_F16: return launch_rows<COMFUSE_DTYPE_F16>(t, p, stream);
    default: return launch_rows<COMFUSE_DTYPE_F32>(t, p, stream);
  }
}

}  // namespace comfuse
