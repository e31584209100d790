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
#include <cstdio>
#include <type_traits>

#include "q8_common.cuh"
#include "q8_params.h"

namespace comfuse {
namespace {

constexpr int kMaxThreads = 512;

// 8 elements of a row
template <int DT>
__device__ __forceinline__ void load_chunk(const char* at, uint32_t* w) {
  ld_16(at, w);
  if constexpr (Elem<DT>::kBytes == 4) ld_16(at + 16, w + 4);
}
template <int DT>
__device__ __forceinline__ void store_chunk(char* at, const float (&v)[8]) {
  uint32_t w[2 * Elem<DT>::kBytes];
  Elem<DT>::pack(v, w);
  st_16(at, w);
  if constexpr (Elem<DT>::kBytes == 4) st_16(at + 16, w + 4);
}

// What a row's codes need, from its sum of squares (negative: in units of 2^192) and the bits of its largest |h gamma|.
struct RowScale {
  float scale, lift, inv, inv_low;
  bool finite;
};
template <bool NORM>
__device__ __forceinline__ RowScale row_scale(float sum, uint32_t top, const QuantizeRowsParams& p) {
  // A row that is not finite: scale NaN.  A maximum so small that 127 / max leaves fp32 is first multiplied by 2^100, exactly.
  RowScale s;
  float amax = __uint_as_float(top);
  s.finite = top < 0x7F800000u;
  s.lift = amax < 0x1p-100f ? 0x1p100f : 1.f;
  s.inv = s.finite && amax > 0.f ? 127.f / (amax * s.lift) : 0.f;
  s.inv_low = !NORM && s.inv > 0.f ? fmaf(-s.inv, amax * s.lift, 127.f) / (amax * s.lift) : 0.f;  // what the division's rounding left out
  if (NORM) {
    const float mean = fabsf(sum) / static_cast<float>(p.N);
    amax = sum < 0.f ? amax * 0x1p-96f * rsqrtf(mean) : amax * rsqrtf(mean + p.eps);  // (eps is nothing beside 2^100 / N)
  }
  s.scale = s.finite ? amax / 127.f : __int_as_float(0x7FFFFFFF);
  return s;
}

__device__ __forceinline__ void largest(float y, uint32_t& top) {
  const uint32_t b = __float_as_uint(y) & 0x7FFFFFFFu;
  top = b > top ? b : top;
}
// A sum of squares that is beyond 2^100 counts in units of 2^192: `part`, or the sum taken anew of scaled values.
template <int N>
__device__ __forceinline__ void add_squares(const float (&h)[N], float& sum, float& high) {
  float part = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) part = fmaf(h[i], h[i], part);
  if (part <= 0x1p100f) {
    sum += part;
  } else {  // (rare; a NaN comes here too, which the largest value will show)
    part = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) part = fmaf(h[i] * 0x1p-96f, h[i] * 0x1p-96f, part);
    high += part;
  }
}

// The warp's statistics.
template <bool NORM>
__device__ __forceinline__ void warp_merge(float& sum, float high, uint32_t& top) {
  top = __reduce_max_sync(0xFFFFFFFFu, top);
  if (NORM) {
    if (__any_sync(0xFFFFFFFFu, high > 0.f)) sum = -fmaf(sum * 0x1p-96f, 0x1p-96f, high);  // in the large unit, which the sign tells
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
  }
}
// The statistics of n warps, or CTAs, added in the same order by everyone.
template <bool NORM>
__device__ __forceinline__ void merge(const float2* part, int n, float& sum, uint32_t& top) {
  float high = 0.f;
  sum = 0.f;
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
}

constexpr float kRound = 12582912.f;  // 1.5 * 2^23: behind its addition the low byte is the rounded number in two's complement
// y's code, as a whole number plus kRound.  Without the norm the quotient is correctly rounded nearly always: rows of 16-bit values meet the exact
// middle of two codes often (their values are few), and 127 / max alone, rounded, would send all of those in a row to one side instead of to
// the even code.  Behind a norm one fused operation rounds y * inv to the whole number (60000 x 256: 26 -> 24 us): a middle may go to either code there, as the
// interface allows.  It is met where h gamma has few values, most often without residual and gains; with both, 92 of 8192 x 4096 bf16 codes are not
// the one that 64 bits give (with a division in fp32 61; without the norm, here, none of 8192 x 16384).
template <bool NORM>
__device__ __forceinline__ float code_of(float y, const RowScale& s) {
  const float v = s.finite ? y * s.lift : 0.f;
  return NORM ? fmaf(v, s.inv, kRound) : fmaf(v, s.inv, v * s.inv_low) + kRound;
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

  constexpr int kWords = 2 * Elem<DT>::kBytes, kChunk = 8 * Elem<DT>::kBytes;
  const int chunks = p.N >> 3, per = (chunks + split - 1) / split;
  const int first = rank * per, last = first + per < chunks ? first + per : chunks;
  const char* xrow = static_cast<const char*>(p.x) + row * p.ldx * Elem<DT>::kBytes;
  const char* rrow = static_cast<const char*>(p.residual) + row * p.ldr * Elem<DT>::kBytes;
  char* hrow = static_cast<char*>(p.h) + row * p.ldh * Elem<DT>::kBytes;
  uint32_t x[CH][kWords], r[NORM ? CH : 1][kWords], g[NORM ? CH : 1][kWords];
#pragma unroll
  for (int j = 0; j < CH; ++j) {
    const int c = first + tid + j * threads;
    if (c < last) {
      load_chunk<DT>(xrow + c * kChunk, x[j]);
      if (NORM && p.residual) load_chunk<DT>(rrow + c * kChunk, r[j]);
      if (NORM && p.gamma) {  // (read by every row: through the L1)
        const uint4* at = reinterpret_cast<const uint4*>(static_cast<const char*>(p.gamma) + c * kChunk);
#pragma unroll
        for (int k = 0; k < kWords / 4; ++k) {
          const uint4 v = at[k];
          g[j][4 * k] = v.x; g[j][4 * k + 1] = v.y; g[j][4 * k + 2] = v.z; g[j][4 * k + 3] = v.w;
        }
      }
    }
  }
  // Without the norm the row stays as it was read (a 16-bit type: half the registers, twice the rows an SM has under way) and is widened for
  // its codes only; the largest of two 16-bit patterns is one instruction.
  constexpr bool kKeepRead = !NORM && DT != COMFUSE_DTYPE_F32;
  float y[kKeepRead ? 1 : CH][8];  // h * gamma
  float sum = 0.f, high = 0.f;     // of the squares: parts of up to 2^100, and larger ones in units of 2^192
  uint32_t top = 0u;
#pragma unroll
  for (int j = 0; j < CH; ++j) {
    const int c = first + tid + j * threads;
    if (c >= last) continue;
    if constexpr (kKeepRead) {
#pragma unroll
      for (int i = 0; i < kWords; ++i) top = __vmaxu2(top, x[j][i] & 0x7FFF7FFFu);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) y[j][i] = Elem<DT>::of(x[j], i);
      if constexpr (NORM) {
        if (p.residual) {
#pragma unroll
          for (int i = 0; i < 8; ++i) y[j][i] += Elem<DT>::of(r[j], i);
        }
        if (p.h && COMFUSE_IN_BOUNDS(row < p.rows && 8 * c + 7 < p.N, p.status)) store_chunk<DT>(hrow + c * kChunk, y[j]);
        add_squares(y[j], sum, high);
        if (p.gamma) {
#pragma unroll
          for (int i = 0; i < 8; ++i) y[j][i] *= Elem<DT>::of(g[j], i);
        }
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) largest(y[j][i], top);
    }
  }
  if constexpr (kKeepRead) {  // (patterns of |x| in order: the larger half, widened)
    const uint32_t w[1] = {(top >> 16) > (top & 0xFFFFu) ? top >> 16 : top & 0xFFFFu};
    top = __float_as_uint(Elem<DT>::of(w, 0));
  }
  // the up to 7 elements behind the last whole chunk, one each for the first threads (of the cluster's first CTA)
  const int behind = 8 * chunks + tid;
  const bool tail = rank == 0 && tid < 8 && behind < p.N;
  float yt[1] = {0.f};
  if (tail) {
    yt[0] = Elem<DT>::get(xrow, behind);
    if constexpr (NORM) {
      if (p.residual) yt[0] += Elem<DT>::get(rrow, behind);
      if (p.h && COMFUSE_IN_BOUNDS(row < p.rows && behind < p.N, p.status)) Elem<DT>::put(hrow, behind, yt[0]);
      add_squares(yt, sum, high);
      if (p.gamma) yt[0] *= Elem<DT>::get(p.gamma, behind);
    }
    largest(yt[0], top);
  }
  warp_merge<NORM>(sum, high, top);
  if constexpr (!WARP) {
    if (lane == 0) s_part[warp] = make_float2(sum, __uint_as_float(top));
    __syncthreads();
    merge<NORM>(s_part, threads >> 5, sum, top);
    if (split > 1) {
      asm volatile("barrier.cluster.wait.acquire;" ::: "memory");  // every CTA of the cluster runs
      if (tid < split) st_cluster_f32x2(map_to_cta(smem_u32(&s_peer[rank]), static_cast<uint32_t>(tid)), sum, __uint_as_float(top));
      cluster_sync_all();  // (behind it nobody writes into another CTA any more)
      merge<NORM>(s_peer, split, sum, top);
    }
  }
  const RowScale s = row_scale<NORM>(sum, top, p);
  if (tid == 0 && rank == 0 && COMFUSE_IN_BOUNDS(row < p.rows, p.status)) p.scale[row] = s.scale;
  int8_t* qrow = p.q + row * p.ldq;
  uint16_t* vrow = p.values + row * p.ldv;
#pragma unroll
  for (int j = 0; j < CH; ++j) {
    const int c = first + tid + j * threads;
    if (c >= last) continue;
    if constexpr (kKeepRead) {
#pragma unroll
      for (int i = 0; i < 8; ++i) y[0][i] = Elem<DT>::of(x[j], i);
    }
    float(&yj)[8] = y[kKeepRead ? 0 : j];
    uint32_t b[8], w[2];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float v = code_of<NORM>(yj[i], s);
      b[i] = __float_as_uint(v);
      yj[i] = (v - kRound) * s.scale;
    }
#pragma unroll
    for (int k = 0; k < 2; ++k)
      w[k] = __byte_perm(__byte_perm(b[4 * k], b[4 * k + 1], 0x0040), __byte_perm(b[4 * k + 2], b[4 * k + 3], 0x0040), 0x5410);
    if (COMFUSE_IN_BOUNDS(row < p.rows && 8 * c + 7 < p.N, p.status)) {
      st_8(qrow + 8 * c, w);
      if (p.values) store_chunk<COMFUSE_DTYPE_BF16>(reinterpret_cast<char*>(vrow + 8 * c), yj);
    }
  }
  if (tail) {
    const float v = code_of<NORM>(yt[0], s);
    if (COMFUSE_IN_BOUNDS(row < p.rows && behind < p.N, p.status)) {
      qrow[behind] = static_cast<int8_t>(__float_as_uint(v) & 0xFFu);
      if (p.values) Elem<COMFUSE_DTYPE_BF16>::put(vrow, behind, (v - kRound) * s.scale);
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
  if (verbose_enabled())
    std::fprintf(stderr, "comfuse: quantize_rows dtype=%d norm=%d: %s, chunks=%d ctas=%d threads=%u\n", DT, NORM, WARP ? "a warp a row" : "CTAs a row", CH, p.split, threads);
  count_launch();
  return cudaLaunchKernelEx(&cfg, quantize_rows_kernel<DT, NORM, CH, WARP>, p);
}

template <int DT, bool NORM>
cudaError_t launch_form(QuantizeRowsParams p, const DeviceInfo& dev, cudaStream_t stream) {
  constexpr bool k16 = DT != COMFUSE_DTYPE_F32;
  const int chunks = p.N >= 8 ? p.N / 8 : 1;
  p.split = 1;
  // A warp per row: up to 256 elements; up to 512, and 1024 without the norm, where there are rows enough to fill the machine so.  us, a warp / a CTA
  // per row (16 bits): 777 x 256 norm 2.2 / 2.3, 777 x 512 3.4 / 2.9, 8192 x 512 10.4 / 11.4, 8192 x 1000 16.6 / 15.6, without norm 9.4 / 10.5, 777 x 1000
  // 2.9 / 2.5.  (The machine starts about one CTA a nanosecond: a CTA for each of 60000 short rows takes 63 us whatever it does.)
  if (chunks <= 32 || (p.rows > 2048 && chunks <= (NORM ? 64 : 128))) {
    constexpr int kWarps = 8;
    const unsigned grid = (static_cast<unsigned>(p.rows) + kWarps - 1) / kWarps;
    if (chunks <= 32) return launch_instance<DT, NORM, 1, true>(p, grid, 32 * kWarps, stream);
    if (chunks <= 64) return launch_instance<DT, NORM, 2, true>(p, grid, 32 * kWarps, stream);
    if constexpr (!NORM) return launch_instance<DT, NORM, 4, true>(p, grid, 32 * kWarps, stream);
  }
  // Rows longer than 16384: at most 8192 elements a CTA, so that an SM holds several (2048 x 65536 norm 233 -> 221 us, fp32 436 -> 413).
  if (chunks > 2048)
    while (chunks > p.split * 1024) p.split *= 2;
  // Few rows: CTAs of 256 .. 512 chunks.  us with 1 / 2 / 4 / 8 a row (norm, bf16): 1 x 16384 4.1 / 3.6 / 2.9 / 2.4, 40 x 8192 3.7 / 4.0 / 3.6 / 3.8, 100 x 16384
  // 7.7 / 6.2 / 5.9 / 5.9; 40 x 4096 2.4 / 2.7 / 2.6 / 2.8, so from 8192 on.
  const bool many = static_cast<long long>(p.rows) * chunks >= 4096ll * dev.sm_count;
  if (!many && chunks >= 1024)
    while (p.split < 8 && static_cast<long long>(p.rows) * p.split <= 4ll * dev.sm_count && chunks >= p.split * 512) p.split *= 2;
  const int per = (chunks + p.split - 1) / p.split;
  // Chunks a thread: few where latency counts, many where bytes under way do.  us with 1 / 2 / 4 / 8 (16 bits): norm 40 x 4096 2.6 / 2.4 / 3.5 / 4.7, 600 x
  // 4096 7.8 / 6.7 / 7.4 / 7.8, 8192 x 4096 66 / 55 / 49 / 51; without norm 8192 x 2048 21.0 / 16.3 / 15.5 / 16.3, 8192 x 16384 - / - / 124 / 109; fp32 norm 8192 x
  // 4096 87 / 78 / 79 / 124, without 8192 x 4096 52 / 40 / 38 / 40.
  int ch = many ? (NORM ? (k16 && per >= 256 ? 4 : 2) : k16 ? (per > 512 ? 8 : 4) : (per >= 512 ? 4 : 2))
                : per > 256 || (per > 128 && static_cast<long long>(p.rows) * p.split > dev.sm_count) ? 2 : 1;
  while (per > ch * kMaxThreads) ch *= 2;
  const unsigned threads = static_cast<unsigned>(((per + ch - 1) / ch + 31) / 32 * 32), grid = static_cast<unsigned>(p.rows) * static_cast<unsigned>(p.split);
  if (ch == 1) return launch_instance<DT, NORM, 1, false>(p, grid, threads, stream);
  if (ch == 2) return launch_instance<DT, NORM, 2, false>(p, grid, threads, stream);
  if constexpr (!NORM && k16) {
    if (ch == 8) return launch_instance<DT, NORM, 8, false>(p, grid, threads, stream);
  }
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
