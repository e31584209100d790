// Rows turned by their positions, written into a paged cache (in 8 bits with a scale each) and read back.
//
//   angle = positions[axis(i)][t] * freqs[i];   (a, b) -> (a cos - b sin, a sin + b cos);   s = max|y| / 127,  code = rint(y / s)
//
// Every element is read and written once: the bytes bound it.  The angles of a token are shared by all of its heads: each CTA computes the sines and cosines of its
// tokens once, into shared memory, and then turns their rows.  A row of D is D / 16 units of two 16-byte pieces (16-bit types), one lane each, so that
// both halves of a pair are in one lane and a row in 4, 8, 16 or 32 lanes of one warp; the largest value of a row is a few shuffles away.
#include <cstdio>

#include "kv_params.h"
#include "q8_common.cuh"

namespace comfuse {
namespace {

constexpr int kThreads = 256;
constexpr int kMostAngles = 1024;  // of a CTA's tokens (one of D = 512 has 256)

// How a row's pairs lie.  kHalvesWhole: (i, i + pairs), pairs a multiple of 8: a unit is a piece of the first half and its partner.  kAdjacent: (2i, 2i + 1): a unit is
// 16 elements in line.  kHalves: any other number of pairs: 16 elements in line, and the partners one by one (from the L1).
enum { kNothing, kHalvesWhole, kAdjacent, kHalves };

// Two pieces of 8 elements, the second of which may lie anywhere, or not be there.
template <int DT>
struct Unit {
  uint32_t w[2][2 * Elem<DT>::kBytes];
  int at[2];  // their first elements; at[1] < 0: one piece
};

template <int DT>
__device__ __forceinline__ void load_piece(const char* row, int at, uint32_t* w) {
  ld_16(row + at * Elem<DT>::kBytes, w);
  if constexpr (Elem<DT>::kBytes == 4) ld_16(row + at * 4 + 16, w + 4);
}
template <int DT>
__device__ __forceinline__ void store_piece(char* row, int at, const float (&v)[8]) {
  uint32_t w[2 * Elem<DT>::kBytes];
  Elem<DT>::pack(v, w);
  st_16(row + at * Elem<DT>::kBytes, w);
  if constexpr (Elem<DT>::kBytes == 4) st_16(row + at * 4 + 16, w + 4);
}

// Which pieces unit u of a row has.
template <int MODE>
__device__ __forceinline__ void unit_pieces(int u, int D, int pairs, int (&at)[2]) {
  if (MODE == kHalvesWhole) {
    const int turned = pairs >> 3;
    if (u < turned) {
      at[0] = 8 * u;
      at[1] = 8 * u + pairs;
      return;
    }
    at[0] = 2 * pairs + 16 * (u - turned);
  } else {
    at[0] = 16 * u;
  }
  at[1] = at[0] + 8 < D ? at[0] + 8 : -1;
}

// Elements of a unit, turned.  `cs`, `sn`: of the row's token.  `row`: where the partners of kHalves stand.
template <int DT, int MODE>
__device__ __forceinline__ void turn(const Unit<DT>& unit, const char* row, const float* cs, const float* sn, int pairs, float (&y)[2][8]) {
#pragma unroll
  for (int k = 0; k < 2; ++k)
#pragma unroll
    for (int i = 0; i < 8; ++i) y[k][i] = Elem<DT>::of(unit.w[k], i);
  if (MODE == kHalvesWhole) {
    if (unit.at[0] < pairs) {
      const float4* c4 = reinterpret_cast<const float4*>(cs + unit.at[0]);
      const float4* s4 = reinterpret_cast<const float4*>(sn + unit.at[0]);
      float c[8], s[8];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float4 a = c4[h], b = s4[h];
        c[4 * h] = a.x; c[4 * h + 1] = a.y; c[4 * h + 2] = a.z; c[4 * h + 3] = a.w;
        s[4 * h] = b.x; s[4 * h + 1] = b.y; s[4 * h + 2] = b.z; s[4 * h + 3] = b.w;
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float a = y[0][i], b = y[1][i];
        y[0][i] = a * c[i] - b * s[i];
        y[1][i] = a * s[i] + b * c[i];
      }
    }
  } else if (MODE == kAdjacent) {
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int pair = unit.at[k] / 2 + i;
        if (unit.at[k] >= 0 && pair < pairs) {
          const float a = y[k][2 * i], b = y[k][2 * i + 1], c = cs[pair], s = sn[pair];
          y[k][2 * i] = a * c - b * s;
          y[k][2 * i + 1] = a * s + b * c;
        }
      }
  } else if (MODE == kHalves) {
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int e = unit.at[k] + i;
        if (unit.at[k] >= 0 && e < 2 * pairs) {
          const bool first = e < pairs;
          const int pair = first ? e : e - pairs;
          const float other = Elem<DT>::get(row, first ? e + pairs : pair), c = cs[pair], s = sn[pair];
          y[k][i] = first ? y[k][i] * c - other * s : other * s + y[k][i] * c;
        }
      }
  }
}

constexpr float kRound = 12582912.f;  // 1.5 * 2^23: behind its addition the low byte is the rounded number in two's complement

// The codes of a unit's elements, from the bits of the row's largest magnitude; returns the scale.  The quotient is correctly rounded nearly always (rows of
// 16-bit values meet the middle of two codes often), a row that is not finite has scale NaN and codes 0, as in rows to int8 elsewhere in the library.
__device__ __forceinline__ float codes_of(const float (&y)[2][8], uint32_t top, uint32_t (&w)[2][2]) {
  float amax = __uint_as_float(top);
  const bool finite = top < 0x7F800000u;
  const float lift = amax < 0x1p-100f ? 0x1p100f : 1.f;  // 127 / max stays in fp32
  const float inv = finite && amax > 0.f ? 127.f / (amax * lift) : 0.f;
  const float inv_low = inv > 0.f ? fmaf(-inv, amax * lift, 127.f) / (amax * lift) : 0.f;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    uint32_t b[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float v = finite ? y[k][i] * lift : 0.f;
      b[i] = __float_as_uint(fmaf(v, inv, v * inv_low) + kRound);
    }
#pragma unroll
    for (int h = 0; h < 2; ++h)
      w[k][h] = __byte_perm(__byte_perm(b[4 * h], b[4 * h + 1], 0x0040), __byte_perm(b[4 * h + 2], b[4 * h + 3], 0x0040), 0x5410);
  }
  return finite ? amax / 127.f : __int_as_float(0x7FFFFFFF);
}

// Lanes of a row: the power of two that holds its units.
__host__ __device__ inline int lanes_of(int D, int pairs, int mode) {
  const int units = mode == kHalvesWhole ? pairs / 8 + (D - 2 * pairs + 15) / 16 : (D + 15) / 16;
  int lanes = 1;
  while (lanes < units) lanes *= 2;
  return lanes;
}

template <int DT, bool CACHED, bool Q8, int MODE>
__global__ void __launch_bounds__(kThreads) rotary_write_kernel(const RotaryWriteParams p, const int lanes) {
  __shared__ __align__(16) float s_cos[kMostAngles], s_sin[kMostAngles];
  griddep_launch_dependents();
  griddep_wait();
  const int pairs = p.pairs;
  const int pitch = (pairs + 3) & ~3;  // of a token's angles
  const int first = blockIdx.x * p.tokens_per_cta;
  const int mine = min(p.tokens_per_cta, p.tokens - first);
  if constexpr (MODE != kNothing) {
    for (int i = threadIdx.x; i < mine * pairs; i += kThreads) {
      const int t = i / pairs, pair = i - t * pairs;
      const int axis = (pair >= p.section_end[0]) + (pair >= p.section_end[1]) + (pair >= p.section_end[2]);
      // Whole turns leave in 64 bits: a position of 2^31 at one radian is 3.4e8 turns, known to 2^-24 of a turn.
      const double turns = p.positions[axis * p.axis_stride + first + t] * (p.freqs[pair] * 0.15915494309189535);
      float s, c;
      sincospif(static_cast<float>(2.0 * (turns - rint(turns))), &s, &c);
      s_cos[t * pitch + pair] = c;
      s_sin[t * pitch + pair] = p.sign * s;
    }
    __syncthreads();
  }
  const int rows = p.q_heads + (CACHED ? 2 * p.kv_heads : 0);
  const int groups = kThreads / lanes, u = threadIdx.x % lanes;
  int at[2];
  unit_pieces<MODE>(u, p.D, pairs, at);
  const bool active = at[0] < p.D;

  // Two rows a round: their loads are on the way together.
  int row = threadIdx.x / lanes, t = 0;
  auto settle = [&](int& r, int& tt) {
    while (r >= rows && tt < mine) {
      r -= rows;
      ++tt;
    }
  };
  settle(row, t);
  while (__any_sync(0xFFFFFFFFu, t < mine)) {
    Unit<DT> unit[2];
    const char* in[2] = {nullptr, nullptr};
    int rr[2], tt[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      rr[j] = row;
      tt[j] = t;
      unit[j].at[0] = at[0];
      unit[j].at[1] = at[1];
      if (t < mine) {
        const long long token = first + t;
        const int h = row;
        in[j] = h < p.q_heads                              ? p.q.in + token * p.q.in_token + h * p.q.in_head
                : !CACHED || h < p.q_heads + p.kv_heads ? p.k.in + token * p.k.in_token + (h - p.q_heads) * p.k.in_head
                                                           : p.v.in + token * p.v.in_token + (h - p.q_heads - p.kv_heads) * p.v.in_head;
        if (active) {
          load_piece<DT>(in[j], at[0], unit[j].w[0]);
          if (at[1] >= 0) load_piece<DT>(in[j], at[1], unit[j].w[1]);
        }
      }
      if (!(t < mine && active && at[1] >= 0)) {
#pragma unroll
        for (int i = 0; i < 2 * Elem<DT>::kBytes; ++i) unit[j].w[1][i] = 0u;
      }
      if (!(t < mine && active)) {
#pragma unroll
        for (int i = 0; i < 2 * Elem<DT>::kBytes; ++i) unit[j].w[0][i] = 0u;
      }
      row += groups;
      settle(row, t);
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const bool there = tt[j] < mine, is_q = rr[j] < p.q_heads, is_k = !is_q && rr[j] < p.q_heads + p.kv_heads;
      float y[2][8];
      if (MODE != kNothing && there && active && (is_q || is_k))
        turn<DT, MODE>(unit[j], in[j], s_cos + tt[j] * pitch, s_sin + tt[j] * pitch, pairs, y);
      else {
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
          for (int i = 0; i < 8; ++i) y[k][i] = Elem<DT>::of(unit[j].w[k], i);
      }
      if (MODE == kHalves) __syncwarp();  // every partner is read before a row is written over itself
      const long long token = first + tt[j];
      if (there && is_q) {
        if (active) {
          char* out = p.q.out + token * p.q.out_token + rr[j] * p.q.out_head;
          if (COMFUSE_IN_BOUNDS(token < p.tokens && at[0] + 8 <= p.D && at[1] + 8 <= p.D, p.status)) {
            store_piece<DT>(out, at[0], y[0]);
            if (at[1] >= 0) store_piece<DT>(out, at[1], y[1]);
          }
        }
      }
      if constexpr (CACHED) {
        uint32_t top = 0u;
        if constexpr (Q8) {
#pragma unroll
          for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(y[k][i]) & 0x7FFFFFFFu);
          for (int o = lanes / 2; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
        }
        if (there && !is_q) {
          const long long slot = p.slots[token];
          if (slot >= 0 && slot < p.capacity) {
            const CacheSide& c = is_k ? p.kc : p.vc;
            const long long page = slot / p.page_size, r = slot - page * p.page_size;
            const int h = is_k ? rr[j] - p.q_heads : rr[j] - p.q_heads - p.kv_heads;
            char* out = c.rows + page * c.page + h * c.head + r * c.row;
            if constexpr (Q8) {
              uint32_t w[2][2];
              const float scale = codes_of(y, top, w);
              if (u == 0 && COMFUSE_IN_BOUNDS(h < p.kv_heads && slot < p.capacity, p.status)) c.scale[page * c.scale_page + h * c.scale_head + r * c.scale_row] = scale;
              if (active && COMFUSE_IN_BOUNDS(h < p.kv_heads && slot < p.capacity && at[0] + 8 <= p.D, p.status)) {
                if (MODE == kHalvesWhole && at[1] != at[0] + 8) {
                  st_8(out + at[0], w[0]);
                  st_8(out + at[1], w[1]);
                } else {  // 16 elements in line (D is a multiple of 16)
                  const uint32_t both[4] = {w[0][0], w[0][1], w[1][0], w[1][1]};
                  st_16(out + at[0], both);
                }
              }
            } else if (active && COMFUSE_IN_BOUNDS(h < p.kv_heads && slot < p.capacity && at[0] + 8 <= p.D, p.status)) {
              store_piece<DT>(out, at[0], y[0]);
              if (at[1] >= 0) store_piece<DT>(out, at[1], y[1]);
            }
          }
        }
      }
    }
  }
}

// A lane of the group of `lanes` that has a token's row of a head (keys, then values) reads and writes 16 elements of it.
template <int DT, bool Q8>
__global__ void __launch_bounds__(kThreads) cache_read_kernel(const CacheReadParams p, const int lanes) {
  constexpr int kRows = 4;  // a lane's rows in flight
  griddep_launch_dependents();
  griddep_wait();
  const int groups = kThreads / lanes, u = threadIdx.x % lanes, at = 16 * u;
  if (at >= p.D) return;
  const bool second = at + 8 < p.D;
  const int rows = 2 * p.heads;
  const long long total = static_cast<long long>(p.tokens) * rows;
  const long long first = static_cast<long long>(blockIdx.x) * groups * kRows + threadIdx.x / lanes;
  uint32_t w[kRows][8];
  float scale[kRows];
  char* out[kRows];
#pragma unroll
  for (int j = 0; j < kRows; ++j) {
    const long long i = first + static_cast<long long>(j) * groups;
    out[j] = nullptr;
    if (i >= total) continue;
    const long long token = i / rows;
    const int r = static_cast<int>(i - token * rows);
    const long long slot = p.slots[token];
    if (slot < 0 || slot >= p.capacity) continue;
    const bool is_k = r < p.heads;
    const CacheSide& c = is_k ? p.kc : p.vc;
    const RowsSide& to = is_k ? p.k : p.v;
    const int h = is_k ? r : r - p.heads;
    const long long page = slot / p.page_size, line = slot - page * p.page_size;
    const char* in = c.rows + page * c.page + h * c.head + line * c.row;
    out[j] = to.out + token * to.out_token + h * to.out_head;
    if constexpr (Q8) {
      ld_16(in + at, w[j]);
      scale[j] = c.scale[page * c.scale_page + h * c.scale_head + line * c.scale_row];
    } else {
      ld_16(in + 2 * at, w[j]);
      if (second) ld_16(in + 2 * at + 16, w[j] + 4);
    }
  }
#pragma unroll
  for (int j = 0; j < kRows; ++j) {
    if (!out[j]) continue;
    if constexpr (Q8) {
      float v[2][8];
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int code = static_cast<int8_t>((w[j][i >> 2] >> (8 * (i & 3))) & 0xFFu);
        v[i >> 3][i & 7] = static_cast<float>(code) * scale[j];
      }
      if (COMFUSE_IN_BOUNDS(at + 16 <= p.D, p.status)) {
        store_piece<DT>(out[j], at, v[0]);
        store_piece<DT>(out[j], at + 8, v[1]);
      }
    } else if (COMFUSE_IN_BOUNDS(at + 8 <= p.D, p.status)) {
      st_16(out[j] + 2 * at, w[j]);
      if (second) st_16(out[j] + 2 * at + 16, w[j] + 4);
    }
  }
}

template <typename Kernel, typename Params>
cudaError_t launch(Kernel kernel, const Params& p, int lanes, unsigned grid, cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[1];
  cfg.gridDim = dim3(grid, 1, 1);
  cfg.blockDim = dim3(kThreads, 1, 1);
  cfg.stream = stream;
  if (programmatic_launch_enabled()) {
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
  }
  count_launch();
  return cudaLaunchKernelEx(&cfg, kernel, p, lanes);
}

template <int DT, bool CACHED, bool Q8>
cudaError_t launch_mode(int mode, const RotaryWriteParams& p, unsigned grid, cudaStream_t stream) {
  const int lanes = lanes_of(p.D, p.pairs, mode);
  switch (mode) {
    case kHalvesWhole: return launch(rotary_write_kernel<DT, CACHED, Q8, kHalvesWhole>, p, lanes, grid, stream);
    case kAdjacent: return launch(rotary_write_kernel<DT, CACHED, Q8, kAdjacent>, p, lanes, grid, stream);
    case kHalves: return launch(rotary_write_kernel<DT, CACHED, Q8, kHalves>, p, lanes, grid, stream);
    default: break;
  }
  if constexpr (CACHED) return launch(rotary_write_kernel<DT, CACHED, Q8, kNothing>, p, lanes, grid, stream);
  return cudaErrorInvalidValue;
}

}  // namespace

cudaError_t launch_rotary_write(int dtype, bool cached, bool quantized, RotaryWriteParams p, const DeviceInfo& dev, cudaStream_t stream) {
  const int mode = !p.positions ? kNothing : p.adjacent ? kAdjacent : p.pairs % 8 == 0 ? kHalvesWhole : kHalves;
  if (mode == kNothing) p.pairs = 0;
  const int pitch = (p.pairs + 3) & ~3;
  // Tokens of a CTA: one where there are few, else as many as give its threads two rows each.
  const int rows = p.q_heads + (cached ? 2 * p.kv_heads : 0), groups = kThreads / lanes_of(p.D, p.pairs, mode);
  int per = 1;
  while (2 * per * pitch <= kMostAngles && per * rows < 2 * groups && static_cast<long long>(p.tokens) >= 8ll * per * dev.sm_count) per *= 2;
  p.tokens_per_cta = per;
  const unsigned grid = static_cast<unsigned>((static_cast<long long>(p.tokens) + per - 1) / per);
  if (verbose_enabled())
    std::fprintf(stderr, "comfuse: rotary_write dtype=%d cached=%d quantized=%d mode=%d tokens a CTA=%d\n", dtype, cached, quantized, mode, per);
  if (!cached) {
    switch (dtype) {
      case COMFUSE_DTYPE_BF16: return launch_mode<COMFUSE_DTYPE_BF16, false, false>(mode, p, grid, stream);
      case COMFUSE_DTYPE_F16: return launch_mode<COMFUSE_DTYPE_F16, false, false>(mode, p, grid, stream);
      default: return launch_mode<COMFUSE_DTYPE_F32, false, false>(mode, p, grid, stream);
    }
  }
  if (dtype == COMFUSE_DTYPE_BF16)
    return quantized ? launch_mode<COMFUSE_DTYPE_BF16, true, true>(mode, p, grid, stream) : launch_mode<COMFUSE_DTYPE_BF16, true, false>(mode, p, grid, stream);
  return quantized ? launch_mode<COMFUSE_DTYPE_F16, true, true>(mode, p, grid, stream) : launch_mode<COMFUSE_DTYPE_F16, true, false>(mode, p, grid, stream);
}

cudaError_t launch_cache_read(int dtype, bool quantized, const CacheReadParams& p, const DeviceInfo&, cudaStream_t stream) {
  const int lanes = lanes_of(p.D, 0, kNothing);
  const long long rows = 2ll * p.heads * p.tokens, per = 4ll * (kThreads / lanes);
  const long long grid = (rows + per - 1) / per;
  if (grid > 0x7FFFFFFF) return cudaErrorInvalidValue;
  const unsigned n = static_cast<unsigned>(grid);
  if (dtype == COMFUSE_DTYPE_BF16)
    return quantized ? launch(cache_read_kernel<COMFUSE_DTYPE_BF16, true>, p, lanes, n, stream) : launch(cache_read_kernel<COMFUSE_DTYPE_BF16, false>, p, lanes, n, stream);
  return quantized ? launch(cache_read_kernel<COMFUSE_DTYPE_F16, true>, p, lanes, n, stream) : launch(cache_read_kernel<COMFUSE_DTYPE_F16, false>, p, lanes, n, stream);
}

}  // namespace comfuse
