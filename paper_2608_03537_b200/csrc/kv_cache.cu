// Rows turned by their positions, written into a paged cache (in 8 bits with a scale each) and read back.
//
//   angle = positions[axis(i)][t] * freqs[i];   (a, b) -> (a cos - b sin, a sin + b cos);   s = max|y| / 127,  code = rint(y / s)
//
// Every element is read and written once: the bytes bound it.  A row of D is D / 16 units of two 16-byte pieces (16-bit types), one lane each, so that both halves of a
// pair are in one lane and a row in a power of two of lanes of one warp; the largest value of a row is a few shuffles away.  The angles of a token are shared by all of its
// heads: a warp computes the sines and cosines of its token once, two pairs a lane, and each lane keeps those of its unit while it turns row after row.  Where there are few tokens
// several warps share one, each with its own sines.
//
// On one B200 (copies run at 6.5 TB/s), replayed as a graph: 16384 x 24 x 128 bf16 turned in 33.5 us = 6.0 TB/s, fp32 in 65.3 = 6.2, with pairs side by side in 81; 8192 tokens, 32 heads of queries
// turned and 2 x 8 of keys and values written, 35 us = 5.8 TB/s, into 8 bits 42.5 = 4.4; one such token 2.1 us: launch and one round trip; 32768 x 8 x 128 read back from 8 bits 36.5 us =
// 5.6 TB/s, from 16 bits 43.7 = 6.1.  Called one by one the short ones take what the host takes (one token 4.3 to 4.7 us), and the read-back from 8 bits 38.6.
#include <cmath>
#include <cstdio>

#include "kv_params.h"
#include "q8_common.cuh"

namespace comfuse {
namespace {

// Two warps a CTA: an SM takes the next one as soon as two are done (256 threads, all as graphs: 32768 x 8 x 128 read back in 38.6 us instead of 36.4, 16384 x 24 x 128 turned with pairs side by side in 39.3 instead
// of 36.2, 777 x 12 x 64 fp32 in 3.7 instead of 3.1).
constexpr int kThreads = 64;
constexpr int kMostPairs = 256;  // (D <= 512)

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

// The sines and cosines of a unit's eight pairs, from the token's; pairs behind the last do not turn.
template <int MODE>
__device__ __forceinline__ void unit_angles(const float2* angles, int first, int pairs, float2 (&cs)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) cs[i] = first + i < pairs ? angles[first + i] : make_float2(1.f, 0.f);
}

// Elements of a unit, turned.  `cs`: of its pairs (kHalvesWhole, kAdjacent); `angles`, `row`: the token's, and where the partners of kHalves stand.
template <int DT, int MODE>
__device__ __forceinline__ void turn(const Unit<DT>& unit, const float2 (&cs)[8], const char* row, const float2* angles, int pairs, float (&y)[2][8]) {
#pragma unroll
  for (int k = 0; k < 2; ++k)
#pragma unroll
    for (int i = 0; i < 8; ++i) y[k][i] = Elem<DT>::of(unit.w[k], i);
  if (MODE == kHalvesWhole) {
    if (unit.at[0] < pairs) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float a = y[0][i], b = y[1][i];
        y[0][i] = a * cs[i].x - b * cs[i].y;
        y[1][i] = a * cs[i].y + b * cs[i].x;
      }
    }
  } else if (MODE == kAdjacent) {
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float a = y[k][2 * i], b = y[k][2 * i + 1];
        const float2 z = cs[4 * k + i];
        // (elements behind the pairs stay as they are, whatever they hold)
        if (unit.at[0] / 2 + 4 * k + i < pairs) {
          y[k][2 * i] = a * z.x - b * z.y;
          y[k][2 * i + 1] = a * z.y + b * z.x;
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
          const float other = Elem<DT>::get(row, first ? e + pairs : pair);
          const float2 z = angles[pair];
          y[k][i] = first ? y[k][i] * z.x - other * z.y : other * z.y + y[k][i] * z.x;
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

// Lanes of a row: the power of two that holds its units (its logarithm).
int lanes_log2_of(int D, int pairs, int mode) {
  const int units = mode == kHalvesWhole ? pairs / 8 + (D - 2 * pairs + 15) / 16 : (D + 15) / 16;
  int n = 0;
  while ((1 << n) < units) ++n;
  return n;
}

// Warps an SM: 8192 tokens (above) 43.2 us with 16, 38.7 with 24, 41.8 with 32, whose registers no longer hold two rows and the sines; fp32 rows are twice as large, and 16 warps hold them.
constexpr int warps_of(int dtype) { return dtype == COMFUSE_DTYPE_F32 ? 16 : 24; }
template <int DT, bool CACHED, bool Q8, int MODE>
__global__ void __launch_bounds__(kThreads, warps_of(DT) * 32 / kThreads) rotary_write_kernel(const RotaryWriteParams p, const int lanes_log2) {
  __shared__ float2 s_angles[MODE == kNothing ? 1 : kThreads / 32][MODE == kNothing ? 1 : kMostPairs];
  griddep_launch_dependents();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const long long item = static_cast<long long>(blockIdx.x) * (kThreads / 32) + warp;
  const long long token = item >> p.slices_log2;
  if (token >= p.tokens) return;  // (whole warps, which share nothing with others)
  const int pairs = p.pairs, lanes = 1 << lanes_log2, u = lane & (lanes - 1);
  const unsigned rows = p.rows, step = (32u >> lanes_log2) << p.slices_log2;
  int at[2];
  unit_pieces<MODE>(u, p.D, pairs, at);
  const bool active = at[0] < p.D, second = at[1] >= 0;
  griddep_wait();

  long long place = -1;
  if constexpr (CACHED) place = p.slots[token];
  // Two rows a round, whose loads are on the way together.
  unsigned next = ((static_cast<unsigned>(item) & ((1u << p.slices_log2) - 1)) << (5 - lanes_log2)) + (lane >> lanes_log2);
  Unit<DT> unit[2];
  const char* in[2];
  unsigned row[2], kind[2];
  bool there[2];
  auto load = [&]() {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      there[j] = next < rows;
      row[j] = next;
      next += step;
      kind[j] = 0;
      if constexpr (CACHED) {
        const unsigned q_heads = p.q_heads, kv_heads = p.kv_heads;
        if (row[j] >= q_heads) {
          kind[j] = row[j] >= q_heads + kv_heads ? 2 : 1;
          row[j] -= kind[j] == 2 ? q_heads + kv_heads : q_heads;
        }
      }
      const RowsSide& side = p.side[kind[j]];
      in[j] = side.in + token * side.in_token + row[j] * side.in_head;
      unit[j].at[0] = at[0];
      unit[j].at[1] = at[1];
      if (there[j] && active) {
        load_piece<DT>(in[j], at[0], unit[j].w[0]);
        if (second) load_piece<DT>(in[j], at[1], unit[j].w[1]);
      }
    }
  };
  load();
  float2* angles = s_angles[MODE == kNothing ? 0 : warp];
  float2 cs[8];
  if constexpr (MODE != kNothing) {  // (under the first rows' loads)
    for (int pair = lane; pair < pairs; pair += 32) {
      const int axis = (pair >= p.section_end[0]) + (pair >= p.section_end[1]) + (pair >= p.section_end[2]);
      // Whole turns leave in 64 bits: a position of 2^31 at one radian is 3.4e8 turns, known to 2^-24 of a turn.
      const double turns = p.positions[axis * p.axis_stride + token] * (p.freqs[pair] * 0.15915494309189535);
      float s, c;
      sincospif(static_cast<float>(2.0 * (turns - rint(turns))), &s, &c);
      angles[pair] = make_float2(c, p.sign * s);
    }
    __syncwarp();
    if constexpr (MODE != kHalves) unit_angles<MODE>(angles, MODE == kAdjacent ? 8 * u : at[0], pairs, cs);
  }
  const int slot = place >= 0 && place < p.capacity ? static_cast<int>(place) : -1;
  unsigned page = 0, line = 0;
  if constexpr (CACHED) {
    page = p.page_size.of(slot);
    line = slot - page * p.page_size.d;
  }
  while (__any_sync(0xFFFFFFFFu, there[0])) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      float y[2][8];
      if (MODE != kNothing && (!CACHED || kind[j] < 2)) {
        if (MODE != kHalves || (there[j] && active)) turn<DT, MODE>(unit[j], cs, in[j], angles, pairs, y);
      } else {
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
          for (int i = 0; i < 8; ++i) y[k][i] = Elem<DT>::of(unit[j].w[k], i);
      }
      if (MODE == kHalves) __syncwarp();  // every partner is read before a row is written over itself
      if (kind[j] == 0) {
        const RowsSide& side = p.side[0];
        char* out = side.out + token * side.out_token + row[j] * side.out_head;
        if (there[j] && active && COMFUSE_IN_BOUNDS(token < p.tokens && at[0] + 8 <= p.D && at[1] + 8 <= p.D, p.status)) {
          store_piece<DT>(out, at[0], y[0]);
          if (second) store_piece<DT>(out, at[1], y[1]);
        }
      }
      if constexpr (CACHED) {
        uint32_t top = 0u;
        if constexpr (Q8) {
          if (active) {
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
              for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(y[k][i]) & 0x7FFFFFFFu);
          }
          for (int o = lanes / 2; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
        }
        if (kind[j] && there[j] && slot >= 0) {
          const CacheSide& c = kind[j] == 1 ? p.kc : p.vc;
          const unsigned h = row[j];
          char* out = c.rows + page * c.page + h * c.head + line * c.row;
          if constexpr (Q8) {
            uint32_t w[2][2];
            const float scale = codes_of(y, top, w);
            if (u == 0 && COMFUSE_IN_BOUNDS(h < p.kv_heads && slot < p.capacity, p.status)) c.scale[page * c.scale_page + h * c.scale_head + line * c.scale_row] = scale;
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
            if (second) store_piece<DT>(out, at[1], y[1]);
          }
        }
      }
    }
    load();
  }
}

// A lane of the group of `lanes` that has a token's row of a head (keys, then values) reads and writes 16 elements of it.  ROWS: of a lane, in flight together.  Neighbouring groups have the
// same head of neighbouring tokens, so that a page is read in line; the rows of a few tokens' heads, which lie in line where they go, are still written by one CTA.
template <int DT, bool Q8, int ROWS>
__global__ void __launch_bounds__(kThreads) cache_read_kernel(const CacheReadParams p, const int lanes_log2) {
  griddep_launch_dependents();
  griddep_wait();
  const int groups = kThreads >> lanes_log2, at = 16 * (threadIdx.x & ((1 << lanes_log2) - 1));
  if (at >= p.D) return;
  const bool second = at + 8 < p.D;
  const unsigned first = blockIdx.x * (groups * ROWS) + (threadIdx.x >> lanes_log2);
  uint32_t w[ROWS][8];
  float scale[ROWS];
  char* out[ROWS];
  unsigned token[ROWS], row[ROWS];
  long long slot[ROWS];
#pragma unroll
  for (int j = 0; j < ROWS; ++j) {
    const unsigned i = first + j * groups;
    const unsigned line = i >> p.tokens_log2, block = p.rows.of(line);
    row[j] = line - block * p.rows.d;
    token[j] = (block << p.tokens_log2) + (i & ((1u << p.tokens_log2) - 1));
    slot[j] = token[j] < static_cast<unsigned>(p.tokens) ? p.slots[token[j]] : -1;
  }
#pragma unroll
  for (int j = 0; j < ROWS; ++j) {
    const unsigned r = row[j];
    out[j] = nullptr;
    if (slot[j] < 0 || slot[j] >= p.capacity) continue;
    const bool is_k = r < static_cast<unsigned>(p.heads);
    const CacheSide& c = is_k ? p.kc : p.vc;
    const RowsSide& to = is_k ? p.k : p.v;
    const unsigned h = is_k ? r : r - p.heads, n = static_cast<unsigned>(slot[j]);
    const long long page = p.page_size.of(n), line = n - page * p.page_size.d;
    const char* in = c.rows + page * c.page + h * c.head + line * c.row;
    out[j] = to.out + token[j] * to.out_token + h * to.out_head;
    if constexpr (Q8) {
      ld_16(in + at, w[j]);
      scale[j] = c.scale[page * c.scale_page + h * c.scale_head + line * c.scale_row];
    } else {
      ld_16(in + 2 * at, w[j]);
      if (second) ld_16(in + 2 * at + 16, w[j] + 4);
    }
  }
#pragma unroll
  for (int j = 0; j < ROWS; ++j) {
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
cudaError_t launch(Kernel kernel, const Params& p, int lanes_log2, unsigned grid, cudaStream_t stream) {
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
  return cudaLaunchKernelEx(&cfg, kernel, p, lanes_log2);
}

template <int DT, bool CACHED, bool Q8>
cudaError_t launch_mode(int mode, const RotaryWriteParams& p, unsigned grid, cudaStream_t stream) {
  const int lanes = lanes_log2_of(p.D, p.pairs, mode);
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
  p.rows = p.q_heads + (cached ? 2 * p.kv_heads : 0);
  // Warps of a token: by how many rounds of warps there are (the last one, which has the memory to itself, counts 0.7 and 0.3 of its share), and what a warp does in one: its sines and start, about as
  // long as two rows a lane, and its rows, two a lane at a time (8192 tokens, 32 + 2 x 8 heads of 128: 36.8 us with one, 34.9 with two, 41 with four; 3000: 15.1 and 17.0; 2000: 12.3 and 11.7;
  // 4096 of 256: 44.1 and 37.7).
  const int groups = 32 >> lanes_log2_of(p.D, p.pairs, mode), at_once = dev.sm_count * warps_of(dtype);
  double least = 0;
  for (int n = 0; n == 0 || (2 * groups) << (n - 1) < p.rows; ++n) {
    const double full = std::ldexp(static_cast<double>(p.tokens), n) / at_once, rounds = full <= 1 ? 1.0 : 0.7 * std::ceil(full) + 0.3 * full;
    const double time = rounds * (1 + (p.rows + (2 * groups << n) - 1) / (2 * groups << n));
    if (n > 0 && time >= least) continue;
    least = time;
    p.slices_log2 = n;
  }
  const long long warps = static_cast<long long>(p.tokens) << p.slices_log2;
  const unsigned grid = static_cast<unsigned>((warps + kThreads / 32 - 1) / (kThreads / 32));
  if (verbose_enabled())
    std::fprintf(stderr, "comfuse: rotary_write dtype=%d cached=%d quantized=%d mode=%d warps a token=%d\n", dtype, cached, quantized, mode, 1 << p.slices_log2);
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

namespace {
template <int DT, bool Q8>
cudaError_t launch_read(CacheReadParams p, const DeviceInfo& dev, cudaStream_t stream) {
  const int lanes = lanes_log2_of(p.D, 0, kNothing), groups = kThreads >> lanes;
  // Eight tokens a block where that leaves no group without one; several rows a lane where they still fill the GPU, four only of 8 bits (as graphs: 32768 x 8 x 128 from 8 bits 38.6 us with two, 36.4 with four;
  // from 16 bits 43.9 and 46.2; 4000 x 8 x 128 from 8 bits 9.1 us with one, 6.7 with two, 8.4 with four).
  while (p.tokens_log2 < 3 && p.tokens % (2 << p.tokens_log2) == 0) ++p.tokens_log2;
  if (p.tokens >= 64) p.tokens_log2 = 3;
  const long long blocks = (p.tokens + (1ll << p.tokens_log2) - 1) >> p.tokens_log2, rows = (blocks << p.tokens_log2) * p.rows.d, ctas = rows / groups;
  const int per = Q8 && ctas >= 128ll * dev.sm_count ? 4 : ctas >= 16ll * dev.sm_count ? 2 : 1;
  const unsigned grid = static_cast<unsigned>((rows + per * groups - 1) / (per * groups));
  if constexpr (Q8)
    if (per == 4) return launch(cache_read_kernel<DT, Q8, 4>, p, lanes, grid, stream);
  return per == 2 ? launch(cache_read_kernel<DT, Q8, 2>, p, lanes, grid, stream) : launch(cache_read_kernel<DT, Q8, 1>, p, lanes, grid, stream);
}
}  // namespace

cudaError_t launch_cache_read(int dtype, bool quantized, const CacheReadParams& p, const DeviceInfo& dev, cudaStream_t stream) {
  if (dtype == COMFUSE_DTYPE_BF16) return quantized ? launch_read<COMFUSE_DTYPE_BF16, true>(p, dev, stream) : launch_read<COMFUSE_DTYPE_BF16, false>(p, dev, stream);
  return quantized ? launch_read<COMFUSE_DTYPE_F16, true>(p, dev, stream) : launch_read<COMFUSE_DTYPE_F16, false>(p, dev, stream);
}

}  // namespace comfuse
