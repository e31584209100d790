// Attention of a few new tokens over a paged cache, split over the cache's length and joined.
//
//   s[n] = cap(alpha q . k[n]) + slope (n - m);   out = sum_n softmax(s)[n] v[n]
//
// Every visible key and value is read once, and for few queries that is all there is to bound it: 2 D (or 4 D) flops an element of a query row against HBM.  So the
// kernel is built around loads in flight.
//
//   * The call's work is a line of units of 64 positions (sequence by sequence, key head by key head), cut into equal shares, one for each of the CTAs that fit on the
//     GPU: whatever the lengths, all finish together.  A CTA finds its share from the lengths themselves.  An item (sequence, key head) that lies in one share is
//     finished there; one that is cut leaves a partial sum, maximum and weighted values for each share, and a second kernel joins them, in order.
//   * A unit is four blocks of 16 positions, one for each warp.  A warp is on its own: it fetches its blocks by 16-byte asynchronous copies, several blocks ahead and across the
//     ends of items, into a ring of its own, and keeps a running maximum, sum and weighted values; no barrier but at the end of an item, where the four are joined.
//   * The keys are the 16-row operand of the warp-wide matrix instruction and the queries the 8-column one: S^T = K Q^T, then O^T += V^T P^T.  The queries that share a key head
//     (tokens x heads of its group) fill eight columns a tile, so that a single query wastes an eighth of what rows of sixteen would.  P^T changes from the accumulators' layout to
//     the operand's by two 8x8 transposes.
//   * 8 bits: the codes become fp16 by two permutes and a subtraction for each four, the key's scale is a factor of its score and the value's scale of its weight.  Codes of a row are
//     taken as they lie in the registers; queries, and the rows of O^T, are permuted alike.
//   * The maximum is renewed only when a score is more than 8 (a factor of 256) above it: a vote instead of a reduction in most blocks.
#pragma once

#include <cstdio>

#include "kv_params.h"
#include "q8_common.cuh"

namespace comfuse {
namespace paged {

cudaError_t launch_bf16(const PagedAttentionPlan& plan, const PagedAttentionParams& p, cudaStream_t stream);
cudaError_t launch_f16(const PagedAttentionPlan& plan, const PagedAttentionParams& p, cudaStream_t stream);
cudaError_t launch_bf16_q8(const PagedAttentionPlan& plan, const PagedAttentionParams& p, cudaStream_t stream);
cudaError_t launch_f16_q8(const PagedAttentionPlan& plan, const PagedAttentionParams& p, cudaStream_t stream);

namespace {

constexpr int kWarps = 4, kThreads = 32 * kWarps;
constexpr int kBlock = 16;              // positions of a warp's step
constexpr int kUnit = kBlock * kWarps;  // of a CTA's
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kSlack = 8.f;           // log2 of what a weight may exceed 1 by

// Sizes of an instance: D up to DH, NT tiles of eight queries.
template <bool Q8, int DH, int NT>
struct Form {
  static constexpr int kRowBytes = DH * (Q8 ? 1 : 2);
  static constexpr int kPieces = kRowBytes / 16;             // of a row
  static constexpr int kSide = kBlock * kRowBytes;           // keys, or values, of a block
  static constexpr int kStage = 2 * kSide + (Q8 ? 128 : 0);  // and their scales
  static constexpr int kJoinColumns = NT == 4 ? 32 : 64;     // where warps are joined, at a time
  static constexpr int kPitch = kJoinColumns + 4;            // floats of a row there: a warp's stores fall on all banks
  static constexpr int kJoin = kWarps * 8 * kPitch * 4;
  static constexpr int kQuery = 8 * NT * DH * 2;
  static constexpr int kSmall = 704 + 64 * 8 * NT;
  static constexpr int kCtasPerSm = DH == 256 && !Q8 ? 1 : 2;
  static constexpr int kSmem = (kCtasPerSm == 2 ? 113 : 226) * 1024;  // what a CTA may take
  static constexpr int kStages = (kSmem - kJoin - kQuery - kSmall) / (kStage * kWarps);
  static constexpr int kBytes = kStages * kStage * kWarps + kJoin + kQuery + kSmall;
};

// Partial results of CTA c: two slots (of the first item of its share, and of the last), each 8 NT rows of kPartRow floats: D values, the maximum, the sum.
__host__ __device__ inline long long part_floats(int rows8, int D) { return 2ll * rows8 * (D + 4); }

// ------------------------------------------------------------------------------------------------ shares
// The line of units.  Sequence b has units(b) units for each of its `hr` items (key heads x row blocks).
struct Line {
  long long total, share, longer;  // the first `longer` CTAs have share + 1 units
  __device__ long long begin(long long cta) const { return cta * share + (cta < longer ? cta : longer); }
  __device__ long long owner(long long unit) const {
    const long long l = longer * (share + 1);
    return unit < l ? unit / (share + 1) : longer + (unit - l) / share;
  }
};
struct Sequence {
  int length, low, units;  // positions low .. length - 1 are visible to some token; units are counted from low rounded down to a block
};
__device__ __forceinline__ Sequence sequence_of(const PagedAttentionParams& p, int b) {
  Sequence s;
  s.length = min(max(p.lengths[b], 0), p.max_length);
  s.low = p.window > 0 ? max(0, s.length - p.tokens + 1 - p.window) : 0;
  s.units = max(1, (s.length - (s.low & ~(kBlock - 1)) + kUnit - 1) / kUnit);  // (an empty sequence has a unit too: its rows are written)
  return s;
}
struct Place {
  int b, hr, unit;
};
// By all of a CTA's threads (the first kThreads of them): the line, and where `n` units given as the function of the line lie.
struct Scan {
  long long warp_sum[kWarps];
  Place place;
};
template <typename UnitOf>
__device__ __forceinline__ Line find(const PagedAttentionParams& p, Scan* s, UnitOf unit_of, Place* place) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int per = (p.batch + kThreads - 1) / kThreads;
  const long long hr = static_cast<long long>(p.heads) * p.row_blocks;
  const int b0 = min(tid * per, p.batch), b1 = min(b0 + per, p.batch);
  long long mine = 0;
  for (int b = b0; b < b1; ++b) mine += sequence_of(p, b).units;
  long long upto = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long v = __shfl_up_sync(0xFFFFFFFFu, upto, o);
    if (lane >= o) upto += v;
  }
  if (lane == 31) s->warp_sum[warp] = upto;
  __syncthreads();
  long long before = 0, total = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    if (w < warp) before += s->warp_sum[w];
    total += s->warp_sum[w];
  }
  before += upto - mine;
  Line line;
  line.total = total * hr;
  line.share = line.total / p.ctas;
  line.longer = line.total - line.share * p.ctas;
  const long long unit = unit_of(line);
  if (unit >= before * hr && unit < (before + mine) * hr) {
    long long rest = unit - before * hr;
    for (int b = b0; b < b1; ++b) {
      const long long n = sequence_of(p, b).units;
      if (rest < n * hr) {
        s->place.b = b;
        s->place.hr = static_cast<int>(rest / n);
        s->place.unit = static_cast<int>(rest - s->place.hr * n);
        break;
      }
      rest -= n * hr;
    }
  }
  __syncthreads();
  *place = s->place;
  return line;
}

// ------------------------------------------------------------------------------------------------ instructions
__device__ __forceinline__ void cp_async_16(uint32_t dst, const void* src, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_async_4(uint32_t dst, const void* src, bool there) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(there ? 4 : 0) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ void ldmatrix_x4(uint32_t at, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void ldmatrix_x4_trans(uint32_t at, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ uint32_t transpose_8x8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
template <bool BF16>
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if constexpr (BF16)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// Two codes of x (chosen by `bytes`, whose even places name them) as fp16: 0x6400 + u is 1024 + u, u = code + 128.
__device__ __forceinline__ uint32_t codes_f16(uint32_t flipped, uint32_t bytes) {
  const uint32_t raw = __byte_perm(flipped, 0x64646464u, bytes);
  uint32_t y;
  asm("sub.f16x2 %0, %1, %2;" : "=r"(y) : "r"(raw), "r"(0x64806480u));
  return y;
}
template <bool BF16>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  return BF16 ? pack_bf16x2_rn(a, b) : pack_f16x2_rn(a, b);
}
template <bool BF16>
__device__ __forceinline__ float2 unpack2(uint32_t w) {
  if constexpr (BF16) return make_float2(bf16_lo(w), bf16_hi(w));
  else return __half22float2(*reinterpret_cast<const __half2*>(&w));
}
// 1 / x for x = 2^n, |n| < 127; anything for 0
__device__ __forceinline__ float reciprocal_of_power(float x) { return __uint_as_float(0x7F000000u - __float_as_uint(x)); }
// log of a sum whose terms were divided by 2^m; nothing: -inf
__device__ __forceinline__ float log_sum(float m, float l) {
  if (m == -INFINITY) return l == 0.f ? -INFINITY : l;  // (else a NaN)
  return m * 0.6931471805599453f + logf(l);
}
// Piece c of row r lies at place c ^ (...): the eight rows that an ldmatrix reads at once are on eight different groups of banks.
template <int PIECES>
__device__ __forceinline__ int place_of(int r, int c) {
  return PIECES >= 8 ? c ^ (r & 7) : c ^ ((r >> 1) & 3);
}

// ------------------------------------------------------------------------------------------------ the kernel
template <int DT, bool Q8, int DH, int NT>
__global__ void __launch_bounds__(kThreads, Form<Q8, DH, NT>::kCtasPerSm) attention_kernel(const PagedAttentionParams p) {
  using F = Form<Q8, DH, NT>;
  constexpr bool kBf16 = DT == COMFUSE_DTYPE_BF16;  // of queries and outputs
  constexpr bool kMmaBf16 = kBf16 && !Q8;           // of the products: 8-bit codes are exact in fp16
  // A weight in 16 bits is off by half a step of its type, which behind a sum over like terms is as much as the output's own rounding.  So the weights go in twice, rounded and what
  // the rounding left.  fp16 weights of bf16 outputs are eight times as fine as those and go in once.
  constexpr bool kTwice = !(Q8 && kBf16);
  constexpr int kSteps = DH / 16;
  constexpr int S = F::kStages;
  static_assert(S >= 2, "a ring of two blocks at least");
  extern __shared__ __align__(128) char smem[];
  char* s_ring = smem;
  float* s_join = reinterpret_cast<float*>(smem + S * F::kStage * kWarps);
  char* s_query = reinterpret_cast<char*>(s_join) + F::kJoin;
  struct Small {
    Scan scan;
    unsigned valid[kWarps][32];         // of the blocks in the ring: positions that are there
    float top[kWarps][8 * NT], sum[kWarps][8 * NT];
    float factor[8 * NT];               // 8 bits: what a query was divided by
    float slope[8 * NT];
    int token[8 * NT];                  // a row's new token
    long long out[8 * NT];              // where its output goes (-1: nowhere)
    int lse[8 * NT];
  };
  static_assert(sizeof(Small) <= F::kSmall && S <= 32, "room for what is small");
  Small& sm = *reinterpret_cast<Small*>(s_query + F::kQuery);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int g = lane >> 2, c = lane & 3;

  griddep_wait();
  griddep_launch_dependents();  // behind the wait: the joining kernel reads the lengths before its own

  Place at;
  const Line line = find(p, &sm.scan, [](const Line& l) { return min(l.begin(blockIdx.x), l.total - 1); }, &at);
  const long long first_unit = line.begin(blockIdx.x);
  const int count = static_cast<int>(line.begin(blockIdx.x + 1) - first_unit);
  if (count <= 0) return;
  const int HR = p.heads * p.row_blocks;

  char* ring = s_ring + warp * S * F::kStage;
  const uint32_t ring_u32 = smem_u32(ring);
  if (p.D < DH) {  // pieces behind D are never fetched and stay zeros
    for (int i = lane; i < S * F::kStage / 16; i += 32) reinterpret_cast<uint4*>(ring)[i] = make_uint4(0, 0, 0, 0);
    __syncwarp();
  }

  // ---- fetching, several blocks ahead
  int f_b = at.b, f_hr = at.hr, f_unit = at.unit, f_left = count;
  Sequence f_seq = sequence_of(p, f_b);
  int f_page = -1;  // of position (lane & 15) of the block that is next
  const bool whole_pages = p.page_size % kBlock == 0;  // a block lies in one page
  auto look_up = [&]() {
    const int pos = (f_seq.low & ~(kBlock - 1)) + f_unit * kUnit + warp * kBlock + (lane & 15);
    f_page = -1;
    if (f_left > 0 && pos >= f_seq.low && pos < f_seq.length) f_page = p.table[f_b * p.table_stride + pos / p.page_size];
  };
  look_up();
  const int D_bytes = p.D * (Q8 ? 1 : 2);
  constexpr int kLoads = F::kPieces / 2, kRowsALoad = 32 / F::kPieces;
  const int my_row = lane / F::kPieces, my_piece = lane % F::kPieces;
  const bool my_piece_there = my_piece * 16 < D_bytes;
  auto fetch = [&](int stage) {
    if (f_left > 0) {
      const bool there = f_page >= 0 && f_page < p.pages;
      const unsigned valid = __ballot_sync(0xFFFFFFFFu, there) & 0xFFFFu;
      if (lane == 0) sm.valid[warp][stage] = valid;
      if (valid) {
        const int head = f_hr / p.row_blocks;
        const int pos = (f_seq.low & ~(kBlock - 1)) + f_unit * kUnit + warp * kBlock + (lane & 15);
        const long long page = there ? f_page : 0, row = there ? pos % p.page_size : 0;
        const uint32_t dst = ring_u32 + stage * F::kStage;
        const long long k_at = page * p.kc.page + head * p.kc.head + row * p.kc.row, v_at = page * p.vc.page + head * p.vc.head + row * p.vc.row;
        if (valid == 0xFFFFu && whole_pages) {
          const char* k = p.kc.rows + __shfl_sync(0xFFFFFFFFu, k_at, 0) + my_row * p.kc.row + my_piece * 16;
          const char* v = p.vc.rows + __shfl_sync(0xFFFFFFFFu, v_at, 0) + my_row * p.vc.row + my_piece * 16;
          if (my_piece_there) {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
              const int r = i * kRowsALoad + my_row;
              const uint32_t to = dst + r * F::kRowBytes + place_of<F::kPieces>(r, my_piece) * 16;
              cp_async_16(to, k + i * kRowsALoad * p.kc.row, true);
              cp_async_16(to + F::kSide, v + i * kRowsALoad * p.vc.row, true);
            }
          }
        } else {
#pragma unroll
          for (int i = 0; i < kLoads; ++i) {
            const int r = i * kRowsALoad + my_row;
            const char* k = p.kc.rows + __shfl_sync(0xFFFFFFFFu, k_at, r) + my_piece * 16;
            const char* v = p.vc.rows + __shfl_sync(0xFFFFFFFFu, v_at, r) + my_piece * 16;
            const bool ok = (valid >> r) & 1u;
            const uint32_t to = dst + r * F::kRowBytes + place_of<F::kPieces>(r, my_piece) * 16;
            if (my_piece_there) {  // (a position that is not there reads as zeros)
              cp_async_16(to, ok ? k : p.kc.rows, ok);
              cp_async_16(to + F::kSide, ok ? v : p.vc.rows, ok);
            }
          }
        }
        if constexpr (Q8) {
          const CacheSide& side = lane < 16 ? p.kc : p.vc;
          const float* s = side.scale + page * side.scale_page + head * side.scale_head + row * side.scale_row;
          cp_async_4(dst + 2 * F::kSide + lane * 4, there ? s : side.scale, there);
        }
      }
      if (--f_left > 0 && ++f_unit == f_seq.units) {
        f_unit = 0;
        if (++f_hr == HR) {
          f_hr = 0;
          f_seq = sequence_of(p, ++f_b);
        }
      }
      look_up();
    }
    cp_async_commit();
  };
  for (int s = 0; s < S - 1; ++s) fetch(s);

  // ---- an item's queries: loaded by pieces of 8 elements, kept in shared memory as rows (8 bits: permuted as the codes lie)
  constexpr int kQueryPieces = DH / 8, kQueryLoads = (8 * NT * kQueryPieces + kThreads - 1) / kThreads;
  uint32_t q_raw[kQueryLoads][4];
  auto load_queries = [&](int b, int hr) {
    const int head = hr / p.row_blocks, row0 = (hr - head * p.row_blocks) * 8 * NT;
#pragma unroll
    for (int i = 0; i < kQueryLoads; ++i) {
      const int n = tid + i * kThreads, r = n / kQueryPieces, piece = n % kQueryPieces, row = row0 + r;
      q_raw[i][0] = q_raw[i][1] = q_raw[i][2] = q_raw[i][3] = 0u;
      if (r < 8 * NT && row < p.rows && piece * 8 < p.D) {
        const int token = row / p.group, h = head * p.group + row % p.group;
        ld_16(p.q + b * p.q_batch + token * p.q_token + h * p.q_head + piece * 16, q_raw[i]);
      }
    }
  };
  auto keep_queries = [&](int b, int hr) {
    const int head = hr / p.row_blocks, row0 = (hr - head * p.row_blocks) * 8 * NT;
#pragma unroll
    for (int i = 0; i < kQueryLoads; ++i) {
      const int n = tid + i * kThreads, r = n / kQueryPieces, piece = n % kQueryPieces;
      if constexpr (Q8 && kBf16) {
        // bf16 to fp16: divided by the power of two below its largest element, a row keeps all of its bits down to 2^-14 of that
        float v[8], most = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          v[j] = Elem<DT>::of(q_raw[i], j);
          most = fmaxf(most, fabsf(v[j]));
        }
#pragma unroll
        for (int o = kQueryPieces / 2; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, o));
        const uint32_t e = __float_as_uint(most) & 0x7F800000u;
        const bool usual = e >= 0x00800000u * 2 && e < 0x00800000u * 253;
        const float down = usual ? reciprocal_of_power(__uint_as_float(e)) : 1.f;
        if (r < 8 * NT && piece == 0) sm.factor[r] = usual ? __uint_as_float(e) : 1.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) q_raw[i][j] = pack_f16x2_rn(v[2 * j] * down, v[2 * j + 1] * down);
      }
      if (r < 8 * NT) {
        // rows of 2 DH bytes, pieces at places as above
        *reinterpret_cast<uint4*>(s_query + r * DH * 2 + place_of<kQueryPieces>(r, piece) * 16) = make_uint4(q_raw[i][0], q_raw[i][1], q_raw[i][2], q_raw[i][3]);
      }
    }
    if (tid < 8 * NT) {
      const int row = row0 + tid, token = min(row / p.group, p.tokens - 1), h = head * p.group + row % p.group;
      sm.token[tid] = token;
      sm.slope[tid] = p.slopes && row < p.rows ? p.slopes[h] * kLog2e : 0.f;
      sm.out[tid] = row < p.rows ? b * p.out_batch + token * p.out_token + h * p.out_head : -1;
      sm.lse[tid] = row < p.rows ? (b * p.tokens + token) * p.heads * p.group + h : 0;
      if constexpr (Q8 && !kBf16) sm.factor[tid] = 1.f;
    }
  };

  // ---- a warp's running state
  float o[kSteps][NT][4], top[NT][2], sum[NT][2];
  // 8 bits: for each row a power of two that the scales of the values it sees are divided by, so that the largest become 64 .. 128: with e up to 2^8 a weight stays below 2^15, and is a
  // normal number of fp16 down to 2^-20 of the largest.
  float unit_v[NT][2];
  auto reset = [&]() {
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      top[n][0] = top[n][1] = -INFINITY;
      sum[n][0] = sum[n][1] = 0.f;
      unit_v[n][0] = unit_v[n][1] = 0.f;
#pragma unroll
      for (int k = 0; k < kSteps; ++k) o[k][n][0] = o[k][n][1] = o[k][n][2] = o[k][n][3] = 0.f;
    }
  };

  constexpr bool kHold = NT == 1;  // the queries' operands stay in registers
  uint32_t q_held[kHold ? kSteps : 1][2];
  // Operand of step k for tile n.  16 bits: ldmatrix of pieces 2k, 2k + 1.  8 bits: elements 16 k + 4 c .. + 3 of row g.
  auto query_operand = [&](int k, int n, uint32_t (&b)[2]) {
    const int r = 8 * n + g;
    const char* row = s_query + r * DH * 2;
    if constexpr (Q8) {
      const uint2 w = *reinterpret_cast<const uint2*>(row + place_of<kQueryPieces>(r, 2 * k + (c >> 1)) * 16 + (c & 1) * 8);
      b[0] = w.x;
      b[1] = w.y;
    } else {
      b[0] = *reinterpret_cast<const uint32_t*>(row + place_of<kQueryPieces>(r, 2 * k) * 16 + c * 4);
      b[1] = *reinterpret_cast<const uint32_t*>(row + place_of<kQueryPieces>(r, 2 * k + 1) * 16 + c * 4);
    }
  };
  float factor[NT][2];  // of a score
  const SoftcapLog2 cap(p.alpha, p.softcap > 0.f ? p.softcap : 1.f);
  auto begin_item = [&]() {
    reset();
    if constexpr (kHold) {
#pragma unroll
      for (int k = 0; k < kSteps; ++k) query_operand(k, 0, q_held[k]);
    }
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        factor[n][j] = p.softcap > 0.f ? 1.f : p.alpha * kLog2e;
        if constexpr (Q8) factor[n][j] *= sm.factor[8 * n + 2 * c + j];
      }
  };

  // ---- one block
  auto block = [&](int stage, const Sequence& seq, int base) {
    const unsigned valid = sm.valid[warp][stage];
    if (!valid) return;
    const uint32_t keys = ring_u32 + stage * F::kStage, values = keys + F::kSide;
    float s[NT][4];
#pragma unroll
    for (int n = 0; n < NT; ++n) s[n][0] = s[n][1] = s[n][2] = s[n][3] = 0.f;
    if constexpr (Q8) {
#pragma unroll
      for (int k = 0; k < kSteps; k += 2) {
        uint32_t r[4];
        const int row = lane & 15, piece = k + (lane >> 4);
        ldmatrix_x4(keys + row * F::kRowBytes + place_of<F::kPieces>(row, piece) * 16, r);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint32_t x = r[2 * h] ^ 0x80808080u, y = r[2 * h + 1] ^ 0x80808080u;
          const uint32_t a[4] = {codes_f16(x, 0x4140), codes_f16(y, 0x4140), codes_f16(x, 0x4342), codes_f16(y, 0x4342)};
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            uint32_t b[2];
            if constexpr (kHold) b[0] = q_held[k + h][0], b[1] = q_held[k + h][1];
            else query_operand(k + h, n, b);
            mma<false>(s[n], a, b[0], b[1]);
          }
        }
      }
    } else {
#pragma unroll
      for (int k = 0; k < kSteps; ++k) {
        uint32_t a[4];
        const int row = lane & 15, piece = 2 * k + (lane >> 4);
        ldmatrix_x4(keys + row * F::kRowBytes + place_of<F::kPieces>(row, piece) * 16, a);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          uint32_t b[2];
          if constexpr (kHold) b[0] = q_held[k][0], b[1] = q_held[k][1];
          else query_operand(k, n, b);
          mma<kMmaBf16>(s[n], a, b[0], b[1]);
        }
      }
    }
    float ks[2] = {1.f, 1.f}, vs[2] = {1.f, 1.f};
    if constexpr (Q8) {
      const float* scales = reinterpret_cast<const float*>(ring + stage * F::kStage + 2 * F::kSide);
      ks[0] = scales[g]; ks[1] = scales[g + 8];
      vs[0] = scales[16 + g]; vs[1] = scales[24 + g];
    }
    const int first = seq.length - p.tokens;  // the first new token's position
    const bool all = valid == 0xFFFFu && base + kBlock - 1 <= first && (p.window <= 0 || base > seq.length - 1 - p.window);
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int j = i & 1, hi = i >> 1;
        float v = Q8 ? s[n][i] * (ks[hi] * factor[n][j]) : s[n][i] * factor[n][j];
        if (p.softcap > 0.f) v = cap(v);
        s[n][i] = v;
      }
    if (p.slopes || !all) {
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int r = 8 * n + 2 * c + (i & 1), k = g + 8 * (i >> 1);
          const int gap = base + k - (first + sm.token[r]);
          if (p.slopes) s[n][i] = fmaf(sm.slope[r], static_cast<float>(gap), s[n][i]);
          if (!all && !(((valid >> k) & 1u) && gap <= 0 && (p.window <= 0 || gap > -p.window))) s[n][i] = -INFINITY;
        }
    }
    // the maximum, where a score is well above it
    bool above = false;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        above |= s[n][i] > top[n][i & 1] + kSlack;
        if constexpr (Q8) above |= fabsf(vs[i >> 1]) > 128.f * unit_v[n][i & 1] && s[n][i] != -INFINITY;
      }
    if (__any_sync(0xFFFFFFFFu, above)) {
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          float m = fmaxf(s[n][j], s[n][j + 2]);
#pragma unroll
          for (int d = 4; d < 32; d <<= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, d));
          m = fmaxf(m, top[n][j]);
          const float less = m == top[n][j] ? 1.f : ex2_approx(top[n][j] - m);
          top[n][j] = m;
          sum[n][j] *= less;
          float both = less;
          if constexpr (Q8) {
            float most = fmaxf(s[n][j] == -INFINITY ? 0.f : fabsf(vs[0]), s[n][j + 2] == -INFINITY ? 0.f : fabsf(vs[1]));
#pragma unroll
            for (int d = 4; d < 32; d <<= 1) most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, d));
            const float unit = fmaxf(unit_v[n][j], __uint_as_float(min(max(__float_as_uint(most) & 0x7F800000u, 0x04000000u), 0x7E000000u) - 0x03000000u));
            both *= unit_v[n][j] / unit;
            unit_v[n][j] = unit;
          }
#pragma unroll
          for (int k = 0; k < kSteps; ++k) {
            o[k][n][j] *= both;
            o[k][n][j + 2] *= both;
          }
        }
    }
    // weights, as the second product's operand
    uint32_t w[NT][2], rest[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      float e[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float m = top[n][i & 1];
        e[i] = ex2_approx(s[n][i] - (m == -INFINITY ? 0.f : m));
      }
      sum[n][0] += e[0] + e[2];
      sum[n][1] += e[1] + e[3];
      if constexpr (Q8) {
        const float inv[2] = {reciprocal_of_power(unit_v[n][0]), reciprocal_of_power(unit_v[n][1])};
#pragma unroll
        for (int i = 0; i < 4; ++i) e[i] = s[n][i] == -INFINITY ? 0.f : e[i] * (vs[i >> 1] * inv[i & 1]);  // (a hidden position's scale may be NaN)
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t x = pack2<kMmaBf16>(e[2 * h], e[2 * h + 1]);
        w[n][h] = transpose_8x8(x);
        if constexpr (kTwice) {
          const float2 r = unpack2<kMmaBf16>(x);
          rest[n][h] = transpose_8x8(pack2<kMmaBf16>(e[2 * h] - r.x, e[2 * h + 1] - r.y));
        }
      }
    }
    if constexpr (!Q8) {
      if (!all && p.tokens > 1) {
        // Some rows see a position and others do not: a value that is not finite must not reach the others as 0 * inf.  Such values are added to the rows that see them, and
        // are zeros for the product.
        bool odd = false;
        for (int i = lane; i < F::kSide / 16; i += 32) {
          const uint4 x = *reinterpret_cast<const uint4*>(ring + stage * F::kStage + F::kSide + i * 16);
          const uint32_t y[4] = {x.x, x.y, x.z, x.w};
          constexpr uint32_t e = kBf16 ? 0x7F80u : 0x7C00u;
#pragma unroll
          for (int j = 0; j < 4; ++j) odd |= (y[j] & e) == e || (y[j] >> 16 & e) == e;
        }
        if (__any_sync(0xFFFFFFFFu, odd)) {
          for (int k = 0; k < kBlock; ++k) {
            const int pos = base + k - first;
#pragma unroll
            for (int d = 0; d < kSteps; ++d)
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                const int e = 16 * d + 8 * h + g;
                uint16_t* at_v = reinterpret_cast<uint16_t*>(ring + stage * F::kStage + F::kSide + k * F::kRowBytes + place_of<F::kPieces>(k, e >> 3) * 16 + (e & 7) * 2);
                const float v = Elem<DT>::get(at_v, 0);
                if (!isfinite(v)) {
#pragma unroll
                  for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                      const int gap = pos - sm.token[8 * n + 2 * c + j];
                      if (gap <= 0 && (p.window <= 0 || gap > -p.window)) o[d][n][2 * h + j] += v;
                    }
                }
              }
          }
          __syncwarp();
          for (int i = lane; i < F::kSide / 2; i += 32) {
            uint16_t* at_v = reinterpret_cast<uint16_t*>(ring + stage * F::kStage + F::kSide) + i;
            if (!isfinite(Elem<DT>::get(at_v, 0))) *at_v = 0;
          }
          __syncwarp();
        }
      }
    }
    if constexpr (Q8) {
#pragma unroll
      for (int k = 0; k < kSteps; k += 2) {
        uint32_t r[4];
        const int row = lane & 15, piece = k + (lane >> 4);
        ldmatrix_x4_trans(values + row * F::kRowBytes + place_of<F::kPieces>(row, piece) * 16, r);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint32_t x = r[2 * h] ^ 0x80808080u, y = r[2 * h + 1] ^ 0x80808080u;
          const uint32_t a[4] = {codes_f16(x, 0x4240), codes_f16(x, 0x4341), codes_f16(y, 0x4240), codes_f16(y, 0x4341)};
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            mma<false>(o[k + h][n], a, w[n][0], w[n][1]);
            if constexpr (kTwice) mma<false>(o[k + h][n], a, rest[n][0], rest[n][1]);
          }
        }
      }
    } else {
#pragma unroll
      for (int k = 0; k < kSteps; ++k) {
        uint32_t a[4];
        const int row = (lane & 7) + ((lane >> 4) << 3), piece = 2 * k + ((lane >> 3) & 1);
        ldmatrix_x4_trans(values + row * F::kRowBytes + place_of<F::kPieces>(row, piece) * 16, a);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          mma<kMmaBf16>(o[k][n], a, w[n][0], w[n][1]);
          mma<kMmaBf16>(o[k][n], a, rest[n][0], rest[n][1]);
        }
      }
    }
  };

  // ---- the end of an item, or of the share: the four warps' results are joined; whole items are finished, cut ones kept
  constexpr int kMine = 8 * F::kJoinColumns / kThreads;
  auto end_item = [&](bool whole, int slot) {
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        float t = sum[n][j];
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) t += __shfl_xor_sync(0xFFFFFFFFu, t, d);
        if (g == 0) {
          sm.top[warp][8 * n + 2 * c + j] = top[n][j];
          sm.sum[warp][8 * n + 2 * c + j] = t;
        }
      }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      float weight[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int r = 8 * n + 2 * c + j;
        float m = sm.top[0][r];
#pragma unroll
        for (int w = 1; w < kWarps; ++w) m = fmaxf(m, sm.top[w][r]);
        weight[j] = top[n][j] == -INFINITY && m == -INFINITY ? 1.f : ex2_approx(top[n][j] - m);
        if constexpr (Q8) weight[j] *= unit_v[n][j];
      }
      // What a thread adds up: columns `col` .. of every kJoinColumns, of row r
      const int r = tid / 16, col = (tid % 16) * kMine, row = 8 * n + r;
      float m = sm.top[0][row], l = 0.f;
#pragma unroll
      for (int w = 1; w < kWarps; ++w) m = fmaxf(m, sm.top[w][row]);
#pragma unroll
      for (int w = 0; w < kWarps; ++w) l += sm.sum[w][row] * (sm.top[w][row] == -INFINITY ? (m == -INFINITY ? 1.f : 0.f) : ex2_approx(sm.top[w][row] - m));
      const float inv = !whole ? 1.f : l == 0.f ? 0.f : 1.f / l;
      const bool there = sm.out[row] >= 0;
      float* part = p.part + blockIdx.x * part_floats(8 * NT, DH) + (slot * 8 * NT + row) * (DH + 4);
      if (there && tid % 16 == 0) {
        if (whole) {
          if (p.lse && COMFUSE_IN_BOUNDS(sm.lse[row] < p.batch * p.tokens * p.heads * p.group, p.status)) p.lse[sm.lse[row]] = log_sum(m, l);
        } else if (COMFUSE_IN_BOUNDS(row < 8 * NT && slot < 2, p.status)) {
          part[DH] = m;
          part[DH + 1] = l;
        }
      }
#pragma unroll
      for (int first = 0; first < DH; first += F::kJoinColumns) {
        if (n > 0 || first > 0) __syncthreads();  // (the last columns are read)
#pragma unroll
        for (int k = 0; k < F::kJoinColumns / 16; ++k)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            float* to = s_join + (warp * 8 + 2 * c + j) * F::kPitch + 16 * k;
            const float* from = o[first / 16 + k][n];
            if constexpr (Q8) {
              *reinterpret_cast<float2*>(to + 2 * g) = make_float2(from[j] * weight[j], from[2 + j] * weight[j]);
            } else {
              to[g] = from[j] * weight[j];
              to[g + 8] = from[2 + j] * weight[j];
            }
          }
        __syncthreads();
        float v[kMine];
#pragma unroll
        for (int j = 0; j < kMine; ++j) v[j] = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w)
#pragma unroll
          for (int j = 0; j < kMine; ++j) v[j] += s_join[(w * 8 + r) * F::kPitch + col + j];
        const int at = first + col;
        if (!there) continue;
        if (whole) {
          if (at < p.D && COMFUSE_IN_BOUNDS(at + kMine <= p.D, p.status)) {
            uint32_t y[kMine / 2];
#pragma unroll
            for (int j = 0; j < kMine; ++j) v[j] *= inv;
            Elem<DT>::pack(v, y);
            char* to = p.out + sm.out[row] + 2 * at;
            if constexpr (kMine == 4) st_8(to, y);
            else *reinterpret_cast<uint32_t*>(to) = y[0];
          }
        } else if (COMFUSE_IN_BOUNDS(row < 8 * NT && slot < 2, p.status)) {
          if constexpr (kMine == 4) st_16(part + at, reinterpret_cast<const uint32_t*>(v));
          else st_8(part + at, reinterpret_cast<const uint32_t*>(v));
        }
      }
    }
  };

  // ---- the share
  int b = at.b, hr = at.hr, unit = at.unit, stage = 0;
  bool from_start = unit == 0;
  int pieces = 0;
  Sequence seq = sequence_of(p, b);
  load_queries(b, hr);
  keep_queries(b, hr);
  __syncthreads();
  begin_item();
  for (int n = 0; n < count; ++n) {
    cp_async_wait<S - 2>();
    __syncwarp();
    fetch(stage == 0 ? S - 1 : stage - 1);
    block(stage, seq, (seq.low & ~(kBlock - 1)) + unit * kUnit + warp * kBlock);
    stage = stage + 1 == S ? 0 : stage + 1;
    ++unit;
    if (unit == seq.units || n + 1 == count) {
      const bool whole = from_start && unit == seq.units, more = n + 1 < count;
      int nb = b, nhr = hr + 1;
      if (nhr == HR) nhr = 0, ++nb;
      if (more) load_queries(nb, nhr);  // on their way under the joining
      end_item(whole, pieces ? 1 : 0);
      if (more) {
        __syncthreads();  // everyone has read the last item's rows
        ++pieces;
        from_start = true;
        unit = 0;
        if (nb != b) seq = sequence_of(p, nb);
        b = nb;
        hr = nhr;
        keep_queries(b, hr);
        __syncthreads();
        begin_item();
      }
    }
  }
  cp_async_wait<0>();
}

// ------------------------------------------------------------------------------------------------ joining
// CTA (i, r): row r of the item that is cut behind share i, if that is its first cut.  Partial results are taken in the order of the shares.
template <int DT, int DH, int NT>
__global__ void __launch_bounds__(kThreads) join_kernel(const PagedAttentionParams p) {
  __shared__ Scan scan;
  __shared__ float s_weight[32];
  griddep_launch_dependents();
  Place at;
  // (the lengths are read in front of the wait: the kernel before this one signals behind its own)
  const Line line = find(p, &scan, [](const Line& l) { return min(l.begin(blockIdx.x + 1), l.total - 1); }, &at);
  griddep_wait();
  const long long cut = line.begin(blockIdx.x + 1), item = cut - at.unit;  // the item's first unit
  if (cut >= line.total || at.unit == 0 || item < line.begin(blockIdx.x)) return;
  const int row0 = (at.hr % p.row_blocks) * 8 * NT, row = row0 + blockIdx.y;
  if (blockIdx.y >= 8 * NT || row >= p.rows) return;
  const int units = sequence_of(p, at.b).units;
  const long long last = line.owner(item + units - 1);
  const int slot = item == line.begin(blockIdx.x) ? 0 : 1;
  const float* first_part = p.part + blockIdx.x * part_floats(8 * NT, DH) + (slot * 8 * NT + blockIdx.y) * (DH + 4);
  const float* next_part = p.part + (blockIdx.x + 1) * part_floats(8 * NT, DH) + blockIdx.y * (DH + 4);
  const int n = static_cast<int>(last - blockIdx.x) + 1;
  auto part = [&](int i) { return i == 0 ? first_part : next_part + (i - 1) * part_floats(8 * NT, DH); };

  constexpr int kMine = DH > kThreads ? DH / kThreads : 1;
  float m = -INFINITY, l = 0.f, v[kMine];
#pragma unroll
  for (int j = 0; j < kMine; ++j) v[j] = 0.f;
  for (int i0 = 0; i0 < n; i0 += 32) {  // 32 parts at a time: their weights first
    const int k = min(32, n - i0);
    const int lane = threadIdx.x & 31;
    const float pm = lane < k ? part(i0 + lane)[DH] : -INFINITY, pl = lane < k ? part(i0 + lane)[DH + 1] : 0.f;
    float most = pm;
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, d));
    most = fmaxf(most, m);
    const float old = m == -INFINITY ? (most == -INFINITY ? 1.f : 0.f) : ex2_approx(m - most);
    const float mine = pm == -INFINITY ? (most == -INFINITY ? 1.f : 0.f) : ex2_approx(pm - most);
    float t = pl * mine;
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) t += __shfl_xor_sync(0xFFFFFFFFu, t, d);
    l = l * old + t;
    m = most;
    __syncthreads();
    if (threadIdx.x < 32) s_weight[lane] = mine;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kMine; ++j) {
      const int d = threadIdx.x + j * kThreads;
      if (d < DH) {
        float a = v[j] * old;
#pragma unroll 8
        for (int i = 0; i < k; ++i) a = fmaf(part(i0 + i)[d], s_weight[i], a);
        v[j] = a;
      }
    }
  }
  const int head = at.hr / p.row_blocks, token = row / p.group, h = head * p.group + row % p.group;
  char* out = p.out + at.b * p.out_batch + token * p.out_token + h * p.out_head;
  const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
  for (int j = 0; j < kMine; ++j) {
    const int d = threadIdx.x + j * kThreads;
    if (d < p.D && COMFUSE_IN_BOUNDS(row < p.rows && at.b < p.batch, p.status)) Elem<DT>::put(out, d, v[j] * inv);
  }
  if (p.lse && threadIdx.x == 0 && COMFUSE_IN_BOUNDS(at.b < p.batch && token < p.tokens, p.status))
    p.lse[(static_cast<long long>(at.b) * p.tokens + token) * p.heads * p.group + h] = log_sum(m, l);
}

// ------------------------------------------------------------------------------------------------ launches
template <int DT, bool Q8, int DH, int NT>
cudaError_t launch_instance(const PagedAttentionPlan& plan, const PagedAttentionParams& p, cudaStream_t stream) {
  using F = Form<Q8, DH, NT>;
  static std::atomic<unsigned long long> ready{0};  // devices on which the kernel may take its shared memory
  int device = 0;
  cudaError_t e = cudaGetDevice(&device);
  if (e != cudaSuccess) return e;
  const unsigned long long bit = 1ull << (device & 63);
  if (device > 63 || !(ready.load(std::memory_order_relaxed) & bit)) {
    e = cudaFuncSetAttribute(attention_kernel<DT, Q8, DH, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, F::kBytes);
    if (e != cudaSuccess) return e;
    ready.fetch_or(bit, std::memory_order_relaxed);
  }
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[1];
  cfg.gridDim = dim3(static_cast<unsigned>(plan.ctas), 1, 1);
  cfg.blockDim = dim3(kThreads, 1, 1);
  cfg.dynamicSmemBytes = F::kBytes;
  cfg.stream = stream;
  if (programmatic_launch_enabled()) {
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
  }
  if (verbose_enabled())
    std::fprintf(stderr, "comfuse: paged_attention dtype=%d quantized=%d D<=%d row tiles=%d row blocks=%d CTAs=%d stages=%d joined=%d\n", DT, Q8, DH, NT, p.row_blocks, plan.ctas, F::kStages,
                 plan.joined);
  count_launch();
  e = cudaLaunchKernelEx(&cfg, attention_kernel<DT, Q8, DH, NT>, p);
  if (e != cudaSuccess || !plan.joined) return e;
  cfg.gridDim = dim3(static_cast<unsigned>(plan.ctas - 1), static_cast<unsigned>(p.rows < 8 * NT ? p.rows : 8 * NT), 1);
  cfg.dynamicSmemBytes = 0;
  count_launch();
  return cudaLaunchKernelEx(&cfg, join_kernel<DT, DH, NT>, p);
}

template <int DT, bool Q8>
cudaError_t launch_type(const PagedAttentionPlan& plan, const PagedAttentionParams& p, cudaStream_t stream) {
  const int nt = plan.row_tiles;
  if (p.D <= 64) return nt == 1 ? launch_instance<DT, Q8, 64, 1>(plan, p, stream) : nt == 2 ? launch_instance<DT, Q8, 64, 2>(plan, p, stream) : launch_instance<DT, Q8, 64, 4>(plan, p, stream);
  if (p.D <= 128) return nt == 1 ? launch_instance<DT, Q8, 128, 1>(plan, p, stream) : nt == 2 ? launch_instance<DT, Q8, 128, 2>(plan, p, stream) : launch_instance<DT, Q8, 128, 4>(plan, p, stream);
  return nt == 1 ? launch_instance<DT, Q8, 256, 1>(plan, p, stream) : launch_instance<DT, Q8, 256, 2>(plan, p, stream);
}

}  // namespace
}  // namespace paged
}  // namespace comfuse
