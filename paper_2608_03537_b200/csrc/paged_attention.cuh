// Attention of a few new tokens over a paged cache, split over the cache's length and joined.
//
//   s[n] = cap(alpha q . k[n]) + slope (n - m);   out = sum_n softmax(s)[n] v[n]
//
// Every visible key and value is read once, and for few queries that is all there is to bound it: 2 D (or 4 D) flops an element of a query row against HBM.  So the
// kernel is built around loads in flight.
//
//   * The call's work is a line of units of some positions (sequence by sequence, key head by key head), cut into equal shares, one for each of the CTAs that fit on the
//     GPU: whatever the lengths, all finish together.  A CTA finds its share from the lengths themselves.  An item (sequence, key head) that lies in one share is
//     finished there; one that is cut leaves a partial sum, maximum and weighted values for each share, and a second kernel joins them, in order.
//   * Calls of few positions, whose time is latency, take clusters instead: each item is one cluster's, its units in equal parts the CTAs', which send one another their results through
//     distributed shared memory, each those of some outputs.  One kernel, no shares to find, no partial results in memory.  (Results that are read from the others instead of sent by them: 1000
//     positions 6.7 us; a read takes 200 ns.)
//   * A unit is a block of 16 or 32 positions for each of the CTA's key warps.  A key warp is on its own: it fetches its blocks by 16-byte asynchronous copies, several blocks ahead and
//     across the ends of items, into a ring of its own, and keeps a running maximum, sum and weighted values; no barrier but at the end of an item, where they are joined.  Where there are
//     more rows of queries than a warp holds, several warps share a ring and its fetching, each with rows of its own, and meet once a block.
//   * The keys are the 16-row operand of the warp-wide matrix instruction and the queries the 8-column one: S^T = K Q^T, then O^T += V^T P^T.  The queries that share a key head
//     (tokens x heads of its group) fill eight columns a tile, so that a single query wastes an eighth of what rows of sixteen would.  P^T changes from the accumulators' layout to
//     the operand's by two 8x8 transposes.
//   * 8 bits: the first product is one of integers.  A query row is a multiple of a power of two, 22 bits and a sign, in three digits of 8 bits, a product each; the sums are exact.
//     The key's scale is a factor of its score, the value's scale one of its weight.  The values' codes become fp16 by five instructions for each four.
//   * The maximum is renewed only when a score is more than 8 (a factor of 256) above it: a vote instead of a reduction in most blocks.
//
// On one B200 (copies run at 6.5 TB/s), replayed as a graph: one sequence of 131072 positions, 8 key heads of 128 for 32 of queries, bf16, 92 us = 5.9 TB/s; 64 sequences of up to 16384 positions over
// 8 bits, 8 heads of 128 for 64, 179 us = 6.0 TB/s on a cold GPU and 199 under its power limit, which is then what bounds it; 1000 positions 6.6 us, most of them start and end; 24 sequences that see
// 512 positions, 16 heads of 64, 13.3 us = 3.5 TB/s; eight sequences of up to 5000 positions with five new tokens each, 2 heads of 256 for 16, 33.9 us = 1.3 TB/s (8 bits: 41): 40 rows of 256 fill
// the registers with eight warps an SM, whose chain from block to block (copies seen, first product, exponentials, second product) is the time; 64 rows of 128 over 80000 positions, 4 heads, 73 us =
// 2.2 TB/s by twelve warps (8 bits: 87; rows of 256: 146 and 178).  Called one by one these take as long, but for the short ones' half a microsecond.
#pragma once

#include <cstdio>
#include <type_traits>

#include "kv_params.h"
#include "q8_common.cuh"

namespace comfuse {
namespace paged {

cudaError_t launch_bf16(const PagedAttentionPlan& plan, const PagedAttentionParams& p, cudaStream_t stream);
cudaError_t launch_f16(const PagedAttentionPlan& plan, const PagedAttentionParams& p, cudaStream_t stream);
cudaError_t launch_bf16_q8(const PagedAttentionPlan& plan, const PagedAttentionParams& p, cudaStream_t stream);
cudaError_t launch_f16_q8(const PagedAttentionPlan& plan, const PagedAttentionParams& p, cudaStream_t stream);

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kSlack = 8.f;  // log2 of what a weight may exceed 1 by
constexpr int kDigits = 3;     // of a query, 8 bits
// log2 of the weight at the running maximum.  fp16 over 16 bits: 2^7, so that with the slack weights stay below 2^15; fp16's steps end at 2^-24, so what both parts of a weight leave is at most
// 2^-32 of the largest (with 1 a weight of e^-16 was off by 6 %, and from e^-17.5 on it was 0, in the product alone).  8 bits have units of their own, and bf16 has fp32's range.
template <int DT, bool Q8>
constexpr int kLiftOf = DT == COMFUSE_DTYPE_F16 && !Q8 ? 7 : 0;

// Sizes of an instance: D up to DH, NT tiles of eight queries a warp, RW warps with rows of their own to a ring.
template <bool Q8, int DH, int NT, int RW, bool CLUSTER>
struct Form {
  static constexpr int kRowBytes = DH * (Q8 ? 1 : 2);
  static constexpr int kPieces = kRowBytes / 16;                  // of a row
  // Groups of 16 positions in a block: two where the registers and the ring hold them (half the votes, meetings and loop a position; 64 rows over 80000 x 4 x 128, 16 bits: 97 us with one, 78 with two).
  static constexpr int kGroups = kRowBytes <= 128 || (!Q8 && DH == 128 && RW > 1) ? 2 : 1;
  static constexpr int kBlock = 16 * kGroups;
  // Rings.  64 rows: eight warps of 255 registers, or, where 168 are enough and the call is not one of latency, twelve (the same call: 78 and 69 us; 64 wide, 8 bits: 65 and 59; 128 wide and
  // 8 bits would spill: 86 and 134; one sequence of 2000 in clusters, 64 wide, 8 bits: 12.3 and 13.8).
  static constexpr int kKeyWarps = RW < 4 ? 4 : !CLUSTER && (Q8 ? DH == 64 : DH == 128) ? 3 : 2;
  static constexpr int kWarps = kKeyWarps * RW, kThreads = 32 * kWarps;
  static constexpr int kUnit = kBlock * kKeyWarps;
  static constexpr int kRows = 8 * NT * RW;                       // of queries
  static constexpr int kSetUp = kUnit < 64 ? 4 : 2;               // what beginning and ending an item costs, in units
  static constexpr int kSide = kBlock * kRowBytes;                // keys, or values, of a block
  static constexpr int kStage = 2 * kSide + (Q8 ? 8 * kBlock : 0);  // and their scales
  static constexpr int kJoinColumns = NT > 1 && RW == 1 ? 32 : 64;  // where warps are joined, at a time
  static constexpr int kPitch = kJoinColumns + 4;                 // floats of a row there: a warp's stores fall on all banks
  static constexpr int kJoin = kWarps * 8 * kPitch * 4;
  static constexpr int kQueryStep = 8 * kRows + (Q8 ? 8 : 0);     // words of a step of all rows (8 bits: steps of a row on other banks)
  static constexpr int kQuery = DH / (Q8 ? 32 : 16) * kQueryStep * 4 * (Q8 ? kDigits : 1);
  static constexpr int kSmall = 256 + 4 * 32 * kKeyWarps + kRows * (8 * kKeyWarps + 24);
  static constexpr int kCtasPerSm = DH == 256 || (RW > 1 && (DH == 128 || Q8)) ? 1 : CLUSTER && DH == 64 && NT == 1 ? 3 : 2;
  // (Three CTAs an SM with rings of two blocks: 24 x 16 items of 512 positions, D = 64, 12.7 us where two take 17.8; one sequence of 131072 by shares 58 us instead of 48.)
  static constexpr int kSmem = kCtasPerSm == 3 ? 75 * 1024 : kCtasPerSm == 2 ? 113 * 1024 : 226 * 1024;  // what a CTA may take
  static constexpr int kMostStages = (kSmem - kJoin - kQuery - kSmall) / (kStage * kKeyWarps);
  static constexpr int kStages = kMostStages < 8 ? kMostStages : 8;
  static constexpr int kBytes = kStages * kStage * kKeyWarps + kJoin + kQuery + kSmall;
};

// Partial results of CTA c: two slots (of the first item of its share, and of the last), each `rows` rows of D + 4 floats: D values, the maximum, the sum.
__host__ __device__ inline long long part_floats(int rows, int D) { return 2ll * rows * (D + 4); }

namespace {

// ------------------------------------------------------------------------------------------------ shares
// The line of units.  Each of a sequence's `hr` items (key heads x row blocks) has the same number of them, and kSetUp more in front that stand for the work of beginning and ending an
// item: shares are equal in both together (64 sequences of 20 .. 1000 positions, 8 heads of 128: the CTA with the most items, 14 of a unit each, took twice as long as the others).
struct Line {
  unsigned total, share, longer;  // the first `longer` CTAs have share + 1
  __device__ unsigned begin(unsigned cta) const { return cta * share + (cta < longer ? cta : longer); }
  __device__ unsigned owner(unsigned unit) const {
    const unsigned l = longer * (share + 1);
    return unit < l ? unit / (share + 1) : longer + (unit - l) / share;
  }
};
struct Sequence {
  int length, low, units;  // positions low .. length - 1 are visible to some token; units are counted from low rounded down to a block
};
template <typename F>
__device__ __forceinline__ Sequence sequence_of(const PagedAttentionParams& p, int b) {
  Sequence s;
  s.length = min(max(p.lengths[b], 0), p.max_length);
  s.low = p.window > 0 ? max(0, s.length - p.tokens + 1 - p.window) : 0;
  s.units = max(1u, static_cast<unsigned>(s.length - (s.low & ~(F::kBlock - 1)) + F::kUnit - 1) / F::kUnit);  // (an empty sequence has a unit too: its rows are written)
  return s;
}
// By each warp on its own, 32 sequences at a time.  The line; then where a unit lies, or which is the first of an item.
template <typename F>
__device__ __forceinline__ Line line_of(const PagedAttentionParams& p, int lane, unsigned* mine) {
  unsigned total = 0;
  for (int b0 = 0; b0 < p.batch; b0 += 32) {
    const unsigned n = b0 + lane < p.batch ? sequence_of<F>(p, b0 + lane).units + F::kSetUp : 0u;
    if (b0 == 0) *mine = n;  // (most calls have no more)
    total += n;
  }
  Line line;
  line.total = __reduce_add_sync(0xFFFFFFFFu, total) * static_cast<unsigned>(p.heads * p.row_blocks);
  line.share = p.shares.of(line.total);
  line.longer = line.total - line.share * p.ctas;
  return line;
}
struct Place {
  int b, hr, at;   // place in the item, kSetUp in front of the first unit
  unsigned real;   // units in front of it, of all items
};
template <typename F>
__device__ __forceinline__ Place place_of_unit(const PagedAttentionParams& p, int lane, unsigned mine, unsigned unit) {
  const unsigned hr = p.heads * p.row_blocks;
  unsigned before = 0;  // of the sequences in front, one item each
  for (int b0 = 0;; b0 += 32) {
    const unsigned n = b0 == 0 ? mine : b0 + lane < p.batch ? sequence_of<F>(p, b0 + lane).units + F::kSetUp : 0u;
    unsigned upto = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const unsigned v = __shfl_up_sync(0xFFFFFFFFu, upto, o);
      if (lane >= o) upto += v;
    }
    const unsigned found = __ballot_sync(0xFFFFFFFFu, unit < (before + upto) * hr);
    if (found || b0 + 32 >= p.batch) {
      const int i = found ? __ffs(found) - 1 : 0;
      const unsigned units = __shfl_sync(0xFFFFFFFFu, n, i), rest = unit - (before + __shfl_sync(0xFFFFFFFFu, upto, i) - units) * hr;
      Place at;
      at.b = b0 + i;
      at.hr = static_cast<int>(__fdividef(static_cast<float>(rest), static_cast<float>(units)));  // (off by one at most)
      if (at.hr * units > rest) --at.hr;
      if ((at.hr + 1) * units <= rest) ++at.hr;
      at.at = rest - at.hr * units;
      at.real = unit - at.at - F::kSetUp * (at.b * hr + at.hr) + max(0, at.at - F::kSetUp);
      return at;
    }
    before += __shfl_sync(0xFFFFFFFFu, upto, 31);
  }
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
__device__ __forceinline__ void mma_s8(int (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+r"(d[0]), "+r"(d[1]), "+r"(d[2]), "+r"(d[3])
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
__device__ __forceinline__ void st_cluster_f32x4(uint32_t at, const float* v) {
  asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(at), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]) : "memory");
}
// cap * tanh(x / cap), x, cap and the result in the log2 domain.  cap - 2 cap / (1 + e^(2x / cap)) is exact to 2^-21 of itself where x is not small beside the cap, but its error is one of the cap; so
// below 0.6 of it x times a polynomial in (x / cap)^2 takes its place (coefficients fitted to tanh(y) / y, 2^-22), which for caps far above x, up to the largest number, is x.
constexpr float kCapNear = 0.6f;
__device__ __forceinline__ float softcap_near(float x, float per_cap) {
  const float y = x * per_cap, t = y * y;
  return fmaf(t, fmaf(t, fmaf(t, fmaf(t, 0.015612628310918808f, -0.05221180245280266f), 0.13313116133213043f), -0.33332598209381104f), 1.f) * x;
}
__device__ __forceinline__ float softcap_any(float x, float cap, float per_cap) {
  const float far = fmaf(-2.f * cap, rcp_approx(1.f + ex2_approx(x * per_cap * (2.f * kLog2e))), cap);
  return fabsf(x * per_cap) < kCapNear ? softcap_near(x, per_cap) : far;
}
// log of a sum whose terms were divided by 2^(m - LIFT); nothing: -inf
template <int LIFT>
__device__ __forceinline__ float log_sum(float m, float l) {
  if (m == -INFINITY) return l == 0.f ? -INFINITY : l;  // (else a NaN)
  return m * 0.6931471805599453f + logf(l * (1.f / (1 << LIFT)));
}
// Piece c of row r lies at place c ^ (...): the eight rows that an ldmatrix reads at once are on eight different groups of banks.
template <int PIECES>
__device__ __forceinline__ int place_of(int r, int c) {
  return PIECES >= 8 ? c ^ (r & 7) : c ^ ((r >> 1) & 3);
}

// ------------------------------------------------------------------------------------------------ the kernel
template <int DT, bool Q8, int DH, int NT, int RW, bool CLUSTER>
__global__ void __launch_bounds__(Form<Q8, DH, NT, RW, CLUSTER>::kThreads, Form<Q8, DH, NT, RW, CLUSTER>::kCtasPerSm) attention_kernel(const PagedAttentionParams p) {
  using F = Form<Q8, DH, NT, RW, CLUSTER>;
  constexpr bool kBf16 = DT == COMFUSE_DTYPE_BF16;  // of queries and outputs
  constexpr bool kMmaBf16 = kBf16 && !Q8;           // of the second product: 8-bit codes are exact in fp16
  // A weight in 16 bits is off by half a step of its type, which behind a sum over like terms is as much as the output's own rounding.  So the weights go in twice, rounded and what
  // the rounding left.  fp16 weights of bf16 outputs are eight times as fine as those and go in once.
  constexpr bool kTwice = !(Q8 && kBf16);
  constexpr int kLift = kLiftOf<DT, Q8>;  // the sums carry it too, so it leaves at the division
  constexpr int kSteps = DH / 16, G = F::kGroups, S = F::kStages;
  static_assert(S >= 2 && S <= 8, "a ring of two blocks at least");
  extern __shared__ __align__(128) char smem[];
  float* s_join = reinterpret_cast<float*>(smem + S * F::kStage * F::kKeyWarps);
  uint32_t* s_query = reinterpret_cast<uint32_t*>(reinterpret_cast<char*>(s_join) + F::kJoin);
  struct Small {
    long long out[F::kRows];                                       // where a row's output goes (-1: nowhere)
    float top[F::kKeyWarps][F::kRows], sum[F::kKeyWarps][F::kRows];
    float factor[F::kRows];                                        // 8 bits: what a query was divided by
    float slope[F::kRows];
    int token[F::kRows];                                           // its new token
    int lse[F::kRows];
    unsigned valid[F::kKeyWarps][8];                               // of the blocks in the ring: positions that are there
  };
  static_assert(sizeof(Small) <= F::kSmall, "room for what is small");
  Small& sm = *reinterpret_cast<Small*>(reinterpret_cast<char*>(s_query) + F::kQuery);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int kw = RW == 1 ? warp : warp / RW, rw = RW == 1 ? 0 : warp % RW;  // which ring, which rows
  const int g = lane >> 2, c = lane & 3;

  griddep_wait();
  griddep_launch_dependents();  // behind the wait: the joining kernel reads the lengths before its own

  const int HR = p.heads * p.row_blocks;
  Place at;
  int count, first_at;
  const int rank = CLUSTER ? blockIdx.x % p.cluster : 0;
  if constexpr (CLUSTER) {
    const int item = blockIdx.x / p.cluster;
    at.b = item / HR;
    at.hr = item - at.b * HR;
    const long long units = sequence_of<F>(p, at.b).units;
    first_at = static_cast<int>(units * rank / p.cluster);
    count = static_cast<int>(units * (rank + 1) / p.cluster) - first_at;
  } else {
    unsigned lane_units;
    const Line line = line_of<F>(p, lane, &lane_units);
    const unsigned share_begin = line.begin(blockIdx.x), share_end = line.begin(blockIdx.x + 1);
    if (share_begin >= share_end) return;
    at = place_of_unit<F>(p, lane, lane_units, share_begin);
    // (the line's last place is a unit: the one behind it has one more in front)
    const Place end = place_of_unit<F>(p, lane, lane_units, min(share_end, line.total - 1));
    count = static_cast<int>(end.real - at.real) + (share_end == line.total);
    if (count <= 0) return;  // (nothing but the front of an item)
    first_at = max(0, at.at - F::kSetUp);
  }

  // ---- an item's queries, kept in shared memory as the product's operands, eight bytes a lane for each step and tile: a step (16 elements; of 8 bits 32) of a row is 32 bytes in line (in
  // each of the digits' planes).  A thread brings a step of a row; of 16 bits neighbours have neighbouring rows, of 8 bits the steps of one, whose largest element they need.
  constexpr int kStepPieces = Q8 ? 4 : 2, kQuerySteps = DH / (8 * kStepPieces), kQueryLoads = (F::kRows * kQuerySteps + F::kThreads - 1) / F::kThreads;
  constexpr int kStepWords = F::kQueryStep, kPlane = kQuerySteps * kStepWords;  // (of a digit)
  uint32_t q_raw[kQueryLoads][kStepPieces][4];
  auto query_row = [&](int i) { return Q8 ? (tid + i * F::kThreads) / kQuerySteps : (tid + i * F::kThreads) % F::kRows; };
  auto query_step = [&](int i) { return Q8 ? (tid + i * F::kThreads) % kQuerySteps : (tid + i * F::kThreads) / F::kRows; };
  auto load_queries = [&](int b, int hr) {
    const int head = p.row_blocks == 1 ? hr : hr / p.row_blocks, row0 = (hr - head * p.row_blocks) * F::kRows;
#pragma unroll
    for (int i = 0; i < kQueryLoads; ++i) {
      const int r = query_row(i), step = query_step(i), row = row0 + r;
      const bool there = r < F::kRows && step < kQuerySteps && row < p.rows;
      const int token = p.groups.of(row), h = head * p.group + row - token * p.group;
      const char* from = p.q + b * p.q_batch + token * p.q_token + h * p.q_head;
#pragma unroll
      for (int j = 0; j < kStepPieces; ++j) {
        const int piece = step * kStepPieces + j;
        q_raw[i][j][0] = q_raw[i][j][1] = q_raw[i][j][2] = q_raw[i][j][3] = 0u;
        if (there && piece * 8 < p.D) ld_16(from + piece * 16, q_raw[i][j]);
      }
    }
  };
  load_queries(at.b, at.hr);

  char* ring = smem + kw * S * F::kStage;
  const uint32_t ring_u32 = smem_u32(ring);
  auto ring_sync = [&]() {  // the warps of a ring
    if constexpr (RW == 1) __syncwarp();
    else named_barrier_sync(1 + kw, 32 * RW);
  };
  if (p.D < DH) {  // pieces behind D are never fetched and stay zeros
    for (int i = lane + 32 * rw; i < S * F::kStage / 16; i += 32 * RW) reinterpret_cast<uint4*>(ring)[i] = make_uint4(0, 0, 0, 0);
    ring_sync();
  }

  // ---- fetching, several blocks ahead.  Lane l knows the page and line of position l of the block that is next, and has piece `my_piece` of rows my_row, my_row + kRowStep, ...
  constexpr int kRowStep = 32 * RW / F::kPieces, kLoads = F::kBlock / kRowStep;
  static_assert(kLoads >= 1 && kLoads * kRowStep == F::kBlock, "rows of a block over the lanes of a ring's warps");
  const int my_piece = lane % F::kPieces, my_row = rw * (32 / F::kPieces) + lane / F::kPieces, my_pos = lane & (F::kBlock - 1);
  const bool my_piece_there = my_piece * 16 < p.D * (Q8 ? 1 : 2);
  const uint32_t my_dst = ring_u32 + my_row * F::kRowBytes + place_of<F::kPieces>(my_row, my_piece) * 16;
  const bool whole_pages = p.page_size.d % F::kBlock == 0;  // a block lies in one page
  const bool dense_rows = p.kc.row == F::kRowBytes && p.vc.row == F::kRowBytes;  // known distances
  const bool same_strides = p.kc.page == p.vc.page && p.kc.row == p.vc.row;
  // (the strides of pages and rows fit in 32 bits)
  auto offset = [](unsigned page, unsigned row, const CacheSide& c) {
    return static_cast<long long>(static_cast<unsigned long long>(page) * static_cast<unsigned>(c.page) + static_cast<unsigned long long>(row) * static_cast<unsigned>(c.row));
  };
  int f_b = at.b, f_hr = at.hr, f_unit = first_at, f_left = count, f_base, f_page, f_line;
  Sequence f_seq = sequence_of<F>(p, f_b);
  const Sequence first_seq = f_seq;
  const int* f_table = p.table + f_b * p.table_stride;
  const char *f_k, *f_v;  // the head's rows, from this lane's piece on
  const float *f_ks, *f_vs;
  auto set_head = [&]() {
    const int head = p.row_blocks == 1 ? f_hr : f_hr / p.row_blocks;
    f_k = p.kc.rows + head * p.kc.head + my_piece * 16;
    f_v = p.vc.rows + head * p.vc.head + my_piece * 16;
    if constexpr (Q8) {
      f_ks = p.kc.scale + head * p.kc.scale_head;
      f_vs = p.vc.scale + head * p.vc.scale_head;
    }
  };
  auto look_up = [&]() {
    f_base = (f_seq.low & ~(F::kBlock - 1)) + f_unit * F::kUnit + kw * F::kBlock;
    const int pos = f_base + my_pos;
    f_page = -1;
    if (pos < f_seq.length) {
      const unsigned n = p.page_size.of(pos);
      f_line = pos - n * p.page_size.d;
      f_page = f_table[n];
    }
  };
  set_head();
  if (count > 0) look_up();
  auto fetch = [&](int stage) {
    if (f_left > 0) {
      const bool there = f_page >= 0 && f_page < p.pages && f_base + my_pos >= f_seq.low;
      constexpr unsigned kAll = F::kBlock == 32 ? 0xFFFFFFFFu : 0xFFFFu;
      const unsigned valid = __ballot_sync(0xFFFFFFFFu, there) & kAll;
      if (lane == 0) sm.valid[kw][stage] = valid;
      if (valid) {
        const uint32_t dst = my_dst + stage * F::kStage;
        if (valid == kAll && whole_pages) {
          const int first = f_line - my_pos + my_row;
          const char* k = f_k + offset(f_page, first, p.kc);
          const char* v = f_v + offset(f_page, first, p.vc);
          if (my_piece_there) {
            if (dense_rows) {
#pragma unroll
              for (int i = 0; i < kLoads; ++i) {
                const uint32_t to = (F::kPieces >= 8 ? dst ^ ((i * kRowStep & 7) << 4) : dst) + i * kRowStep * F::kRowBytes;
                cp_async_16(to, k + i * kRowStep * F::kRowBytes, true);
                cp_async_16(to + F::kSide, v + i * kRowStep * F::kRowBytes, true);
              }
            } else {
              const long long k_step = kRowStep * p.kc.row, v_step = kRowStep * p.vc.row;
#pragma unroll
              for (int i = 0; i < kLoads; ++i) {
                const uint32_t to = (F::kPieces >= 8 ? dst ^ ((i * kRowStep & 7) << 4) : dst) + i * kRowStep * F::kRowBytes;
                cp_async_16(to, k, true);
                cp_async_16(to + F::kSide, v, true);
                k += k_step;
                v += v_step;
              }
            }
          }
        } else {
          // each position's offset by the lane that knows it, then to those that fetch it
          const long long k_mine = there ? offset(f_page, f_line, p.kc) : 0, v_mine = same_strides ? k_mine : there ? offset(f_page, f_line, p.vc) : 0;
#pragma unroll
          for (int i = 0; i < kLoads; ++i) {
            const int r = i * kRowStep + my_row;
            const long long k_at = __shfl_sync(0xFFFFFFFFu, k_mine, r);
            long long v_at = k_at;
            if (!same_strides) v_at = __shfl_sync(0xFFFFFFFFu, v_mine, r);
            const bool ok = (valid >> r) & 1u;  // (a position that is not there reads as zeros)
            const uint32_t to = (F::kPieces >= 8 ? dst ^ ((i * kRowStep & 7) << 4) : dst) + i * kRowStep * F::kRowBytes;
            if (my_piece_there) {
              cp_async_16(to, f_k + k_at, ok);
              cp_async_16(to + F::kSide, f_v + v_at, ok);
            }
          }
        }
        if constexpr (Q8) {
          const long long page = there ? f_page : 0, row = there ? f_line : 0;
          const uint32_t to = ring_u32 + stage * F::kStage + 2 * F::kSide + my_pos * 4;
          // (16 positions: the upper lanes take the values' scales)
          if (rw == 0 && (F::kBlock == 32 || lane < 16)) cp_async_4(to, f_ks + page * p.kc.scale_page + row * p.kc.scale_row, there);
          if (rw == 0 && (F::kBlock == 32 || lane >= 16)) cp_async_4(to + 4 * F::kBlock, f_vs + page * p.vc.scale_page + row * p.vc.scale_row, there);
        }
      }
      if (--f_left > 0) {
        if (++f_unit == f_seq.units) {
          f_unit = 0;
          if (++f_hr == HR) {
            f_hr = 0;
            f_seq = sequence_of<F>(p, ++f_b);
            f_table = p.table + f_b * p.table_stride;
          }
          set_head();
        }
        look_up();
      }
    }
    cp_async_commit();
  };
  auto keep_queries = [&](int b, int hr) {
    const int head = p.row_blocks == 1 ? hr : hr / p.row_blocks, row0 = (hr - head * p.row_blocks) * F::kRows;
#pragma unroll
    for (int i = 0; i < kQueryLoads; ++i) {
      const int r = query_row(i), step = query_step(i);
      const bool mine = r < F::kRows && step < kQuerySteps;
      uint32_t* to = s_query + step * kStepWords + r * 8;
      if constexpr (Q8) {
        // A multiple of 2^-21 of the power of two at or below the row's largest element, below 2^22 of them, in three digits: exact for bf16 down to 2^-14 of that, for fp16 to 2^-11.
        uint32_t top = 0u;  // of the bits: infinities and NaNs are above every number
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(Elem<DT>::of(q_raw[i][j], e)) & 0x7FFFFFFFu);
#pragma unroll
        for (int o = kQuerySteps / 2; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
        const bool odd = top >= 0x7F800000u;  // (such a row has no digits: NaN)
        const uint32_t e = min(max(top & 0x7F800000u, 0x10000000u), 0x7F000000u);  // (2^-95: a row below that is zero beside any other; 2^127: the largest numbers')
        const float up = __uint_as_float(0x89800000u - e);  // 2^21 / e, a normal number for all of them
        if (mine && step == 0) sm.factor[r] = odd ? __int_as_float(0x7FFFFFFF) : __uint_as_float(e) * 0x1p-21f;
        // elements 4w .. 4w + 3 of the step are word 2 (w mod 4) + w / 4 of its row: lane c's first four, and 16 further its second
        uint32_t digit[kDigits][8];
#pragma unroll
        for (int w = 0; w < 8; ++w) {
          uint32_t word[kDigits] = {};
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int n = 4 * w + j;
            int x = odd ? 0 : __float2int_rn(Elem<DT>::of(q_raw[i][n >> 3], n & 7) * up);
#pragma unroll
            for (int d = kDigits - 1; d > 0; --d) {
              const int low = static_cast<int8_t>(x & 0xFF);
              word[d] |= (low & 0xFFu) << (8 * j);
              x = (x - low) >> 8;
            }
            word[0] |= (x & 0xFFu) << (8 * j);
          }
#pragma unroll
          for (int d = 0; d < kDigits; ++d) digit[d][2 * (w & 3) + (w >> 2)] = word[d];
        }
        if (mine) {
#pragma unroll
          for (int d = 0; d < kDigits; ++d)
#pragma unroll
            for (int w = 0; w < 8; w += 4) *reinterpret_cast<uint4*>(to + d * kPlane + w) = make_uint4(digit[d][w], digit[d][w + 1], digit[d][w + 2], digit[d][w + 3]);
        }
      } else if (mine) {
#pragma unroll
        for (int w = 0; w < 4; w += 2) *reinterpret_cast<uint4*>(to + 2 * w) = make_uint4(q_raw[i][0][w], q_raw[i][1][w], q_raw[i][0][w + 1], q_raw[i][1][w + 1]);
      }
    }
    if (tid < F::kRows) {
      const int row = row0 + tid, turn = p.groups.of(row), token = min(turn, p.tokens - 1), h = head * p.group + row - turn * p.group;
      sm.token[tid] = token;
      sm.slope[tid] = p.slopes && row < p.rows ? p.slopes[h] * kLog2e : 0.f;
      sm.out[tid] = row < p.rows ? b * p.out_batch + token * p.out_token + h * p.out_head : -1;
      sm.lse[tid] = row < p.rows ? (b * p.tokens + token) * p.heads * p.group + h : 0;
    }
  };
  // Tile n of a warp is tile n RW + rw of the CTA, so that few rows are spread over its warps; columns 2c, 2c + 1 are this lane's.  Tiles behind the rows are left out.
  const int row_of_mine = 8 * rw + 2 * c;
  int tiles = NT;
  auto query_operand = [&](int digit, int step, int n) {
    return *reinterpret_cast<const uint2*>(s_query + digit * kPlane + step * kStepWords + (n * RW + rw) * 64 + lane * 2);
  };
  constexpr bool kHold = NT == 1 && DH <= 128;  // operands of the queries stay in registers
  uint2 q_held[kHold ? (Q8 ? kDigits : 1) : 1][kHold ? kQuerySteps : 1];

  int b = at.b, hr = at.hr, unit = first_at;  // where the blocks are

  // ---- a warp's running state
  float o[kSteps][NT][4], top[NT][2], sum[NT][2];
  // 8 bits: for each row a power of two that the scales of the values it sees are divided by, so that the largest become 64 .. 128: with e up to 2^8 a weight stays below 2^15, and is a
  // normal number of fp16 down to 2^-20 of the largest.
  float unit_v[NT][2];
  float factor[NT][2];  // of a score
  auto begin_item = [&]() {
    if constexpr (RW > 1) {
      const int here = p.row_blocks == 1 ? p.rows : min(F::kRows, p.rows - (hr - hr / p.row_blocks * p.row_blocks) * F::kRows);
      tiles = max(0, min(NT, (here - 8 * rw + 8 * RW - 1) / (8 * RW)));
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      top[n][0] = top[n][1] = -INFINITY;
      sum[n][0] = sum[n][1] = 0.f;
      unit_v[n][0] = unit_v[n][1] = 0.f;
#pragma unroll
      for (int k = 0; k < kSteps; ++k) o[k][n][0] = o[k][n][1] = o[k][n][2] = o[k][n][3] = 0.f;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        // (alpha and the query's together first: a tiny alpha and a large query make an ordinary factor)
        factor[n][j] = Q8 ? p.alpha * sm.factor[row_of_mine + 8 * RW * n + j] * kLog2e : p.alpha_log2;
      }
    }
    if constexpr (kHold) {
#pragma unroll
      for (int d = 0; d < (Q8 ? kDigits : 1); ++d)
#pragma unroll
        for (int k = 0; k < kQuerySteps; ++k) q_held[d][k] = query_operand(d, k, 0);
    }
  };
  auto query = [&](int digit, int step, int n) {
    if constexpr (kHold) return q_held[digit][step];
    else return query_operand(digit, step, n);
  };

  // ---- one block
  // Where this lane reads of a row's pieces for ldmatrix; piece `k` (even) of the rows is at this address ^ (k << 4), pieces from 8 on 128 bytes further.
  const int low_row = lane & 15, v_row = Q8 ? low_row : (lane & 7) + ((lane >> 4) << 3), v_piece = Q8 ? lane >> 4 : (lane >> 3) & 1;
  const uint32_t k_lane = low_row * F::kRowBytes + place_of<F::kPieces>(low_row, lane >> 4) * 16;
  const uint32_t v_lane = F::kSide + v_row * F::kRowBytes + place_of<F::kPieces>(v_row, v_piece) * 16;
  auto at_piece = [](uint32_t base, int k) { return (base ^ ((k & 7) << 4)) + (k >> 3) * 128; };
  // The products and the softmax of a block, for this warp's first TN tiles.
  auto products = [&](auto tn, int stage, const Sequence& seq, int base, unsigned valid, bool all) {
    constexpr int TN = decltype(tn)::value;
    const int first = seq.length - p.tokens;  // the first new token's position
    const uint32_t keys = ring_u32 + stage * F::kStage + k_lane, values = ring_u32 + stage * F::kStage + v_lane;
    float s[G][TN][4];
    if constexpr (Q8) {
      uint32_t a[kQuerySteps][G][4];
#pragma unroll
      for (int k = 0; k < kQuerySteps; ++k)
#pragma unroll
        for (int h = 0; h < G; ++h) ldmatrix_x4(at_piece(keys + h * 16 * F::kRowBytes, 2 * k), a[k][h]);
#pragma unroll
      for (int n = 0; n < TN; ++n) {
        int sd[kDigits][G][4];
#pragma unroll
        for (int d = 0; d < kDigits; ++d)
#pragma unroll
          for (int h = 0; h < G; ++h) sd[d][h][0] = sd[d][h][1] = sd[d][h][2] = sd[d][h][3] = 0;
#pragma unroll
        for (int k = 0; k < kQuerySteps; ++k)
#pragma unroll
          for (int d = 0; d < kDigits; ++d) {
            const uint2 b = query(d, k, n);
#pragma unroll
            for (int h = 0; h < G; ++h) mma_s8(sd[d][h], a[k][h], b.x, b.y);
          }
#pragma unroll
        for (int h = 0; h < G; ++h)
#pragma unroll
          for (int i = 0; i < 4; ++i)  // (a digit's sum is at most 128 * 128 * 256: the upper two in 32 bits)
            s[h][n][i] = fmaf(static_cast<float>(sd[0][h][i] * 256 + sd[1][h][i]), 256.f, static_cast<float>(sd[2][h][i]));
      }
    } else {
#pragma unroll
      for (int h = 0; h < G; ++h)
#pragma unroll
        for (int n = 0; n < TN; ++n) s[h][n][0] = s[h][n][1] = s[h][n][2] = s[h][n][3] = 0.f;
#pragma unroll
      for (int k = 0; k < kQuerySteps; ++k) {
        uint32_t a[G][4];
#pragma unroll
        for (int h = 0; h < G; ++h) ldmatrix_x4(at_piece(keys + h * 16 * F::kRowBytes, 2 * k), a[h]);
#pragma unroll
        for (int n = 0; n < TN; ++n) {
          const uint2 b = query(0, k, n);
#pragma unroll
          for (int h = 0; h < G; ++h) mma<kMmaBf16>(s[h][n], a[h], b.x, b.y);
        }
      }
    }
    [[maybe_unused]] float ks[G][2], vs[G][2];
    if constexpr (Q8) {
      const float* scales = reinterpret_cast<const float*>(ring + stage * F::kStage + 2 * F::kSide);
#pragma unroll
      for (int h = 0; h < G; ++h)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          ks[h][i] = scales[16 * h + 8 * i + g];
          vs[h][i] = scales[F::kBlock + 16 * h + 8 * i + g];
        }
    }
    // s: scores in the log2 domain less the running maximum, raised by kLift (no maximum yet: the scores)
    float ref[TN][2], limit[TN][2];
#pragma unroll
    for (int n = 0; n < TN; ++n)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const bool none = top[n][j] == -INFINITY;
        ref[n][j] = none ? 0.f : top[n][j] - kLift;
        limit[n][j] = none ? -INFINITY : kSlack + kLift;
      }
    if (p.cap > 0.f) {
      auto far_of = [&](int h, int n) {
        bool far = false;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          s[h][n][i] *= Q8 ? factor[n][i & 1] * ks[h][i >> 1] : factor[n][i & 1];
          far |= fabsf(s[h][n][i] * p.per_cap) >= kCapNear;
        }
        return far;
      };
      auto capped_any = [&](int h, int n) {
#pragma unroll
        for (int i = 0; i < 4; ++i) s[h][n][i] = softcap_any(s[h][n][i], p.cap, p.per_cap) - ref[n][i & 1];
      };
      auto capped_near = [&](int h, int n) {  // (most blocks of most calls: no exponentials)
#pragma unroll
        for (int i = 0; i < 4; ++i) s[h][n][i] = softcap_near(s[h][n][i], p.per_cap) - ref[n][i & 1];
      };
      // One look at all of the block's scores (five new tokens of 8 sequences, D = 256: 34.3 us, with one a tile 35.4), or, where 168 registers or fewer would not hold what lies between (64 rows
      // of 128 over 20000 positions, 8 heads: 48.5 us instead of 53.1), at a tile's.
      if constexpr (F::kThreads * F::kCtasPerSm > 256) {
#pragma unroll
        for (int h = 0; h < G; ++h)
#pragma unroll
          for (int n = 0; n < TN; ++n) {
            if (__any_sync(0xFFFFFFFFu, far_of(h, n))) capped_any(h, n);
            else capped_near(h, n);
          }
      } else {
        bool far = false;
#pragma unroll
        for (int h = 0; h < G; ++h)
#pragma unroll
          for (int n = 0; n < TN; ++n) far |= far_of(h, n);
        const bool any = __any_sync(0xFFFFFFFFu, far);
        if (any) {
#pragma unroll
          for (int h = 0; h < G; ++h)
#pragma unroll
            for (int n = 0; n < TN; ++n) capped_any(h, n);
        } else {
#pragma unroll
          for (int h = 0; h < G; ++h)
#pragma unroll
            for (int n = 0; n < TN; ++n) capped_near(h, n);
        }
      }
    } else {
#pragma unroll
      for (int h = 0; h < G; ++h)
#pragma unroll
        for (int n = 0; n < TN; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i) s[h][n][i] = fmaf(s[h][n][i], Q8 ? factor[n][i & 1] * ks[h][i >> 1] : factor[n][i & 1], -ref[n][i & 1]);
    }
    if (p.slopes) {  // slope (n - m), from the distance of the block's first position on
#pragma unroll
      for (int n = 0; n < TN; ++n)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int r = row_of_mine + 8 * RW * n + j;
          const float slope = sm.slope[r], from = static_cast<float>(base + g - (first + sm.token[r])) * slope;
#pragma unroll
          for (int h = 0; h < G; ++h)
#pragma unroll
            for (int i = 0; i < 2; ++i) s[h][n][2 * i + j] += fmaf(slope, static_cast<float>(16 * h + 8 * i), from);
        }
    }
    if (!all) {
#pragma unroll
      for (int n = 0; n < TN; ++n)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int last = first + sm.token[row_of_mine + 8 * RW * n + j] - base;  // the row sees positions of the block up to this one
#pragma unroll
          for (int h = 0; h < G; ++h)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const int k = 16 * h + 8 * i + g;
              if (!((valid >> k) & 1u) || k > last || (p.window > 0 && k <= last - p.window)) s[h][n][2 * i + j] = -INFINITY;
            }
        }
    }
    // the maximum, where a score is well above it
    bool above = false;
#pragma unroll
    for (int n = 0; n < TN; ++n)
#pragma unroll
      for (int h = 0; h < G; ++h)
#pragma unroll
        for (int i = 0; i < 4; ++i) above |= s[h][n][i] > limit[n][i & 1];
    if constexpr (Q8) {
      float least = unit_v[0][0];
#pragma unroll
      for (int n = 0; n < TN; ++n) least = fminf(fminf(least, unit_v[n][0]), unit_v[n][1]);
#pragma unroll
      for (int h = 0; h < G; ++h) above |= fmaxf(fabsf(vs[h][0]), fabsf(vs[h][1])) > 128.f * least;
    }
    if (__any_sync(0xFFFFFFFFu, above)) {
#pragma unroll
      for (int n = 0; n < TN; ++n)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          float m = -INFINITY;
          [[maybe_unused]] float most = 0.f;
#pragma unroll
          for (int h = 0; h < G; ++h)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const float v = s[h][n][2 * i + j];
              m = fmaxf(m, v);
              if constexpr (Q8) most = fmaxf(most, v == -INFINITY ? 0.f : fabsf(vs[h][i]));
            }
#pragma unroll
          for (int d = 4; d < 32; d <<= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, d));
          // (s is relative to ref: the maximum rises by m, where that is positive or there was none)
          const bool none = top[n][j] == -INFINITY;
          const float rise = none ? m : fmaxf(m - kLift, 0.f), shift = !none ? rise : rise == -INFINITY ? 0.f : rise - kLift;
          const float less = none ? 1.f : ex2_approx(-rise);  // (without a maximum there is nothing yet to make less)
          top[n][j] = none ? rise : top[n][j] + rise;
          sum[n][j] *= less;
          float both = less;
          if constexpr (Q8) {
#pragma unroll
            for (int d = 4; d < 32; d <<= 1) most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, d));
            const float unit = fmaxf(unit_v[n][j], __uint_as_float(min(max(__float_as_uint(most) & 0x7F800000u, 0x04000000u), 0x7E000000u) - 0x03000000u));
            both *= unit_v[n][j] / unit;
            unit_v[n][j] = unit;
          }
#pragma unroll
          for (int h = 0; h < G; ++h)
#pragma unroll
            for (int i = 0; i < 2; ++i) s[h][n][2 * i + j] -= shift;
#pragma unroll
          for (int k = 0; k < kSteps; ++k) {
            o[k][n][j] *= both;
            o[k][n][j + 2] *= both;
          }
        }
    }
    // weights, as the second product's operand
    uint32_t w[G][TN][2];
    [[maybe_unused]] uint32_t rest[G][TN][2];
#pragma unroll
    for (int n = 0; n < TN; ++n) {
      const float inv[2] = {reciprocal_of_power(unit_v[n][0]), reciprocal_of_power(unit_v[n][1])};
#pragma unroll
      for (int h = 0; h < G; ++h) {
        float e[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) e[i] = ex2_approx(s[h][n][i]);
        sum[n][0] += e[0] + e[2];
        sum[n][1] += e[1] + e[3];
        if constexpr (Q8) {
#pragma unroll
          for (int i = 0; i < 4; ++i) e[i] *= vs[h][i >> 1] * inv[i & 1];
          if (!all) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (s[h][n][i] == -INFINITY) e[i] = 0.f;  // (a hidden position's scale may be NaN)
          }
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const uint32_t x = pack2<kMmaBf16>(e[2 * i], e[2 * i + 1]);
          w[h][n][i] = transpose_8x8(x);
          if constexpr (kTwice) {
            const float2 r = unpack2<kMmaBf16>(x);
            rest[h][n][i] = transpose_8x8(pack2<kMmaBf16>(e[2 * i] - r.x, e[2 * i + 1] - r.y));
          }
        }
      }
    }
#pragma unroll
    for (int h = 0; h < G; ++h) {
      const uint32_t rows = values + h * 16 * F::kRowBytes;
      if constexpr (Q8) {
#pragma unroll
        for (int k = 0; k < kSteps; k += 2) {
          uint32_t r[4];
          ldmatrix_x4_trans(at_piece(rows, k), r);
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const uint32_t x = r[2 * i] ^ 0x80808080u, y = r[2 * i + 1] ^ 0x80808080u;
            const uint32_t a[4] = {codes_f16(x, 0x4240), codes_f16(x, 0x4341), codes_f16(y, 0x4240), codes_f16(y, 0x4341)};
#pragma unroll
            for (int n = 0; n < TN; ++n) {
              mma<false>(o[k + i][n], a, w[h][n][0], w[h][n][1]);
              if constexpr (kTwice) mma<false>(o[k + i][n], a, rest[h][n][0], rest[h][n][1]);
            }
          }
        }
      } else {
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
          uint32_t a[4];
          ldmatrix_x4_trans(at_piece(rows, 2 * k), a);
#pragma unroll
          for (int n = 0; n < TN; ++n) {
            mma<kMmaBf16>(o[k][n], a, w[h][n][0], w[h][n][1]);
            mma<kMmaBf16>(o[k][n], a, rest[h][n][0], rest[h][n][1]);
          }
        }
      }
    }
  };
  auto block = [&](int stage, const Sequence& seq, int base) {
    const unsigned valid = sm.valid[kw][stage];
    if (!valid) return;
    const int first = seq.length - p.tokens;  // the first new token's position
    constexpr unsigned kAll = F::kBlock == 32 ? 0xFFFFFFFFu : 0xFFFFu;
    const bool all = valid == kAll && base + F::kBlock - 1 <= first && (p.window <= 0 || base > seq.length - 1 - p.window);
    if constexpr (!Q8) {
      if (!all && p.tokens > 1) {
        // Some rows see a position and others do not: a value that is not finite must not reach the others as 0 * inf.  Such values are added to the rows that see them, and
        // are zeros for the product.
        const char* block_v = ring + stage * F::kStage + F::kSide;
        bool odd = false;
        for (int i = lane; i < F::kSide / 16; i += 32) {
          const uint4 x = *reinterpret_cast<const uint4*>(block_v + i * 16);
          const uint32_t y[4] = {x.x, x.y, x.z, x.w};
          constexpr uint32_t e = kBf16 ? 0x7F80u : 0x7C00u;
#pragma unroll
          for (int j = 0; j < 4; ++j) odd |= (y[j] & e) == e || (y[j] >> 16 & e) == e;
        }
        // (all warps of a ring come here, find the same, and clear it together)
        if (__any_sync(0xFFFFFFFFu, odd)) {
          for (int k = 0; k < F::kBlock; ++k) {
            const int pos = base + k - first;
#pragma unroll
            for (int d = 0; d < kSteps; ++d)
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                const int e = 16 * d + 8 * h + g;
                const float v = Elem<DT>::get(block_v + k * F::kRowBytes + place_of<F::kPieces>(k, e >> 3) * 16 + (e & 7) * 2, 0);
                if (!isfinite(v)) {
#pragma unroll
                  for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                      const int gap = pos - sm.token[row_of_mine + 8 * RW * n + j];
                      if (gap <= 0 && (p.window <= 0 || gap > -p.window)) o[d][n][2 * h + j] += v;
                    }
                }
              }
          }
          ring_sync();
          for (int i = lane; i < F::kSide / 2; i += 32) {
            uint16_t* at_v = reinterpret_cast<uint16_t*>(ring + stage * F::kStage + F::kSide) + i;
            if (!isfinite(Elem<DT>::get(at_v, 0))) *at_v = 0;
          }
          ring_sync();
        }
      }
    }
    if (RW == 1 || tiles == NT) products(std::integral_constant<int, NT>(), stage, seq, base, valid, all);
    else if (NT > 1 && tiles > 0) products(std::integral_constant<int, 1>(), stage, seq, base, valid, all);
  };

  // ---- the end of an item, or of the share: the rings' results are joined; whole items are finished, cut ones kept
  // A thread adds up kMine columns of every kJoinColumns, of one of the 8 RW rows that a tile of each row warp makes.
  constexpr int kSumThreads = F::kThreads < 256 ? F::kThreads : 256;
  constexpr int kMine = 8 * RW * F::kJoinColumns / kSumThreads, kAcross = F::kJoinColumns / kMine;
  // `parts`: where the rows of a cut item go.  A cluster: pieces of four columns to the CTAs in turn, statistics to all.
  struct Sent {
    float2 stats[CLUSTER ? 16 : 1][F::kRows];       // by sender
    float4 values[CLUSTER ? F::kRows * DH / 4 + 16 : 1];  // by sender, its pieces for this CTA
  };
  static_assert(sizeof(Sent) <= S * F::kStage * F::kKeyWarps, "what a cluster's CTAs send lies where the rings were");
  Sent& sent = *reinterpret_cast<Sent*>(smem);
  int here = 0, sent_each = 0;  // rows, pieces of a sender
  auto end_item = [&](bool whole, float* parts) {
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        float t = sum[n][j];
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) t += __shfl_xor_sync(0xFFFFFFFFu, t, d);
        if (g == 0) {
          sm.top[kw][row_of_mine + 8 * RW * n + j] = top[n][j];
          sm.sum[kw][row_of_mine + 8 * RW * n + j] = t;
        }
      }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      float weight[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int r = row_of_mine + 8 * RW * n + j;
        float m = sm.top[0][r];
#pragma unroll
        for (int w = 1; w < F::kKeyWarps; ++w) m = fmaxf(m, sm.top[w][r]);
        weight[j] = top[n][j] == -INFINITY && m == -INFINITY ? 1.f : ex2_approx(top[n][j] - m);
        if constexpr (Q8) weight[j] *= unit_v[n][j];
      }
      const int r = min(tid / kAcross, 8 * RW - 1), col = (tid % kAcross) * kMine, row = n * 8 * RW + r;
      float m = sm.top[0][row], l = 0.f;
#pragma unroll
      for (int w = 1; w < F::kKeyWarps; ++w) m = fmaxf(m, sm.top[w][row]);
#pragma unroll
      for (int w = 0; w < F::kKeyWarps; ++w) l += sm.sum[w][row] * (sm.top[w][row] == -INFINITY ? (m == -INFINITY ? 1.f : 0.f) : ex2_approx(sm.top[w][row] - m));
      const float inv = !whole ? 1.f : l == 0.f ? 0.f : 1.f / l;
      const bool there = tid < kSumThreads && sm.out[row] >= 0;
      float* part = parts + row * (DH + 4);
      if (there && tid % kAcross == 0) {
        if (whole) {
          if (p.lse && COMFUSE_IN_BOUNDS(sm.lse[row] < p.batch * p.tokens * p.heads * p.group, p.status)) p.lse[sm.lse[row]] = log_sum<kLiftOf<DT, Q8>>(m, l);
        } else if constexpr (CLUSTER) {
          for (int k = 0; k < p.cluster; ++k) st_cluster_f32x2(map_to_cta(smem_u32(&sent.stats[rank][row]), k), m, l);
        } else if (COMFUSE_IN_BOUNDS(row < F::kRows, p.status)) {
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
            float* to = s_join + ((kw * RW + rw) * 8 + 2 * c + j) * F::kPitch + 16 * k;
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
        for (int w = 0; w < F::kKeyWarps; ++w)
#pragma unroll
          for (int j = 0; j < kMine; ++j) v[j] += s_join[(w * RW * 8 + r) * F::kPitch + col + j];
        const int at = first + col;
        if (!there) continue;
        if (whole) {
          if (at < p.D && COMFUSE_IN_BOUNDS(at + kMine <= p.D, p.status)) {
            uint32_t y[kMine / 2];
#pragma unroll
            for (int j = 0; j < kMine; ++j) v[j] *= inv;
            Elem<DT>::pack(v, y);
            char* to = p.out + sm.out[row] + 2 * at;
            if constexpr (kMine == 8) st_16(to, y);
            else if constexpr (kMine == 4) st_8(to, y);
            else *reinterpret_cast<uint32_t*>(to) = y[0];
          }
        } else if constexpr (CLUSTER) {
#pragma unroll
          for (int j = 0; j < kMine; j += 4) {
            const int piece = (row * DH + at + j) / 4, to = piece % p.cluster;
            const uint32_t where = map_to_cta(smem_u32(&sent.values[rank * sent_each + piece / p.cluster]), to);
            if constexpr (kMine >= 4) st_cluster_f32x4(where, v + j);
            else st_cluster_f32x2(where + (at & 2) * 4, v[0], v[1]);
          }
        } else if (COMFUSE_IN_BOUNDS(row < F::kRows, p.status)) {
#pragma unroll
          for (int j = 0; j < kMine; j += 2) *reinterpret_cast<float2*>(part + at + j) = make_float2(v[j], v[j + 1]);
        }
      }
    }
  };

  // ---- the share: S - 1 rounds that only fetch, then a block each
  int stage = 0;
  bool from_start = unit == 0, fresh = true;
  int pieces = 0;
  Sequence seq = first_seq;
  for (int n = 1 - S; n < (CLUSTER ? max(count, 1) : count); ++n) {
    if (n >= 0) {
      if (fresh) {
        keep_queries(b, hr);
        __syncthreads();
        begin_item();
        fresh = false;
      }
      cp_async_wait<S - 2>();
      ring_sync();
    }
    fetch(n < 0 ? n + S - 1 : stage == 0 ? S - 1 : stage - 1);
    if (n < 0) continue;
    if (!CLUSTER || count > 0) block(stage, seq, (seq.low & ~(F::kBlock - 1)) + unit * F::kUnit + kw * F::kBlock);
    stage = stage + 1 == S ? 0 : stage + 1;
    ++unit;
    if constexpr (CLUSTER) {
      if (n + 1 < count) continue;
      if (p.cluster == 1) {
        end_item(true, nullptr);
        break;
      }
      cp_async_wait<0>();
      const int head = p.row_blocks == 1 ? hr : hr / p.row_blocks;
      here = min(F::kRows, p.rows - (hr - head * p.row_blocks) * F::kRows);
      sent_each = (here * (DH / 4) + p.cluster - 1) / p.cluster;
      cluster_sync_all();  // every CTA's rings are done with
      end_item(false, nullptr);
      cluster_sync_all();  // (behind it nobody writes into another CTA's shared memory)
      for (int i = tid; i < sent_each; i += F::kThreads) {
        const int piece = i * p.cluster + rank, r = piece / (DH / 4), col = (piece % (DH / 4)) * 4;
        if (r >= here) continue;
        float m = -INFINITY, l = 0.f;
        for (int k = 0; k < p.cluster; ++k) m = fmaxf(m, sent.stats[k][r].x);
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
        for (int k = 0; k < p.cluster; ++k) {
          const float2 s = sent.stats[k][r];
          const float4 x = sent.values[k * sent_each + i];
          const float w = s.x == -INFINITY ? (m == -INFINITY ? 1.f : 0.f) : ex2_approx(s.x - m);
          l = fmaf(s.y, w, l);
          v.x = fmaf(x.x, w, v.x); v.y = fmaf(x.y, w, v.y); v.z = fmaf(x.z, w, v.z); v.w = fmaf(x.w, w, v.w);
        }
        const float inv = l == 0.f ? 0.f : 1.f / l;
        const float y[4] = {v.x * inv, v.y * inv, v.z * inv, v.w * inv};
        uint32_t packed[2];
        Elem<DT>::pack(y, packed);
        if (col < p.D && COMFUSE_IN_BOUNDS(col + 4 <= p.D && r < here, p.status)) st_8(p.out + sm.out[r] + 2 * col, packed);
        if (p.lse && col == 0 && COMFUSE_IN_BOUNDS(sm.lse[r] < p.batch * p.tokens * p.heads * p.group, p.status)) p.lse[sm.lse[r]] = log_sum<kLiftOf<DT, Q8>>(m, l);
      }
      break;
    }
    if (unit == seq.units || n + 1 == count) {
      const bool whole = from_start && unit == seq.units, more = n + 1 < count;
      int nb = b, nhr = hr + 1;
      if (nhr == HR) nhr = 0, ++nb;
      if (more) load_queries(nb, nhr);  // on their way under the joining
      end_item(whole, p.part + blockIdx.x * part_floats(F::kRows, DH) + (pieces ? F::kRows * (DH + 4) : 0));
      if (more) {
        __syncthreads();  // everyone has read the last item's rows
        ++pieces;
        fresh = from_start = true;
        unit = 0;
        if (nb != b) seq = sequence_of<F>(p, nb);
        b = nb;
        hr = nhr;
      }
    }
  }
  cp_async_wait<0>();
}

// ------------------------------------------------------------------------------------------------ joining
// CTA (i, r): row r of item i (few items), or of the item that is cut behind share i, if that is its first cut.  Partial results are added up in the order of the shares.
constexpr int kJoinThreads = 256;
template <int DT, bool Q8, int DH, int NT, int RW>
__global__ void __launch_bounds__(kJoinThreads) join_kernel(const PagedAttentionParams p, const int by_item) {
  using F = Form<Q8, DH, NT, RW, false>;
  constexpr int kAcross = DH / 4, kStripes = kJoinThreads / kAcross;  // threads of a row, four columns each; every kStripes-th part is one stripe's
  constexpr int kMost = 296;                                          // parts
  __shared__ float s_weight[kMost];
  __shared__ float4 s_sum[kStripes][kAcross];
  griddep_launch_dependents();
  const int tid = threadIdx.x, lane = tid & 31;
  // (the lengths are read in front of the wait: the kernel before this one signals behind its own)
  unsigned lane_units;
  const Line line = line_of<F>(p, lane, &lane_units);
  Place at;
  unsigned item, first, units;  // where the item begins, its first share
  bool cut;
  if (by_item) {
    const int HR = p.heads * p.row_blocks;
    at.b = blockIdx.x / HR;
    at.hr = blockIdx.x - at.b * HR;
    unsigned before = 0;
    for (int b0 = 0; b0 < at.b; b0 += 32) before += b0 + lane < at.b ? (b0 == 0 ? lane_units : sequence_of<F>(p, b0 + lane).units + F::kSetUp) : 0u;
    units = sequence_of<F>(p, at.b).units;
    item = __reduce_add_sync(0xFFFFFFFFu, before) * HR + at.hr * (units + F::kSetUp);
    first = line.owner(item + F::kSetUp);
    cut = line.owner(item + F::kSetUp + units - 1) != first;
  } else {
    const unsigned behind = line.begin(blockIdx.x + 1);
    at = place_of_unit<F>(p, lane, lane_units, min(behind, line.total - 1));
    units = sequence_of<F>(p, at.b).units;
    item = behind - at.at;
    first = blockIdx.x;
    cut = behind < line.total && at.at > F::kSetUp && item + F::kSetUp >= line.begin(blockIdx.x);
  }
  const int r = blockIdx.y, row = (at.hr % p.row_blocks) * F::kRows + r;
  const bool mine = cut && row < p.rows;
  const int n = mine ? static_cast<int>(line.owner(item + F::kSetUp + units - 1) - first) + 1 : 0;  // parts
  const int slot = item <= line.begin(first) ? 0 : 1;  // (a share that begins in front of the item has some of another's first)
  const float* first_part = p.part + first * part_floats(F::kRows, DH) + (slot * F::kRows + r) * (DH + 4);
  const float* next_part = p.part + (first + 1) * part_floats(F::kRows, DH) + r * (DH + 4);
  auto part = [&](int i) { return i == 0 ? first_part : next_part + (i - 1) * part_floats(F::kRows, DH); };
  const int stripe = tid / kAcross, col = (tid % kAcross) * 4;
  const int head = at.hr / p.row_blocks, token = p.groups.of(row), h = head * p.group + row - token * p.group;
  char* out = p.out + at.b * p.out_batch + token * p.out_token + h * p.out_head;
  float* lse = p.lse ? p.lse + (static_cast<long long>(at.b) * p.tokens + token) * p.heads * p.group + h : nullptr;
  griddep_wait();
  if (!mine) return;

  // the first parts of this thread's stripe are on their way while the weights are worked out
  constexpr int kEarly = 4;
  float4 early[kEarly];
#pragma unroll
  for (int i = 0; i < kEarly; ++i) early[i] = stripe + i * kStripes < n ? *reinterpret_cast<const float4*>(part(stripe + i * kStripes) + col) : make_float4(0.f, 0.f, 0.f, 0.f);
  float2 stats = lane < n ? *reinterpret_cast<const float2*>(part(lane) + DH) : make_float2(-INFINITY, 0.f);  // (of the first 32: more are read again)
  float m = stats.x;
  for (int i = lane + 32; i < n; i += 32) m = fmaxf(m, part(i)[DH]);
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, d));
  float l = 0.f;
  for (int i = lane; i < n; i += 32) {
    if (i >= 32) stats = *reinterpret_cast<const float2*>(part(i) + DH);
    const float w = stats.x == -INFINITY ? (m == -INFINITY ? 1.f : 0.f) : ex2_approx(stats.x - m);
    l = fmaf(stats.y, w, l);
    if (tid < 32) s_weight[i] = w;
  }
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) l += __shfl_xor_sync(0xFFFFFFFFu, l, d);
  const float inv = l == 0.f ? 0.f : 1.f / l;
  __syncthreads();
  float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
  auto add = [&](const float4& x, float w) {
    v.x = fmaf(x.x, w, v.x); v.y = fmaf(x.y, w, v.y); v.z = fmaf(x.z, w, v.z); v.w = fmaf(x.w, w, v.w);
  };
#pragma unroll
  for (int i = 0; i < kEarly; ++i)
    if (stripe + i * kStripes < n) add(early[i], s_weight[stripe + i * kStripes]);
#pragma unroll 8
  for (int i = stripe + kEarly * kStripes; i < n; i += kStripes) add(*reinterpret_cast<const float4*>(part(i) + col), s_weight[i]);
  s_sum[stripe][tid % kAcross] = v;
  __syncthreads();
  if (stripe > 0) return;
#pragma unroll
  for (int i = 1; i < kStripes; ++i) {
    const float4 x = s_sum[i][tid];
    v.x += x.x; v.y += x.y; v.z += x.z; v.w += x.w;
  }
  const float y[4] = {v.x * inv, v.y * inv, v.z * inv, v.w * inv};
  uint32_t packed[2];
  Elem<DT>::pack(y, packed);
  if (col < p.D && COMFUSE_IN_BOUNDS(col + 4 <= p.D && row < p.rows && at.b < p.batch, p.status)) st_8(out + 2 * col, packed);
  if (lse && tid == 0 && COMFUSE_IN_BOUNDS(at.b < p.batch && token < p.tokens, p.status)) *lse = log_sum<kLiftOf<DT, Q8>>(m, l);
}

// ------------------------------------------------------------------------------------------------ launches
// Dynamic shared memory, and clusters of 16, are asked for once a device.
cudaError_t make_ready(const void* kernel, int bytes, bool clusters, std::atomic<unsigned long long>* ready) {
  int device = 0;
  cudaError_t e = cudaGetDevice(&device);
  if (e != cudaSuccess) return e;
  const unsigned long long bit = 1ull << (device & 63);
  if (device < 64 && (ready->load(std::memory_order_relaxed) & bit)) return cudaSuccess;
  e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == cudaSuccess && clusters) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  if (e == cudaSuccess) ready->fetch_or(bit, std::memory_order_relaxed);
  return e;
}

template <int DT, bool Q8, int DH, int NT, int RW, bool CLUSTER>
cudaError_t launch_instance(const PagedAttentionPlan& plan, const PagedAttentionParams& p, cudaStream_t stream) {
  using F = Form<Q8, DH, NT, RW, CLUSTER>;
  static std::atomic<unsigned long long> ready{0};
  const auto kernel = attention_kernel<DT, Q8, DH, NT, RW, CLUSTER>;
  cudaError_t e = make_ready(reinterpret_cast<const void*>(kernel), F::kBytes, CLUSTER, &ready);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[2];
  cfg.gridDim = dim3(static_cast<unsigned>(plan.ctas), 1, 1);
  cfg.blockDim = dim3(F::kThreads, 1, 1);
  cfg.dynamicSmemBytes = F::kBytes;
  cfg.stream = stream;
  cfg.attrs = attr;
  if (programmatic_launch_enabled()) {
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.numAttrs = 1;
  }
  if (CLUSTER && plan.cluster > 1) {
    attr[cfg.numAttrs].id = cudaLaunchAttributeClusterDimension;
    attr[cfg.numAttrs].val.clusterDim.x = static_cast<unsigned>(plan.cluster);
    attr[cfg.numAttrs].val.clusterDim.y = 1;
    attr[cfg.numAttrs++].val.clusterDim.z = 1;
  }
  if (verbose_enabled())
    std::fprintf(stderr, "comfuse: paged_attention dtype=%d quantized=%d D<=%d row tiles=%d x %d row blocks=%d CTAs=%d cluster=%d stages=%d joined=%d\n", DT, Q8, DH, NT, RW, p.row_blocks, plan.ctas,
                 plan.cluster, F::kStages, plan.joined);
  count_launch();
  e = cudaLaunchKernelEx(&cfg, kernel, p);
  if constexpr (!CLUSTER) {
    if (e != cudaSuccess || !plan.joined) return e;
    const long long items = static_cast<long long>(p.batch) * p.heads * p.row_blocks;
    const int by_item = items < plan.ctas - 1;
    cfg.gridDim = dim3(static_cast<unsigned>(by_item ? items : plan.ctas - 1), static_cast<unsigned>(p.rows < F::kRows ? p.rows : F::kRows), 1);
    cfg.blockDim = dim3(kJoinThreads, 1, 1);
    cfg.dynamicSmemBytes = 0;
    count_launch();
    e = cudaLaunchKernelEx(&cfg, join_kernel<DT, Q8, DH, NT, RW>, p, by_item);
  }
  return e;
}

template <int DT, bool Q8, int DH>
cudaError_t launch_rows(const PagedAttentionPlan& plan, const PagedAttentionParams& p, cudaStream_t stream) {
  if (plan.rows == 8) return plan.cluster ? launch_instance<DT, Q8, DH, 1, 1, true>(plan, p, stream) : launch_instance<DT, Q8, DH, 1, 1, false>(plan, p, stream);
  if (plan.rows == 16) return plan.cluster ? launch_instance<DT, Q8, DH, 2, 1, true>(plan, p, stream) : launch_instance<DT, Q8, DH, 2, 1, false>(plan, p, stream);
  if (plan.rows == 32) return plan.cluster ? launch_instance<DT, Q8, DH, 2, 2, true>(plan, p, stream) : launch_instance<DT, Q8, DH, 2, 2, false>(plan, p, stream);
  return plan.cluster ? launch_instance<DT, Q8, DH, 2, 4, true>(plan, p, stream) : launch_instance<DT, Q8, DH, 2, 4, false>(plan, p, stream);
}
template <int DT, bool Q8>
cudaError_t launch_type(const PagedAttentionPlan& plan, const PagedAttentionParams& p, cudaStream_t stream) {
  if (p.D <= 64) return launch_rows<DT, Q8, 64>(plan, p, stream);
  if (p.D <= 128) return launch_rows<DT, Q8, 128>(plan, p, stream);
  return launch_rows<DT, Q8, 256>(plan, p, stream);
}

// What a plan needs to know of the instance that runs it.
struct FormFacts {
  int unit, block, ctas_per_sm, set_up, unit_bytes;
  int cluster_unit, cluster_ctas_per_sm, cluster_unit_bytes;
};
template <bool Q8, int DH, int NT, int RW>
constexpr FormFacts facts_of() {
  using F = Form<Q8, DH, NT, RW, false>;
  using C = Form<Q8, DH, NT, RW, true>;
  return {F::kUnit, F::kBlock, F::kCtasPerSm, F::kSetUp, F::kStage * F::kKeyWarps, C::kUnit, C::kCtasPerSm, C::kStage * C::kKeyWarps};
}
template <bool Q8, int DH>
FormFacts facts(int rows) {
  return rows == 8 ? facts_of<Q8, DH, 1, 1>() : rows == 16 ? facts_of<Q8, DH, 2, 1>() : rows == 32 ? facts_of<Q8, DH, 2, 2>() : facts_of<Q8, DH, 2, 4>();
}
template <bool Q8>
FormFacts facts(int D, int rows) {
  return D <= 64 ? facts<Q8, 64>(rows) : D <= 128 ? facts<Q8, 128>(rows) : facts<Q8, 256>(rows);
}

}  // namespace
}  // namespace paged
}  // namespace comfuse
