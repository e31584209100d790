// Parameter blocks and launchers of the key-value cache (plain data).  Strides are in BYTES unless said otherwise.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "host_common.h"

namespace comfuse {

// Division of numbers below 2^31 by a divisor known on the host: with l = ceil(log2 d) and m = floor(2^(31 + l) / d) + 1 the quotient is floor(n m / 2^(31 + l)), since
// n m exceeds 2^(31 + l) n / d by at most n < 2^31, less than 2^(31 + l) / d.  m fits in 32 bits; d = 1 stands apart.
struct Divisor {
  unsigned m, shift, d;
  Divisor() = default;
  explicit Divisor(unsigned by) : m(0), shift(0), d(by) {
    if (by < 2) return;
    unsigned l = 1;
    while ((1ull << l) < by) ++l;
    m = static_cast<unsigned>((1ull << (31 + l)) / by + 1);
    shift = l - 1;
  }
  __host__ __device__ __forceinline__ unsigned of(unsigned n) const {
#ifdef __CUDA_ARCH__
    const unsigned upper = __umulhi(n, m);
#else
    const unsigned upper = static_cast<unsigned>((static_cast<unsigned long long>(n) * m) >> 32);
#endif
    return m ? upper >> shift : n;
  }
};

// Where a cached row lies: base + page * page_stride + head * head_stride + row * row_stride.
struct CacheSide {
  char* rows;
  float* scale;
  long long page, head, row;                    // bytes
  long long scale_page, scale_head, scale_row;  // elements
};

struct RowsSide {
  const char* in;
  char* out;
  long long in_token, in_head, out_token, out_head;
};

struct RotaryWriteParams {
  int tokens, q_heads, kv_heads, D;
  int rows;              // of a token: what is to turn or store
  int slices_log2;       // warps that share a token
  RowsSide side[3];      // queries, keys, values (the latter two: in only)
  CacheSide kc, vc;
  const long long* slots;
  long long capacity;    // slots of the cache, below 2^31
  Divisor page_size;
  const int* positions;  // null: nothing is turned
  const double* freqs;
  long long axis_stride; // elements
  int pairs, adjacent;
  int section_end[4];    // the first pair behind each axis
  float sign;            // of the sine
  unsigned int* status;
};
// dtype: of q, k, v; cached: keys and values go into the cache; quantized: in 8 bits
cudaError_t launch_rotary_write(int dtype, bool cached, bool quantized, RotaryWriteParams p, const DeviceInfo& dev, cudaStream_t stream);

struct CacheReadParams {
  int tokens, heads, D;
  Divisor page_size, rows;  // rows: 2 * heads of a token
  int tokens_log2;          // of a block of tokens, whose rows of one head lie side by side in a warp
  CacheSide kc, vc;
  RowsSide k, v;         // (out only)
  const long long* slots;
  long long capacity;
  unsigned int* status;
};
cudaError_t launch_cache_read(int dtype, bool quantized, const CacheReadParams& p, const DeviceInfo& dev, cudaStream_t stream);

struct PagedAttentionParams {
  int batch, tokens, heads, group, D;   // group: query heads of a key head
  int rows;                             // tokens * group: the queries of a sequence that read the same keys
  int row_blocks;                       // CTAs' worth of them
  int pages, max_length, window;
  Divisor page_size, groups, shares;    // groups: divides by `group`, shares: by `ctas`
  const char* q;
  char* out;
  long long q_batch, q_token, q_head, out_batch, out_token, out_head;
  CacheSide kc, vc;
  const int* table;
  long long table_stride;               // elements
  const int* lengths;
  const float* slopes;
  float* lse;
  float alpha, alpha_log2;              // alpha log2 e
  float cap, per_cap;                   // in the log2 domain, and 1 / cap; 0: no soft-cap
  float* part;                          // partial results, see paged_attention.cuh
  int ctas, cluster;                    // cluster: CTAs of an item (0: shares)
  unsigned int* status;
};
// How a call is cut: query rows of a CTA (8, 16, 32 or 64), row blocks, CTAs, bytes of partial results.
struct PagedAttentionPlan {
  int rows, row_blocks, ctas;
  int cluster;                          // CTAs of an item, 0: items are cut where equal shares end
  bool joined;                          // items may be cut: a second kernel joins them
  size_t workspace;
};
PagedAttentionPlan paged_attention_plan(int batch, int rows, int heads, int D, bool quantized, int max_length, int window, int tokens);
cudaError_t launch_paged_attention(int dtype, bool quantized, const PagedAttentionPlan& plan, const PagedAttentionParams& p, cudaStream_t stream);

}  // namespace comfuse
