// C entry points of the key-value cache: argument checks, choice of the form.
#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstdlib>

#include "kv_params.h"
#include "paged_attention.cuh"

namespace comfuse {
namespace {

bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
bool type_16(int dtype) { return dtype == COMFUSE_DTYPE_BF16 || dtype == COMFUSE_DTYPE_F16; }
constexpr int64_t kMostStride = int64_t{1} << 44;  // elements: with the sizes' limits, products of strides and indices stay in 64 bits

// Strides that address something: not negative, no overlap of neighbours along the innermost one.
template <int N>
bool strides_ok(const int64_t (&s)[N], const int64_t (&sizes)[N], int64_t D) {
  for (int i = 0; i < N; ++i) {
    if (sizes[i] == 1) continue;  // (not used)
    if (s[i] < D || s[i] > kMostStride) return false;
  }
  return true;
}
template <int N>
bool strides_aligned(const int64_t (&s)[N], const int64_t (&sizes)[N], int bytes) {
  for (int i = 0; i < N; ++i)
    if (sizes[i] != 1 && (s[i] * bytes) % 16 != 0) return false;
  return true;
}
#define CHECK_STRIDES(s, bytes, ...)                                                   \
  do {                                                                                 \
    const int64_t sizes_[] = {__VA_ARGS__};                                            \
    if (!strides_ok(s, sizes_, d_)) return COMFUSE_ERR_INVALID_ARG;                    \
    if (!strides_aligned(s, sizes_, bytes)) return COMFUSE_ERR_ALIGNMENT;              \
  } while (0)

comfuse_status_t check_rotary(const comfuse_rotary_t* r, int D) {
  if (r->pairs < 1 || 2 * static_cast<int64_t>(r->pairs) > D || r->axes < 1 || r->axes > 4 || !r->positions || !r->freqs) return COMFUSE_ERR_INVALID_ARG;
  if ((r->adjacent & ~1) || (r->inverse & ~1) || (r->axes > 1 && (r->axis_stride < 0 || r->axis_stride > kMostStride))) return COMFUSE_ERR_INVALID_ARG;
  int64_t sum = 0;
  for (int i = 0; i < 4; ++i) {
    if (r->sections[i] < 0 || (i >= r->axes && r->sections[i] != 0)) return COMFUSE_ERR_INVALID_ARG;
    sum += r->sections[i];
  }
  if (sum != r->pairs) return COMFUSE_ERR_INVALID_ARG;
  return aligned(r->positions, 4) && aligned(r->freqs, 8) ? COMFUSE_OK : COMFUSE_ERR_ALIGNMENT;
}

comfuse_status_t check_cache(const comfuse_kv_cache_t* c) {
  if (!c) return COMFUSE_ERR_INVALID_ARG;
  if (c->pages < 1 || c->heads < 1 || c->page_size < 1 || c->D < 1 || !type_16(c->dtype) || (c->quantized & ~1)) return COMFUSE_ERR_INVALID_ARG;
  if (!c->k || !c->v || (c->quantized ? !c->k_scale || !c->v_scale : c->k_scale || c->v_scale)) return COMFUSE_ERR_INVALID_ARG;
  if (c->D % (c->quantized ? 16 : 8) != 0) return COMFUSE_ERR_ALIGNMENT;
  if (c->D > 256 || c->page_size > 65536 || c->heads > 65536 || static_cast<int64_t>(c->pages) * c->page_size > 0x7FFFFFFF) return COMFUSE_ERR_UNSUPPORTED;
  const int64_t d_ = c->D;
  const int bytes = c->quantized ? 1 : 2;
  CHECK_STRIDES(c->k_strides, bytes, c->pages, c->heads, c->page_size);
  CHECK_STRIDES(c->v_strides, bytes, c->pages, c->heads, c->page_size);
  if (!aligned(c->k, 16) || !aligned(c->v, 16)) return COMFUSE_ERR_ALIGNMENT;
  // (offsets within a page, and of pages, are products of 32-bit numbers)
  for (const int64_t* s : {c->k_strides, c->v_strides})
    if ((c->pages > 1 && s[0] * bytes > 0x7FFFFFFF) || (c->page_size > 1 && s[2] * bytes > 0x7FFFFFFF)) return COMFUSE_ERR_UNSUPPORTED;
  if (c->quantized) {
    const int64_t sizes[] = {c->pages, c->heads, c->page_size};
    if (!strides_ok(c->k_scale_strides, sizes, 1) || !strides_ok(c->v_scale_strides, sizes, 1)) return COMFUSE_ERR_INVALID_ARG;
    if (!aligned(c->k_scale, 4) || !aligned(c->v_scale, 4)) return COMFUSE_ERR_ALIGNMENT;
  }
  return COMFUSE_OK;
}

comfuse_status_t check_rotary_call(const comfuse_rotary_desc_t* d, const comfuse_rotary_t* r, const void* x, const void* out) {
  if (!d || !r || !x || !out) return COMFUSE_ERR_INVALID_ARG;
  if (d->tokens < 1 || d->heads < 1 || d->D < 1 || (!type_16(d->dtype) && d->dtype != COMFUSE_DTYPE_F32)) return COMFUSE_ERR_INVALID_ARG;
  if (d->D % 8 != 0) return COMFUSE_ERR_ALIGNMENT;
  if (d->D > 512 || d->heads > 65536) return COMFUSE_ERR_UNSUPPORTED;
  comfuse_status_t s = check_rotary(r, d->D);
  if (s != COMFUSE_OK) return s;
  const int64_t d_ = d->D;
  const int bytes = d->dtype == COMFUSE_DTYPE_F32 ? 4 : 2;
  CHECK_STRIDES(d->x_strides, bytes, d->tokens, d->heads);
  CHECK_STRIDES(d->out_strides, bytes, d->tokens, d->heads);
  if (x == out && ((d->tokens > 1 && d->x_strides[0] != d->out_strides[0]) || (d->heads > 1 && d->x_strides[1] != d->out_strides[1]))) return COMFUSE_ERR_INVALID_ARG;
  return aligned(x, 16) && aligned(out, 16) ? COMFUSE_OK : COMFUSE_ERR_ALIGNMENT;
}

comfuse_status_t check_write(const comfuse_cache_write_desc_t* d, const comfuse_kv_cache_t* c, const comfuse_rotary_t* r, const void* k, const void* v, const void* q,
                             const void* q_out, const int64_t* slots) {
  if (!d || !k || !v || !slots || d->tokens < 1 || d->q_heads < 0) return COMFUSE_ERR_INVALID_ARG;
  comfuse_status_t s = check_cache(c);
  if (s != COMFUSE_OK) return s;
  if ((d->q_heads > 0) != (q != nullptr) || (q != nullptr) != (q_out != nullptr) || (q && !r)) return COMFUSE_ERR_INVALID_ARG;
  if (d->q_heads > 65536) return COMFUSE_ERR_UNSUPPORTED;
  if (r) {
    if (r->inverse) return COMFUSE_ERR_INVALID_ARG;
    s = check_rotary(r, c->D);
    if (s != COMFUSE_OK) return s;
  }
  const int64_t d_ = c->D;
  CHECK_STRIDES(d->k_strides, 2, d->tokens, c->heads);
  CHECK_STRIDES(d->v_strides, 2, d->tokens, c->heads);
  if (q) {
    CHECK_STRIDES(d->q_strides, 2, d->tokens, d->q_heads);
    CHECK_STRIDES(d->q_out_strides, 2, d->tokens, d->q_heads);
    if (q == q_out && ((d->tokens > 1 && d->q_strides[0] != d->q_out_strides[0]) || (d->q_heads > 1 && d->q_strides[1] != d->q_out_strides[1]))) return COMFUSE_ERR_INVALID_ARG;
  }
  return aligned(k, 16) && aligned(v, 16) && aligned(q, 16) && aligned(q_out, 16) && aligned(slots, 8) ? COMFUSE_OK : COMFUSE_ERR_ALIGNMENT;
}

comfuse_status_t check_read(const comfuse_cache_read_desc_t* d, const comfuse_kv_cache_t* c, const int64_t* slots, const void* k, const void* v) {
  if (!d || !k || !v || !slots || d->tokens < 1 || d->reserved != 0) return COMFUSE_ERR_INVALID_ARG;
  const comfuse_status_t s = check_cache(c);
  if (s != COMFUSE_OK) return s;
  const int64_t d_ = c->D;
  CHECK_STRIDES(d->k_strides, 2, d->tokens, c->heads);
  CHECK_STRIDES(d->v_strides, 2, d->tokens, c->heads);
  if (static_cast<int64_t>(d->tokens) * c->heads >= (int64_t{1} << 30)) return COMFUSE_ERR_UNSUPPORTED;  // (rows, of keys and of values, are counted in 32 bits)
  return aligned(k, 16) && aligned(v, 16) && aligned(slots, 8) ? COMFUSE_OK : COMFUSE_ERR_ALIGNMENT;
}

// COMFUSE_ATTENTION_CLUSTER: CTAs of an item (1, 2, 4, 8, 16), 0 = equal shares and a second kernel; otherwise the sizes decide.
int forced_cluster() {
  static const int n = [] {
    const char* e = std::getenv("COMFUSE_ATTENTION_CLUSTER");
    const int v = e ? std::atoi(e) : -1;
    return v == 0 || v == 1 || v == 2 || v == 4 || v == 8 || v == 16 ? v : -1;
  }();
  return n;
}

// The longest sequence a call may meet, 0 where that is out of range.
int64_t longest(const comfuse_paged_attention_desc_t* d, const comfuse_kv_cache_t* c) {
  const int64_t room = static_cast<int64_t>(d->table_width) * c->page_size;
  const int64_t n = d->max_length > 0 && d->max_length < room ? d->max_length : room;
  return n <= 0x7FFFF000 ? n : 0;  // (positions are counted in 32 bits)
}
comfuse_status_t check_attention_sizes(const comfuse_paged_attention_desc_t* d, const comfuse_kv_cache_t* c) {
  if (!d || !c) return COMFUSE_ERR_INVALID_ARG;
  if (c->pages < 1 || c->heads < 1 || c->page_size < 1 || c->D < 1 || !type_16(c->dtype) || (c->quantized & ~1)) return COMFUSE_ERR_INVALID_ARG;
  if (d->batch < 1 || d->tokens < 1 || d->q_heads < 1 || d->table_width < 1 || d->max_length < 0 || d->window < 0 || d->q_heads % c->heads != 0) return COMFUSE_ERR_INVALID_ARG;
  if (!std::isfinite(d->alpha) || !std::isfinite(d->softcap) || d->softcap < 0.f) return COMFUSE_ERR_INVALID_ARG;
  if (c->D % (c->quantized ? 16 : 8) != 0) return COMFUSE_ERR_ALIGNMENT;
  if (c->D > 256 || c->page_size > 65536 || d->tokens > 64 || d->q_heads > 65536 || longest(d, c) == 0) return COMFUSE_ERR_UNSUPPORTED;
  if (static_cast<int64_t>(d->batch) * d->tokens * d->q_heads > 0x7FFFFFFF) return COMFUSE_ERR_UNSUPPORTED;  // (rows are counted in 32 bits)
  return COMFUSE_OK;
}
PagedAttentionPlan plan_of(const comfuse_paged_attention_desc_t* d, const comfuse_kv_cache_t* c) {
  return paged_attention_plan(d->batch, d->tokens * (d->q_heads / c->heads), c->heads, c->D, c->quantized != 0, static_cast<int>(longest(d, c)), d->window, d->tokens);
}
comfuse_status_t check_attention(const comfuse_paged_attention_desc_t* d, const comfuse_kv_cache_t* c, const void* q, const int32_t* table, const int32_t* lengths, const float* slopes,
                                 const void* out, const float* lse) {
  comfuse_status_t s = check_attention_sizes(d, c);
  if (s != COMFUSE_OK) return s;
  s = check_cache(c);
  if (s != COMFUSE_OK) return s;
  if (!q || !table || !lengths || !out || (d->batch > 1 && (d->table_stride < d->table_width || d->table_stride > kMostStride))) return COMFUSE_ERR_INVALID_ARG;
  const int64_t d_ = c->D;
  CHECK_STRIDES(d->q_strides, 2, d->batch, d->tokens, d->q_heads);
  CHECK_STRIDES(d->out_strides, 2, d->batch, d->tokens, d->q_heads);
  if (q == out && ((d->batch > 1 && d->q_strides[0] != d->out_strides[0]) || (d->tokens > 1 && d->q_strides[1] != d->out_strides[1]) || (d->q_heads > 1 && d->q_strides[2] != d->out_strides[2])))
    return COMFUSE_ERR_INVALID_ARG;
  return aligned(q, 16) && aligned(out, 16) && aligned(table, 4) && aligned(lengths, 4) && aligned(slopes, 4) && aligned(lse, 4) ? COMFUSE_OK : COMFUSE_ERR_ALIGNMENT;
}

void fill_rotary(const comfuse_rotary_t* r, RotaryWriteParams* p) {
  p->sign = 1.f;
  if (!r) return;
  p->positions = r->positions;
  p->freqs = r->freqs;
  p->axis_stride = r->axes > 1 ? r->axis_stride : 0;
  p->pairs = r->pairs;
  p->adjacent = r->adjacent;
  p->sign = r->inverse ? -1.f : 1.f;
  int end = 0;
  for (int i = 0; i < 4; ++i) p->section_end[i] = end += r->sections[i];
}
void fill_cache(const comfuse_kv_cache_t& c, CacheSide* k, CacheSide* v) {
  const int bytes = c.quantized ? 1 : 2;
  auto used = [](int64_t stride, int64_t size) { return size > 1 ? stride : 0; };  // (of a dimension of one element: anything)
  *k = {static_cast<char*>(c.k), c.k_scale, used(c.k_strides[0], c.pages) * bytes, used(c.k_strides[1], c.heads) * bytes, used(c.k_strides[2], c.page_size) * bytes, c.k_scale_strides[0], c.k_scale_strides[1], c.k_scale_strides[2]};
  *v = {static_cast<char*>(c.v), c.v_scale, used(c.v_strides[0], c.pages) * bytes, used(c.v_strides[1], c.heads) * bytes, used(c.v_strides[2], c.page_size) * bytes, c.v_scale_strides[0], c.v_scale_strides[1], c.v_scale_strides[2]};
}
RowsSide rows_side(const void* in, const int64_t* in_strides, void* out, const int64_t* out_strides, int bytes) {
  RowsSide r = {};
  r.in = static_cast<const char*>(in);
  r.out = static_cast<char*>(out);
  if (in_strides) r.in_token = in_strides[0] * bytes, r.in_head = in_strides[1] * bytes;
  if (out_strides) r.out_token = out_strides[0] * bytes, r.out_head = out_strides[1] * bytes;
  return r;
}
comfuse_status_t launched(cudaError_t e) { return e == cudaSuccess ? COMFUSE_OK : COMFUSE_ERR_CUDA; }

}  // namespace

// A CTA takes up to 64 query rows, more are further row blocks, which read the same keys a second time (from the L2).  There are as many CTAs as fit on the 148 SMs of the GPU, and never more than
// there may be units.
PagedAttentionPlan paged_attention_plan(int batch, int rows, int heads, int D, bool quantized, int max_length, int window, int tokens) {
  PagedAttentionPlan plan = {};
  const int DH = D <= 64 ? 64 : D <= 128 ? 128 : 256;
  plan.rows = rows <= 8 ? 8 : rows <= 16 ? 16 : rows <= 32 ? 32 : 64;
  plan.row_blocks = (rows + plan.rows - 1) / plan.rows;
  const paged::FormFacts f = quantized ? paged::facts<true>(D, plan.rows) : paged::facts<false>(D, plan.rows);
  int64_t seen = max_length;  // positions of a sequence that may be visible, from the block of the first on
  if (window > 0) seen = std::min<int64_t>(seen, static_cast<int64_t>(window) + tokens - 1 + f.block - 1);
  const int64_t units = std::max<int64_t>(1, (seen + f.unit - 1) / f.unit), cluster_units = std::max<int64_t>(1, (seen + f.cluster_unit - 1) / f.cluster_unit);
  const int64_t items = static_cast<int64_t>(batch) * heads * plan.row_blocks;
  if (items > 0x7FFFFFFF / (units + f.set_up)) return plan;  // (units are counted in 32 bits: no CTAs)
  const int64_t slots = 148 * f.ctas_per_sm;
  // Items by clusters, or equal shares and a second kernel?  By estimated times (us): a CTA's start and end, and a unit alone, as measured on one sequence of 100 .. 16000 positions (rows: 16, 8 bits;
  // D up to 64, 128, 256; columns: 8, 16, 32, 64 query rows); where CTAs share SMs a unit takes a quarter longer, where they take all of HBM its bytes at 6 TB/s.  A second kernel costs 2.9, a
  // cluster's joining 1.2; clusters of 8 and 16 leave some SMs idle, and clusters that do not fit at once are not taken.  Of a batch's lengths only the largest is known: 0.6 of it is
  // taken for the mean.  Over 300 calls of 1 .. 64 sequences of 100 .. 16000 positions, lengths spread below the longest, the choice is 1.4 % slower than the best of the six would be, in the geometric
  // mean; shares alone 15 %.  Over 120 calls of 2 .. 64 sequences of 200 .. 4000 positions it is 1.6 % slower, and where all are equally long 1.4 % (the worst 27 and 29 %); over 30 that see
  // windows of 512, 3.6 and 3.2 % (19 %).
  static constexpr float kStart[2][3][4] = {{{3.1f, 3.9f, 4.1f, 4.4f}, {3.1f, 4.6f, 5.7f, 7.4f}, {4.4f, 6.3f, 6.6f, 6.6f}}, {{4.4f, 6.3f, 6.5f, 6.7f}, {4.9f, 6.9f, 6.9f, 6.9f}, {5.4f, 8.3f, 8.0f, 10.7f}}};
  static constexpr float kUnit[2][3][4] = {{{0.79f, 0.97f, 1.27f, 1.39f}, {0.83f, 0.94f, 1.47f, 1.49f}, {1.08f, 1.22f, 1.57f, 1.90f}},
                                           {{0.85f, 1.07f, 1.36f, 1.35f}, {1.01f, 1.37f, 1.90f, 2.00f}, {0.95f, 1.58f, 2.01f, 2.12f}}};
  constexpr double kLaunch = 2.5;  // of the start: once, however many rounds of CTAs there are
  const int di = DH == 64 ? 0 : DH == 128 ? 1 : 2, ri = plan.rows == 8 ? 0 : plan.rows == 16 ? 1 : plan.rows == 32 ? 2 : 3;
  const double start = kStart[quantized][di][ri], unit = kUnit[quantized][di][ri], mean = batch > 1 ? 0.6 : 1.0;
  auto unit_us = [](double alone, int bytes, int64_t ctas) {
    const double n = static_cast<double>(ctas);
    return std::max(alone * (1.0 + 0.25 * std::max(0.0, n / 148 - 1.0)), bytes * n / 6e6);
  };
  // (three rings instead of two do half as much again in a third more time)
  const double share_unit = f.unit == f.cluster_unit ? unit : unit * 1.33;
  double best = start + 2.9 + std::max(1.0, static_cast<double>(items) * (static_cast<double>(units) * mean + 2 * f.set_up) / static_cast<double>(slots)) * unit_us(share_unit, f.unit_bytes, std::min(slots, items * units));
  for (int c = 1; c <= 16; c *= 2) {
    const int64_t ctas = items * c, fit = f.cluster_ctas_per_sm * (c == 16 ? 112 : c == 8 ? 120 : 148), rounds = (ctas + fit - 1) / fit;
    if ((c > 1 && (c > cluster_units || rounds > 1)) || ctas > 0x7FFFFFFF) break;
    const double each = static_cast<double>((cluster_units + c - 1) / c) * unit_us(unit, f.cluster_unit_bytes, std::min(ctas, fit)) * (rounds == 1 ? 1.0 : mean);
    const double us = kLaunch + static_cast<double>(rounds) * (start - kLaunch + each) + (c > 1 ? 1.2 : 0.0);
    if (us < best) plan.cluster = c, best = us;
  }
  if (forced_cluster() >= 0 && items * 16 <= 0x7FFFFFFF) plan.cluster = forced_cluster();
  if (plan.cluster > 0) {
    plan.ctas = static_cast<int>(items * plan.cluster);
    return plan;
  }
  plan.ctas = static_cast<int>(std::min<int64_t>(slots, items * (units + f.set_up)));
  plan.joined = units > 1 && plan.ctas > 1;
  plan.workspace = plan.joined ? static_cast<size_t>(plan.ctas) * paged::part_floats(plan.rows, DH) * sizeof(float) : 0;
  return plan;
}

cudaError_t launch_paged_attention(int dtype, bool quantized, const PagedAttentionPlan& plan, const PagedAttentionParams& p, cudaStream_t stream) {
  if (dtype == COMFUSE_DTYPE_BF16) return quantized ? paged::launch_bf16_q8(plan, p, stream) : paged::launch_bf16(plan, p, stream);
  return quantized ? paged::launch_f16_q8(plan, p, stream) : paged::launch_f16(plan, p, stream);
}

}  // namespace comfuse

using namespace comfuse;

extern "C" {

comfuse_status_t comfuse_rotary(const comfuse_rotary_desc_t* desc, const comfuse_rotary_t* rotary, const void* x, void* out, void* cuda_stream) {
  comfuse_status_t s = check_rotary_call(desc, rotary, x, out);
  if (s != COMFUSE_OK) return s;
  const DeviceInfo* dev = nullptr;
  s = check_device(&dev);
  if (s != COMFUSE_OK) return s;
  RotaryWriteParams p = {};
  p.tokens = desc->tokens; p.q_heads = desc->heads; p.D = desc->D;
  p.side[0] = rows_side(x, desc->x_strides, out, desc->out_strides, desc->dtype == COMFUSE_DTYPE_F32 ? 4 : 2);
  fill_rotary(rotary, &p);
  p.status = dev->status_word;
  return launched(launch_rotary_write(desc->dtype, false, false, p, *dev, static_cast<cudaStream_t>(cuda_stream)));
}

comfuse_status_t comfuse_cache_write(const comfuse_cache_write_desc_t* desc, const comfuse_kv_cache_t* cache, const comfuse_rotary_t* rotary, const void* k, const void* v, const void* q,
                                     void* q_out, const int64_t* slots, void* cuda_stream) {
  comfuse_status_t s = check_write(desc, cache, rotary, k, v, q, q_out, slots);
  if (s != COMFUSE_OK) return s;
  const DeviceInfo* dev = nullptr;
  s = check_device(&dev);
  if (s != COMFUSE_OK) return s;
  RotaryWriteParams p = {};
  p.tokens = desc->tokens; p.q_heads = desc->q_heads; p.kv_heads = cache->heads; p.D = cache->D;
  p.side[0] = rows_side(q, desc->q_strides, q_out, desc->q_out_strides, 2);
  p.side[1] = rows_side(k, desc->k_strides, nullptr, nullptr, 2);
  p.side[2] = rows_side(v, desc->v_strides, nullptr, nullptr, 2);
  fill_cache(*cache, &p.kc, &p.vc);
  p.slots = reinterpret_cast<const long long*>(slots);
  p.page_size = Divisor(cache->page_size);
  p.capacity = static_cast<long long>(cache->pages) * cache->page_size;
  fill_rotary(rotary, &p);
  p.status = dev->status_word;
  return launched(launch_rotary_write(cache->dtype, true, cache->quantized != 0, p, *dev, static_cast<cudaStream_t>(cuda_stream)));
}

comfuse_status_t comfuse_cache_read(const comfuse_cache_read_desc_t* desc, const comfuse_kv_cache_t* cache, const int64_t* slots, void* k, void* v, void* cuda_stream) {
  comfuse_status_t s = check_read(desc, cache, slots, k, v);
  if (s != COMFUSE_OK) return s;
  const DeviceInfo* dev = nullptr;
  s = check_device(&dev);
  if (s != COMFUSE_OK) return s;
  CacheReadParams p = {};
  p.tokens = desc->tokens; p.heads = cache->heads; p.D = cache->D;
  p.page_size = Divisor(cache->page_size);
  p.rows = Divisor(2 * cache->heads);
  fill_cache(*cache, &p.kc, &p.vc);
  p.k = rows_side(nullptr, nullptr, k, desc->k_strides, 2);
  p.v = rows_side(nullptr, nullptr, v, desc->v_strides, 2);
  p.slots = reinterpret_cast<const long long*>(slots);
  p.capacity = static_cast<long long>(cache->pages) * cache->page_size;
  p.status = dev->status_word;
  return launched(launch_cache_read(cache->dtype, cache->quantized != 0, p, *dev, static_cast<cudaStream_t>(cuda_stream)));
}

comfuse_status_t comfuse_paged_attention_workspace_size(const comfuse_paged_attention_desc_t* desc, const comfuse_kv_cache_t* cache, size_t* bytes) {
  if (!bytes) return COMFUSE_ERR_INVALID_ARG;
  const comfuse_status_t s = check_attention_sizes(desc, cache);
  if (s != COMFUSE_OK) return s;
  const PagedAttentionPlan plan = plan_of(desc, cache);
  if (plan.ctas == 0) return COMFUSE_ERR_UNSUPPORTED;
  *bytes = plan.workspace;
  return COMFUSE_OK;
}

comfuse_status_t comfuse_paged_attention(const comfuse_paged_attention_desc_t* desc, const comfuse_kv_cache_t* cache, const void* q, const int32_t* table, const int32_t* lengths,
                                         const float* slopes, void* out, float* lse, void* workspace, size_t workspace_bytes, void* cuda_stream) {
  comfuse_status_t s = check_attention(desc, cache, q, table, lengths, slopes, out, lse);
  if (s != COMFUSE_OK) return s;
  const PagedAttentionPlan plan = plan_of(desc, cache);
  if (plan.ctas == 0) return COMFUSE_ERR_UNSUPPORTED;
  if (plan.workspace > 0) {
    if (!workspace || workspace_bytes < plan.workspace) return COMFUSE_ERR_WORKSPACE;
    if (!aligned(workspace, 16)) return COMFUSE_ERR_ALIGNMENT;
  }
  const DeviceInfo* dev = nullptr;
  s = check_device(&dev);
  if (s != COMFUSE_OK) return s;
  const comfuse_paged_attention_desc_t& d = *desc;
  PagedAttentionParams p = {};
  p.batch = d.batch; p.tokens = d.tokens; p.heads = cache->heads; p.group = d.q_heads / cache->heads; p.D = cache->D;
  p.rows = d.tokens * p.group;
  p.row_blocks = plan.row_blocks;
  p.pages = cache->pages; p.page_size = Divisor(cache->page_size);
  p.max_length = static_cast<int>(longest(desc, cache));
  p.window = d.window < p.max_length + d.tokens ? d.window : 0;  // (one that hides nothing)
  p.q = static_cast<const char*>(q);
  p.out = static_cast<char*>(out);
  p.q_batch = 2 * d.q_strides[0]; p.q_token = 2 * d.q_strides[1]; p.q_head = 2 * d.q_strides[2];
  p.out_batch = 2 * d.out_strides[0]; p.out_token = 2 * d.out_strides[1]; p.out_head = 2 * d.out_strides[2];
  fill_cache(*cache, &p.kc, &p.vc);
  p.table = table; p.table_stride = d.table_stride; p.lengths = lengths;
  p.slopes = slopes; p.lse = lse;
  p.alpha = d.alpha; p.alpha_log2 = d.alpha * paged::kLog2e;
  p.cap = std::min(d.softcap * paged::kLog2e, FLT_MAX);  // (caps near the largest number and below the normal ones stay finite)
  p.per_cap = p.cap > 0.f ? std::min(1.f / p.cap, FLT_MAX) : 0.f;
  p.part = static_cast<float*>(workspace);
  p.ctas = plan.ctas;
  p.cluster = plan.cluster;
  p.groups = Divisor(p.group);
  p.shares = Divisor(plan.ctas);
  p.status = dev->status_word;
  return launched(launch_paged_attention(cache->dtype, cache->quantized != 0, plan, p, static_cast<cudaStream_t>(cuda_stream)));
}

}  // extern "C"
