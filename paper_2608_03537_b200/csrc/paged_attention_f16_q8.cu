// Instances of the paged attention: f16 queries over a cache of 8-bit values.
#include "paged_attention.cuh"

namespace comfuse {
namespace paged {

cudaError_t launch_f16_q8(const PagedAttentionPlan& plan, const PagedAttentionParams& p, cudaStream_t stream) { return launch_type<COMFUSE_DTYPE_F16, true>(plan, p, stream); }

}  // namespace paged
}  // namespace comfuse
