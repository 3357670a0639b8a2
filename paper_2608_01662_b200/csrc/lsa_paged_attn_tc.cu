#include "lsa_paged.cuh"
namespace lsa {
cudaError_t launch_paged_attn_tc(const PagedAttnArgs&, cudaStream_t, int64_t*) { return cudaErrorNotSupported; }
}
