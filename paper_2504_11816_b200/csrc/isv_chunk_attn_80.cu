// The chunk attention's kernels for head_dim 80.
#include "isv_chunk_attn.cuh"

namespace isv {
namespace chunk {
template cudaError_t attn_configure<80>(bool bf16);
template cudaError_t launch_attn<80>(const AttnParams &p, bool bf16, int grid, cudaStream_t st, const char **what);
}  // namespace chunk
}  // namespace isv
