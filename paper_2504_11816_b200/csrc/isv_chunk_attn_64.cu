// The chunk attention's kernels for head_dim 64.
#include "isv_chunk_attn.cuh"

namespace isv {
namespace chunk {
template cudaError_t attn_configure<64>(bool bf16);
template cudaError_t launch_attn<64>(const AttnParams &p, bool bf16, int grid, cudaStream_t st, const char **what);
}  // namespace chunk
}  // namespace isv
