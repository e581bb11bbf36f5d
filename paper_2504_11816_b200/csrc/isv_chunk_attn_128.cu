// The chunk attention's kernels for head_dim 128.
#include "isv_chunk_attn.cuh"

namespace isv {
namespace chunk {
template cudaError_t attn_configure<128>(bool bf16);
template cudaError_t launch_attn<128>(const AttnParams &p, bool bf16, int grid, cudaStream_t st, const char **what);
}  // namespace chunk
}  // namespace isv
