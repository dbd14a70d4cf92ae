// The sparse decode kernel over 3-bit pages.
#include "sparse_kernel.cuh"

namespace wushkv {
int launch_sparse_3bit(const SparseParams& P, cudaStream_t st) { return launch_sparse<3>(P, st); }
}  // namespace wushkv
