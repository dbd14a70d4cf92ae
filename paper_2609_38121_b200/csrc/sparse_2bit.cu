// The sparse decode kernel over 2-bit pages.
#include "sparse_kernel.cuh"

namespace wushkv {
int launch_sparse_2bit(const SparseParams& P, cudaStream_t st) { return launch_sparse<2>(P, st); }
}  // namespace wushkv
