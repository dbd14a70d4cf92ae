// The sparse decode kernel over 4-bit pages.
#include "sparse_kernel.cuh"

namespace wushkv {
int launch_sparse_4bit(const SparseParams& P, cudaStream_t st) { return launch_sparse<4>(P, st); }
}  // namespace wushkv
