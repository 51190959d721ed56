// The kernel of fluxbin_kv_tree.cuh for head dimension 64.
#include "fluxbin_kv_tree.cuh"

cudaError_t fbd::launch_tree_64(const AttendArgs &a, bool bf16, cudaStream_t s) { return run_tree_of<64>(a, bf16, s); }
