// The kernel of fluxbin_kv_tree.cuh for head dimension 256.
#include "fluxbin_kv_tree.cuh"

cudaError_t fbd::launch_tree_256(const AttendArgs &a, bool bf16, cudaStream_t s) { return run_tree_of<256>(a, bf16, s); }
