// Block norms with rows in registers: any types, rows on any boundary.
#include "block_rows.cuh"

namespace ceca {

cudaError_t block_rows_any(const BlockArgs &p, bool grad, cudaStream_t s) { return launch_rows<1, kAnyType, kAnyType>(p, grad, s); }

}  // namespace ceca
