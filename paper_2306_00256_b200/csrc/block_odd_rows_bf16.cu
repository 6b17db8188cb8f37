// Block norms with rows in registers: bf16 throughout, rows on any boundary.
#include "block_rows.cuh"

namespace ceca {

cudaError_t block_odd_rows_bf16(const BlockArgs &p, bool grad, cudaStream_t s) { return launch_rows<1, DSGD_BF16, DSGD_BF16>(p, grad, s); }

}  // namespace ceca
