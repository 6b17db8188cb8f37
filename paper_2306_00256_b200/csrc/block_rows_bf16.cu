// Block norms with rows in registers: bf16 throughout, rows on 16-byte boundaries.
#include "block_rows.cuh"

namespace ceca {

cudaError_t block_rows_bf16(const BlockArgs &p, bool grad, cudaStream_t s) { return launch_rows<8, DSGD_BF16, DSGD_BF16>(p, grad, s); }

}  // namespace ceca
