// Block norms with rows in registers: an fp32 stream and bf16 activations, rows on 16-byte boundaries.
#include "block_rows.cuh"

namespace ceca {

cudaError_t block_rows_mixed(const BlockArgs &p, bool grad, cudaStream_t s) { return launch_rows<4, DSGD_F32, DSGD_BF16>(p, grad, s); }

}  // namespace ceca
