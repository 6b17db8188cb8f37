// Block norms with rows in registers: fp32 throughout, rows on 16-byte boundaries.
#include "block_rows.cuh"

namespace ceca {

cudaError_t block_rows_f32(const BlockArgs &p, bool grad, cudaStream_t s) { return launch_rows<4, DSGD_F32, DSGD_F32>(p, grad, s); }

}  // namespace ceca
