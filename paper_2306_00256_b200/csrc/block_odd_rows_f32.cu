// Block norms with rows in registers: fp32 throughout, rows on any boundary.
#include "block_rows.cuh"

namespace ceca {

cudaError_t block_odd_rows_f32(const BlockArgs &p, bool grad, cudaStream_t s) { return launch_rows<1, DSGD_F32, DSGD_F32>(p, grad, s); }

}  // namespace ceca
