// Block norms with rows in registers: an fp32 stream and bf16 activations, rows on any boundary; the types that no other has.
#include "block_rows.cuh"

namespace ceca {

cudaError_t block_odd_rows_mixed(const BlockArgs &p, bool grad, cudaStream_t s) { return launch_rows<1, DSGD_F32, DSGD_BF16>(p, grad, s); }
cudaError_t block_odd_rows_any(const BlockArgs &p, bool grad, cudaStream_t s) { return launch_rows<1, kAnyType, kAnyType>(p, grad, s); }

}  // namespace ceca
