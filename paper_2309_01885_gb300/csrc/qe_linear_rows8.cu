// Few-rows products with codes held in 8 bits.
#include "qe_linear_rows.cuh"

namespace qe {

cudaError_t launch_linear_rows_8(const LinearArgs &a, cudaStream_t s) { return launch_rows_bits<8>(a, s); }

}  // namespace qe
