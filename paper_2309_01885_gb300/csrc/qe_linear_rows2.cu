// Few-rows products with codes held in 2 bits.
#include "qe_linear_rows.cuh"

namespace qe {

cudaError_t launch_linear_rows_2(const LinearArgs &a, cudaStream_t s) { return launch_rows_bits<2>(a, s); }

}  // namespace qe
