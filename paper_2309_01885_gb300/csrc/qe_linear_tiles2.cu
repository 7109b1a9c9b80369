// Many-rows products with codes held in 2 bits.
#include "qe_linear_tiles.cuh"

namespace qe {

cudaError_t launch_linear_tiles_2(const LinearArgs &a, cudaStream_t s) { return launch_tiles_bits<2>(a, s); }

}  // namespace qe
