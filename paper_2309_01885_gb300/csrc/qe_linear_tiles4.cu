// Many-rows products with codes held in 4 bits.
#include "qe_linear_tiles.cuh"

namespace qe {

cudaError_t launch_linear_tiles_4(const LinearArgs &a, cudaStream_t s) { return launch_tiles_bits<4>(a, s); }

}  // namespace qe
