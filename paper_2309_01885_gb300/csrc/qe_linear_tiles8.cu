// Many-rows products with codes held in 8 bits.
#include "qe_linear_tiles.cuh"

namespace qe {

cudaError_t launch_linear_tiles_8(const LinearArgs &a, cudaStream_t s) { return launch_tiles_bits<8>(a, s); }

}  // namespace qe
