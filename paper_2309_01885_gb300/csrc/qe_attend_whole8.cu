// The few-rows attention kernel with a CTA of eight warps for each item, for short contexts:
// compiled apart from the other forms so that none holds up the build.
#include "qe_attend_rows.cuh"

namespace qe {

cudaError_t launch_attend_whole8(const AttendArgs &a, int tiles, cudaStream_t s) {
    return launch_rows_any<8, true>(a, tiles, s);
}

}  // namespace qe
