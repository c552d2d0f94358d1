// The attention kernel of few rows for masks among the newest tokens.
#include "pdkv_attend_warp.cuh"

namespace pdkv {

cudaError_t launch_attend_masked(const AttnParams &p, const void *map, int dtype, cudaStream_t stream) { return launch_warp_kernel<kMasked>(p, map, dtype, stream); }

}  // namespace pdkv
