// The attention kernel of few rows for capped scores.
#include "pdkv_attend_warp.cuh"

namespace pdkv {

cudaError_t launch_attend_capped(const AttnParams &p, const void *map, int dtype, cudaStream_t stream) { return launch_warp_kernel<kCapped>(p, map, dtype, stream); }

}  // namespace pdkv
