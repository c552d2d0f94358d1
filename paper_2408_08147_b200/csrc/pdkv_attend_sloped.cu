// The attention kernel of few rows for scores biased by distance, capped or not.
#include "pdkv_attend_warp.cuh"

namespace pdkv {

cudaError_t launch_attend_sloped(const AttnParams &p, const void *map, int dtype, cudaStream_t stream) { return launch_warp_kernel<kSloped>(p, map, dtype, stream); }

}  // namespace pdkv
