// The gather form of the layer products for bf16 values (layer_gather.cuh): a unit per type, so that they compile side by side.
#include "layer_gather.cuh"

namespace comet {
template comet_status_t layer_gather_typed<__nv_bfloat16>(Context *, const GatherCall &, cudaStream_t);
}  // namespace comet
