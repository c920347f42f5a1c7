// The gather form of the layer products for f16 values (layer_gather.cuh): a unit per type, so that they compile side by side.
#include "layer_gather.cuh"

namespace comet {
template comet_status_t layer_gather_typed<__half>(Context *, const GatherCall &, cudaStream_t);
}  // namespace comet
