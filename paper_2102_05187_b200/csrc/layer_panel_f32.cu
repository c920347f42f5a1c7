// The few-columns form of the layer products for f32 values (layer_panel.cuh).
#include "layer_panel.cuh"

namespace comet {
template comet_status_t layer_panel_typed<float>(Context *, const GatherCall &, cudaStream_t);
}  // namespace comet
