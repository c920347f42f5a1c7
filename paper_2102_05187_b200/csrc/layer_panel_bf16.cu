// The few-columns form of the layer products for bf16 values (layer_panel.cuh).
#include "layer_panel.cuh"

namespace comet {
template comet_status_t layer_panel_typed<__nv_bfloat16>(Context *, const GatherCall &, cudaStream_t);
}  // namespace comet
