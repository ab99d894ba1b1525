// Layers on the tiled and the staged kernels, f16 inputs.
#include "linear_tiled.hpp"

namespace sp24 {

template sp24_status layer_tiled<SP24_F16>(const LinearArgs& a, LayerTile tile, hipStream_t st);
template sp24_status layer_staged<SP24_F16>(const LinearArgs& a, hipStream_t st);

} // namespace sp24
