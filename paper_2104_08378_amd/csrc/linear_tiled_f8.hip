// Layers on the tiled kernels, f8 inputs.
#include "linear_tiled.hpp"

namespace sp24 {

template sp24_status layer_tiled<SP24_F8>(const LinearArgs& a, LayerTile tile, hipStream_t st);

} // namespace sp24
