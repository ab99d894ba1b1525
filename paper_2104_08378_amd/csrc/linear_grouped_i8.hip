// Rows of experts on the tiled and the staged kernels, i8 inputs.
#include "linear_tiled.hpp"

namespace sp24 {

template sp24_status layer_tiled<SP24_I8>(const GroupedArgs& a, LayerTile tile, hipStream_t st);
template sp24_status layer_staged<SP24_I8>(const GroupedArgs& a, hipStream_t st);

} // namespace sp24
