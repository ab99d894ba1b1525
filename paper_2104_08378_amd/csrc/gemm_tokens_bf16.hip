// The weights' gradient from tokens' rows of type SP24_BF16.
#include "gemm_tokens.hpp"

namespace sp24 {

template sp24_status gemm_tokens<SP24_BF16, SP24_F32>(const TokenArgs&, int, hipStream_t);
template sp24_status gemm_tokens<SP24_BF16, SP24_BF16>(const TokenArgs&, int, hipStream_t);

} // namespace sp24
