// attn_cross.hip -- the attention kernel over an encoder's key and value rows.
#include "attention.hpp"

namespace mnmt {
template hipError_t launch_attn_kernel<false>(const AttnArgs&, int, hipStream_t);
}  // namespace mnmt
