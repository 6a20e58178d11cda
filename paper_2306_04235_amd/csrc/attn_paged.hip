// attn_paged.hip -- the attention kernel over the pages of a cache.
#include "attention.hpp"

namespace mnmt {
template hipError_t launch_attn_kernel<true>(const AttnArgs&, int, hipStream_t);
}  // namespace mnmt
