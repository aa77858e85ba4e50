// paged_attention.hip — attention over the pages of a cache, also of trees of drafted
// tokens (attention.hpp has the kernels).
#include "attention.hpp"

namespace mezo {

hipError_t launch_paged_attention(const PagedArgs& args, hipStream_t stream) { return launch_any(args, stream); }

}  // namespace mezo
