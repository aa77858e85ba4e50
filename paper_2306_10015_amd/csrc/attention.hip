// attention.hip — attention over the keys and values of packed documents or of their
// caches, contiguous in memory (attention.hpp has the kernels).
#include "attention.hpp"

namespace mezo {

hipError_t launch_attention(const AttentionArgs& args, hipStream_t stream) { return launch_any(args, stream); }

}  // namespace mezo
