// attn_sparse_bf16.hip -- bf16 instantiations of the attention over selected key
// blocks (attn_sparse.h).
#include "attn_sparse.h"

namespace sdattn {

hipError_t launch_attn_sparse_bf16(const SparseArgs& a) { return dispatch_sparse<kBF16>(a, SparseWidths{}); }

}  // namespace sdattn
