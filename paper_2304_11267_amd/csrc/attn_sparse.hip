// attn_sparse.hip -- entry point of the attention over selected key blocks and its
// fp16 instantiations; the kernel is in attn_fwd_kernel.h, its use in attn_sparse.h.
#include "attn_sparse.h"

namespace sdattn {

hipError_t launch_attn_sparse(const SparseArgs& a) {
    if (a.Lq == 1) return launch_attn_sparse_row(a);
    return a.dtype == kF16 ? dispatch_sparse<kF16>(a, SparseWidths{}) : launch_attn_sparse_bf16(a);
}

}  // namespace sdattn
