// attn_span_row_paged_bf16.hip -- instantiations of attn_span_row.h: bf16, 8-bit pages.
#include "attn_span_row.h"

namespace sdattn {

hipError_t launch_span_row_paged_bf16(const SpanKernel& a, hipStream_t stream) {
    return span_row_dispatch<kBF16, true>(a, stream, SpanRowWidths{});
}

}  // namespace sdattn
