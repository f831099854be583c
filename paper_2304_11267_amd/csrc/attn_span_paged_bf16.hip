// attn_span_paged_bf16.hip -- instantiations of attn_span.h: bf16, 8-bit pages.
#include "attn_span.h"

namespace sdattn {

hipError_t launch_span_paged_bf16(const SpanKernel& a, hipStream_t stream) {
    return span_dispatch<kBF16, true>(a, stream, SpanWidths{});
}

}  // namespace sdattn
