// attn_span_paged_f16.hip -- instantiations of attn_span.h: fp16, 8-bit pages.
#include "attn_span.h"

namespace sdattn {

hipError_t launch_span_paged_f16(const SpanKernel& a, hipStream_t stream) {
    return span_dispatch<kF16, true>(a, stream, SpanWidths{});
}

}  // namespace sdattn
