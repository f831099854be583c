// attn_span_dense_bf16.hip -- instantiations of attn_span.h: bf16, 16-bit keys and values.
#include "attn_span.h"

namespace sdattn {

hipError_t launch_span_dense_bf16(const SpanKernel& a, hipStream_t stream) {
    return span_dispatch<kBF16, false>(a, stream, SpanWidths{});
}

}  // namespace sdattn
