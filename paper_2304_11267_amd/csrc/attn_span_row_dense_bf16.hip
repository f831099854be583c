// attn_span_row_dense_bf16.hip -- instantiations of attn_span_row.h: bf16, 16-bit keys and values.
#include "attn_span_row.h"

namespace sdattn {

hipError_t launch_span_row_dense_bf16(const SpanKernel& a, hipStream_t stream) {
    return span_row_dispatch<kBF16, false>(a, stream, SpanRowWidths{});
}

}  // namespace sdattn
