// attn_span_dense_f16.hip -- instantiations of attn_span.h: fp16, 16-bit keys and values.
#include "attn_span.h"

namespace sdattn {

hipError_t launch_span_dense_f16(const SpanArgs& s) { return span_launch<kF16, false>(s); }

}  // namespace sdattn
