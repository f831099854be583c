// attn_span.hip -- how a call of attn_span.h is cut up, its entry point, and the join of the
// parts of its keys.
#include "attn_geom.h"
#include "attn_span_seq.h"

namespace sdattn {

namespace {

// 8 values of a row a thread: O = sum_s 2^(m_s - M) O_s / sum_s 2^(m_s - M) l_s, in the order of
// the splits.  A split without keys has l = 0, and its O is not written.
template <int ET>
__global__ __launch_bounds__(256) void span_join_kernel(const SpanKernel a) {
    const int pieces = a.D / 8;
    const long long R = (long long)a.Lq * a.G, rows = a.B * (long long)a.Hk * R;
    const long long id = (long long)blockIdx.x * 256 + threadIdx.x;
    const long long at = id / pieces;
    if (at >= rows) return;
    const int d = (int)(id - at * pieces) * 8;
    const long long bh = at / R;
    const int row = (int)(at - bh * R), b = (int)(bh / a.Hk), hk = (int)(bh - (long long)b * a.Hk);
    const int token = row / a.G, head = hk * a.G + row % a.G;
    if (token >= span_seq(a, b).count) return;
    const float* const ml = a.part + (size_t)a.splits * rows * a.D + at * 2;
    float top = kSpanNone;
    for (int s = 0; s < a.splits; ++s)
        if (ml[s * rows * 2 + 1] != 0.0f) top = fmaxf(top, ml[s * rows * 2]);
    float sum = 0.0f, o[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = 0.0f;
    for (int s = 0; s < a.splits; ++s) {
        const float ls = ml[s * rows * 2 + 1];
        if (ls == 0.0f) continue;
        const float w = fast_exp2(ml[s * rows * 2] - top);
        const float* const p = a.part + ((size_t)s * rows + at) * a.D + d;
        const f32x4 x = *(const f32x4*)p, y = *(const f32x4*)(p + 4);
        sum = fmaf(w, ls, sum);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = fmaf(w, x[e], o[e]), o[4 + e] = fmaf(w, y[e], o[4 + e]);
    }
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    *(u32x4*)(a.out + b * a.ob + head * a.oh + token * a.ol + d) =
        u32x4{pack2<ET>(o[0] * inv, o[1] * inv), pack2<ET>(o[2] * inv, o[3] * inv), pack2<ET>(o[4] * inv, o[5] * inv),
              pack2<ET>(o[6] * inv, o[7] * inv)};
}

}  // namespace

static hipError_t launch_span_join(const SpanKernel& a, int type, hipStream_t stream) {
    const long long threads = (long long)a.B * a.Hk * a.Lq * a.G * (a.D / 8);
    if (!grid_fits((threads + 255) / 256, 256)) return kGridTooLarge;
    auto k = type == kF16 ? span_join_kernel<kF16> : span_join_kernel<kBF16>;
    hipLaunchKernelGGL(k, dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, stream, a);
    return hipGetLastError();
}

SpanPlan span_plan(const SpanArgs& a) {
    SpanPlan p{};
    const int G = a.H / a.Hk;
    const long long rows = (long long)a.Lq * G;
    p.single = rows <= kSpanRows;
    const long long heads = (long long)a.B * a.Hk;
    const int block = p.single ? kSpanRows : a.D > kSpanNarrow ? 256 : 128, tile = p.single ? 32 : 64;
    p.row_blocks = (int)((rows + block - 1) / block);
    const long long wgs = heads * p.row_blocks;
    // the most tiles that a block can see
    long long tiles = ((long long)a.Lk + tile - 1) / tile;
    if (a.window > 0) {
        const long long spread = (long long)block / G + a.frame;   // of the block's hi
        const long long seen = ((long long)a.sinks + tile - 1) / tile + ((long long)a.window + spread) / tile + 2;
        if (seen < tiles) tiles = seen;
    }
    // workgroups that the card holds at once
    const long long most = tiles / (p.single ? 16 : 8), room = p.single ? 1024 : a.D > kSpanNarrow ? kCus : 2 * kCus;
    p.splits = (int)(room / wgs < most ? room / wgs : most);
    if (p.splits < 1) p.splits = 1;
    if (p.splits > 1) {
        const __int128 bytes = (__int128)p.splits * a.B * a.Hk * rows * (a.D + 2) * 4;
        p.workspace = bytes < ((__int128)1 << 62) ? (long long)bytes : -1;
    }
    return p;
}

hipError_t launch_span(const SpanArgs& s) {
    const SpanPlan p = span_plan(s);
    SpanKernel a{};
    a.q = (const uint16_t*)s.q, a.out = (uint16_t*)s.out;
    a.k = (const char*)s.k, a.v = (const char*)s.v;
    a.ks = s.k_scales, a.vs = s.v_scales, a.table = s.table, a.starts = s.starts, a.counts = s.counts;
    a.part = (float*)s.workspace;
    auto strides = [](bool heads, int H, int L, int D, long long* sb, long long* sh, long long* sl) {
        *sb = (long long)H * L * D;
        *sh = heads ? (long long)L * D : D;
        *sl = heads ? D : (long long)H * D;
    };
    strides(s.x_heads, s.H, s.Lq, s.D, &a.qb, &a.qh, &a.ql);
    strides(s.y_heads, s.H, s.Lq, s.D, &a.ob, &a.oh, &a.ol);
    strides(s.x_heads, s.Hk, s.Lk, s.D, &a.kb, &a.kh, &a.kl);
    a.B = s.B, a.Hk = s.Hk, a.G = s.H / s.Hk, a.Lq = s.Lq, a.Lk = s.Lk, a.D = s.D;
    a.pages = s.pages, a.slots = s.slots;
    a.frame = s.frame, a.window = s.window, a.sinks = s.sinks;
    a.row_blocks = p.row_blocks, a.splits = p.splits;
    a.zero = s.scale == 0.0f, a.neg = s.scale < 0;
    a.c = a.zero ? 1.0f : (a.neg ? -s.scale : s.scale) * kLog2e;
    const hipStream_t stream = (hipStream_t)s.stream;
    const bool f16 = s.dtype == kF16;
    hipError_t r;
    if (p.single)
        r = s.table ? (f16 ? launch_span_row_paged_f16(a, stream) : launch_span_row_paged_bf16(a, stream))
                    : (f16 ? launch_span_row_dense_f16(a, stream) : launch_span_row_dense_bf16(a, stream));
    else
        r = s.table ? (f16 ? launch_span_paged_f16(a, stream) : launch_span_paged_bf16(a, stream))
                    : (f16 ? launch_span_dense_f16(a, stream) : launch_span_dense_bf16(a, stream));
    if (r == hipSuccess && p.splits > 1) r = launch_span_join(a, s.dtype, stream);
    return r;
}

}  // namespace sdattn
