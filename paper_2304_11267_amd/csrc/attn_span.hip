// attn_span.hip -- how a call of attn_span.h is cut up, its entry point, and the join of the
// parts of its keys.
#include <cmath>

#include "attn_geom.h"
#include "attn_span_seq.h"

namespace sdattn {

namespace {

// O = sum_s 2^(m_s - M) O_s / sum_s 2^(m_s - M) l_s for a row of part s's sums O_s, l_s and reference m_s, always
// in the same order.  A part without keys has l = 0.
struct SpanJoin {
    const float* part;   // of a row: O_s
    const float* ml;
    uint16_t* out;
    size_t apart;        // rows from one part to the next
    bool live;
};
__device__ __forceinline__ SpanJoin span_join_row(const SpanKernel& a, long long at) {
    const int R = a.Lq * a.G;
    const size_t rows = (size_t)a.B * a.Hk * R;
    const int bh = (int)(at / R), row = (int)(at - (long long)bh * R), b = bh / a.Hk, hk = bh - b * a.Hk;
    const int token = row / a.G, head = hk * a.G + row - token * a.G;
    return SpanJoin{a.part + at * a.D, a.part + a.splits * rows * a.D + at * 2,
                    a.out + b * a.ob + head * a.oh + token * a.ol, rows, token < span_seq(a, b).count};
}
template <int ET>
__device__ __forceinline__ void span_join_store(uint16_t* out, const float* o, float sum) {
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    *(u32x4*)out = u32x4{pack2<ET>(o[0] * inv, o[1] * inv), pack2<ET>(o[2] * inv, o[3] * inv),
                         pack2<ET>(o[4] * inv, o[5] * inv), pack2<ET>(o[6] * inv, o[7] * inv)};
}

// Many rows and two or three parts: 8 values of a row a thread.  Bound by memory: 21600 rows of 128 in two parts 7.6 us,
// 3.6 TB/s.
template <int ET>
__global__ __launch_bounds__(256) void span_join_kernel(const SpanKernel a) {
    const int pieces = a.D / 8;
    const long long id = (long long)blockIdx.x * 256 + threadIdx.x, at = id / pieces;
    if (at >= (long long)a.B * a.Hk * a.Lq * a.G) return;
    const int d = (int)(id - at * pieces) * 8;
    const SpanJoin r = span_join_row(a, at);
    if (!r.live) return;
    float top = kSpanNone, sum = 0.0f, o[8];
    for (int s = 0; s < a.splits; ++s)
        if (r.ml[s * r.apart * 2 + 1] != 0.0f) top = fmaxf(top, r.ml[s * r.apart * 2]);
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = 0.0f;
#pragma unroll 2
    for (int s = 0; s < a.splits; ++s) {
        const float l = r.ml[s * r.apart * 2 + 1], w = l == 0.0f ? 0.0f : fast_exp2(r.ml[s * r.apart * 2] - top);
        const float* const p = r.part + s * r.apart * a.D + d;
        const f32x4 x = *(const f32x4*)p, y = *(const f32x4*)(p + 4);
        sum = fmaf(w, l, sum);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = fmaf(w, x[e], o[e]), o[4 + e] = fmaf(w, y[e], o[4 + e]);
    }
    span_join_store<ET>(r.out + d, o, sum);
}

// Few rows and many parts: a wave for a row's 64 values from 64 blockIdx.y on, 8 of them a lane, every eighth part,
// all of them on their way at once: 256 rows of 128 in four parts 4.7 us, a launch's latency.  (64 parts and more: in
// runs.)
template <int ET>
__global__ __launch_bounds__(64) void span_join_wide_kernel(const SpanKernel a) {
    constexpr int kRun = 64;
    const int lane = lane_id(), g = lane >> 3, d = blockIdx.y * 64 + (lane & 7) * 8;
    const SpanJoin r = span_join_row(a, blockIdx.x);
    if (!r.live) return;
    const bool in = d < a.D;
    float m = kSpanNone, sum = 0.0f, o[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = 0.0f;
    for (int s0 = 0; s0 < a.splits; s0 += kRun) {
        const int s = s0 + lane;
        float ms = kSpanNone, ls = 0.0f;
        if (s < a.splits) ms = r.ml[s * r.apart * 2], ls = r.ml[s * r.apart * 2 + 1];
        f32x4 x[kRun / 8][2];
#pragma unroll
        for (int i = 0; i < kRun / 8; ++i) {
            const int p = s0 + 8 * i + g;
            x[i][0] = x[i][1] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
            if (p < a.splits && in) {
                const float* const q = r.part + p * r.apart * a.D + d;
                x[i][0] = *(const f32x4*)q;
                x[i][1] = *(const f32x4*)(q + 4);
            }
        }
        float top = fmaxf(m, ls == 0.0f ? kSpanNone : ms);
#pragma unroll
        for (int k = 1; k < 64; k <<= 1) top = fmaxf(top, __shfl_xor(top, k, 64));
        const float w = ls == 0.0f ? 0.0f : fast_exp2(ms - top), before = fast_exp2(m - top);
        m = top;
        float part = w * ls;
#pragma unroll
        for (int k = 1; k < 64; k <<= 1) part += __shfl_xor(part, k, 64);
        sum = fmaf(sum, before, part);
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] *= before;
#pragma unroll
        for (int i = 0; i < kRun / 8; ++i) {
            const float f = __shfl(w, 8 * i + g, 64);
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = fmaf(f, x[i][0][e], o[e]), o[4 + e] = fmaf(f, x[i][1][e], o[4 + e]);
        }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
#pragma unroll
        for (int k = 8; k < 64; k <<= 1) o[e] += __shfl_xor(o[e], k, 64);
    if (g == 0 && in) span_join_store<ET>(r.out + d, o, sum);
}

}  // namespace

static hipError_t launch_span_join(const SpanKernel& a, int type, hipStream_t stream) {
    const long long rows = (long long)a.B * a.Hk * a.Lq * a.G;
    if (a.splits > 3) {
        const int blocks = (a.D + 63) / 64;
        if (!grid_fits(rows * blocks, 64)) return kGridTooLarge;
        auto k = type == kF16 ? span_join_wide_kernel<kF16> : span_join_wide_kernel<kBF16>;
        hipLaunchKernelGGL(k, dim3((unsigned)rows, (unsigned)blocks), dim3(64), 0, stream, a);
        return hipGetLastError();
    }
    const long long threads = rows * (a.D / 8);
    if (!grid_fits((threads + 255) / 256, 256)) return kGridTooLarge;
    auto k = type == kF16 ? span_join_kernel<kF16> : span_join_kernel<kBF16>;
    hipLaunchKernelGGL(k, dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, stream, a);
    return hipGetLastError();
}

// A way to cut a call up, and the time that it is taken for, in us.
struct SpanWay {
    int row_blocks, splits;
    long long tiles;   // the most that a block can see
    double time;
};

// By the time of a part's tiles one after another and of the join: 4.5 us for its launch, and each part's rows through
// memory.  A tile's time, in us: for few rows its bytes at what one CU reads alone, 50 KB a us, and 0.12 at least; else
// what a workgroup of few takes (paged, D = 128 1.6 to 2.3; 16-bit, D = 128 / 64 / 40 1.3 / 0.94 / 0.8),
// or 1.6 times that where two share a CU.
static SpanWay span_way(const SpanArgs& a, bool single) {
    const int G = a.H / a.Hk;
    const long long rows = (long long)a.Lq * G, heads = (long long)a.B * a.Hk;
    const int block = single ? kSpanRows : span_block((a.D + 15) / 16 * 16, a.slots > 0), tile = single ? 32 : 64;
    SpanWay w{(int)((rows + block - 1) / block), 1, 0, 0.0};
    const long long wgs = heads * w.row_blocks;
    // the most tiles that a block can see
    long long tiles = ((long long)a.Lk + tile - 1) / tile;
    if (a.window > 0) {
        const long long spread = (long long)block / G + a.frame;   // of the block's hi
        const long long seen = ((long long)a.sinks + tile - 1) / tile + ((long long)a.window + spread) / tile + 2;
        if (seen < tiles) tiles = seen;
    }
    w.tiles = tiles;
    const double cost = single ? fmax(32.0 * 2 * a.D * (a.slots > 0 ? 1 : 2) / 50e3, 0.12)
                      : block == 256 ? 1.0 + 0.01 * a.D : (0.55 + 0.006 * a.D) * (a.slots > 0 ? 1.25 : 1.0);
    const double part = (double)rows * heads * a.D * 8 / 4e6 + 0.1;
    const bool pairs = !single && block == 128;   // two workgroups a CU
    const long long most = tiles / (single ? 4 : 2);
    auto rounds = [&](long long room) { return (double)((wgs + room - 1) / room); };
    w.time = pairs && wgs > kCus ? rounds(2 * kCus) * (double)tiles * cost * 1.6 : rounds(kCus) * (double)tiles * cost;
    auto consider = [&](long long room, double slower) {
        const double ideal = sqrt((double)tiles * cost * slower / part);
        long long s = single ? (room + wgs / 2) / wgs : room / wgs;
        if (s > most) s = most;
        if ((double)s > ideal) s = (long long)ideal;
        if (s < 2) return;
        const double t = (double)((tiles + s - 1) / s) * cost * slower + 4.5 + (double)s * part;
        if (t < w.time) w.time = t, w.splits = (int)s;
    };
    consider(kCus, 1.0);
    if (pairs) consider(2 * kCus, 1.6);
    return w;
}

SpanPlan span_plan(const SpanArgs& a) {
    const long long rows = (long long)a.Lq * (a.H / a.Hk), heads = (long long)a.B * a.Hk;
    SpanPlan p{};
    SpanWay w = span_way(a, true);
    p.single = true;
    if (rows > kSpanRows) {
        // Blocks of 32 rows whose eight waves share out the keys, where there is a CU for each (110 calls drawn at random, at
        // most 3000 such blocks: 13.7 us in the geometric mean, 16.0 tiled; where there are up to 512 blocks 14.0, all 16.7; 754 tokens of
        // 8 heads D = 80, windows of 162, 19.5 -> 9.0; 29 tokens of two heads 7.6 -> 8.4).
        const SpanWay tiled = span_way(a, false);
        if (heads * w.row_blocks > kCus || tiled.time < w.time) w = tiled, p.single = false;
    }
    p.row_blocks = w.row_blocks, p.splits = w.splits;
    p.part_tiles = (int)((w.tiles + w.splits - 1) / w.splits);
    if (p.splits > 1) {
        const __int128 bytes = (__int128)p.splits * heads * rows * (a.D + 2) * 4;
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
    a.row_blocks = p.row_blocks, a.splits = p.splits, a.part_tiles = p.part_tiles;
    a.zero = s.scale == 0.0f, a.neg = s.scale < 0;
    a.c = a.zero ? 1.0f : fminf((a.neg ? -s.scale : s.scale) * kLog2e, __FLT_MAX__);   // (zero times it stays that)
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
