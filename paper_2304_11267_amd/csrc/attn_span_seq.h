// attn_span_seq.h -- what the kernels of attn_span.h and the join of their parts share: a call's
// arguments, the place of a sequence, and the keys that its tokens see (attn_span.h says which).
#pragma once

#include "device.h"
#include "launch.h"

namespace sdattn {

constexpr int kSpanRows = 32;          // rows of a block of attn_span_row.h
// Rows of a block of the tiled kernel for heads of D (a multiple of 16).  Wide heads have no registers for the codes of
// pages beside 128 rows.
constexpr int span_block(int D, bool paged) { return D > (paged ? 96 : 128) ? 256 : 128; }
constexpr float kSpanNone = -__FLT_MAX__;   // the exponent's reference before the first key: no finite score is below it

struct SpanKernel {
    const uint16_t* q;
    uint16_t* out;
    const char* k;             // 16-bit values, or pages of codes
    const char* v;
    const float* ks;           // [pages, Hk]
    const float* vs;
    const int* table;          // [B, slots]
    const int* starts;         // [B] or null: Lk - Lq
    const int* counts;         // [B] or null: Lq
    float* part;               // splits > 1: O [splits, B, Hk, Lq G, D], then (m, l) [.., 2]
    long long qb, qh, ql, ob, oh, ol, kb, kh, kl;   // elements between batch items, heads, tokens
    int B, Hk, G, Lq, Lk, D;
    int pages, slots;
    int frame, window, sinks;
    int row_blocks, splits;    // blocks of a key head's rows, parts of their keys
    int part_tiles, waves;     // attn_span_row.h: the most tiles of a part, waves of a workgroup
    uint32_t per_wave;         // 2^32 / waves, rounded up
    float c;                   // |scale| log2(e), finite and not 0; with scale 0, 1 and Q is taken for zeros
    int neg;                   // scale < 0
    int zero;                  // scale = 0
};

// A sequence's place: what is on the device is taken as it is and kept in bounds.
struct SpanSeq {
    long long start;
    int count, n;
};
__device__ __forceinline__ SpanSeq span_seq(const SpanKernel& a, int b) {
    SpanSeq s;
    s.start = a.starts ? a.starts[b] : a.Lk - a.Lq;
    s.count = a.counts ? min(max(a.counts[b], 0), a.Lq) : a.Lq;
    const long long n = s.start + s.count;
    s.n = n < 0 ? 0 : n > a.Lk ? a.Lk : (int)n;
    return s;
}
__device__ __forceinline__ int span_hi(const SpanKernel& a, const SpanSeq& s, int token) {
    if (a.frame == 0) return s.n;
    const long long p = s.start + token;
    if (p < 0) return 0;
    if (p >= s.n) return s.n;
    const uint32_t f = (uint32_t)a.frame;
    const uint32_t end = f == 1 ? (uint32_t)p + 1 : ((uint32_t)p / f + 1) * f;   // below 2^30 + 2^31
    return (int)min(end, (uint32_t)s.n);
}
__device__ __forceinline__ int span_lo(const SpanKernel& a, int hi) { return a.window ? max(hi - a.window, 0) : 0; }

// The tiles of `tk` keys that a run of tokens reads: the first `first` ones, then those from `from` on.
struct SpanTiles {
    int first, from, count;
    __device__ __forceinline__ int at(int i) const { return i < first ? i : from + (i - first); }
};
__device__ __forceinline__ SpanTiles span_tiles(const SpanKernel& a, const SpanSeq& s, int token0, int token1, int tk) {
    const int lo = span_lo(a, span_hi(a, s, token0)), hi = span_hi(a, s, token1);
    SpanTiles t;
    t.first = (min(a.sinks, hi) + tk - 1) / tk;
    t.from = max(lo / tk, t.first);
    t.count = t.first + max(0, (hi + tk - 1) / tk - t.from);
    return t;
}

// The kernel's arguments and its workgroup's number, read anew: what a rare path at a kernel's end derives from them
// takes no registers before it.
struct SpanAnew {
    SpanKernel a;
    int wg;
};
__device__ __forceinline__ SpanAnew span_anew() {
    const __attribute__((address_space(4))) void* p = (const __attribute__((address_space(4))) void*)__builtin_amdgcn_kernarg_segment_ptr();
    int wg = blockIdx.x;
    asm volatile("" : "+s"(p), "+s"(wg));
    return SpanAnew{*(const SpanKernel*)p, wg};
}

// What every query of a run of tokens sees of a tile.
struct SpanRun {
    int lo0, lo1, hi0, hi1, sinks;   // of the first and the last token
    __device__ __forceinline__ bool all(int key0, int tk) const {
        return key0 + tk <= hi0 && (key0 >= lo1 || key0 + tk <= sinks);
    }
    __device__ __forceinline__ bool none(int key0, int tk) const {
        return key0 >= hi1 || (key0 + tk <= lo0 && key0 >= sinks);
    }
};
__device__ __forceinline__ SpanRun span_run(const SpanKernel& a, const SpanSeq& s, int token0, int token1) {
    SpanRun r;
    r.hi0 = span_hi(a, s, token0), r.hi1 = span_hi(a, s, token1);
    r.lo0 = span_lo(a, r.hi0), r.lo1 = span_lo(a, r.hi1);
    r.sinks = a.sinks;
    return r;
}

// The instantiations (a translation unit each): attn_span.h's, and for few rows attn_span_row.h's.
hipError_t launch_span_dense_f16(const SpanKernel& a, hipStream_t stream);
hipError_t launch_span_dense_bf16(const SpanKernel& a, hipStream_t stream);
hipError_t launch_span_paged_f16(const SpanKernel& a, hipStream_t stream);
hipError_t launch_span_paged_bf16(const SpanKernel& a, hipStream_t stream);
hipError_t launch_span_row_dense_f16(const SpanKernel& a, hipStream_t stream);
hipError_t launch_span_row_dense_bf16(const SpanKernel& a, hipStream_t stream);
hipError_t launch_span_row_paged_f16(const SpanKernel& a, hipStream_t stream);
hipError_t launch_span_row_paged_bf16(const SpanKernel& a, hipStream_t stream);

}  // namespace sdattn
