// attn_span.h -- attention over the keys that a query's place in its sequence lets it see,
// from 16-bit tensors or from the 8-bit pages of kv_cache.hip.
//
// Token l of batch item b is at position p = start + l; the sequence has n = start + count
// keys.  With frames of F tokens (F = 1: token by token; 0: no order), a window of W keys (0:
// no limit) and S first keys that stay visible:
//   hi(p) = n (F = 0), or min(n, (floor(p / F) + 1) F);   lo(p) = max(0, hi(p) - W)  (W = 0: 0)
//   key j is seen where j < hi(p) and (j >= lo(p) or j < S)
// Both ends grow with p, so a block of queries reads two runs of key tiles: the first ones up
// to S, and those from its first query's lo to its last one's hi.  Only the tiles at the ends
// of these runs are looked at key by key.
//
// The G = H / Hk query heads of a key head are rows of one block: row r is head r % G of token
// r / G, so keys are read once for all of them.
#pragma once

#include "attn_geom.h"
#include "attn_span_seq.h"

namespace sdattn {

namespace {

constexpr int kSpanTile = 64;          // keys of a tile: a page of the cache
// The exponent's reference m is moved when a weight would pass 2^span_limit, to span_bias
// below the largest score, 7 octaves that few tiles move it in.  fp16: weights near 2^8 keep the small ones above its
// subnormals' end (it holds values below 2^16).  bf16, which has 32 bits' range: below 2^-17, so that the sums of values at that
// range's end over 2^17 keys stay within it.
template <int ET>
constexpr float span_bias = ET == kF16 ? 8.0f : -24.0f;
template <int ET>
constexpr float span_limit = span_bias<ET> + 7.0f;
// c s - m is one operation, exact in c s, where m came from a c s that was rounded.  Up to 2^23 that is a quarter of an octave
// of a weight at most; from 2^28 on a row's largest weight would be anything from 0 to infinity.  Rows whose m has
// been past 2^23 are computed again at the end (span_again); the largest |m| is noted where m is moved.  (A row whose m is
// infinite is one of no numbers already.)
constexpr float kSpanFar = 8388608.0f;
__device__ __forceinline__ bool span_far(float worst, float m) { return worst >= kSpanFar && m <= __FLT_MAX__; }
__device__ __forceinline__ float span_worst(float worst, float m) { return fmaxf(worst, m == kSpanNone ? 0.0f : fabsf(m)); }

// 8 codes as 8 values of the 16-bit type times s, a power of two (v_cvt_scalef32_pk_f16_fp8 /
// _bf16_fp8)
template <int ET>
__device__ __forceinline__ u32x4 decode8(uint32_t lo, uint32_t hi, float s) {
    u32x4 r;
    if constexpr (ET == kF16) {
        r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)lo, s, false));
        r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)lo, s, true));
        r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)hi, s, false));
        r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)hi, s, true));
    } else {
        r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)lo, s, false));
        r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)lo, s, true));
        r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)hi, s, false));
        r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)hi, s, true));
    }
    return r;
}

// Keeps the compiler from moving v's computation into a later block of code that alone uses it.
template <typename T>
__device__ __forceinline__ void computed_here(T& v) { asm volatile("" : "+v"(v)); }

// Of the 32 keys from key0 on those that a query with these ends sees, one a bit.
__device__ __forceinline__ uint32_t span_seen(int key0, int hi, int lo, int sinks) {
    auto below = [&](int end) __attribute__((always_inline)) {
        const int n = min(max(end - key0, 0), 32);
        return (uint32_t)((1ull << n) - 1);
    };
    return below(hi) & (~below(lo) | below(sinks));
}
// Scores of keys whose bit is not set as minus infinity: register r is key 8 (r / 4) + r % 4.
__device__ __forceinline__ void span_hide(f32x16& st, uint32_t seen) {
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        const uint32_t in = (uint32_t)((int)(seen << (31 - (8 * (r >> 2) + (r & 3)))) >> 31);
        st[r] = __uint_as_float((__float_as_uint(st[r]) & in) | (0xff800000u & ~in));
    }
}

// The bits of those 16-bit values of two that are infinite or no number.
template <int ET>
__device__ __forceinline__ uint32_t bad2(uint32_t w) {
    constexpr uint32_t kInf = ET == kF16 ? 0x7c00u : 0x7f80u;
    return ((w & kInf) == kInf ? 0xffffu : 0u) | ((w & (kInf << 16)) == (kInf << 16) ? 0xffff0000u : 0u);
}
// The bits of those codes of four that are no number (0x7f and 0xff).
__device__ __forceinline__ uint32_t bad_codes(uint32_t c) { return (((c & 0x7f7f7f7fu) + 0x01010101u) >> 7 & 0x01010101u) * 255u; }

// Values of V that are no numbers, or infinite, are zeros in the products of a tile that not all queries see whole: a
// weight of 0 would not keep them out.  For the queries that do see one, this adds it to the sums (acc as the
// products leave it), at the end, where key by key costs no time that counts: `vt` is the tile's first row in memory,
// `row` bytes from one to the next, `seen` this lane's keys of the 32.
template <int ET, bool PAGED, int DN>
__device__ __forceinline__ void span_add_bad(f32x16 (&acc)[DN], const char* vt, long long row, uint32_t seen, int D, int half) {
    for (uint32_t left = seen; __any(left != 0); left &= left - 1) {
        if (!left) continue;
        const char* const v = vt + (__ffs((int)left) - 1) * row;
#pragma unroll
        for (int n = 0; n < DN; ++n)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int d = 32 * n + 8 * g + 4 * half;
                if (d >= D) continue;
                uint32_t w[2];
                if constexpr (PAGED) {
                    const uint32_t c = bad_codes(*(const uint32_t*)(v + d));   // (the type's no number is all ones too)
                    w[0] = (c & 0xff ? 0xffffu : 0u) | (c & 0xff00 ? 0xffff0000u : 0u);
                    w[1] = (c & 0xff0000 ? 0xffffu : 0u) | (c & 0xff000000u ? 0xffff0000u : 0u);
                } else {
                    const u32x2 x = *(const u32x2*)(v + 2 * d);
                    w[0] = x[0] & bad2<ET>(x[0]), w[1] = x[1] & bad2<ET>(x[1]);
                }
                if (!(w[0] | w[1])) continue;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float x = to_float<ET>((uint16_t)(w[e >> 1] >> (16 * (e & 1))));
                    computed_here(x);   // (this file's floats are taken for numbers: neither side of the sum is known to be one)
                    x += acc[n][4 * g + e];
                    computed_here(x);
                    acc[n][4 * g + e] = x;
                }
            }
    }
}

// A row whose scores are far from zero, by a wave, key by key: its largest score, rounded as all of them are, and then
// the weights and sums relative to it, in 32 bits.  `row` is its query, [lo, hi) and a.sinks what it sees, tile_of(i) the i-th
// of n tiles of TK keys.  What comes here is far from what a model makes: the time does not count.
struct SpanAgain {
    float o[3], m, l;   // of the columns lane + 64 i
};
template <int ET, bool PAGED, int TK, typename F>
__device__ __forceinline__ SpanAgain span_again(const SpanKernel& a, int b, int hk, const uint16_t* row, int hi, int lo, int n, F tile_of) {
    const int lane = lane_id();
    const long long bytes = PAGED ? a.D : 2 * a.kl;   // from one key to the next
    auto scores = [&](auto use) __attribute__((always_inline)) {
        for (int i = 0; i < n; ++i) {
            const int t = tile_of(i), key = t * TK + lane;
            long long at = 2 * (b * a.kb + hk * a.kh + (long long)t * TK * a.kl);
            float ct = a.c, vs = 1.0f;
            if constexpr (PAGED) {
                const int page = a.table[(size_t)b * a.slots + t / (kCachePage / TK)];
                if (page < 0 || page >= a.pages) continue;
                at = (((long long)page * a.Hk + hk) * kCachePage + t % (kCachePage / TK) * TK) * a.D;
                ct = __builtin_amdgcn_fmed3f(ct * a.ks[(size_t)page * a.Hk + hk], __FLT_MIN__, __FLT_MAX__);
                vs = a.vs[(size_t)page * a.Hk + hk];
            }
            const bool seen = lane < TK && key < hi && (key >= lo || key < a.sinks);
            float x = 0.0f;
            if (seen) {
                const char* const k = a.k + at + lane * bytes;
                for (int d = 0; d < a.D; d += 8) {
                    u32x4 q = *(const u32x4*)(row + d), w;
                    if (a.neg) q ^= 0x80008000u;
                    if (a.zero) q = u32x4{0u, 0u, 0u, 0u};
                    if constexpr (PAGED) {
                        const u32x2 c = *(const u32x2*)(k + d);
                        w = decode8<ET>(c[0], c[1], 1.0f);
                    } else {
                        w = *(const u32x4*)(k + 2 * d);
                    }
                    x = dot8<ET>(w, q, x);
                }
                x *= ct;
                computed_here(x);   // (rounded)
            }
            use(seen, x, a.v + at, vs);
        }
    };
    float top = -__builtin_inff();
    bool bad = false;   // no number, or infinite and not below zero
    scores([&](bool seen, float x, const char*, float) __attribute__((always_inline)) {
        if (!seen) return;
        top = fmaxf(top, x);
        bad |= __float_as_uint(x) != 0xff800000u && (__float_as_uint(x) & 0x7f800000u) == 0x7f800000u;
    });
    if (__any(bad)) {
        const float none = __uint_as_float(0x7fc00000u);
        return SpanAgain{{none, none, none}, kSpanNone, none};
    }
#pragma unroll
    for (int k = 1; k < 64; k <<= 1) top = fmaxf(top, __shfl_xor(top, k, 64));
    SpanAgain r{{0.0f, 0.0f, 0.0f}, kSpanNone, 0.0f};
    if (top == -__builtin_inff()) return r;
    r.m = top;
    scores([&](bool seen, float x, const char* v, float vs) __attribute__((always_inline)) {
        const float w = seen ? fast_exp2(x - top) : 0.0f;
        r.l += w;
        for (uint64_t left = __ballot(seen); left; left &= left - 1) {
            const int j = __builtin_ctzll(left);
            const float f = __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(w), j));
#pragma unroll
            for (int c = 0; c < 3; ++c) {
                const int d = lane + 64 * c;
                if (d >= a.D) continue;
                if constexpr (PAGED) r.o[c] = fmaf(f, __builtin_amdgcn_cvt_f32_fp8((int)*(const uint8_t*)(v + j * bytes + d), 0) * vs, r.o[c]);
                else r.o[c] = fmaf(f, to_float<ET>(*(const uint16_t*)(v + j * bytes + 2 * d)), r.o[c]);
            }
        }
    });
#pragma unroll
    for (int k = 1; k < 64; k <<= 1) r.l += __shfl_xor(r.l, k, 64);
    return r;
}

// ---------------------------------------------------------------- the tiled kernel

// Workgroups of NW waves of 32 rows: four, and two or three workgroups a CU, whose waves share the SIMDs without
// waiting for each other at barriers (eight waves of one workgroup, D = 128: one of a SIMD's two ends its tile first, and
// the other's products then have no exponentials beside them); eight past D = 128, and over pages past 96, where registers
// and LDS leave no room for that.  K and V tiles of 64 keys lie as 16-bit values in LDS buffers, two or three of K and two
// of V, rows of DP values whose 16-byte chunks are permuted where rows would share banks (chunk c of row r in the place of
// c ^ swap(r)).
//
// The pass is one stream over 32-key sub-tiles p = 0, 1, ...: step p issues
//   S^T = K Q^T of sub-tile p + 1,  the weights 2^(c s - m) of p,  O^T += V^T P^T of p - 1
// which do not depend on each other, a few operations of the vector unit behind each matrix product, in the order
// written here (sched_barrier keeps it: a wave issues in order, and a run of either leaves the other unit
// to the SIMD's other wave alone).  An operand of K or V is read from LDS again, for the next step,
// behind the product that it has fed.  m is moved with a sub-tile's maximum where a weight would pass its limit.
//
// The matrix core bounds it past D = 96, the vector unit beside it below: 17550 tokens, 16 heads of 128, windows of four
// frames of 1350 and the first: 890 to 930 us by the card, 880 to 920 TFLOP/s of the visible keys, where a library's product
// reaches 1300.  4096 tokens of D = 40, windows of 1024 and 77: 29.6 us; a tile takes 1.1 us of it on two
// workgroups of a CU, of which the products alone are 0.58, the exponentials and sums 0.3 to 0.4, copies and LDS reads
// the rest.  Pages, 1350 tokens over 6750 keys, D = 128: 132 us and a join of 7.6.

// Waves of a SIMD that the registers are cut for: three where that costs none (D = 40 in pages, 2665 tokens of 16 sequences
// 99 -> 83 us; D = 64, 64 heads of 4096 tokens 370 -> 345; 64 in pages spills, 99 -> 101).
constexpr int span_waves(int DP, bool paged) { return DP <= 48 || (DP == 64 && !paged) ? 3 : 2; }

template <int DP, int NW>
struct SpanTile {
    static constexpr int kThreads = 64 * NW, kRows = 32 * NW;
    static constexpr int KC = DP / 8;                          // chunks of a row
    static constexpr int kLow = KC & -KC;
    static constexpr int kSwap = kLow > 16 ? 16 : kLow;
    static constexpr int DK = DP / 16;                         // 16-deep steps of S
    static constexpr int DN = (DP + 31) / 32;                  // 32-row tiles of O^T
    static constexpr int kTileBytes = kSpanTile * DP * 2;
    // operands of K read ahead of their products: a sub-tile's, or what registers there are
    static constexpr int kAhead = NW == 4 || DP <= 112 ? DK : DP == 144 ? 3 : 2;
    static_assert(DK % kAhead == 0, "a step ends where the ring does");
    static constexpr int kBufsK = kAhead == DK ? 2 : 3;        // (with fewer, a tile's K is read while it is used)
    // With columns to spare in the last 32 rows of O^T, one of them is of ones: the row sum of the weights comes out
    // of the matrix core.  Its lanes read a constant block: a one and zeros, where 16 rows of a tile begin.
    static constexpr bool kOnes = DP % 32 == 16;
    static_assert(!kOnes || kSwap == 2, "the last 32 columns lie 4 n chunks on, whatever the swap");
    static constexpr int kWords = (kBufsK + 2) * kTileBytes;   // after K and V: four words of keys,
    static constexpr int kConst = kWords + 32;                 // and the constant block
    static constexpr int kLdsBytes = kConst + (kOnes ? 3 * 16 * DP * 2 + 16 : 0);
    static __device__ __forceinline__ int swap(int row) { return kSwap > 1 ? row / (16 / kSwap) & (kSwap - 1) : 0; }
};

// The tiles that all queries of a run of tokens see whole: below `sinks`, or in [from, to).
struct SpanWhole {
    int from, to, sinks;
    __device__ __forceinline__ bool has(int t) const { return t < to && (t >= from || t < sinks); }
};
__device__ __forceinline__ SpanWhole span_whole(const SpanRun& r) {
    constexpr int TK = kSpanTile;
    return SpanWhole{(r.lo1 + TK - 1) / TK, r.hi0 / TK, r.sinks / TK};
}

// Blocks of the last rows, which see most, first; where all workgroups are on the card at once, for the next head
// last, so that the two of a CU differ (causal, 16 heads of 4096 tokens D = 40 77 -> 65 us; 8192 tokens D = 128, four
// rounds, 307 -> 374).
struct SpanPlace {
    int rb, bh, split;
};
__device__ __forceinline__ SpanPlace span_place(const SpanKernel& a, int wg) {
    const int item = xcd_remap(wg, gridDim.x), turn = item / a.row_blocks;
    int rb = item - turn * a.row_blocks;
    if (!(turn & 1) || gridDim.x > 2 * kCus) rb = a.row_blocks - 1 - rb;
    const int bh = turn / a.splits;
    return SpanPlace{rb, bh, turn - bh * a.splits};
}

// The rows of a wave whose bits are set, by span_again, and stored.
template <int ET, int DP, int NW, bool PAGED>
__device__ __forceinline__ void span_tile_again(uint32_t rows, int wave) {
    using G = SpanTile<DP, NW>;
    const SpanAnew anew = span_anew();
    const SpanKernel& a = anew.a;
    const SpanPlace at = span_place(a, anew.wg);
    const int b = at.bh / a.Hk, hk = at.bh - b * a.Hk, R = a.Lq * a.G, r0 = at.rb * G::kRows, lane = lane_id();
    const SpanSeq seq = span_seq(a, b);
    const SpanTiles tiles = span_tiles(a, seq, r0 / a.G, min((r0 + G::kRows - 1) / a.G, seq.count - 1), kSpanTile);
    const int per = (tiles.count + a.splits - 1) / a.splits, begin = at.split * per, n = min(per, tiles.count - begin);
    for (; rows; rows &= rows - 1) {
        const int row = r0 + 32 * wave + __builtin_ctz(rows), token = row / a.G, head = hk * a.G + row - token * a.G;
        const int hi = span_hi(a, seq, token), lo = span_lo(a, hi);
        const SpanAgain x = span_again<ET, PAGED, kSpanTile>(a, b, hk, a.q + b * a.qb + head * a.qh + token * a.ql, hi, lo, n,
                                                             [&](int i) { return tiles.at(begin + i); });
        const float inv = x.l == 0.0f ? 0.0f : 1.0f / x.l;
        const size_t all = (size_t)a.B * a.Hk * R, to = at.split * all + (size_t)at.bh * R + row;
#pragma unroll
        for (int c = 0; c < 3; ++c) {
            const int d = lane + 64 * c;
            if (d >= a.D) continue;
            if (a.splits > 1) a.part[to * a.D + d] = x.o[c];
            else a.out[b * a.ob + head * a.oh + token * a.ol + d] = from_float<ET>(x.o[c] * inv);
        }
        if (a.splits > 1 && lane == 0) {
            float* const ml = a.part + a.splits * all * a.D + to * 2;
            ml[0] = x.m;
            ml[1] = x.l;
        }
    }
}

template <int ET, int DP, int NW, bool PAGED>
__global__ __launch_bounds__((SpanTile<DP, NW>::kThreads), span_waves(DP, PAGED)) void span_tile_kernel(const SpanKernel a) {
    using G = SpanTile<DP, NW>;
    constexpr int DK = G::DK, DN = G::DN, KC = G::KC, TK = kSpanTile, NKB = G::kBufsK;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const int tid = threadIdx.x;
    const int lane = lane_id(), l32 = lane & 31, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int D = a.D;

    const SpanPlace at = span_place(a, blockIdx.x);
    const int rb = at.rb, bh = at.bh, split = at.split, b = bh / a.Hk, hk = bh - b * a.Hk;
    auto token_of = [&](int row) __attribute__((always_inline)) { return a.G == 1 ? row : row / a.G; };
    // this lane's row, and its query, which waits for nothing
    const int R = a.Lq * a.G, r0 = rb * G::kRows, w0 = r0 + 32 * wave;
    const int row = min(w0 + l32, R - 1), token = token_of(row), head = hk * a.G + row - token * a.G;
    u32x4 qreg[DK];
#pragma unroll
    for (int s = 0; s < DK; ++s) {
        const int d0 = 16 * s + 8 * half;
        qreg[s] = u32x4{0u, 0u, 0u, 0u};
        if (d0 < D) qreg[s] = *(const u32x4*)(a.q + b * a.qb + head * a.qh + token * a.ql + d0);
    }
    const SpanSeq seq = span_seq(a, b);
    // tokens of this block and of this wave, the ones past `count` left out
    const int token0 = token_of(r0), token1 = min(token_of(r0 + G::kRows - 1), seq.count - 1);
    if (token0 >= seq.count) return;
    const int wtoken0 = min(token_of(w0), token1), wtoken1 = max(min(token_of(w0 + 31), seq.count - 1), wtoken0);
    const SpanTiles tiles = span_tiles(a, seq, token0, token1, TK);
    const SpanWhole block = span_whole(span_run(a, seq, token0, token1));
    const SpanWhole whole = span_whole(span_run(a, seq, wtoken0, wtoken1));

    const bool valid = token < seq.count && w0 + l32 < R, live = w0 < R && token_of(w0) < seq.count;
    const int hi = span_hi(a, seq, min(token, seq.count - 1)), lo = span_lo(a, hi), sinks = a.sinks;
#pragma unroll
    for (int s = 0; s < DK; ++s) {
        if (a.neg) qreg[s] ^= 0x80008000u;   // a negative scale (exact)
        if (a.zero) qreg[s] = u32x4{0u, 0u, 0u, 0u};
    }

    // this split's tiles
    const int per = (tiles.count + a.splits - 1) / a.splits;
    const int i_begin = split * per, i_end = min(i_begin + per, tiles.count);
    int i = i_begin;

    // ---- tiles into LDS
    const uint32_t lds0 = lds_offset(smem);
    // keys of tile c whose V is no number, in word c % 4: cleared three tiles before it is written, so that no
    // barrier is needed for it
    uint64_t* const bad = (uint64_t*)(smem + G::kWords);
    // 16-bit tensors: 1 KB copies, KC of them over the waves
    constexpr int kCopies = (KC + NW - 1) / NW;
    [[maybe_unused]] const char* Kb = nullptr;
    [[maybe_unused]] const char* Vb = nullptr;
    [[maybe_unused]] const uint32_t row_bytes = (uint32_t)a.kl * 2;
    [[maybe_unused]] uint32_t copy_off[kCopies];
    [[maybe_unused]] bool copy_k[kCopies];     // a chunk of K, too (past D its values meet zeros of Q: they are zeros)
    // pages: pieces of 16 codes over the threads
    constexpr int kPieces = (4 * DP + G::kThreads - 1) / G::kThreads;
    [[maybe_unused]] u32x4 kraw[kPieces], vraw[kPieces];
    [[maybe_unused]] int place[kPieces][2];    // of its two chunks in a tile; -1: none
    if constexpr (PAGED) {
#pragma unroll
        for (int p = 0; p < kPieces; ++p)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int q = 2 * (p * G::kThreads + tid) + e, r = q / (D / 8), c = q - r * (D / 8);
                place[p][e] = r < TK ? (r * KC + (c ^ G::swap(r))) * 16 : -1;
            }
        if (D != DP) {   // values past D are never written and meet zeros of Q
            for (int z = tid; z < (NKB + 2) * G::kTileBytes / 16; z += G::kThreads) *(u32x4*)(smem + z * 16) = u32x4{0u, 0u, 0u, 0u};
        }
    } else {
        Kb = a.k + 2 * (b * a.kb + hk * a.kh);
        Vb = a.v + 2 * (b * a.kb + hk * a.kh);
#pragma unroll
        for (int p = 0; p < kCopies; ++p) {
            const int q = (wave + p * NW) * 64 + lane, r = q / KC;
            const int c = (q - r * KC) ^ G::swap(r);
            copy_k[p] = c < D / 8;
            copy_off[p] = (uint32_t)r * row_bytes + min(c, D / 8 - 1) * 16;
        }
        if (DP != D) {
            for (int z = tid; z < NKB * TK; z += G::kThreads) {
                const int r = z % TK;
                *(u32x4*)(smem + z / TK * G::kTileBytes + (r * KC + ((KC - 1) ^ G::swap(r))) * 16) = u32x4{0u, 0u, 0u, 0u};
            }
        }
    }
    if (tid < 4) bad[tid] = 0;
    if (G::kOnes && tid < 4) *(u32x4*)(smem + G::kConst + tid * 16 * DP * 2) = u32x4{(uint32_t)from_float<ET>(1.0f), 0u, 0u, 0u};
    __syncthreads();

    // Pages and scales of places `base` .. base + 63 of the list of tiles, one a lane.
    [[maybe_unused]] int base = i - 64, pages = 0;
    [[maybe_unused]] float kss = 0.0f, vss = 0.0f;
    [[maybe_unused]] uint64_t present = 0;
    struct Tile {
        int t, page;       // t < 0: none
        float ks, vs;
    };
    // the tile at the first place from i on that has a page, with i past it
    auto next_tile = [&]() __attribute__((always_inline)) -> Tile {
        Tile x{-1, 0, 1.0f, 1.0f};
        if constexpr (PAGED) {
            while (i < i_end) {
                if (i - base >= 64) {
                    base = i;
                    const int at = min(i + lane, i_end - 1);
                    const int page = a.table[(size_t)b * a.slots + tiles.at(at)];
                    const bool there = page >= 0 && page < a.pages;
                    pages = there ? page : 0;
                    kss = a.ks[(size_t)pages * a.Hk + hk];
                    vss = a.vs[(size_t)pages * a.Hk + hk];
                    present = __ballot(there && i + lane < i_end);
                }
                const uint64_t left = present >> (i - base);
                if (left) {
                    i += __builtin_ctzll(left);
                    const int at = i - base;
                    x.t = tiles.at(i);
                    x.page = __builtin_amdgcn_readlane(pages, at);
                    x.ks = __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(kss), at));
                    x.vs = __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(vss), at));
                    ++i;
                    return x;
                }
                i = base + 64;
            }
        } else if (i < i_end) {
            x.t = tiles.at(i);
            ++i;
        }
        return x;
    };
    // A tile of K or of V, from `from` (its batch item's and head's, or the pages), into buffer buf; pages: into
    // registers, as codes.
    auto load = [&](const Tile& x, const char* from, u32x4 (&raw)[kPieces], int buf, bool k) __attribute__((always_inline)) {
        if constexpr (PAGED) {
            const char* const at = from + ((size_t)x.page * a.Hk + hk) * TK * D;
#pragma unroll
            for (int p = 0; p < kPieces; ++p)
                if (place[p][0] >= 0) raw[p] = *(const u32x4*)(at + (p * G::kThreads + tid) * 16);
        } else {
            const char* const at = from + (long long)x.t * TK * row_bytes;
            const int last = seq.n - 1 - x.t * TK;   // keys past the last one repeat it
            auto copy = [&](auto some) __attribute__((always_inline)) {
#pragma unroll
                for (int p = 0; p < kCopies; ++p) {
                    const int ci = wave + p * NW;
                    if (ci < KC) {
                        uint32_t off = copy_off[p];
                        if (last < TK - 1) {
                            const int r = (ci * 64 + lane) / KC;
                            if (r > last) off -= (uint32_t)(r - last) * row_bytes;
                        }
                        if (!decltype(some)::value || copy_k[p]) copy16_to_lds(at, off, lds0 + buf * G::kTileBytes + ci * 1024);
                    }
                }
            };
            if (k && D != DP) copy(std::true_type{});
            else copy(std::false_type{});
        }
    };
    auto load_k = [&](const Tile& x, int buf) __attribute__((always_inline)) { load(x, PAGED ? a.k : Kb, kraw, buf, true); };
    auto load_v = [&](const Tile& x, int buf) __attribute__((always_inline)) { load(x, PAGED ? a.v : Vb, vraw, NKB + buf, false); };
    // pages: the codes read by load as 16-bit values in buffer buf, V's times its scale
    auto store_k = [&](int buf) __attribute__((always_inline)) {
        if constexpr (PAGED) {
#pragma unroll
            for (int p = 0; p < kPieces; ++p)
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    if (place[p][e] >= 0)
                        *(u32x4*)(smem + buf * G::kTileBytes + place[p][e]) = decode8<ET>(kraw[p][2 * e], kraw[p][2 * e + 1], 1.0f);
        }
    };
    auto store_v = [&](const Tile& x, int buf, uint64_t* word) __attribute__((always_inline)) {
        if constexpr (PAGED) {
            const bool end = !block.has(x.t);
#pragma unroll
            for (int p = 0; p < kPieces; ++p)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    if (place[p][e] < 0) continue;
                    uint32_t lo4 = vraw[p][2 * e], hi4 = vraw[p][2 * e + 1];
                    if (end) {
                        const int r = place[p][e] / (KC * 16);
                        const uint32_t lob = bad_codes(lo4), hib = bad_codes(hi4);
                        const bool past = x.t * TK + r >= seq.n;   // (whatever the page holds there; nobody sees it)
                        if ((lob | hib) && !past) atomicOr((unsigned long long*)word, 1ull << r);
                        lo4 = past ? 0 : lo4 & ~lob;
                        hi4 = past ? 0 : hi4 & ~hib;
                    }
                    *(u32x4*)(smem + (NKB + buf) * G::kTileBytes + place[p][e]) = decode8<ET>(lo4, hi4, x.vs);
                }
        }
    };
    // 16-bit tensors: values of V in an end tile that are no numbers, as zeros, with their keys
    auto scan = [&](int buf, uint64_t* word) __attribute__((always_inline)) {
        char* const vt = smem + (NKB + buf) * G::kTileBytes;
        for (int q = tid; q < TK * KC; q += G::kThreads) {
            const u32x4 w = *(const u32x4*)(vt + q * 16);
            const u32x4 b = {bad2<ET>(w[0]), bad2<ET>(w[1]), bad2<ET>(w[2]), bad2<ET>(w[3])};
            if (b[0] | b[1] | b[2] | b[3]) {
                *(u32x4*)(vt + q * 16) = w & ~b;
                atomicOr((unsigned long long*)word, 1ull << (q / KC));
            }
        }
    };

    // ---- per-lane places in a buffer (as in attn_fwd_kernel.h).  Where the swap has bits that chunks of one row
    // differ in (kXor), they come into an address by exclusive or, else by addition, as part of the instruction.
    constexpr int kXor = G::kSwap;   // a power of two: bits below it are a chunk's in its group
    const int k_at = (l32 * KC + (half ^ G::swap(l32))) * 16;
    const int v_key = 4 * (lane >> 5) + ((lane & 15) >> 2), v_d = 16 * (lane >> 4 & 1) + 4 * (lane & 3);
    const int v_at = NKB * G::kTileBytes + (v_key * KC + ((v_d / 8) ^ G::swap(v_key))) * 16 + v_d % 8 * 2;
    const int v_up = NKB * G::kTileBytes + ((v_key + 8) * KC + ((v_d / 8) ^ G::swap(v_key + 8))) * 16 + v_d % 8 * 2;
    // the last 32 columns, of which DP has 16: past D the constant block, the one at D
    const int c_d = 32 * (DN - 1) + v_d, c_mask = G::kOnes && c_d >= D ? 0 : -1;
    const int c_at = c_mask ? v_at + 64 * (DN - 1) : G::kConst + (c_d == D ? 0 : 8), c_up = c_mask ? v_up + 64 * (DN - 1) : c_at;
    // chunk `more` on from the place at an address, `more` a constant that shares no bit with the chunk there
    auto chunk_on = [&](int at, int more) __attribute__((always_inline)) {
        return (at ^ ((more & (kXor - 1)) * 16)) + (more & -kXor) * 16;
    };

    f32x16 acc[DN];
    float m = kSpanNone, l = 0.0f, alpha = 1.0f;
    int spoiled = 0;   // this lane's query sees a value that is no number
    float worst = 0.0f;   // the largest |m| that this row has had
#pragma unroll
    for (int n = 0; n < DN; ++n)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[n][r] = 0.0f;

    constexpr int NQ = DK, NP = 2 * DN, NM = NQ + NP;   // matrix products of S^T, of O^T and of a step
    constexpr int NA = NM / 4;                          // beside the maximum
    constexpr int KR = G::kAhead;                       // operands of K read ahead
    u32x4 kf[KR], vf[2][DN], pk[2][2];
    f32x16 st[2];
    auto read_k = [&](int buf, int sub, int s) __attribute__((always_inline)) {
        kf[s % KR] = *(const u32x4*)(smem + chunk_on(buf + k_at, 2 * s) + 32 * sub * KC * 16);
    };
    auto read_v = [&](int buf, int sub, int h) __attribute__((always_inline)) {
        const int u = h / DN, n = h % DN, rows = (32 * sub + 16 * u) * KC * 16;
        const bool ones = G::kOnes && n == DN - 1;   // (kXor is 2 then: 4 n is added)
        const char* const xp = smem + (ones ? (buf & c_mask) + c_at : chunk_on(buf + v_at, 4 * n)) + rows;
        const char* const yp = smem + (ones ? (buf & c_mask) + c_up : chunk_on(buf + v_up, 4 * n)) + rows;
        const u32x2 x = lds_read_tr(xp), y = lds_read_tr(yp);
        vf[u][n] = u32x4{x[0], x[1], y[0], y[1]};
    };
    const f32x16 zero = {};
    auto s_mfma = [&](int x, int s) __attribute__((always_inline)) { st[x] = mfma32x32x16<ET>(kf[s % KR], qreg[s], s == 0 ? zero : st[x]); };
    auto o_mfma = [&](int x, int h) __attribute__((always_inline)) {
        acc[h % DN] = mfma32x32x16<ET>(vf[h / DN][h % DN], pk[x][h / DN], acc[h % DN]);
    };
    // The scores of the sub-tile at `key0` that this lane's query does not see, as minus infinity
    auto mask = [&](int x, int key0, const uint64_t* word) __attribute__((always_inline)) {
        const uint32_t seen = span_seen(key0, hi, lo, sinks);
        span_hide(st[x], seen >> (4 * half));
        // a query that sees a key of which a V is no number
        if (seen & (uint32_t)(*word >> (key0 & 32))) spoiled = 1;
    };
    // m moved for st[x], where it has to be, and what that makes of the sums so far
    auto look = [&](int x, float ct) __attribute__((always_inline)) {
        float p = st[x][0], q = st[x][1];
#pragma unroll
        for (int r = 2; r < 14; r += 4) {
            p = fmaxf(fmaxf(p, st[x][r]), st[x][r + 1]);
            q = fmaxf(fmaxf(q, st[x][r + 2]), st[x][r + 3]);
        }
        p = fmaxf(fmaxf(p, st[x][14]), st[x][15]);
        const float mx = half_max(fmaxf(p, q)) * ct;
        const float m_new = mx - m > span_limit<ET> ? mx - span_bias<ET> : m;
        alpha = fast_exp2(m - m_new);
        if (!G::kOnes) l *= alpha;
        m = m_new;
    };
    // The weights of st[x] as a list of operations, 2 scores at a time, each stage one unit behind the one before:
    // c s - m, 2^, rounding and the row sum
    constexpr int kOut = G::kOnes ? 1 : 2, kOps = 8 * (4 + kOut);
    auto weights = [&](int x, int i, float ct) __attribute__((always_inline)) {
        int at = 0;
#pragma unroll
        for (int t = 0; t < 10; ++t) {
            if (t < 8) {
                if (i == at) st[x][2 * t] = fmaf(st[x][2 * t], ct, -m);
                if (i == at + 1) st[x][2 * t + 1] = fmaf(st[x][2 * t + 1], ct, -m);
                at += 2;
            }
            if (t >= 1 && t < 9) {
                if (i == at) st[x][2 * t - 2] = fast_exp2(st[x][2 * t - 2]);
                if (i == at + 1) st[x][2 * t - 1] = fast_exp2(st[x][2 * t - 1]);
                at += 2;
            }
            if (t >= 2) {
                const int w = t - 2;
                if (i == at) pk[x][w / 4][w % 4] = pack2<ET>(st[x][2 * w], st[x][2 * w + 1]);
                if (!G::kOnes && i == at + 1) l = add_pair<ET>(pk[x][w / 4][w % 4], l);
                at += kOut;
            }
        }
    };
    // Step of sub-tile SUB at `key0` (`end`: key by key); its tile's V lies at vbuf and K at kbuf, the next one's K at next.
    auto step = [&](auto sub_c, int vbuf, int kbuf, int next, bool end, int key0, const uint64_t* word, float ct) __attribute__((always_inline)) {
        constexpr int X = decltype(sub_c)::value, Y = 1 - X;
        auto product = [&](int g) __attribute__((always_inline)) {
            // S^T and O^T in turn: each is a chain on one accumulator, which two in a row would wait on
            const int q = (g * NQ + NM - 1) / NM, h = g - q;
            if ((g + 1) * NQ > q * NM) {
                s_mfma(Y, q);
                __builtin_amdgcn_sched_barrier(0);   // (the operand's registers are free now)
                // (of sub-tile p + 1, or of the one after: X 0 has p + 1 in its own tile)
                if (q + KR < NQ) read_k(X == 0 ? kbuf : next, Y, q + KR);
                else read_k(next, X, q + KR - NQ);
            } else {
                o_mfma(Y, h);
                __builtin_amdgcn_sched_barrier(0);
                read_v(vbuf, X, h);
            }
        };
        if (end) mask(X, key0, word);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int g = 0; g < NA; ++g) {
            product(g);
            __builtin_amdgcn_sched_barrier(0);
        }
        look(X, ct);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int g = NA; g < NM; ++g) {
            product(g);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = (g - NA) * kOps / (NM - NA); i < (g - NA + 1) * kOps / (NM - NA); ++i) weights(X, i, ct);
            __builtin_amdgcn_sched_barrier(0);
        }
        computed_here(pk[X][0]);
        computed_here(pk[X][1]);
        if (!G::kOnes) computed_here(l);
        // the products of the sub-tile before were for the m before
        if (__any(alpha != 1.0f)) {
            worst = span_worst(worst, m);
#pragma unroll
            for (int n = 0; n < DN; ++n)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[n][r] *= alpha;
        }
    };
    std::integral_constant<int, 0> c0;
    std::integral_constant<int, 1> c1;

    // ---- the stream.  While tile c is used its V and the next one's K are read from LDS (its own K is in
    // registers by then), and the next one's V and the K of the one after that are on their way.
    const Tile none{-1, 0, 1.0f, 1.0f};
    Tile t0 = next_tile(), t1 = none, t2;
    if (t0.t >= 0) {
        load_k(t0, 0);
        load_v(t0, 0);
        store_k(0);
        store_v(t0, 0, &bad[0]);
        t1 = next_tile();
        if (t1.t >= 0) {
            load_k(t1, 1);
            store_k(1);
        }
        wait_copies<0>();
        __syncthreads();
        // the first sub-tile's scores; nothing before it
#pragma unroll
        for (int s = 0; s < KR; ++s) read_k(0, 0, s);
#pragma unroll
        for (int s = 0; s < NQ; ++s) {
            s_mfma(0, s);
            if (s + KR < NQ) read_k(0, 0, s + KR);
        }
#pragma unroll
        for (int s = 0; s < KR; ++s) read_k(0, 1, s);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            pk[1][u] = u32x4{0u, 0u, 0u, 0u};
#pragma unroll
            for (int n = 0; n < DN; ++n) vf[u][n] = u32x4{0u, 0u, 0u, 0u};
        }
        for (int c = 0, kbuf = 0;; ++c) {
            const int knext = kbuf + 1 == NKB ? 0 : kbuf + 1, kfree = NKB == 2 ? kbuf : knext + 1 == NKB ? 0 : knext + 1;
            const int even = c & 1;
            uint64_t* const word = &bad[c & 3];
            // the tiles to read are in LDS for every wave, and the other buffers free
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            wait_copies<0>();
            __syncthreads();
            if (!PAGED && !block.has(t0.t)) {
                scan(even, word);
                __syncthreads();
            }
            if (tid == 0) bad[(c + 3) & 3] = 0;
            t2 = t1.t >= 0 ? next_tile() : none;
            if (t1.t >= 0) load_v(t1, even ^ 1);
            if (t2.t >= 0) load_k(t2, kfree);
            const bool end = !whole.has(t0.t) || (!block.has(t0.t) && *word != 0);
            // (zero and infinities times it stay that)
            const float ct = PAGED ? __builtin_amdgcn_fmed3f(a.c * t0.ks, __FLT_MIN__, __FLT_MAX__) : a.c;
            if (live) {   // (waves without rows copy tiles for the others)
                step(c0, even * G::kTileBytes, kbuf * G::kTileBytes, knext * G::kTileBytes, end, t0.t * TK, word, ct);
                step(c1, even * G::kTileBytes, kbuf * G::kTileBytes, knext * G::kTileBytes, end, t0.t * TK + 32, word, ct);
            }
            if (t1.t < 0) break;
            store_v(t1, even ^ 1, &bad[(c + 1) & 3]);
            if (t2.t >= 0) store_k(kfree);
            t0 = t1;
            t1 = t2;
            kbuf = knext;
        }
#pragma unroll
        for (int h = 0; h < NP; ++h) o_mfma(1, h);
    }
    if (__any(spoiled)) {
        for (int at = i_begin; at < i_end; ++at) {
            const int t = tiles.at(at);
            if (block.has(t)) continue;   // (of these the values went into the products)
            const char* vt = Vb + (long long)t * TK * row_bytes;
            if constexpr (PAGED) {
                const int page = a.table[(size_t)b * a.slots + t];
                if (page < 0 || page >= a.pages) continue;
                vt = a.v + ((size_t)page * a.Hk + hk) * TK * D;
            }
            const long long bytes = PAGED ? D : row_bytes;
            for (int k = 0; k < TK; k += 32)
                span_add_bad<ET, PAGED, DN>(acc, vt + k * bytes, bytes, span_seen(t * TK + k, hi, lo, sinks), D, half);
        }
    }

    float sum;
    if constexpr (G::kOnes) {
        const float own = D == DP ? acc[DN - 1][8] : acc[DN - 1][4];   // column D, row 16 or 8 of the tile: lanes below 32
        const float other = half_partner(own, half);
        sum = half ? other : own;
    } else {
        sum = half_sum(l);
    }
    const bool far = span_far(worst, m);
    if (const uint32_t again = (uint32_t)__ballot(valid && far); __builtin_expect(again != 0, 0)) span_tile_again<ET, DP, NW, PAGED>(again, wave);
    if (!valid || far) return;
    if (a.splits > 1) {
        const size_t at = ((size_t)split * a.B * a.Hk + bh) * R + row;
        float* const o = a.part + at * D;
#pragma unroll
        for (int n = 0; n < DN; ++n)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                if (32 * n + 8 * g < D)
                    *(f32x4*)(o + 32 * n + 8 * g + 4 * half) = f32x4{acc[n][4 * g], acc[n][4 * g + 1], acc[n][4 * g + 2], acc[n][4 * g + 3]};
        if (half == 0) {
            float* const ml = a.part + (size_t)a.splits * a.B * a.Hk * R * D + at * 2;
            ml[0] = m;
            ml[1] = sum;
        }
        return;
    }
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;   // 0 where no key is seen
    uint16_t* const o = a.out + b * a.ob + head * a.oh + token * a.ol;
#pragma unroll
    for (int n = 0; n < DN; ++n)
#pragma unroll
        for (int g = 0; g < 4; ++g)
            if (32 * n + 8 * g < D)
                *(u32x2*)(o + 32 * n + 8 * g + 4 * half) = u32x2{pack2<ET>(acc[n][4 * g] * inv, acc[n][4 * g + 1] * inv),
                                                                pack2<ET>(acc[n][4 * g + 2] * inv, acc[n][4 * g + 3] * inv)};
}

template <int ET, int DP, int NW, bool PAGED>
hipError_t launch_span_tile(const SpanKernel& a, hipStream_t stream) {
    using G = SpanTile<DP, NW>;
    const long long wgs = (long long)a.B * a.Hk * a.splits * a.row_blocks;
    if (!grid_fits(wgs, G::kThreads)) return kGridTooLarge;
    auto kern = span_tile_kernel<ET, DP, NW, PAGED>;
    static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(kern),
                                                       hipFuncAttributeMaxDynamicSharedMemorySize, G::kLdsBytes);
    if (attr != hipSuccess) return attr;
    hipLaunchKernelGGL(kern, dim3((unsigned)wgs), dim3(G::kThreads), G::kLdsBytes, stream, a);
    return hipGetLastError();
}

// ---------------------------------------------------------------- choice

template <int ET, bool PAGED, int... I>
hipError_t span_dispatch(const SpanKernel& a, hipStream_t stream, std::integer_sequence<int, I...>) {
    hipError_t r = hipErrorInvalidValue;
    const int dp = (a.D + 15) / 16 * 16;
    ((dp == 32 + 16 * I ? (void)(r = launch_span_tile<ET, 32 + 16 * I, span_block(32 + 16 * I, PAGED) / 32, PAGED>(a, stream)) : (void)0), ...);
    return r;
}
using SpanWidths = std::make_integer_sequence<int, 9>;   // 32, 48, ..., 160

}  // namespace

}  // namespace sdattn
