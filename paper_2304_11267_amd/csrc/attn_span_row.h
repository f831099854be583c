// attn_span_row.h -- the attention of attn_span.h in blocks of at most 32 rows of a key head (the query heads of one
// new token, or of a few), for calls that have a CU for each block.
//
// What counts is reading the visible keys and values once.  A workgroup takes one block, or a
// part of its keys, and each of its waves every eighth tile of 32 of them (wide heads: every fourth or third),
// through a ring of LDS buffers of its own: direct global->LDS copies of the tiles to come are in flight while one is used, and no
// wave waits for another before the end.  The page and the scales of a wave's tiles lie in its
// lanes, 64 tiles at a time.  Codes stay codes in LDS; a lane turns the 8 that it needs for a matrix product
// into 16-bit values on their way there (4 instructions), V's through the transposing read of bytes
// (ds_read_b64_tr_b8).  Rows past R are columns of the products that nobody looks at: the matrix core has
// time for them.  At the end the waves' parts are joined through LDS.  One token of eight sequences of 11000 to 32768
// keys in pages, 32 heads of 128 over 8: 79 us and a join of 4.8, 4.8 TB/s where a copy reaches 5.14; a token of 16
// windows of 1088 16-bit keys, D = 64, 4 key heads: 8.6, a launch and a chain of five tiles a wave on 64
// CUs; two prompts of 77 in pages, D = 40: 5.2.
#pragma once

#include "attn_span.h"

namespace sdattn {

namespace {

constexpr int kRowKeys = 32;       // keys of a tile

template <int D, bool PAGED>
struct SpanRow {
    static constexpr int kElem = PAGED ? 1 : 2;
    static constexpr int kRowBytes = D * kElem;
    // 16-byte chunks of a row (with D % 16 == 8 pages' rows do not begin at one: they lie as they come)
    static constexpr bool kChunks = kRowBytes % 16 == 0;
    static constexpr int KC = kRowBytes / 16;
    static constexpr int kLow = kChunks ? KC & -KC : 1;
    static constexpr int kSwap = kLow > 16 ? 16 : kLow;
    static constexpr int DK = (D + 15) / 16;
    static constexpr int DN = (D + 31) / 32;
    static constexpr int kTileBytes = kRowKeys * kRowBytes;          // of K, and of V
    static constexpr int kCopies = (kTileBytes + 1023) / 1024;       // 1 KB each
    static constexpr int kBufBytes = 2 * kCopies * 1024;
    static constexpr int kRoom = 160 * 1024 - 2048;
    static constexpr int kWaves = 8 * 2 * kBufBytes <= kRoom ? 8 : 4 * 2 * kBufBytes <= kRoom ? 4 : 3;
    static constexpr int kThreads = 64 * kWaves;
    static constexpr int kFit = kRoom / (kWaves * kBufBytes);
    static constexpr int kBufs = kFit > 4 ? 4 : kFit;                // tiles in LDS or on their way
    static constexpr int kRing = kBufs * kBufBytes;                  // of a wave
    static constexpr int kJoin = kSpanRows * (D + 4) * 4;            // O of a row, then m and l
    // (a read of V's last 16 columns may end past a row)
    static constexpr int lds_bytes(int waves) { return kRing + 16 > kJoin ? waves * kRing + 16 : waves * kJoin; }
    static constexpr int kAhead = (kBufs - 1) * 2 * kCopies;         // copies in flight behind a tile that is used
    static_assert(kAhead < 64, "vmcnt");
    static __device__ __forceinline__ int swap(int row) { return kSwap > 1 ? row / (16 / kSwap) & (kSwap - 1) : 0; }
    // byte of column d (a multiple of 8) of a row in a tile
    static __device__ __forceinline__ int at(int row, int d) {
        if constexpr (!kChunks) return row * kRowBytes + d * kElem;
        const int byte = d * kElem;
        return (row * KC + ((byte / 16) ^ swap(row))) * 16 + byte % 16;
    }
};

// The rows of a wave whose bits are set, by span_again: O and m, l in `parts`.
template <int ET, int D, bool PAGED>
__device__ __forceinline__ void span_row_again(uint32_t rows, int wave, float* parts) {
    const SpanAnew anew = span_anew();
    const SpanKernel& a = anew.a;
    const int item = a.row_blocks > 1 ? xcd_remap(anew.wg, gridDim.x) : anew.wg, list = item / a.splits, split = item - list * a.splits;
    const int bh = list / a.row_blocks, b = bh / a.Hk, hk = bh - b * a.Hk, R = a.Lq * a.G, r0 = (list - bh * a.row_blocks) * kSpanRows;
    const SpanSeq seq = span_seq(a, b);
    const SpanTiles tiles = span_tiles(a, seq, r0 / a.G, min(min(r0 + kSpanRows - 1, R - 1) / a.G, seq.count - 1), kRowKeys);
    const int per = (tiles.count + a.splits - 1) / a.splits, first = split * per + wave, last = min(split * per + per, tiles.count);
    const int lane = lane_id();
    for (; rows; rows &= rows - 1) {
        const int j = __builtin_ctz(rows), row = r0 + j, token = min(row / a.G, seq.count - 1), head = hk * a.G + row % a.G;
        const int hi = span_hi(a, seq, token), lo = span_lo(a, hi);
        const SpanAgain x = span_again<ET, PAGED, kRowKeys>(a, b, hk, a.q + b * a.qb + head * a.qh + token * a.ql, hi, lo,
                                                            first < last ? (last - first + a.waves - 1) / a.waves : 0,
                                                            [&](int i) { return tiles.at(first + i * a.waves); });
        float* const o = parts + j * (D + 4);
#pragma unroll
        for (int c = 0; c < 3; ++c)
            if (lane + 64 * c < D) o[lane + 64 * c] = x.o[c];
        if (lane == 0) {
            o[D] = x.m;
            o[D + 1] = x.l;
        }
    }
}

template <int ET, int D, bool PAGED>
__global__ __launch_bounds__((SpanRow<D, PAGED>::kThreads)) void span_row_kernel(const SpanKernel a) {
    using G = SpanRow<D, PAGED>;
    constexpr int DK = G::DK, DN = G::DN, TK = kRowKeys, NB = G::kBufs;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const int tid = threadIdx.x;
    const int lane = lane_id(), l32 = lane & 31, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);

    // (blocks of one head on one XCD, whose L2 they share)
    const int item = a.row_blocks > 1 ? xcd_remap(blockIdx.x, gridDim.x) : (int)blockIdx.x, list = item / a.splits;
    const int split = item - list * a.splits;
    const int bh = list / a.row_blocks, b = bh / a.Hk, hk = bh - b * a.Hk;
    const SpanSeq seq = span_seq(a, b);
    const int R = a.Lq * a.G, r0 = (list - bh * a.row_blocks) * kSpanRows;
    const int token0 = r0 / a.G, token1 = min(min(r0 + kSpanRows - 1, R - 1) / a.G, seq.count - 1);
    if (token0 >= seq.count) return;
    const int row = min(r0 + l32, R - 1);
    const int token = min(row / a.G, seq.count - 1), head = hk * a.G + row % a.G;

    u32x4 qreg[DK];
#pragma unroll
    for (int s = 0; s < DK; ++s) {
        const int d0 = 16 * s + 8 * half;
        u32x4 w = {0u, 0u, 0u, 0u};
        if (d0 < D) w = *(const u32x4*)(a.q + b * a.qb + head * a.qh + token * a.ql + d0);
        if (a.neg) w ^= 0x80008000u;
        if (a.zero) w = u32x4{0u, 0u, 0u, 0u};
        qreg[s] = w;
    }

    const SpanTiles tiles = span_tiles(a, seq, token0, token1, TK);
    const SpanRun run = span_run(a, seq, token0, token1);
    const int hi = span_hi(a, seq, token), lo = span_lo(a, hi), sinks = a.sinks;
    // this split's tiles, and of these every `waves`-th
    const int per = (tiles.count + a.splits - 1) / a.splits;
    const int waves = a.waves;
    const int first = split * per + wave, last = min(split * per + per, tiles.count);
    const int left = first < last ? last - first + waves - 1 : 0;
    const int mine = waves == 1 ? left : (int)__umulhi((uint32_t)left, a.per_wave);   // left / waves
    auto tile_of = [&](int i) __attribute__((always_inline)) { return tiles.at(first + i * waves); };

    // pages: of this wave's tiles 64 k .. 64 k + 63, one a lane
    [[maybe_unused]] int pages = 0;
    [[maybe_unused]] float kss = 0.0f, vss = 0.0f;   // of K: times a.c
    auto look_up = [&](int i) __attribute__((always_inline)) {
        if constexpr (PAGED) {
            const int j = min(i + lane, mine - 1);
            const int page = a.table[(size_t)b * a.slots + tile_of(j) / (kCachePage / TK)];
            const bool there = page >= 0 && page < a.pages;
            const size_t at = (size_t)(there ? page : 0) * a.Hk + hk;
            pages = there ? page : -1;
            kss = __builtin_amdgcn_fmed3f(a.c * a.ks[at], __FLT_MIN__, __FLT_MAX__);   // (zero and infinities times it stay that)
            vss = a.vs[at];
        }
    };
    const uint32_t ring = lds_offset(smem) + wave * NB * G::kBufBytes;
    const char* const buf0 = smem + wave * NB * G::kBufBytes;
    // the next `kBufs` tiles' pages may belong to the next 64: page, scales as they were at the copy
    [[maybe_unused]] int slot_page[NB];
    float slot_ks[NB] = {}, slot_vs[NB] = {};
    auto copy = [&](int i, auto slot_c) __attribute__((always_inline)) {
        constexpr int slot = decltype(slot_c)::value;
        const int t = tile_of(i);
        const char *Kt, *Vt;
        if constexpr (PAGED) {
            if (i % 64 == 0) look_up(i);
            const int page = __builtin_amdgcn_readlane(pages, i % 64);
            slot_page[slot] = page;
            slot_ks[slot] = __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(kss), i % 64));
            slot_vs[slot] = __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(vss), i % 64));
            // (a page that is not there: some other, whose tile is left alone)
            const size_t at = (((size_t)max(page, 0) * a.Hk + hk) * kCachePage + t % (kCachePage / TK) * TK) * D;
            Kt = a.k + at;
            Vt = a.v + at;
        } else {
            const long long at = 2 * (b * a.kb + hk * a.kh + (long long)t * TK * a.kl);
            Kt = a.k + at;
            Vt = a.v + at;
        }
        const int end = seq.n - 1 - t * TK;   // 16-bit rows past the last key repeat it
#pragma unroll
        for (int p = 0; p < G::kCopies; ++p) {
            const int q = min(p * 64 + lane, G::kTileBytes / 16 - 1);   // (past the tile: its last chunk)
            uint32_t off;
            if constexpr (G::kChunks) {
                const int r = q / G::KC, c = (q - r * G::KC) ^ G::swap(r);
                off = PAGED ? r * G::kRowBytes + c * 16 : (uint32_t)min(r, end) * (uint32_t)(a.kl * 2) + c * 16;
            } else {
                off = q * 16;
            }
            copy16_to_lds(Kt, off, ring + slot * G::kBufBytes + p * 1024);
            copy16_to_lds(Vt, off, ring + slot * G::kBufBytes + (G::kCopies + p) * 1024);
        }
    };

    f32x16 acc[DN];
    float m = kSpanNone, l = 0.0f, worst = 0.0f;
    int spoiled = 0;
#pragma unroll
    for (int n = 0; n < DN; ++n)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[n][r] = 0.0f;

    // lanes' places in a tile: 8 values of K's row l32, and for V as the products' operand wants its
    // keys (key 8 (e / 4) + 4 half + e % 4 of 16 in slot e)
    int k_off[DK], v_off[DN], v_hi[DN];
#pragma unroll
    for (int s = 0; s < DK; ++s) {
        const int d0 = 16 * s + 8 * half;
        k_off[s] = G::at(l32, d0 < D ? d0 : 0);   // (past D: any values, for Q's zeros; codes are no number only where column 0 is)
    }
    {
        const int g = lane >> 4, e = lane & 15;
#pragma unroll
        for (int n = 0; n < DN; ++n) {
            if constexpr (PAGED) {
                const int key = 8 * (e >> 3) + 4 * (g >> 1) + (e >> 1 & 3);
                int d = 32 * n + 16 * (g & 1) + 8 * (e & 1);
                if (d >= D) d = 32 * n + 8 * (e & 1);   // rows of O^T that are not stored
                if (d >= D) d = 0;
                v_off[n] = G::kCopies * 1024 + G::at(key, d);
                v_hi[n] = 0;
            } else {
                const int key = 4 * (g >> 1) + (e >> 2);
                int d = 32 * n + 16 * (g & 1) + 4 * (e & 3);
                if (d >= D) d = 32 * n + 4 * (e & 1);
                v_off[n] = G::kCopies * 1024 + G::at(key, d / 8 * 8) + d % 8 * 2;
                v_hi[n] = G::kCopies * 1024 + G::at(key + 8, d / 8 * 8) + d % 8 * 2;
            }
        }
    }

    auto use = [&](auto end_c, const char* kt, int key0, float ct, [[maybe_unused]] float vs) __attribute__((always_inline)) {
        constexpr bool END = decltype(end_c)::value;
        f32x16 st;
#pragma unroll
        for (int r = 0; r < 16; ++r) st[r] = 0.0f;
#pragma unroll
        for (int s = 0; s < DK; ++s) {
            u32x4 w;
            if constexpr (PAGED) {
                const u32x2 c = *(const u32x2*)(kt + k_off[s]);
                w = decode8<ET>(c[0], c[1], 1.0f);
            } else {
                w = *(const u32x4*)(kt + k_off[s]);
                if (16 * s + 16 > D && half) w = u32x4{0u, 0u, 0u, 0u};   // (Q's zeros there may meet an infinity of a seen key)
            }
            st = mfma32x32x16<ET>(w, qreg[s], st);
        }
        [[maybe_unused]] u32x4 hold[2] = {{~0u, ~0u, ~0u, ~0u}, {~0u, ~0u, ~0u, ~0u}};   // of 2 keys each: those that count
        if constexpr (END) {
            const uint32_t seen = span_seen(key0, hi, lo, sinks);
            span_hide(st, seen >> (4 * half));
            if (a.Lq == 1) {
                // all queries see the same: values of keys that they do not see are zeros, whatever they hold
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int k = 16 * (i >> 2) + 8 * (i >> 1 & 1) + 4 * half + 2 * (i & 1);
                    hold[i >> 2][i & 3] = (seen >> k & 1 ? 0xffffu : 0u) | (seen >> k & 2 ? 0xffff0000u : 0u);
                }
            } else {
                // values that are no numbers as zeros, and those of keys past the end; added afterwards where they are seen
                uint32_t keys = 0;
                char* const vt = (char*)kt + G::kCopies * 1024;
                if constexpr (PAGED) {
                    for (int q = lane; q < G::kTileBytes / 8; q += 64) {
                        const int r = q / (D / 8);
                        const u32x2 w = *(const u32x2*)(vt + q * 8), bad = {bad_codes(w[0]), bad_codes(w[1])};
                        if (key0 + r >= seq.n) *(u32x2*)(vt + q * 8) = u32x2{0u, 0u};
                        else if (bad[0] | bad[1]) *(u32x2*)(vt + q * 8) = w & ~bad;
                        if (bad[0] | bad[1]) keys |= 1u << r;
                    }
                } else {
                    for (int q = lane; q < G::kTileBytes / 16; q += 64) {
                        const u32x4 w = *(const u32x4*)(vt + q * 16);
                        const u32x4 bad = {bad2<ET>(w[0]), bad2<ET>(w[1]), bad2<ET>(w[2]), bad2<ET>(w[3])};
                        if (bad[0] | bad[1] | bad[2] | bad[3]) {
                            *(u32x4*)(vt + q * 16) = w & ~bad;
                            keys |= 1u << (q / G::KC);
                        }
                    }
                }
#pragma unroll
                for (int o = 1; o < 64; o <<= 1) keys |= (uint32_t)__shfl_xor((int)keys, o, 64);
                if (keys & seen) spoiled = 1;
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                __builtin_amdgcn_wave_barrier();
            }
        }
        float mx = st[0];
#pragma unroll
        for (int r = 1; r < 16; ++r) mx = fmaxf(mx, st[r]);
        mx = half_max(mx) * ct;
        if (__any(mx - m > span_limit<ET>)) {
            const float m_new = fmaxf(m, mx - span_bias<ET>);
            const float alpha = fast_exp2(m - m_new);
#pragma unroll
            for (int n = 0; n < DN; ++n)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[n][r] *= alpha;
            l *= alpha;
            m = m_new;
            worst = span_worst(worst, m);
        }
        float p[16];
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            p[r] = fast_exp2(fmaf(st[r], ct, -m));
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            u32x4 pk;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                pk[w] = pack2<ET>(p[8 * u + 2 * w], p[8 * u + 2 * w + 1]);
                l = add_pair<ET>(pk[w], l);
            }
#pragma unroll
            for (int n = 0; n < DN; ++n) {
                const int at = 16 * u * G::kRowBytes;   // (16 rows on: the same places of their chunks)
                u32x4 w;
                if constexpr (PAGED) {
                    const u32x2 c = lds_read_tr8(kt + v_off[n] + at);
                    w = decode8<ET>(c[0], c[1], vs);
                } else {
                    const u32x2 x = lds_read_tr(kt + v_off[n] + at), y = lds_read_tr(kt + v_hi[n] + at);
                    w = u32x4{x[0], x[1], y[0], y[1]};
                }
                if constexpr (END) w &= hold[u];
                acc[n] = mfma32x32x16<ET>(w, pk, acc[n]);
            }
        }
    };
    std::integral_constant<bool, false> whole_c;
    std::integral_constant<bool, true> end_c;

    auto each_slot = [&](auto f) __attribute__((always_inline)) {
        f(std::integral_constant<int, 0>{});
        f(std::integral_constant<int, 1>{});
        if constexpr (NB > 2) f(std::integral_constant<int, 2>{});
        if constexpr (NB > 3) f(std::integral_constant<int, 3>{});
    };
    each_slot([&](auto c) __attribute__((always_inline)) {
        if (decltype(c)::value < NB - 1 && decltype(c)::value < mine) copy(decltype(c)::value, c);
    });
    for (int i0 = 0; i0 < mine; i0 += NB) {
        each_slot([&](auto c) __attribute__((always_inline)) {
            constexpr int slot = decltype(c)::value;
            const int i = i0 + slot;
            if (i >= mine) return;
            // the buffer of the tile before this one is free: its reads have returned
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            if (i + NB - 1 < mine) {
                copy(i + NB - 1, std::integral_constant<int, (slot + NB - 1) % NB>{});
                wait_copies<G::kAhead>();
            } else if (NB > 2 && i + NB - 2 < mine) {
                wait_copies<(NB > 2 ? NB - 2 : 0) * 2 * G::kCopies>();
            } else if (NB > 3 && i + NB - 3 < mine) {
                wait_copies<(NB > 3 ? NB - 3 : 0) * 2 * G::kCopies>();
            } else {
                wait_copies<0>();
            }
            const int t = tile_of(i);
            if (PAGED && slot_page[slot] < 0) return;
            const float ct = PAGED ? slot_ks[slot] : a.c;
            if (run.all(t * TK, TK)) use(whole_c, buf0 + slot * G::kBufBytes, t * TK, ct, slot_vs[slot]);
            else use(end_c, buf0 + slot * G::kBufBytes, t * TK, ct, slot_vs[slot]);
        });
    }

    if (__any(spoiled)) {
        for (int i = 0; i < mine; ++i) {
            const int t = tile_of(i);
            if (run.all(t * TK, TK)) continue;   // (of these the values went into the products)
            const char* vt = a.v + 2 * (b * a.kb + hk * a.kh + (long long)t * TK * a.kl);
            if constexpr (PAGED) {
                const int page = a.table[(size_t)b * a.slots + t / (kCachePage / TK)];
                if (page < 0 || page >= a.pages) continue;
                vt = a.v + (((size_t)page * a.Hk + hk) * kCachePage + t % (kCachePage / TK) * TK) * D;
            }
            span_add_bad<ET, PAGED, DN>(acc, vt, PAGED ? D : 2 * a.kl, span_seen(t * TK, hi, lo, sinks), D, half);
        }
    }

    // ---- the waves' parts: O [row][D], then m, l
    constexpr int kO = D + 4;
    l = half_sum(l);
    __syncthreads();   // every wave is done with its buffers
    float* const parts = (float*)smem;
    if (r0 + l32 < R) {
        float* const o = parts + (wave * kSpanRows + l32) * kO;
#pragma unroll
        for (int n = 0; n < DN; ++n)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                if (32 * n + 8 * g < D)
                    *(f32x4*)(o + 32 * n + 8 * g + 4 * half) = f32x4{acc[n][4 * g], acc[n][4 * g + 1], acc[n][4 * g + 2], acc[n][4 * g + 3]};
        if (half == 0) {
            o[D] = m;
            o[D + 1] = l;
        }
    }
    if (const uint32_t again = (uint32_t)__ballot(span_far(worst, m) && r0 + l32 < R); __builtin_expect(again != 0, 0))
        span_row_again<ET, D, PAGED>(again, wave, parts + wave * kSpanRows * kO);
    __syncthreads();
    const size_t rows = (size_t)a.B * a.Hk * R;
    for (int z = tid; z < min(R - r0, kSpanRows) * (D / 4); z += 64 * waves) {
        const int r = z / (D / 4), d = (z - r * (D / 4)) * 4, tk = (r0 + r) / a.G;
        if (tk >= seq.count) break;   // (rows of later tokens follow)
        const float* const o = parts + r * kO;
        float top = kSpanNone, sum = 0.0f;
        f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
        auto highest = [&](int w) __attribute__((always_inline)) { top = fmaxf(top, o[w * kSpanRows * kO + D]); };
        auto add = [&](int w) __attribute__((always_inline)) {
            const float* const ow = o + w * kSpanRows * kO;
            const float f = fast_exp2(ow[D] - top);
            sum = fmaf(ow[D + 1], f, sum);
            const f32x4 x = *(const f32x4*)(ow + d);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = fmaf(x[e], f, v[e]);
        };
        if (waves == G::kWaves) {
#pragma unroll
            for (int w = 0; w < G::kWaves; ++w) highest(w);
#pragma unroll
            for (int w = 0; w < G::kWaves; ++w) add(w);
        } else {
            for (int w = 0; w < waves; ++w) highest(w);
            for (int w = 0; w < waves; ++w) add(w);
        }
        if (a.splits > 1) {
            const size_t at = (split * rows + (size_t)bh * R + r0 + r);
            *(f32x4*)(a.part + at * D + d) = v;
            if (d == 0) {
                float* const ml = a.part + a.splits * rows * D + at * 2;
                ml[0] = top;
                ml[1] = sum;
            }
        } else {
            const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
            *(u32x2*)(a.out + b * a.ob + (hk * a.G + r0 + r - tk * a.G) * a.oh + tk * a.ol + d) =
                u32x2{pack2<ET>(v[0] * inv, v[1] * inv), pack2<ET>(v[2] * inv, v[3] * inv)};
        }
    }
}

template <int ET, int D, bool PAGED>
hipError_t launch_span_row_d(const SpanKernel& a, hipStream_t stream) {
    using G = SpanRow<D, PAGED>;
    const long long wgs = (long long)a.B * a.Hk * a.row_blocks * a.splits;
    if (!grid_fits(wgs, G::kThreads)) return kGridTooLarge;
    // With more workgroups than CUs no more waves than there are tiles, or than a join of 16 values a thread takes, where
    // two workgroups then fit a CU (a token of 64 sequences of 8 heads, one tile, D = 64: 9.9 -> 6.2 us; 8 tokens of 64
    // sequences, 64 heads over 16, one tile, D = 128 32 -> 20).
    SpanKernel k = a;
    k.waves = G::kWaves;
    if (wgs > kCus) {
        const int rows = a.Lq * a.G < kSpanRows ? a.Lq * a.G : kSpanRows, join = (rows * (D / 4) + 255) / 256;
        const int need = a.part_tiles > join ? a.part_tiles : join;
        if (need < k.waves && G::lds_bytes(need) <= 80 * 1024) k.waves = need;
    }
    k.per_wave = (uint32_t)(((1ull << 32) + k.waves - 1) / k.waves);   // (exact up to 2^29 tiles)
    auto kern = span_row_kernel<ET, D, PAGED>;
    static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(kern),
                                                       hipFuncAttributeMaxDynamicSharedMemorySize, G::lds_bytes(G::kWaves));
    if (attr != hipSuccess) return attr;
    hipLaunchKernelGGL(kern, dim3((unsigned)wgs), dim3(64 * k.waves), G::lds_bytes(k.waves), stream, k);
    return hipGetLastError();
}

template <int ET, bool PAGED, int... I>
hipError_t span_row_dispatch(const SpanKernel& a, hipStream_t stream, std::integer_sequence<int, I...>) {
    hipError_t r = hipErrorInvalidValue;
    ((a.D == kSpanMinD + 8 * I ? (void)(r = launch_span_row_d<ET, kSpanMinD + 8 * I, PAGED>(a, stream)) : (void)0), ...);
    return r;
}
using SpanRowWidths = std::make_integer_sequence<int, (kSpanMaxD - kSpanMinD) / 8 + 1>;

}  // namespace

}  // namespace sdattn
