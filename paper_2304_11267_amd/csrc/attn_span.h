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

#include "attn_span_seq.h"

namespace sdattn {

namespace {

constexpr int kSpanTile = 64;          // keys of a tile: a page of the cache
// The exponent's reference m is moved when a weight would pass 2^kSpanLimit, to kSpanBias
// below the largest score: weights near 2^8 keep fp16's small ones above its subnormals' end,
// and few tiles move it (fp16 holds values below 2^16).
constexpr float kSpanBias = 8.0f;
constexpr float kSpanLimit = 15.0f;

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

// whether any of 8 16-bit values is infinite or no number
template <int ET>
__device__ __forceinline__ bool bad8(u32x4 w) {
    constexpr uint32_t kInf = ET == kF16 ? 0x7c00u : 0x7f80u;
    bool bad = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) bad = bad || (w[i] & kInf) == kInf || (w[i] & (kInf << 16)) == (kInf << 16);
    return bad;
}

// ---------------------------------------------------------------- the tiled kernel

// Workgroups of 4 waves of 32 rows; K and V tiles of 64 keys as 16-bit values in two LDS
// buffers each, rows of DP values whose 16-byte chunks lie permuted where rows would share
// banks (chunk c of row r in the place of c ^ swap(r)).
template <int DP>
struct SpanTile {
    static constexpr int kWaves = 4, kThreads = 64 * kWaves, kRows = 32 * kWaves;
    static constexpr int KC = DP / 8;                          // chunks of a row
    static constexpr int kLow = KC & -KC;
    static constexpr int kSwap = kLow > 16 ? 16 : kLow;
    static constexpr int DK = DP / 16;                         // 16-deep steps of S
    static constexpr int DN = (DP + 31) / 32;                  // 32-row tiles of O^T
    static constexpr int kTileBytes = kSpanTile * DP * 2;
    static constexpr int kBufBytes = 2 * kTileBytes;
    static constexpr int kLdsBytes = 2 * kBufBytes + 32;       // and three words of keys
    static constexpr int kWavesPerSimd = 2 * kLdsBytes <= 160 * 1024 ? 2 : 1;
    static __device__ __forceinline__ int swap(int row) { return kSwap > 1 ? row / (16 / kSwap) & (kSwap - 1) : 0; }
};

template <int ET, int DP, bool PAGED>
__global__ __launch_bounds__(SpanTile<DP>::kThreads, SpanTile<DP>::kWavesPerSimd) void span_tile_kernel(const SpanKernel a) {
    using G = SpanTile<DP>;
    constexpr int DK = G::DK, DN = G::DN, KC = G::KC, TK = kSpanTile;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const int tid = threadIdx.x;
    const int lane = lane_id(), l32 = lane & 31, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int D = a.D;

    int item = xcd_remap(blockIdx.x, gridDim.x);
    const int rb = a.row_blocks - 1 - item % a.row_blocks;   // the last rows, which see most, first
    item /= a.row_blocks;
    const int split = item % a.splits;
    const int bh = item / a.splits, b = bh / a.Hk, hk = bh - b * a.Hk;
    const SpanSeq seq = span_seq(a, b);
    const int R = a.Lq * a.G, r0 = rb * G::kRows;
    // tokens of this block and of this wave, the ones past `count` left out
    const int token0 = r0 / a.G, token1 = min((r0 + G::kRows - 1) / a.G, seq.count - 1);
    if (token0 >= seq.count) return;
    const int w0 = r0 + 32 * wave;
    const int wtoken0 = w0 / a.G, wtoken1 = min((w0 + 31) / a.G, seq.count - 1);
    const bool idle = wtoken0 >= seq.count;
    const SpanTiles tiles = span_tiles(a, seq, token0, token1, TK);
    const SpanRun block = span_run(a, seq, token0, token1);
    const SpanRun run = span_run(a, seq, min(wtoken0, token1), wtoken1);
    // this lane's row
    const int row = w0 + l32;
    const int token = min(row / a.G, seq.count - 1), head = hk * a.G + row % a.G;
    const bool valid = row / a.G < seq.count && row < R;
    const int hi = span_hi(a, seq, token), lo = span_lo(a, hi), sinks = a.sinks;

    // this split's tiles
    const int per = (tiles.count + a.splits - 1) / a.splits;
    int i = split * per;
    const int i_end = min(i + per, tiles.count);

    u32x4 qreg[DK];
#pragma unroll
    for (int s = 0; s < DK; ++s) {
        const int d0 = 16 * s + 8 * half;
        u32x4 w = {0u, 0u, 0u, 0u};
        if (valid && d0 < D) w = *(const u32x4*)(a.q + b * a.qb + head * a.qh + token * a.ql + d0);
        if (a.neg) w ^= 0x80008000u;   // a negative scale (exact)
        qreg[s] = w;
    }

    // ---- tiles into LDS
    const uint32_t lds0 = lds_offset(smem);
    // keys whose V is no number, of this tile, the next one and the one after that: a word is
    // cleared two tiles before it is written, so that no barrier is needed for it
    uint64_t* const bad = (uint64_t*)(smem + 2 * G::kBufBytes);
    // 16-bit tensors: 1 KB copies, 2 KC of them over the waves; a lane's chunk in its row
    constexpr int kCopies = (2 * KC + G::kWaves - 1) / G::kWaves;
    [[maybe_unused]] const char* Kb = nullptr;
    [[maybe_unused]] const char* Vb = nullptr;
    // pages: pieces of 16 codes over the threads
    constexpr int kPieces = (DP + 63) / 64;
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
            for (int z = tid; z < 2 * G::kBufBytes / 16; z += G::kThreads) *(u32x4*)(smem + z * 16) = u32x4{0u, 0u, 0u, 0u};
        }
    } else {
        Kb = a.k + 2 * (b * a.kb + hk * a.kh);
        Vb = a.v + 2 * (b * a.kb + hk * a.kh);
    }
    if (tid < 3) bad[tid] = 0;
    __syncthreads();

    // the page of tile t, or -1
    auto page_of = [&](int t) __attribute__((always_inline)) -> int {
        const int page = __builtin_amdgcn_readfirstlane(a.table[(size_t)b * a.slots + t]);
        return page >= 0 && page < a.pages ? page : -1;
    };
    // the next tile from place i on that has a page; its place in *at
    auto next_tile = [&](int from, int* page) __attribute__((always_inline)) -> int {
        *page = 0;
        if constexpr (PAGED) {
            for (; from < i_end; ++from) {
                *page = page_of(tiles.at(from));
                if (*page >= 0) break;
            }
        }
        return from;
    };
    auto load = [&](int t, int page, int buf) __attribute__((always_inline)) {
        if constexpr (PAGED) {
            const size_t at = ((size_t)page * a.Hk + hk) * TK * D;
#pragma unroll
            for (int p = 0; p < kPieces; ++p) {
                if (place[p][0] >= 0) {
                    kraw[p] = *(const u32x4*)(a.k + at + (p * G::kThreads + tid) * 16);
                    vraw[p] = *(const u32x4*)(a.v + at + (p * G::kThreads + tid) * 16);
                }
            }
        } else {
            const char *Kt = Kb + (long long)t * TK * a.kl * 2, *Vt = Vb + (long long)t * TK * a.kl * 2;
            const int last = seq.n - 1 - t * TK;   // keys past the last one repeat it
#pragma unroll
            for (int p = 0; p < kCopies; ++p) {
                const int ci = wave + p * G::kWaves;
                if (ci < 2 * KC) {
                    const bool isv = ci >= KC;
                    const int q = (isv ? ci - KC : ci) * 64 + lane, r = q / KC;
                    int c = (q - r * KC) ^ G::swap(r);
                    if (DP != D) c = min(c, D / 8 - 1);
                    copy16_to_lds(isv ? Vt : Kt, (uint32_t)min(r, last) * (uint32_t)(a.kl * 2) + c * 16,
                                  lds0 + buf * G::kBufBytes + ci * 1024);
                }
            }
        }
    };
    // pages: the codes read by load as 16-bit values (V times its scale) in buffer `buf`
    auto store = [&](int t, float vscale, int buf, uint64_t* word) __attribute__((always_inline)) {
        if constexpr (PAGED) {
            char* const kt = smem + buf * G::kBufBytes;
            char* const vt = kt + G::kTileBytes;
            const bool edge = !block.all(t * TK, TK);
#pragma unroll
            for (int p = 0; p < kPieces; ++p)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    if (place[p][e] < 0) continue;
                    uint32_t lo4 = vraw[p][2 * e], hi4 = vraw[p][2 * e + 1];
                    *(u32x4*)(kt + place[p][e]) = decode8<ET>(kraw[p][2 * e], kraw[p][2 * e + 1], 1.0f);
                    if (edge) {
                        const int r = place[p][e] / (KC * 16);
                        // a code that is no number: 0x7f or 0xff
                        const uint64_t w = lo4 | (uint64_t)hi4 << 32, n7 = (w & 0x7f7f7f7f7f7f7f7full) + 0x0101010101010101ull;
                        const bool nan = (n7 & 0x8080808080808080ull) != 0;
                        if (nan || t * TK + r >= seq.n) lo4 = hi4 = 0;
                        if (nan) atomicOr((unsigned long long*)word, 1ull << r);
                    }
                    *(u32x4*)(vt + place[p][e]) = decode8<ET>(lo4, hi4, vscale);
                }
        }
    };
    // 16-bit tensors: chunks of V in an end tile that hold no number, as zeros, with their keys
    auto scan = [&](int buf, uint64_t* word) __attribute__((always_inline)) {
        char* const vt = smem + buf * G::kBufBytes + G::kTileBytes;
        for (int q = tid; q < TK * KC; q += G::kThreads) {
            if (bad8<ET>(*(const u32x4*)(vt + q * 16))) {
                *(u32x4*)(vt + q * 16) = u32x4{0u, 0u, 0u, 0u};
                atomicOr((unsigned long long*)word, 1ull << (q / KC));
            }
        }
    };

    // ---- per-lane places in a buffer (as in attn_fwd_kernel.h)
    int k_off[DK], v_off[DN], v_hi[DN];
#pragma unroll
    for (int s = 0; s < DK; ++s) k_off[s] = (l32 * KC + ((2 * s + half) ^ G::swap(l32))) * 16;
    {
        const int g = lane >> 4, e = lane & 15;
        const int key = 4 * (g >> 1) + (e >> 2);
#pragma unroll
        for (int n = 0; n < DN; ++n) {
            int d = 32 * n + 16 * (g & 1) + 4 * (e & 3);
            if (d >= DP) d -= 16;   // rows of O^T that are not stored
            v_off[n] = G::kTileBytes + (key * KC + ((d / 8) ^ G::swap(key))) * 16 + d % 8 * 2;
            v_hi[n] = G::kTileBytes + ((key + 8) * KC + ((d / 8) ^ G::swap(key + 8))) * 16 + d % 8 * 2;
        }
    }

    f32x16 acc[DN];
    float m = kSpanNone, l = 0.0f;
    int spoiled = 0;   // this lane's query sees a value that is no number
#pragma unroll
    for (int n = 0; n < DN; ++n)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[n][r] = 0.0f;

    // S^T = K Q^T, p = 2^(c s - m), O^T += V^T P^T for the tile at `key0` in buffer `buf`;
    // ct = c times the page's scale
    auto consume = [&](auto end_c, int buf, int key0, float ct, const uint64_t* word) __attribute__((always_inline)) {
        constexpr bool END = decltype(end_c)::value;
        const char* const kt = smem + buf * G::kBufBytes;
        f32x16 st[2];
#pragma unroll
        for (int sub = 0; sub < 2; ++sub) {
#pragma unroll
            for (int r = 0; r < 16; ++r) st[sub][r] = 0.0f;
#pragma unroll
            for (int s = 0; s < DK; ++s)
                st[sub] = mfma32x32x16<ET>(*(const u32x4*)(kt + k_off[s] + 32 * sub * KC * 16), qreg[s], st[sub]);
        }
        uint32_t seen = ~0u;
        if constexpr (END) {
            seen = 0;
#pragma unroll
            for (int sub = 0; sub < 2; ++sub)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int key = key0 + 32 * sub + 8 * (r >> 2) + 4 * half + (r & 3);
                    const bool in = key < hi && (key >= lo || key < sinks);
                    seen |= in ? 1u << (16 * sub + r) : 0u;
                    if (!in) st[sub][r] = -__builtin_inff();
                }
        }
        float mx = fmaxf(st[0][0], st[1][0]);
#pragma unroll
        for (int r = 1; r < 16; ++r) mx = fmaxf(mx, fmaxf(st[0][r], st[1][r]));
        mx = half_max(mx);
        mx = mx == -__builtin_inff() ? mx : mx * ct;   // (ct may be 0)
        if (__any(mx - m > kSpanLimit)) {
            const float m_new = fmaxf(m, mx - kSpanBias);
            const float alpha = fast_exp2(m - m_new);
#pragma unroll
            for (int n = 0; n < DN; ++n)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[n][r] *= alpha;
            l *= alpha;
            m = m_new;
        }
        u32x4 pk[2][2];
#pragma unroll
        for (int sub = 0; sub < 2; ++sub) {
            float p[16];
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                p[r] = fast_exp2(fmaf(st[sub][r], ct, -m));
                if (END) p[r] = seen >> (16 * sub + r) & 1 ? p[r] : 0.0f;
            }
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    pk[sub][u][w] = pack2<ET>(p[8 * u + 2 * w], p[8 * u + 2 * w + 1]);
                    l = add_pair<ET>(pk[sub][u][w], l);
                }
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int n = 0; n < DN; ++n) {
                    const int at = (32 * sub + 16 * u) * KC * 16;
                    const u32x2 x = lds_read_tr(kt + v_off[n] + at), y = lds_read_tr(kt + v_hi[n] + at);
                    acc[n] = mfma32x32x16<ET>(u32x4{x[0], x[1], y[0], y[1]}, pk[sub][u], acc[n]);
                }
        }
        if constexpr (END) {
            const uint64_t keys = *word;
            if (keys) {   // a query that sees one of them has no number to give
#pragma unroll
                for (int sub = 0; sub < 2; ++sub)
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if ((seen >> (16 * sub + r) & 1) && (keys >> (32 * sub + 8 * (r >> 2) + 4 * half + (r & 3)) & 1))
                            spoiled = 1;
            }
        }
    };
    std::integral_constant<bool, false> whole_c;
    std::integral_constant<bool, true> end_c;

    int page = 0;
    i = next_tile(i, &page);
    int buf = 0, now = 0;   // buffer and word of this tile
    float kscale = 1.0f, vscale = 1.0f;
    auto scales = [&](int page) __attribute__((always_inline)) {
        if constexpr (PAGED) {
            kscale = a.ks[(size_t)page * a.Hk + hk];
            vscale = a.vs[(size_t)page * a.Hk + hk];
        }
    };
    if (i < i_end) {
        load(tiles.at(i), page, 0);
        scales(page);
        store(tiles.at(i), vscale, 0, &bad[0]);
    }
    while (i < i_end) {
        const int t = tiles.at(i);
        const float ct = a.c * kscale;
        // this tile is in LDS for every wave, and the other buffer free
        wait_copies<0>();
        __syncthreads();
        const int next = now == 2 ? 0 : now + 1, after = next == 2 ? 0 : next + 1;
        if (tid == 0) bad[after] = 0;
        const bool block_end = !block.all(t * TK, TK);
        if (!PAGED && block_end) {
            scan(buf, &bad[now]);
            __syncthreads();
        }
        i = next_tile(i + 1, &page);
        if (i < i_end) {
            load(tiles.at(i), page, buf ^ 1);
            scales(page);
        }
        if (!idle && !run.none(t * TK, TK)) {
            if (run.all(t * TK, TK)) {
                consume(whole_c, buf, t * TK, ct, &bad[now]);
                if (block_end && bad[now] != 0) spoiled = 1;   // (its queries see all of the tile)
            } else {
                consume(end_c, buf, t * TK, ct, &bad[now]);
            }
        }
        if (PAGED && i < i_end) store(tiles.at(i), vscale, buf ^ 1, &bad[next]);
        buf ^= 1;
        now = next;
    }

    if (idle) return;
    const float sum = half_sum(l);
    // (this file's floats are taken for numbers by the compiler: no number is made of bits)
    spoiled |= __shfl_xor(spoiled, 32, 64);
    if (a.splits > 1) {
        if (!valid) return;
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
            ((uint32_t*)ml)[1] = spoiled ? 0x7fc00000u : __float_as_uint(sum);
        }
        return;
    }
    if (!valid) return;
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;   // 0 where no key is seen
    const uint32_t nan = spoiled ? 0x7fff7fffu : 0u;     // (no number in both types)
    uint16_t* const o = a.out + b * a.ob + head * a.oh + token * a.ol;
#pragma unroll
    for (int n = 0; n < DN; ++n)
#pragma unroll
        for (int g = 0; g < 4; ++g)
            if (32 * n + 8 * g < D)
                *(u32x2*)(o + 32 * n + 8 * g + 4 * half) = u32x2{pack2<ET>(acc[n][4 * g] * inv, acc[n][4 * g + 1] * inv) | nan,
                                                                pack2<ET>(acc[n][4 * g + 2] * inv, acc[n][4 * g + 3] * inv) | nan};
}

template <int ET, int DP, bool PAGED>
hipError_t launch_span_tile(const SpanKernel& a, hipStream_t stream) {
    using G = SpanTile<DP>;
    const long long wgs = (long long)a.B * a.Hk * a.splits * a.row_blocks;
    if (!grid_fits(wgs, G::kThreads)) return kGridTooLarge;
    auto kern = span_tile_kernel<ET, DP, PAGED>;
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
    ((dp == 32 + 16 * I ? (void)(r = launch_span_tile<ET, 32 + 16 * I, PAGED>(a, stream)) : (void)0), ...);
    return r;
}
using SpanWidths = std::make_integer_sequence<int, 9>;   // 32, 48, ..., 160

}  // namespace

}  // namespace sdattn
