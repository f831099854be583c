// linear.hip -- the projections around the attention in SD's transformer
// blocks: y = x w^T + bias with weights stored [out, in], and the head
// split / merge folded into the addressing of the rows.
//
// A token row m = b*L + l of x (or y) lives either in rows layout [B, L, C]
// or in heads layout [B, H, L, C/H] (channel c = h*(C/H) + d at
// ((b*H + h)*L + l)*(C/H) + d).  Writing Q, K and V in heads layout is the
// head split before Eq. 3; reading O in heads layout is the head merge before
// the output projection -- neither needs a transpose of its own.
//
// Two kernels: linear_kernel shares 128x64 tiles among a workgroup's waves
// (below); linear_ksplit_kernel, for few tiles or few token rows, splits the
// reduced dimension over them (launch_group_e has the rule).
//
// One launch may carry up to three independent products (the block's Q, K
// and V projections, whose inputs differ for cross-attention), each possibly
// a batch of equal-sized products at fixed strides (the 36 products of a
// Winograd convolution); each workgroup finds its product and batch item
// from its tile index, so the small context projections run beside the
// large latent one instead of after it.
//
// Workgroup tile: 128 token rows x 64 output channels, four waves of 32 rows.
// Each 64-channel slice of the x and w tiles is copied global -> LDS with
// global_load_lds (16 bytes per lane, whole 128-byte rows per instruction,
// no registers), into a ring of kStages slices so that kStages - 1 copies are
// in flight while one slice is multiplied.  Inside a slice, row r's 16-byte
// chunk c sits at chunk position c ^ swz(r), which keeps the MFMA operand
// reads (ds_read_b128, one row per lane) free of bank conflicts.  The product
// runs as y^T = w x^T on 32x32x16 MFMAs: A = 32 weight rows x 16 channels,
// B = 16 channels x 32 token rows, one token row per lane; each lane ends with
// 4 consecutive output channels per register group; the tile goes out through
// LDS so that each lane stores 16 contiguous bytes.
//
// Low-rank adapters of many requests ride beside the shared product: row m of batch
// item b adds s_i up_i (down_i x_m), i = ids[b], in one of two ways (launch_adapters_e).
// AdapterFused, ranks up to 32 and requests of 32 rows and more (not of many rows and
// many channels): tiles of one request
// each, whose slices carry the 16 or 32 rows of down_i beside those of w, so that x is read
// once and T = s_i down_i x ends in the registers that the last product, up_i T, takes.
// AdapterSet, all others: a first launch (adapter_down_kernel) writes T, and both kernels
// above add T up_i^T to the rows of each request.
#include "device.h"
#include "launch.h"

namespace sdattn {

namespace {

constexpr int kBM = 128;                          // token rows per workgroup
constexpr int kBN = 64;                           // output channels per workgroup
constexpr int kBK = 64;                           // input channels per slice
constexpr int kUnits = (kBM + kBN) * kBK / 8;     // 16-byte chunks per slice (1536)
constexpr int kSliceBytes = kUnits * 16;          // 24 KiB
constexpr int kCopies = kUnits / 64 / 4;          // copy instructions per wave per slice (6)
constexpr int kStages = 3;
constexpr int kRuns = 4;                          // partial sums over the input channels
constexpr int kSplitMinK = 512;                   // fewest channels (exclusive) summed that way
constexpr int kLdsBytes = kStages * kSliceBytes;  // 72 KiB: two workgroups per CU

struct LinProblem {
    const uint16_t* x;
    const uint16_t* w;
    const uint16_t* bias;   // null: no bias
    uint16_t* y;
    int M, K, N, L;         // M = B*L token rows
    int xhw, yhw;           // head widths of the heads layouts (1 for rows layout)
    int nnt, tile0;         // channel tiles; first tile index of this product
    int per_batch;          // tiles of one batch item
    long long sx, sw, sy;   // element strides between batch items
};
struct LinGroup {
    LinProblem p[kMaxLinearProblems];
    int n;
};

// chunk-position swizzle of row r: distinct for any 8 consecutive rows, and
// (r & 1, swz) distinct for any 16 consecutive rows
__device__ __forceinline__ int swz(int r) { return (r & 7) ^ ((r >> 3) & 1); }

// c / hw for 0 <= c < 2^16 and 8 <= hw: the fp32 quotient is within one of
// the true one, and one correction step makes it exact.
__device__ __forceinline__ int div_small(int c, int hw, float inv_hw) {
    int h = (int)((float)c * inv_hw);
    h -= (h * hw > c) ? 1 : 0;
    h += ((h + 1) * hw <= c) ? 1 : 0;
    return h;
}

// Element offset of token row m = b*L + l (channel 0, head 0) in a tensor of
// C channels, and of channel c relative to it.
template <bool HEADS>
__device__ __forceinline__ size_t row_base(int m, int L, int C, int hw) {
    if constexpr (HEADS) {
        const int b = m / L, l = m - b * L;
        return ((size_t)b * (C / hw) * L + l) * hw;
    } else {
        return (size_t)m * C;
    }
}
template <bool HEADS>
__device__ __forceinline__ size_t chan_offset(int c, int L, int hw, float inv_hw) {
    if constexpr (HEADS) {
        const int h = div_small(c, hw, inv_hw);
        return (size_t)h * L * hw + (c - h * hw);
    } else {
        return (size_t)c;
    }
}

// The adapters of a product's rows: T holds their rows' inner products.
struct AdapterSet {
    const uint16_t* t;      // [M, Rp]; rows without an adapter unwritten
    const uint16_t* up;     // [count, N, R]
    const int* ids;         // [B]: the adapter of a batch item; none outside [0, count)
    int count, R, Rp;
};
template <int RR>           // rows of down beside a slice's rows of w: 16 or 32, at least R
struct AdapterFused {
    static constexpr int kRows = RR;
    const uint16_t* down;   // [count, R, K]
    const uint16_t* up;     // [count, N, R]
    const int* ids;         // [batch items]
    const float* scales;    // [count] or null
    int count, R;
};
struct AdapterNone {};
__device__ __forceinline__ AdapterNone adapters_of() { return AdapterNone{}; }
template <typename A>
__device__ __forceinline__ A adapters_of(const A& a) { return a; }
template <typename A, typename... AD>
constexpr bool adapters_are = sizeof...(AD) == 1 && (std::is_same<A, AD>::value && ...);
template <typename... AD>
struct FusedRows {
    static constexpr int value = 0;
};
template <int RR>
struct FusedRows<AdapterFused<RR>> {
    static constexpr int value = RR;
};
template <typename... AD>
constexpr int fused_rows = FusedRows<AD...>::value;   // 0: no AdapterFused

constexpr int kFusedMaxN = 768, kFusedMaxRows = 256;   // see launch_adapters_e

// The operands of the last product of AdapterFused, Y^T += up T^T, on an MFMA of 16 ranks from
// `base` on: T^T comes as a 32x32 accumulator whose registers hold ranks 8 (r / 4) + 4 half +
// r % 4 of token l32 (with 16 rows the last 8 repeat them), so up is read in that order.
template <int ET>
__device__ __forceinline__ u32x4 fused_t(const float* t, float scale, int base, int R, int half) {
    u32x4 v;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        float f[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int r = 2 * w + e, rank = base + 8 * (r >> 2) + 4 * half + (r & 3);
            f[e] = rank < R ? t[r] * scale : 0.0f;   // (rows past R repeat the last one)
        }
        v[w] = pack2<ET>(f[0], f[1]);   // rounded to the type that the matrix core multiplies
    }
    return v;
}
__device__ __forceinline__ u32x4 fused_up(const uint16_t* row, int base, int R, int half) {
    u32x4 v = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        const int r0 = base + 8 * q + 4 * half;
        if (R % 4 == 0) {
            if (r0 < R) {
                const u32x2 w = *(const u32x2*)(row + r0);
                v[2 * q] = w[0];
                v[2 * q + 1] = w[1];
            }
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (r0 + e < R) v[2 * q + (e >> 1)] |= (uint32_t)row[r0 + e] << (16 * (e & 1));
        }
    }
    return v;
}

// Ranks r0 .. r0 + 7 of an adapter's row of R, zeros from R on, in reads of W values (R is
// a multiple of W).
template <int W>
__device__ __forceinline__ u32x4 adapter_chunk(const uint16_t* row, int r0, int R) {
    u32x4 v = {0u, 0u, 0u, 0u};
    if constexpr (W == 8) {
        if (r0 < R) v = *(const u32x4*)(row + r0);
    } else if constexpr (W == 4) {
#pragma unroll
        for (int e = 0; e < 2; ++e)
            if (r0 + 4 * e < R) {
                const u32x2 w = *(const u32x2*)(row + r0 + 4 * e);
                v[2 * e] = w[0];
                v[2 * e + 1] = w[1];
            }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (r0 + e < R) v[e >> 1] |= (uint32_t)row[r0 + e] << (16 * (e & 1));
    }
    return v;
}

// sum[g][e] = the product of T's row t with the rows of up for channels n + dn g + e: 16
// reads of up in flight.
template <int ET, int W, int NG>
__device__ __forceinline__ void adapter_dots(const uint16_t* up, const uint16_t* t, int R, int n, int dn, int N,
                                             float (&sum)[NG][4]) {
    constexpr int CH = 4 / NG;   // chunks of 8 ranks at a time
    const uint16_t* p[NG];
#pragma unroll
    for (int g = 0; g < NG; ++g) {
        p[g] = up + (size_t)min(n + dn * g, N - 4) * R;   // (groups of 4 channels end together with N)
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[g][e] = 0.0f;
    }
    for (int r0 = 0; r0 < R; r0 += 8 * CH) {
        u32x4 tf[CH], u[CH][NG][4];
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            tf[c] = u32x4{0u, 0u, 0u, 0u};
            if (r0 + 8 * c < R) tf[c] = *(const u32x4*)(t + r0 + 8 * c);
#pragma unroll
            for (int g = 0; g < NG; ++g)
#pragma unroll
                for (int e = 0; e < 4; ++e) u[c][g][e] = adapter_chunk<W>(p[g] + e * R, r0 + 8 * c, R);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int g = 0; g < NG; ++g)
#pragma unroll
                for (int e = 0; e < 4; ++e) sum[g][e] = dot8<ET>(u[c][g][e], tf[c], sum[g][e]);
    }
}
// f(W) with the widest reads that R leaves aligned
template <typename F>
__device__ __forceinline__ void adapter_width(int R, F f) {
    if (R % 8 == 0) f(std::integral_constant<int, 8>{});
    else if (R % 4 == 0) f(std::integral_constant<int, 4>{});
    else f(std::integral_constant<int, 1>{});
}

// up T^T for the token rows and channels of a tile, the last addend of their sums.  Every
// row sees its own request's adapter alone, infinities and all, and a request's bits do not
// depend on its neighbours in a tile.
//   Requests of 32 rows and more: adapter_sums, 16 ranks a step on the matrix core, one
// request's rows at a time (at most two in 32 rows), the others' T as zeros and their sums
// dropped.
//   Shorter ones: adapter_dots, each lane multiplies its row's T with its own channels' rows
// of up (16 tokens of 16 requests, K = N = 1280, R = 8: one request after the other took 9
// us more).
constexpr int kAdapterRows = 32;
constexpr int kUpSteps = 4;   // steps of 16 ranks in flight

// This lane's row's adapter, its up and its T (false: none)
__device__ __forceinline__ bool adapter_of_row(const AdapterSet& ad, int row, int M, int N, int L, const uint16_t** up,
                                               const uint16_t** t) {
    if (row >= M) return false;
    const int id = ad.ids[row / L];
    if (id < 0 || id >= ad.count) return false;
    *up = ad.up + (size_t)id * N * ad.R;
    *t = ad.t + (size_t)row * ad.Rp;
    return true;
}

// sum[b] for the 32 token rows from row0 and the 32 channels from n0 + 32 b, in the
// accumulators' layout
template <int ET, int NB, int W>
__device__ __forceinline__ void adapter_sums_w(const AdapterSet& ad, int row0, int n0, int M, int N, int L,
                                               f32x16 (&sum)[NB]) {
    const int l32 = lane_id() & 31, half = lane_id() >> 5;
    if (L < kAdapterRows) {
        const uint16_t *up, *t;
        if (!adapter_of_row(ad, row0 + l32, M, N, L, &up, &t)) return;
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                float d[2][4];
                adapter_dots<ET, W, 2>(up, t, ad.R, n0 + 32 * b + 16 * q + 4 * half, 8, N, d);
#pragma unroll
                for (int g = 0; g < 2; ++g)
#pragma unroll
                    for (int e = 0; e < 4; ++e) sum[b][8 * q + 4 * g + e] = d[g][e];
            }
        return;
    }
    const int row = min(row0 + l32, M - 1);
    const int last = min(row0 + 31, M - 1) / L;
    for (int b = row0 / L; b <= last; ++b) {
        const int id = __builtin_amdgcn_readfirstlane(ad.ids[b]);
        if (id < 0 || id >= ad.count) continue;
        const bool mine = (long long)row >= (long long)b * L && (long long)row < (long long)(b + 1) * L;
        f32x16 own[NB];
#pragma unroll
        for (int t = 0; t < NB; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) own[t][r] = 0.0f;
        const uint16_t* up[NB];
#pragma unroll
        for (int t = 0; t < NB; ++t) up[t] = ad.up + ((size_t)id * N + min(n0 + 32 * t + l32, N - 1)) * ad.R;
        for (int s0 = 0; s0 < ad.Rp / 16; s0 += kUpSteps) {
            u32x4 tf[kUpSteps], uf[kUpSteps][NB];
#pragma unroll
            for (int s = 0; s < kUpSteps; ++s) {
                const int r0 = 16 * (s0 + s) + 8 * half;   // from R on: zeros
                tf[s] = u32x4{0u, 0u, 0u, 0u};
                if (mine && r0 < ad.Rp) tf[s] = *(const u32x4*)(ad.t + (size_t)row * ad.Rp + r0);
#pragma unroll
                for (int t = 0; t < NB; ++t) uf[s][t] = adapter_chunk<W>(up[t], r0, ad.R);
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int s = 0; s < kUpSteps; ++s)
#pragma unroll
                for (int t = 0; t < NB; ++t) own[t] = mfma32x32x16<ET>(uf[s][t], tf[s], own[t]);
        }
#pragma unroll
        for (int t = 0; t < NB; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) sum[t][r] = mine ? own[t][r] : sum[t][r];
    }
}
template <int ET, int NB>
__device__ __forceinline__ void adapter_sums(const AdapterSet& ad, int row0, int n0, int M, int N, int L,
                                             f32x16 (&sum)[NB]) {
#pragma unroll
    for (int t = 0; t < NB; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) sum[t][r] = 0.0f;
    if (row0 >= M) return;
    adapter_width(ad.R, [&](auto w) __attribute__((always_inline)) {
        adapter_sums_w<ET, NB, decltype(w)::value>(ad, row0, n0, M, N, L, sum);
    });
}

// Wait until at most `ahead` slices of this wave's copies are still in flight.
template <int COPIES = kCopies>
__device__ __forceinline__ void wait_slices(int ahead) {
    static_assert(kStages == 3, "wait_slices covers ahead = 0 and 1");
    if (ahead >= 1) __builtin_amdgcn_s_waitcnt(vm_wait(COPIES));
    else __builtin_amdgcn_s_waitcnt(vm_wait(0));
}

// Workgroup barrier after this wave's LDS reads have returned.  The slice
// copies are waited for explicitly (wait_slices); a fence here would drain
// every copy still in flight, since they count as LDS writes.  The memory
// clobber keeps the compiler from moving LDS reads across the barrier.
__device__ __forceinline__ void lds_barrier() {
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// The slices of linear_kernel's ring.  With an adapter's rows in them and few channels, two: three
// workgroups then share a CU (8 requests of 4096 rows, K = N = 320, R 16: 24.2 -> 21.4 us; past
// kSplitMinK channels their registers leave room for two either way), or two with 32 such rows.
template <bool FOLD, typename... AD>
constexpr int linear_stages = (fused_rows<AD...> > 0 && !FOLD) || fused_rows<AD...> > 16 ? 2 : kStages;
template <bool FOLD, typename... AD>
constexpr int linear_lds = linear_stages<FOLD, AD...> * (kSliceBytes + fused_rows<AD...> * kBK * 2);
// AD: nothing, an AdapterSet (one product with batch 1), or an AdapterFused (one product,
// a batch item for each request)
template <int ET, bool XH, bool YH, bool FOLD, typename... AD>
__global__ __launch_bounds__(256) void linear_kernel(const LinGroup grp, const AD... ad) {
    constexpr int RR = fused_rows<AD...>;
    constexpr bool FUSED = RR > 0;
    constexpr int kSlot = kSliceBytes + RR * kBK * 2;   // of the ring
    constexpr int ST = linear_stages<FOLD, AD...>;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const int lane = lane_id();
    const int l32 = lane & 31;
    const int half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

    const int tile = xcd_remap(blockIdx.x, gridDim.x);
    const int pi = (grp.n > 2 && tile >= grp.p[2].tile0) ? 2 : (grp.n > 1 && tile >= grp.p[1].tile0) ? 1 : 0;
    const LinProblem& P = grp.p[pi];
    const int bi = (tile - P.tile0) / P.per_batch;     // batch item
    const int local = tile - P.tile0 - bi * P.per_batch;
    const uint16_t* __restrict__ X = P.x + bi * P.sx;
    const uint16_t* __restrict__ W = P.w + bi * P.sw;
    const int M = P.M, K = P.K, N = P.N, L = P.L, xhw = P.xhw;
    const int nt = local % P.nnt;        // consecutive workgroups share the token rows
    const int m0 = (local / P.nnt) * kBM;
    const int n0 = nt * kBN;
    const int nk = (K + kBK - 1) / kBK;

    // Copy j of this wave moves 16-byte chunk c of tile row r (x rows first,
    // then w rows); rows past M or N repeat the last row (their outputs are
    // never stored), channels past K repeat the last chunk (their operands are
    // zeroed before use).  Row bases are fixed across slices.
    size_t cbase[kCopies];
    int cch[kCopies];
#pragma unroll
    for (int j = 0; j < kCopies; ++j) {
        const int u0 = (wave * kCopies + j) * 64;
        const int u = u0 + lane;
        if (u0 < kBM * 8) {
            const int r = u >> 3;
            cch[j] = 8 * ((u & 7) ^ swz(r));
            cbase[j] = row_base<XH>(min(m0 + r, M - 1), L, K, xhw);
        } else {
            const int r = (u >> 3) - kBM;
            cch[j] = 8 * ((u & 7) ^ swz(r));
            cbase[j] = (size_t)min(n0 + r, N - 1) * K;
        }
    }
    const float inv_xhw = 1.0f / (float)xhw;

    // FUSED: the request's adapter (the first one's addresses where it has none), the quarter
    // of down's rows that this wave copies with 8 lanes each, and its operands of up
    [[maybe_unused]] bool adapted = false;
    [[maybe_unused]] float t_scale = 1.0f;
    [[maybe_unused]] const uint16_t* d_row = nullptr;
    [[maybe_unused]] int d_ch = 0, offd[4];
    [[maybe_unused]] u32x4 upf[RR > 0 ? RR / 16 : 1][2];
    [[maybe_unused]] int rank = 0;
    if constexpr (FUSED) {
        const auto a = adapters_of(ad...);
        const int named = __builtin_amdgcn_readfirstlane(a.ids[bi]);
        adapted = named >= 0 && named < a.count;
        const int id = adapted ? named : 0;
        rank = a.R;
        if (a.scales) t_scale = a.scales[id];
        const int r = RR / 4 * wave + (lane % (2 * RR) >> 3);
        d_ch = 8 * ((lane & 7) ^ swz(r));
        d_row = a.down + ((size_t)id * a.R + min(r, a.R - 1)) * K;
#pragma unroll
        for (int q = 0; q < RR / 16; ++q)
#pragma unroll
            for (int t = 0; t < 2; ++t)
                upf[q][t] = fused_up(a.up + ((size_t)id * N + min(n0 + 32 * t + l32, N - 1)) * a.R, 16 * q, a.R, half);
#pragma unroll
        for (int s = 0; s < 4; ++s)
            offd[s] = kSliceBytes + (l32 & (RR - 1)) * kBK * 2 + ((2 * s + half) ^ swz(l32 & (RR - 1))) * 16;
    }

    // slice i (channels 64i .. 64i + 63) into ring slot i % ST
    auto issue = [&](int i) __attribute__((always_inline)) {
        const int k0 = i * kBK;
        char* st = smem + (i % ST) * kSlot;
#pragma unroll
        for (int j = 0; j < kCopies; ++j) {
            const int u0 = (wave * kCopies + j) * 64;
            const int ch = min(k0 + cch[j], K - 8);
            const char* src = u0 < kBM * 8
                                  ? (const char*)(X + cbase[j] + chan_offset<XH>(ch, L, xhw, inv_xhw))
                                  : (const char*)(W + cbase[j] + ch);
            __builtin_amdgcn_global_load_lds(src, (lds_void_t*)(st + u0 * 16), 16, 0, 0);
        }
        if constexpr (FUSED) {
            if (lane < 2 * RR)
                __builtin_amdgcn_global_load_lds((const char*)(d_row + min(k0 + d_ch, K - 8)),
                                                 (lds_void_t*)(st + kSliceBytes + wave * (RR * 32)), 16, 0, 0);
        }
    };
    constexpr int kIssued = kCopies + (FUSED ? 1 : 0);   // copies of a wave and slice

    // operand offsets inside a slice: B = x row 32*wave + l32, A_t = w row
    // 32t + l32, chunk 2s + half for k-step s (rows 32t + l32 share swz(l32))
    const int hx = swz(l32);
    int offx[4], offw[2][4];
#pragma unroll
    for (int s = 0; s < 4; ++s) {
        const int cpos = (2 * s + half) ^ hx;
        offx[s] = ((32 * wave + l32) * 8 + cpos) * 16;
#pragma unroll
        for (int t = 0; t < 2; ++t) offw[t][s] = ((kBM + 32 * t + l32) * 8 + cpos) * 16;
    }

    // bias of this lane's output channels (8-byte aligned groups of 4),
    // fetched before the product
    const uint16_t* __restrict__ Bias = P.bias;
    u32x2 bias[2][4];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int g = 0; g < 4; ++g) bias[t][g] = u32x2{0u, 0u};
    if (Bias) {
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int n = min(n0 + 32 * t + 8 * g + 4 * half, N - 4);
                bias[t][g] = *(const u32x2*)(Bias + n);
            }
    }

    // acc += slice i (FIRST: acc = slice i); before() is issued while the slice's
    // operands come from LDS
    f32x16 zero;
#pragma unroll
    for (int r = 0; r < 16; ++r) zero[r] = 0.0f;
    [[maybe_unused]] f32x16 dacc = zero, dtot = zero;   // FUSED: T^T, as acc and tot
    // the slice's down rows at st, on the x operands of k-step s
    [[maybe_unused]] auto down_step = [&](const char* st, int s, u32x4 xf, int kval) __attribute__((always_inline)) {
        u32x4 df = *(const u32x4*)(st + offd[s]);
        if (8 * (2 * s + half) >= kval) df = u32x4{0u, 0u, 0u, 0u};
        dacc = mfma32x32x16<ET>(df, xf, dacc);
    };
    auto slice = [&](int i, auto first_c, f32x16 (&acc)[2], auto before) __attribute__((always_inline)) {
        constexpr bool FIRST = decltype(first_c)::value;
        wait_slices<kIssued>(min(nk - 1 - i, ST - 2));
        lds_barrier();   // slice i is in LDS for every wave; slot (i - 1) % ST is free
        if (i + ST - 1 < nk) issue(i + ST - 1);
        const char* st = smem + (i % ST) * kSlot;
        const int kval = K - i * kBK;    // channels of this slice inside K (uniform)
        // all twelve operand reads first, so their latencies overlap
        u32x4 bf[4], af[2][4];
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            bf[s] = *(const u32x4*)(st + offx[s]);
            af[0][s] = *(const u32x4*)(st + offw[0][s]);
            af[1][s] = *(const u32x4*)(st + offw[1][s]);
        }
        before();
        if (kval < kBK) {
#pragma unroll
            for (int s = 0; s < 4; ++s)
                if (8 * (2 * s + half) >= kval) {
                    bf[s] = u32x4{0u, 0u, 0u, 0u};
                    af[0][s] = bf[s];
                    af[1][s] = bf[s];
                }
        }
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            acc[0] = mfma32x32x16<ET>(af[0][s], bf[s], FIRST && s == 0 ? zero : acc[0]);
            acc[1] = mfma32x32x16<ET>(af[1][s], bf[s], FIRST && s == 0 ? zero : acc[1]);
        }
        if constexpr (FUSED) {
            if (FIRST) dacc = zero;
#pragma unroll
            for (int s = 0; s < 4; ++s) down_step(st, s, bf[s], kval);
        }
    };

#pragma unroll
    for (int i = 0; i < ST - 1; ++i)
        if (i < nk) issue(i);

    // With FOLD, acc sums a run of slices and tot the runs before it.  Past
    // kSplitMinK channels that is the split-K kernel's order of summation, so a
    // row has the same bits whichever kernel takes it, alone or in a batch of any
    // size; up to there the split kernel is not taken and one run does (the 64x64
    // level's convolution 27 us against 28).  The additions cost a wave that has its
    // SIMD to itself 5 clocks each, beside MFMAs too: without / with them 2048x640x640
    // 7.2 / 7.5 us (7.9 with them in the loop of every slice), 1024x1280x1280 11.3 /
    // 11.4 (12.0), 2048x2560x640 19.4 / 19.0 (20.0).
    f32x16 acc[2] = {zero, zero}, tot[2] = {zero, zero};
    // the adapters' part, the last addend: AdapterSet's while the first slices are on their way
    [[maybe_unused]] f32x16 more[2] = {zero, zero};
    if constexpr (adapters_are<AdapterSet, AD...>)
        adapter_sums<ET>(adapters_of(ad...), m0 + 32 * wave, n0, M, N, L, more);
    const int run = K > kSplitMinK ? (nk + kRuns - 1) / kRuns : nk;
    if constexpr (!FOLD) {
        // (a loop of its own: as slices opened by a run's first one, products with a
        // ragged last slice were slower, 8192x328x320 8.7 -> 9.1 us)
        for (int i = 0; i < nk; ++i) {
            wait_slices<kIssued>(min(nk - 1 - i, ST - 2));
            lds_barrier();   // slice i is in LDS for every wave; slot (i - 1) % ST is free
            if (i + ST - 1 < nk) issue(i + ST - 1);
            const char* st = smem + (i % ST) * kSlot;
            const int kval = K - i * kBK;    // channels of this slice inside K (uniform)
            // all twelve operand reads first, so their latencies overlap
            u32x4 bf[4], af[2][4];
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                bf[s] = *(const u32x4*)(st + offx[s]);
                af[0][s] = *(const u32x4*)(st + offw[0][s]);
                af[1][s] = *(const u32x4*)(st + offw[1][s]);
            }
            if (kval < kBK) {
#pragma unroll
                for (int s = 0; s < 4; ++s)
                    if (8 * (2 * s + half) >= kval) {
                        bf[s] = u32x4{0u, 0u, 0u, 0u};
                        af[0][s] = bf[s];
                        af[1][s] = bf[s];
                    }
            }
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                acc[0] = mfma32x32x16<ET>(af[0][s], bf[s], acc[0]);
                acc[1] = mfma32x32x16<ET>(af[1][s], bf[s], acc[1]);
            }
            if constexpr (FUSED) {
#pragma unroll
                for (int s = 0; s < 4; ++s) down_step(st, s, bf[s], kval);
            }
        }
    } else
    for (int i0 = 0; i0 < nk; i0 += run) {
        slice(i0, std::true_type{}, acc, [&]() __attribute__((always_inline)) {
            if (i0 > 0) {
                __builtin_amdgcn_sched_barrier(0);
                tot[0] += acc[0];
                tot[1] += acc[1];
                if constexpr (FUSED) dtot += dacc;
                __builtin_amdgcn_sched_barrier(0);
            }
        });
        for (int i = i0 + 1; i < min(i0 + run, nk); ++i) slice(i, std::false_type{}, acc, [] {});
    }

    // FUSED: up T^T
    if constexpr (FUSED) {
        if (adapted) {
            float t[16];
#pragma unroll
            for (int r = 0; r < 16; ++r) t[r] = FOLD ? dtot[r] + dacc[r] : dacc[r];
#pragma unroll
            for (int q = 0; q < RR / 16; ++q) {
                const u32x4 tf = fused_t<ET>(t + 8 * q, t_scale, 16 * q, rank, half);
#pragma unroll
                for (int b = 0; b < 2; ++b) more[b] = mfma32x32x16<ET>(upf[q][b], tf, more[b]);
            }
        }
    }

    // Stage the 128 x 64 output tile (bias added, rounded) in LDS, rows of
    // kOutStride bytes: lane (l32, half) holds channels 32t + 8g + 4*half + (0..3)
    // of tile row 32*wave + l32.
    constexpr int kOutStride = kBN * 2 + 16;
    static_assert(kBM * kOutStride <= kLdsBytes, "output tile fits in the slice ring");
    lds_barrier();   // every wave is done with the slices
    {
        char* orow = smem + (32 * wave + l32) * kOutStride;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                float v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float f = FOLD ? tot[t][4 * g + e] + acc[t][4 * g + e] : acc[t][4 * g + e];
                    if constexpr (sizeof...(AD) > 0) f += more[t][4 * g + e];
                    v[e] = f + to_float<ET>((uint16_t)(bias[t][g][e >> 1] >> (16 * (e & 1))));
                }
                u32x2 w;
                w[0] = pack2<ET>(v[0], v[1]);
                w[1] = pack2<ET>(v[2], v[3]);
                *(u32x2*)(orow + (32 * t + 8 * g + 4 * half) * 2) = w;
            }
    }
    lds_barrier();
    // 16 bytes per lane: chunk q = tid + 256j is tile row q / 8 + 32j, channels
    // n = n0 + 8 (q % 8) .. + 7 (inside one head, as head widths are multiples
    // of 8).  The channel offset is the same for all j; the row's batch and
    // token advance by 32 tokens per j.
    const int c8 = threadIdx.x & 7;
    const int n = n0 + 8 * c8;
    const int r0 = threadIdx.x >> 3;
    if (n < N) {
        const int yhw = P.yhw;
        uint16_t* __restrict__ Yc = P.y + bi * P.sy + chan_offset<YH>(n, L, yhw, 1.0f / (float)yhw);
        int b = (m0 + r0) / L, l = (m0 + r0) - b * L;   // token row m = b*L + l
#pragma unroll
        for (int j = 0; j < kBM * kBN / 8 / 256; ++j) {
            const int r = r0 + 32 * j;
            if (m0 + r < M) {
                const u32x4 v = *(const u32x4*)(smem + r * kOutStride + c8 * 16);
                const size_t row = YH ? ((size_t)b * (N / yhw) * L + l) * yhw : (size_t)(m0 + r) * N;
                *(u32x4*)(Yc + row) = v;
            }
            l += 32;
            while (l >= L) {
                l -= L;
                ++b;
            }
        }
    }
}

// The same product for grids of few tiles (few token rows): the reduced
// dimension is split over the workgroup's four waves instead of the tile.  Each
// wave multiplies the whole TM x TN tile over its own run of channels, through
// a private LDS ring of ST slices of 64 channels that no other wave touches,
// so the main loop has no workgroup barrier and a chain of K/64 slices becomes
// four chains of a quarter of the length; the partial tiles meet once in LDS.
// Bound by the latency of those chains and each CU's copy rate (a 64x64 tile of
// K = 1280 is 328 KB through one CU); with one slice per wave (ST = 1) two or
// three workgroups share a CU and cover each other's waits, which measured
// faster than deeper rings (512x1280x1280: 9.1 against 9.4 us with ST = 2).
template <int TM, int TN, int ST, typename... AD>
struct KsGeom {
    static constexpr int RR = fused_rows<AD...>;                  // rows of down in a slice
    static constexpr int kSlice = (TM + TN + RR) * kBK * 2;       // bytes
    static constexpr int kCopies = kSlice / 1024;                 // copy instructions per slice
    static constexpr int kOutRow = TN * 4 + 16;                   // bytes per row of a partial tile
    static constexpr int kRing = kRuns * ST * kSlice;
    static constexpr int kMore = kRuns * TM * kOutRow;            // partial tiles, then the adapters' tile, then T's parts
    static constexpr int kT = kMore + (sizeof...(AD) > 0 ? TM * kOutRow : 0);
    static constexpr int kPart = kT + kRuns * TM * RR * 4;
    static constexpr int kLds = kRing > kPart ? kRing : kPart;
    static_assert(kLds <= 160 * 1024 && TM % 32 == 0 && TN % 32 == 0, "geometry");
    static_assert(kCopies * (ST - 1) < 64, "copies in flight fit vmcnt");
};

// Wait until at most n (<= N) slices of this wave's copies are in flight.
template <int COPIES, int N>
__device__ __forceinline__ void ks_wait(int n) {
    if constexpr (N > 0) {
        if (n < N) {
            ks_wait<COPIES, N - 1>(n);
            return;
        }
    }
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(COPIES * N) : "memory");
}

template <int ET, bool YH, int TM, int TN, int ST, typename... AD>
__global__ __launch_bounds__(256, sizeof...(AD) > 0 ? 2 : 1) void linear_ksplit_kernel(const LinGroup grp, const AD... ad) {
    constexpr int RR = fused_rows<AD...>;
    constexpr bool FUSED = RR > 0;
    using G = KsGeom<TM, TN, ST, AD...>;
    constexpr int MB = TM / 32, NB = TN / 32, KS = kBK / 16;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const int lane = lane_id();
    const int l32 = lane & 31;
    const int half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

    const int tile = xcd_remap(blockIdx.x, gridDim.x);
    const int pi = (grp.n > 2 && tile >= grp.p[2].tile0) ? 2 : (grp.n > 1 && tile >= grp.p[1].tile0) ? 1 : 0;
    const LinProblem& P = grp.p[pi];
    const int bi = (tile - P.tile0) / P.per_batch;
    const int local = tile - P.tile0 - bi * P.per_batch;
    const uint16_t* __restrict__ X = P.x + bi * P.sx;
    const uint16_t* __restrict__ W = P.w + bi * P.sw;
    const int M = P.M, K = P.K, N = P.N, L = P.L;
    const int nmt = (M + TM - 1) / TM;
    const int mt = local % nmt;          // consecutive workgroups share the weight rows
    const int m0 = mt * TM;
    const int n0 = (local / nmt) * TN;

    // this wave's slices
    const int ns = (K + kBK - 1) / kBK;
    const int per = (ns + kRuns - 1) / kRuns;
    const int first = wave * per;
    const int count = max(0, min(per, ns - first));
    char* ring = smem + wave * (ST * G::kSlice);

    // Copy j moves chunk cch[j] / 8 of tile row r (x rows, then w rows); rows
    // past M or N repeat the last row (their outputs are never stored).
    const uint16_t* src[G::kCopies];
    int cch[G::kCopies];
    // FUSED: the request's adapter (the first one's addresses where it has none)
    [[maybe_unused]] bool adapted = false;
    [[maybe_unused]] int id = 0;
    [[maybe_unused]] const uint16_t* down = nullptr;
    [[maybe_unused]] int rank = 1;
    if constexpr (FUSED) {
        const auto a = adapters_of(ad...);
        const int named = __builtin_amdgcn_readfirstlane(a.ids[bi]);
        adapted = named >= 0 && named < a.count;
        id = adapted ? named : 0;
        down = a.down + (size_t)id * a.R * K;
        rank = a.R;
    }
#pragma unroll
    for (int j = 0; j < G::kCopies; ++j) {
        const int u = j * 64 + lane;
        const int r = u / 8;
        cch[j] = 8 * ((u % 8) ^ swz(r)) + first * kBK;
        src[j] = j * 64 < TM * 8 ? X + (size_t)min(m0 + r, M - 1) * K
                                 : W + (size_t)min(n0 + r - TM, N - 1) * K;
        if (FUSED && j * 64 >= (TM + TN) * 8) src[j] = down + (size_t)min(r - TM - TN, rank - 1) * K;
    }
    auto issue = [&](int i) __attribute__((always_inline)) {
        char* st = ring + (i % ST) * G::kSlice;
#pragma unroll
        for (int j = 0; j < G::kCopies; ++j)   // channels past K repeat the last chunk (zeroed below)
            __builtin_amdgcn_global_load_lds((const char*)(src[j] + min(cch[j] + i * kBK, K - 8)),
                                             (lds_void_t*)(st + j * 1024), 16, 0, 0);
    };

    int offx[KS], offw[KS];   // row l32, chunk 2s + half; rows 32 apart share the swizzle
    [[maybe_unused]] int offd[KS];
#pragma unroll
    for (int s = 0; s < KS; ++s) {
        const int cpos = (2 * s + half) ^ swz(l32);
        offx[s] = (l32 * 8 + cpos) * 16;
        offw[s] = ((TM + l32) * 8 + cpos) * 16;
        if constexpr (FUSED) offd[s] = ((TM + TN + (l32 & (RR - 1))) * 8 + ((2 * s + half) ^ swz(l32 & (RR - 1)))) * 16;
    }

    f32x16 acc[MB][NB];
#pragma unroll
    for (int a = 0; a < MB; ++a)
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[a][b][r] = 0.0f;

#pragma unroll
    for (int i = 0; i < ST; ++i)
        if (i < count) issue(i);

    [[maybe_unused]] f32x16 dacc[MB];       // FUSED: T^T of this run
#pragma unroll
    for (int a = 0; a < MB; ++a)
#pragma unroll
        for (int r = 0; r < 16; ++r) dacc[a][r] = 0.0f;
    // AdapterSet: the adapters' part while the first slices are on their way; a wave takes a
    // quarter of the channels, or a block of 32 x 32
    constexpr bool APART = adapters_are<AdapterSet, AD...>;
    constexpr int kWaveN = TN / kRuns, NG = kWaveN / 8;
    [[maybe_unused]] float dots[MB][NG][4];
    [[maybe_unused]] f32x16 block[1];
    if constexpr (APART) {
        const AdapterSet set = adapters_of(ad...);
        if (L < kAdapterRows) {
#pragma unroll
            for (int a = 0; a < MB; ++a) {
#pragma unroll
                for (int g = 0; g < NG; ++g)
#pragma unroll
                    for (int e = 0; e < 4; ++e) dots[a][g][e] = 0.0f;
                const uint16_t *up, *t;
                if (adapter_of_row(set, m0 + 32 * a + l32, M, N, L, &up, &t))
                    adapter_width(set.R, [&](auto w) __attribute__((always_inline)) {
                        adapter_dots<ET, decltype(w)::value, NG>(up, t, set.R, n0 + kWaveN * wave + 4 * half, 8, N, dots[a]);
                    });
            }
        } else if (wave < MB * NB) {
            adapter_sums<ET>(set, m0 + 32 * (wave / NB), n0 + 32 * (wave % NB), M, N, L, block);
        }
    }

    for (int i = 0; i < count; ++i) {
        ks_wait<G::kCopies, ST - 1>(count - 1 - i);
        const char* st = ring + (i % ST) * G::kSlice;
        u32x4 xf[MB][KS], wf[NB][KS];
        [[maybe_unused]] u32x4 df[KS];
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            if constexpr (FUSED) df[s] = *(const u32x4*)(st + offd[s]);
#pragma unroll
            for (int a = 0; a < MB; ++a) xf[a][s] = *(const u32x4*)(st + offx[s] + a * 32 * kBK * 2);
#pragma unroll
            for (int b = 0; b < NB; ++b) wf[b][s] = *(const u32x4*)(st + offw[s] + b * 32 * kBK * 2);
        }
        // the slot is read out: its next slice may be copied in
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (i + ST < count) issue(i + ST);
        const int kval = K - (first + i) * kBK;   // channels of this slice inside K
        if (kval < kBK) {
#pragma unroll
            for (int s = 0; s < KS; ++s)
                if (8 * (2 * s + half) >= kval) {
#pragma unroll
                    for (int a = 0; a < MB; ++a) xf[a][s] = u32x4{0u, 0u, 0u, 0u};
#pragma unroll
                    for (int b = 0; b < NB; ++b) wf[b][s] = u32x4{0u, 0u, 0u, 0u};
                    if constexpr (FUSED) df[s] = u32x4{0u, 0u, 0u, 0u};
                }
        }
        if constexpr (FUSED) {
#pragma unroll
            for (int s = 0; s < KS; ++s)
#pragma unroll
                for (int a = 0; a < MB; ++a) dacc[a] = mfma32x32x16<ET>(df[s], xf[a][s], dacc[a]);
        }
#pragma unroll
        for (int s = 0; s < KS; ++s)
#pragma unroll
            for (int a = 0; a < MB; ++a)
#pragma unroll
                for (int b = 0; b < NB; ++b) acc[a][b] = mfma32x32x16<ET>(wf[b][s], xf[a][s], acc[a][b]);
    }

    // 16 bytes per lane: chunk q = tid + 256j is tile row q / (TN / 8), channels
    // n = n0 + 8 (q % (TN / 8)) .. + 7, the same n for every j
    constexpr int kCols = TN / 8;
    const int c8 = threadIdx.x % kCols;
    const int n = n0 + 8 * c8;
    u32x2 bias[2] = {u32x2{0u, 0u}, u32x2{0u, 0u}};
    if (P.bias && n < N) {
        bias[0] = *(const u32x2*)(P.bias + n);
        bias[1] = *(const u32x2*)(P.bias + n + 4);
    }

    // partial tiles: lane (l32, half) holds channels 32b + 8g + 4*half + (0..3)
    // of row 32a + l32
    __syncthreads();   // every wave is done with its ring
    {
        char* part = smem + wave * (TM * G::kOutRow);
#pragma unroll
        for (int a = 0; a < MB; ++a)
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const f32x4 v = {acc[a][b][4 * g], acc[a][b][4 * g + 1], acc[a][b][4 * g + 2],
                                     acc[a][b][4 * g + 3]};
                    *(f32x4*)(part + (32 * a + l32) * G::kOutRow + (32 * b + 8 * g + 4 * half) * 4) = v;
                }
        if constexpr (FUSED) {   // T's part, [TM][RR ranks]
            char* tp = smem + G::kT + wave * (TM * RR * 4);
#pragma unroll
            for (int a = 0; a < MB; ++a)
#pragma unroll
                for (int q = 0; q < RR / 8; ++q)
                    *(f32x4*)(tp + (32 * a + l32) * RR * 4 + (8 * q + 4 * half) * 4) =
                        f32x4{dacc[a][4 * q], dacc[a][4 * q + 1], dacc[a][4 * q + 2], dacc[a][4 * q + 3]};
        }
    }
    if constexpr (APART) {
        if (L < kAdapterRows) {
#pragma unroll
            for (int a = 0; a < MB; ++a)
#pragma unroll
                for (int g = 0; g < NG; ++g)
                    *(f32x4*)(smem + G::kMore + (32 * a + l32) * G::kOutRow + (kWaveN * wave + 8 * g + 4 * half) * 4) =
                        f32x4{dots[a][g][0], dots[a][g][1], dots[a][g][2], dots[a][g][3]};
        } else if (wave < MB * NB) {
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *(f32x4*)(smem + G::kMore + (32 * (wave / NB) + l32) * G::kOutRow + (32 * (wave % NB) + 8 * g + 4 * half) * 4) =
                    f32x4{block[0][4 * g], block[0][4 * g + 1], block[0][4 * g + 2], block[0][4 * g + 3]};
        }
    }
    if constexpr (FUSED) {
        // T whole, the runs in the shared tiles' order, then up T^T by a wave for each 32 x 32
        const auto f = adapters_of(ad...);
        static_assert(MB * NB <= kRuns, "a block a wave");
        const bool mine = wave < MB * NB;
        const int a = wave / NB, b = wave % NB;
        u32x4 upf[RR / 16];
#pragma unroll
        for (int q = 0; q < RR / 16; ++q)
            upf[q] = fused_up(f.up + ((size_t)id * N + min(n0 + 32 * b + l32, N - 1)) * f.R, 16 * q, f.R, half);
        __syncthreads();
        if (mine) {
            float t[RR / 2];
#pragma unroll
            for (int r = 0; r < RR / 2; ++r) t[r] = 0.0f;
#pragma unroll
            for (int w = 0; w < kRuns; ++w)
#pragma unroll
                for (int q = 0; q < RR / 8; ++q) {
                    const f32x4 p = *(const f32x4*)(smem + G::kT + w * (TM * RR * 4) + (32 * a + l32) * RR * 4 +
                                                    (8 * q + 4 * half) * 4);
#pragma unroll
                    for (int e = 0; e < 4; ++e) t[4 * q + e] += p[e];
                }
            f32x16 sum;
#pragma unroll
            for (int r = 0; r < 16; ++r) sum[r] = 0.0f;
            if (adapted) {
                const float scale = f.scales ? f.scales[id] : 1.0f;
#pragma unroll
                for (int q = 0; q < RR / 16; ++q)
                    sum = mfma32x32x16<ET>(upf[q], fused_t<ET>(t + 8 * q, scale, 16 * q, f.R, half), sum);
            }
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *(f32x4*)(smem + G::kMore + (32 * a + l32) * G::kOutRow + (32 * b + 8 * g + 4 * half) * 4) =
                    f32x4{sum[4 * g], sum[4 * g + 1], sum[4 * g + 2], sum[4 * g + 3]};
        }
    }
    __syncthreads();
    if (n >= N) return;
    const int yhw = P.yhw;
    uint16_t* __restrict__ Yc = P.y + bi * P.sy + chan_offset<YH>(n, L, yhw, 1.0f / (float)yhw);
#pragma unroll
    for (int j = 0; j < (TM * kCols + 256 - 1) / (256); ++j) {
        const int r = (threadIdx.x + 256 * j) / kCols;
        if (r < TM && m0 + r < M) {
            f32x4 lo = {0.0f, 0.0f, 0.0f, 0.0f}, hi = lo;
#pragma unroll
            for (int w = 0; w < kRuns; ++w) {
                const char* p = smem + w * (TM * G::kOutRow) + r * G::kOutRow + c8 * 32;
                lo += *(const f32x4*)p;
                hi += *(const f32x4*)(p + 16);
            }
            if constexpr (sizeof...(AD) > 0) {
                const char* p = smem + G::kMore + r * G::kOutRow + c8 * 32;
                lo += *(const f32x4*)p;
                hi += *(const f32x4*)(p + 16);
            }
            u32x4 v;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const u32x2 bb = bias[e >> 1];
                const float b0 = to_float<ET>((uint16_t)bb[e & 1]);
                const float b1 = to_float<ET>((uint16_t)(bb[e & 1] >> 16));
                v[e] = e < 2 ? pack2<ET>(lo[2 * e] + b0, lo[2 * e + 1] + b1)
                             : pack2<ET>(hi[2 * e - 4] + b0, hi[2 * e - 3] + b1);
            }
            *(u32x4*)(Yc + row_base<YH>(m0 + r, L, N, yhw)) = v;
        }
    }
}

// T = s_i down_i x for the rows of the batch items that have an adapter: a workgroup
// takes 16 TB rows of one item and 16 RB ranks, its four waves a quarter of the channels
// each.  T^T = down x^T on 16x16x32 MFMAs, whose operands come straight from memory, 16
// bytes a lane: a row's 64 bytes meet in one instruction, and the next one takes the
// other half of its cache lines.  Bound by reading x once where there are few ranks, by the
// caches' reads of down where there are many (4 requests of 1024 rows, K = N = 1280, R 128:
// 51.3 us in all with TB = 1, 49.4 with 2).  T is rounded to the tensors' type, the type that
// the second product's matrix instructions take; the scale goes in before, in fp32.
constexpr int kDownSteps = 4;   // steps of 32 channels in flight
struct DownKernel {
    const uint16_t* x;
    const uint16_t* down;   // [count, R, K]
    const int* ids;
    const float* scales;    // [count] or null
    uint16_t* t;            // [B L, Rp]
    int L, K, xhw, R, Rp, count;
    int tiles;              // row tiles of an item
};

template <int ET>
__device__ __forceinline__ f32x4 mfma16x16x32(u32x4 a, u32x4 b, f32x4 c) {
    if constexpr (ET == kF16)
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

template <int ET, bool XH, int RB, int TB>
__global__ __launch_bounds__(256) void adapter_down_kernel(const DownKernel a) {
    __shared__ f32x4 part[kRuns - 1][RB * TB][64];
    const int lane = lane_id();
    const int l16 = lane & 15, quad = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int b = blockIdx.x / a.tiles, l0 = (blockIdx.x - b * a.tiles) * 16 * TB;
    const int r0 = blockIdx.y * 16 * RB;
    const int id = a.ids[b];
    if (id < 0 || id >= a.count) return;
    const float inv_xhw = 1.0f / (float)a.xhw;
    const uint16_t* x[TB];
    const uint16_t* d[RB];
#pragma unroll
    for (int t = 0; t < TB; ++t) x[t] = a.x + row_base<XH>(b * a.L + min(l0 + 16 * t + l16, a.L - 1), a.L, a.K, a.xhw);
#pragma unroll
    for (int j = 0; j < RB; ++j) d[j] = a.down + ((size_t)id * a.R + min(r0 + 16 * j + l16, a.R - 1)) * a.K;

    f32x4 acc[RB][TB];
#pragma unroll
    for (int j = 0; j < RB; ++j)
#pragma unroll
        for (int t = 0; t < TB; ++t) acc[j][t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    const int steps = (a.K + 31) / 32;
    const int per = (steps + kRuns - 1) / kRuns;
    const int first = wave * per, end = min(first + per, steps);
    for (int s0 = first; s0 < end; s0 += kDownSteps) {
        u32x4 xv[kDownSteps][TB], dv[kDownSteps][RB];
#pragma unroll
        for (int u = 0; u < kDownSteps; ++u) {
            const int c = 32 * (s0 + u) + 8 * quad, cc = min(c, a.K - 8);
#pragma unroll
            for (int t = 0; t < TB; ++t) xv[u][t] = *(const u32x4*)(x[t] + chan_offset<XH>(cc, a.L, a.xhw, inv_xhw));
#pragma unroll
            for (int j = 0; j < RB; ++j) dv[u][j] = *(const u32x4*)(d[j] + cc);
        }
#pragma unroll
        for (int u = 0; u < kDownSteps; ++u) {
            // past this wave's channels both factors are zeros (a zero and a NaN are no zero)
            const bool out = s0 + u >= end || 32 * (s0 + u) + 8 * quad >= a.K;
            const u32x4 zero = {0u, 0u, 0u, 0u};
#pragma unroll
            for (int j = 0; j < RB; ++j)
#pragma unroll
                for (int t = 0; t < TB; ++t)
                    acc[j][t] = mfma16x16x32<ET>(out ? zero : dv[u][j], out ? zero : xv[u][t], acc[j][t]);
        }
    }
    if (wave > 0) {
#pragma unroll
        for (int j = 0; j < RB; ++j)
#pragma unroll
            for (int t = 0; t < TB; ++t) part[wave - 1][j * TB + t][lane] = acc[j][t];
    }
    __syncthreads();
    if (wave > 0) return;
    const float scale = a.scales ? a.scales[id] : 1.0f;
#pragma unroll
    for (int j = 0; j < RB; ++j)
#pragma unroll
        for (int t = 0; t < TB; ++t) {
#pragma unroll
            for (int w = 0; w < kRuns - 1; ++w) acc[j][t] += part[w][j * TB + t][lane];
            // this lane's 4 ranks of its row; ranks from R on are zeros
            const int r = r0 + 16 * j + 4 * quad, l = l0 + 16 * t + l16;
            if (l < a.L && r < a.Rp) {
                float v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = r + e < a.R ? acc[j][t][e] * scale : 0.0f;
                *(u32x2*)(a.t + (size_t)(b * a.L + l) * a.Rp + r) = u32x2{pack2<ET>(v[0], v[1]), pack2<ET>(v[2], v[3])};
            }
        }
}

// tm x tn tiles of one batch item
long long tiles_of(const LinearArgs& a, int tm, int tn) {
    return ((long long)a.B * a.L + tm - 1) / tm * ((a.N + tn - 1) / tn);
}

template <int ET, bool XH, bool YH, bool FOLD, typename... AD>
hipError_t launch_t(const LinGroup& g, long long nblk, void* stream, const AD&... ad) {
    auto k = linear_kernel<ET, XH, YH, FOLD, AD...>;
    constexpr int lds = linear_lds<FOLD, AD...>;
    static_assert(2 * lds <= 160 * 1024, "two workgroups a CU");
    static const hipError_t attr = hipFuncSetAttribute(
        reinterpret_cast<const void*>(k), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (attr != hipSuccess) return attr;
    hipLaunchKernelGGL(k, dim3((unsigned)nblk), dim3(256), lds, (hipStream_t)stream, g, ad...);
    return hipGetLastError();
}

template <int ET, bool XH, bool YH, typename... AD>
hipError_t launch_f(const LinGroup& g, long long nblk, bool fold, void* stream, const AD&... ad) {
    return fold ? launch_t<ET, XH, YH, true>(g, nblk, stream, ad...)
                : launch_t<ET, XH, YH, false>(g, nblk, stream, ad...);
}

// Number the TM x TN tiles of the group's products (tile0, per_batch, nnt);
// returns how many there are.
long long number_tiles(LinGroup& g, const LinearArgs* a, int tm, int tn) {
    long long nblk = 0;
    for (int i = 0; i < g.n; ++i) {
        g.p[i].nnt = (a[i].N + tn - 1) / tn;
        g.p[i].tile0 = (int)nblk;
        g.p[i].per_batch = (int)tiles_of(a[i], tm, tn);
        nblk += tiles_of(a[i], tm, tn) * a[i].batch;
        if (nblk > 0x7fffffff) return nblk;
    }
    return nblk;
}

template <int ET, bool YH, int TM, int TN, int ST, typename... AD>
hipError_t launch_ks(LinGroup& g, const LinearArgs* a, const AD&... ad) {
    using G = KsGeom<TM, TN, ST, AD...>;
    const long long nblk = number_tiles(g, a, TM, TN);
    if (nblk > 0x7fffffff) return hipErrorInvalidValue;
    auto k = linear_ksplit_kernel<ET, YH, TM, TN, ST, AD...>;
    static const hipError_t attr = hipFuncSetAttribute(
        reinterpret_cast<const void*>(k), hipFuncAttributeMaxDynamicSharedMemorySize, G::kLds);
    if (attr != hipSuccess) return attr;
    hipLaunchKernelGGL(k, dim3((unsigned)nblk), dim3(256), G::kLds, (hipStream_t)a[0].stream, g, ad...);
    return hipGetLastError();
}

// The tile of the split-K kernel: 32 x 32 while those tiles fit the CUs once,
// 64 x 64 where rows past 32 would read the weights twice and there are tiles
// enough (two per CU), 32 x 64 between.  Measured (us, 32x32 / 32x64 / 64x64):
// 128x1280x1280 5.1 / 6.0 / 7+; 512x1280x1280 10.0 / 9.2 / 9.1; 36 products
// 48x1280x1280 - / 34.5 / 30.3; 36 of 64x640x640 12.2 / 9.5 / 10.3.
template <int ET, bool YH, typename... AD>
hipError_t launch_ksplit(LinGroup& g, const LinearArgs* a, const AD&... ad) {
    long long n32 = 0, n64 = 0, rows = 0;
    for (int i = 0; i < g.n; ++i) {
        n32 += tiles_of(a[i], 32, 32) * a[i].batch;
        n64 += tiles_of(a[i], 64, 64) * a[i].batch;
        rows = rows > g.p[i].M ? rows : g.p[i].M;
    }
    if (n32 <= 256) return launch_ks<ET, YH, 32, 32, 2>(g, a, ad...);
    // (with an adapter's tile and T beside the partial tiles one 64 x 64 workgroup fills a CU)
    if constexpr (fused_rows<AD...> == 0) {
        if (rows > 32 && n64 >= 512) return launch_ks<ET, YH, 64, 64, 1>(g, a, ad...);
    }
    return launch_ks<ET, YH, 32, 64, 1>(g, a, ad...);
}

template <int ET, typename... AD>
hipError_t launch_group_e(LinGroup& g, const LinearArgs* a, const AD&... ad) {
    const bool xh = a[0].x_heads, yh = a[0].y_heads;
    // Split K over the waves where 128-row tiles leave the chip idle (at most
    // 128 of them: half of the CUs) or mostly compute padding (at most 64 rows):
    // 512x1280x1280 (80 tiles) 12.1 -> 9.2 us, 768x1280x1280 (120) 12.1 -> 9.8,
    // 1280x640x640 (100) 7.7 -> 7.2, 36 products 32x1280x1280 31.3 -> 25.8.  From
    // there on the shared tiles are as fast or faster: 1024x1280x1280 (160 tiles)
    // 12.3 against 13.2, 3328x320x320 (130) 5.8 against 6.1, 36 products
    // 72x1280x1280 34.4 against 41.9.  Products split only past kSplitMinK
    // channels, where the shared tiles sum in the same order (FOLD): a row's bits
    // depend neither on its company in a launch nor on the other images of a batch.
    if (!xh) {
        long long tiles = 0;
        bool few_rows = true, may = true;
        for (int i = 0; i < g.n; ++i) {
            tiles += tiles_of(a[i], kBM, kBN) * a[i].batch;
            few_rows = few_rows && g.p[i].M <= 64;
            may = may && a[i].K > kSplitMinK;
        }
        if (may && (tiles <= 128 || few_rows))
            return yh ? launch_ksplit<ET, true>(g, a, ad...) : launch_ksplit<ET, false>(g, a, ad...);
    }
    const long long nblk = number_tiles(g, a, kBM, kBN);
    if (nblk > 0x7fffffff) return hipErrorInvalidValue;
    bool fold = false;
    for (int i = 0; i < g.n; ++i) fold = fold || a[i].K > kSplitMinK;
    void* s = a[0].stream;
    if (xh)
        return yh ? launch_f<ET, true, true>(g, nblk, fold, s, ad...) : launch_f<ET, true, false>(g, nblk, fold, s, ad...);
    return yh ? launch_f<ET, false, true>(g, nblk, fold, s, ad...) : launch_f<ET, false, false>(g, nblk, fold, s, ad...);
}

// The group's products; an error for those that cannot share a launch.
hipError_t make_group(LinGroup& g, const LinearArgs* a, int n) {
    if (n < 1 || n > kMaxLinearProblems) return hipErrorInvalidValue;
    g.n = n;
    for (int i = 0; i < n; ++i) {
        if (a[i].dtype != a[0].dtype || a[i].x_heads != a[0].x_heads ||
            a[i].y_heads != a[0].y_heads || a[i].stream != a[0].stream || a[i].batch < 1)
            return hipErrorInvalidValue;
        LinProblem& p = g.p[i];
        p.x = (const uint16_t*)a[i].x;
        p.w = (const uint16_t*)a[i].w;
        p.bias = (const uint16_t*)a[i].bias;
        p.y = (uint16_t*)a[i].y;
        p.M = a[i].B * a[i].L;
        p.K = a[i].K;
        p.N = a[i].N;
        p.L = a[i].L;
        p.xhw = a[i].x_heads ? a[i].K / a[i].H : 1;
        p.yhw = a[i].y_heads ? a[i].N / a[i].H : 1;
        p.sx = a[i].sx;
        p.sw = a[i].sw;
        p.sy = a[i].sy;
    }
    return hipSuccess;
}

template <int ET, bool XH>
hipError_t launch_down(const LinearArgs& a, const AdapterArgs& d) {
    DownKernel k{(const uint16_t*)a.x, (const uint16_t*)d.down, d.ids, d.scales, (uint16_t*)d.t,
                 a.L, a.K, a.x_heads ? a.K / a.H : 1, d.R, adapter_rank_padded(d.R), d.count, 0};
    auto rows_of = [&](int rb) { return rb > 1 && a.L >= 32 ? 32 : 16; };
    auto groups = [&](int rb) {
        return (long long)a.B * ((a.L + rows_of(rb) - 1) / rows_of(rb)) * ((d.R + 16 * rb - 1) / (16 * rb));
    };
    // 64 ranks a workgroup read x least often; fewer while the workgroups are too few to have enough of
    // down in flight (a T's sum is the same either way).  The whole call with 64 / 32 / 16 ranks, us: 64
    // tokens of 64 requests, K = N = 1280, R 64 (64 / 128 / 256 workgroups) 18.1 / 15.1 / 13.5; 8 of 77, 768,
    // 640, R 64 (24 / 48 / 160) 17.3 / 14.4 / 12.3; 16 of 77, 1280, 1280, R 64 (48 / 96 / 320) 28.6 / 24.3 / 23.4;
    // 2 of 1024, 1280, 1280, R 64 (64 / 128 / 512) 31.8 / 28.0 / 27.0, 640, 640 19.8 / 16.9 / 16.6; 4 of 1024,
    // 1280, 1280, R 64 (128 / 256 / 1024) 42.7 / 39.1 / 43.0; 8 of 1024, 640, 640, R 64 (256 / 512 / 2048) 31.0 /
    // 31.5 / 37.6; 4096 rows, 640, 640, R 128 (as many) 25.7 / 26.3 / 32.8.
    int rb = d.R <= 16 ? 1 : d.R <= 32 ? 2 : 4;
    if (groups(1) <= 512) rb = 1;
    else if (rb > 2 && groups(2) < 512) rb = 2;
    const int rows = rows_of(rb);
    const bool two = rows == 32;
    k.tiles = (a.L + rows - 1) / rows;
    const dim3 grid((unsigned)(a.B * k.tiles), (unsigned)((d.R + 16 * rb - 1) / (16 * rb)));
    auto f = rb == 1   ? adapter_down_kernel<ET, XH, 1, 1>
             : rb == 2 ? (two ? adapter_down_kernel<ET, XH, 2, 2> : adapter_down_kernel<ET, XH, 2, 1>)
                       : (two ? adapter_down_kernel<ET, XH, 4, 2> : adapter_down_kernel<ET, XH, 4, 1>);
    hipLaunchKernelGGL(f, grid, dim3(256), 0, (hipStream_t)a.stream, k);
    return hipGetLastError();
}

template <int ET>
hipError_t launch_adapters_e(LinGroup& g, const LinearArgs& a, const AdapterArgs& d) {
    // Fused, the down rows cost every tile of 64 channels a fifth of its time (up to kSplitMinK input
    // channels) or a third; apart, x is read once more, and a launch waits for another.  us, plain product /
    // fused / apart: 8 requests of 77 rows, K 768, N 640, R 4 4.7 / 6.0 / 9.9; 8 of 4096, 320, 320, 16
    // 17.8 / 21.4 / 30.9; 8 of 4096, 320, 1280, 16 60 / 73 / 72; 4 of 1024, 1280, 1280, 16 26.2 / 35.8 / 33.4.
    // With 17 to 32 ranks: 2 of 64, 1280, 1280, 32 4.5 / 7.0 / 9.8; 8 of 77, 768, 640, 24 4.6 / 6.9 / 10.0; 2 of
    // 4096, 320, 320, 32 7.7 / 10.0 / 13.6; 8 of 1024, 640, 640, 32 16.7 / 22.9 / 26.9; 8 of 4096, 320, 1280, 32
    // 60 / 79 / 81; worst where many requests' rows end early in a tile, 64 of 40, 640, 640, 32 7.6 / 19.6 / 15.5.
    // The choice is by a request's own sizes, so that its bits do not depend on the others of its batch.
    if (a.L >= kAdapterRows && d.R <= 32 &&
        (a.K <= kSplitMinK || a.N <= kFusedMaxN || a.L <= kFusedMaxRows)) {
        // tiles of launch_group_e at most
        const int rows = a.L <= 64 && a.K > kSplitMinK ? 32 : kBM;
        if (!grid_fits(a.B * (((long long)a.L + rows - 1) / rows) * ((a.N + kBN - 1) / kBN), 256)) return kGridTooLarge;
        LinearArgs one = a;   // a batch item for each request
        one.B = 1;
        one.batch = a.B;
        one.sx = (long long)a.L * a.K;
        one.sy = (long long)a.L * a.N;
        const hipError_t e = make_group(g, &one, 1);
        if (e != hipSuccess) return e;
        auto with = [&](auto rows) {
            return launch_group_e<ET>(g, &one, AdapterFused<decltype(rows)::value>{
                (const uint16_t*)d.down, (const uint16_t*)d.up, d.ids, d.scales, d.count, d.R});
        };
        return d.R <= 16 ? with(std::integral_constant<int, 16>{}) : with(std::integral_constant<int, 32>{});
    }
    if (!grid_fits(a.B * (((long long)a.L + 15) / 16), 256) || !grid_fits(tiles_of(a, kBM, kBN), 256))
        return kGridTooLarge;
    const hipError_t e = a.x_heads ? launch_down<ET, true>(a, d) : launch_down<ET, false>(a, d);
    if (e != hipSuccess) return e;
    const AdapterSet set{(const uint16_t*)d.t, (const uint16_t*)d.up, d.ids, d.count, d.R, adapter_rank_padded(d.R)};
    return launch_group_e<ET>(g, &a, set);
}

}  // namespace

long long linear_grid(int B, int L, int N) {
    // (the split-K kernel's smaller tiles are taken for at most 128 of these, or 64 rows)
    LinearArgs a{};
    a.B = B;
    a.L = L;
    a.N = N;
    return tiles_of(a, kBM, kBN);
}

hipError_t launch_linear_group(const LinearArgs* a, int n) {
    LinGroup g{};
    const hipError_t e = make_group(g, a, n);
    if (e != hipSuccess) return e;
    return a[0].dtype == kF16 ? launch_group_e<kF16>(g, a) : launch_group_e<kBF16>(g, a);
}

hipError_t launch_linear(const LinearArgs& a) { return launch_linear_group(&a, 1); }

hipError_t launch_linear_adapters(const LinearArgs& a, const AdapterArgs& d) {
    LinGroup g{};
    const hipError_t e = make_group(g, &a, 1);
    if (e != hipSuccess) return e;
    return a.dtype == kF16 ? launch_adapters_e<kF16>(g, a, d) : launch_adapters_e<kBF16>(g, a, d);
}

}  // namespace sdattn
