// kv_cache.hip -- keys and values quantised to e4m3 as they are written into pages of 64
// tokens, and read back.
//
// A page holds, for each key head, 64 tokens of D codes and one scale 2^e:
//   e = the least whole number with max |x| <= 448 * 2^e over the page's tokens,
//   code = x 2^-e rounded to nearest even.
// Powers of two make both steps exact but for that rounding, so a page that a larger token
// joins is coded again (2^(e_old - e) times the old codes) without dividing anything, and
// its codes lose nothing but what falls below the smallest code's half.
//
// Both directions move bytes: 2 read and 1 written for a value, or the reverse.  A team of
// threads takes one (page, key head) of K or V, holds its new values in registers between the
// maximum and the codes, and writes 8 codes (8 bytes) at a time.  17550 tokens of 16 heads of 128: written in
// 46 us, 4.66 TB/s where a copy reaches 5.14; eight sequences of 1365 to 4096 tokens, 8 heads of 80, read back in 20.3,
// 4.4 TB/s; a token of each of 64 sequences 4.1, a launch and the chain from its place to its page's scale.
#include "device.h"
#include "launch.h"

namespace sdattn {

namespace {

constexpr int kPage = kCachePage;
constexpr int kCacheThreads = 256;
constexpr int kMinExp = -100, kMaxExp = 120;

struct CacheKernel {
    const uint16_t* x[2];      // (read: null) new keys, values
    uint16_t* y[2];            // (write: null)
    uint8_t* codes[2];         // [pages, Hk, 64, D]
    float* scales[2];          // [pages, Hk]
    const int* table;          // [B, slots]
    const int* starts;         // [B]
    const int* counts;         // [B] or null
    int B, Hk, L, D, pages, slots;
    int blocks;                // pages (write) or runs of 64 tokens (read) of a sequence
    long long sb, sh, sl;      // elements from one batch item, head and token to the next
};

// v with what is not finite as 0
__device__ __forceinline__ uint16_t finite16(uint16_t v, uint16_t inf) { return (v & inf) == inf ? 0 : v & 0x7fff; }

// the largest |x| of 8 values that is finite, as the bits of its type (which sort as the values do)
template <int ET>
__device__ __forceinline__ uint32_t top8(u32x4 w) {
    constexpr uint16_t kInf = ET == kF16 ? 0x7c00 : 0x7f80;
    uint32_t t = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        t = max(t, (uint32_t)finite16((uint16_t)w[i], kInf));
        t = max(t, (uint32_t)finite16((uint16_t)(w[i] >> 16), kInf));
    }
    return t;
}

// The least e with top <= 448 * 2^e (448 = 1.75 * 2^8), for top >= 0.
__device__ __forceinline__ int scale_exponent(float top) {
    if (!(top > 0.0f)) return kMinExp;
    int x;
    const float m = frexpf(top, &x);   // top = m 2^x, 0.5 <= m < 1
    const int e = x - 9 + (m > 0.875f ? 1 : 0);
    return min(max(e, kMinExp), kMaxExp);
}

// 2^e for |e| <= 126
__device__ __forceinline__ float pow2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// 8 values times s (a power of two) as codes.  Finite values past 1.875 2^15 (fp16) or 2^127
// (bf16) are held as that: rounded to e4m3 they would come back infinite.  Inf and NaN become NaN.
template <int ET>
__device__ __forceinline__ u32x2 encode8(u32x4 w, float s) {
    constexpr uint16_t kInf = ET == kF16 ? 0x7c00 : 0x7f80;
    constexpr uint16_t kMost = ET == kF16 ? 0x7b80 : 0x7f70;
    float f[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        uint16_t v = (uint16_t)(w[i >> 1] >> (16 * (i & 1)));
        const uint16_t a = v & 0x7fff;
        if (a > kMost && a < kInf) v = (v & 0x8000) | kMost;
        f[i] = a >= kInf ? __builtin_nanf("") : to_float<ET>(v) * s;
    }
    u32x2 c;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        int p = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * i], f[4 * i + 1], 0, false);
        p = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * i + 2], f[4 * i + 3], p, true);
        c[i] = (uint32_t)p;
    }
    return c;
}

// 4 codes times r <= 1 (a power of two) as codes
__device__ __forceinline__ uint32_t recode4(uint32_t c, float r) {
    int p = __builtin_amdgcn_cvt_pk_fp8_f32(__builtin_amdgcn_cvt_f32_fp8((int)c, 0) * r, __builtin_amdgcn_cvt_f32_fp8((int)c, 1) * r, 0, false);
    p = __builtin_amdgcn_cvt_pk_fp8_f32(__builtin_amdgcn_cvt_f32_fp8((int)c, 2) * r, __builtin_amdgcn_cvt_f32_fp8((int)c, 3) * r, p, true);
    return (uint32_t)p;
}

// A team of TEAM threads takes one (page of a sequence, key head) of K or V: CH pieces of 8
// values a thread.
template <int ET, int TEAM, int CH>
__global__ __launch_bounds__(kCacheThreads) void cache_write_kernel(const CacheKernel a) {
    constexpr int kTeams = kCacheThreads / TEAM;
    __shared__ uint32_t tops[kCacheThreads / 64];
    const int t = threadIdx.x % TEAM;
    const long long items = 2LL * a.B * a.blocks * a.Hk;
    const long long item = (long long)blockIdx.x * kTeams + (TEAM == 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x / TEAM) : 0);
    if (TEAM == 64 && item >= items) return;   // (no barriers in teams of one wave; the others' items are the workgroups)
    // key heads change first, as a token's heads lie side by side in rows
    const int h = (int)(item % a.Hk);
    long long rest = item / a.Hk;
    const int block = (int)(rest % a.blocks);
    rest /= a.blocks;
    const int b = (int)(rest % a.B), which = (int)(rest / a.B);
    const int D = a.D, pieces = D / 8;

    const long long start = a.starts[b];
    const long long count = a.counts ? min(max(a.counts[b], 0), a.L) : a.L;
    // the sequence's first touched page (positions below 0 have none) and this team's
    const long long slot = (start < 0 ? 0 : start / kPage) + block;
    const long long p0 = slot * kPage;                            // its first position
    const long long from = start > p0 ? start : p0;
    const long long to = start + count < p0 + kPage ? start + count : p0 + kPage;
    if (from >= to || slot >= a.slots) return;                    // (the same for the whole team)
    const int page = a.table[(long long)b * a.slots + slot];
    if (page < 0 || page >= a.pages) return;
    const int row0 = (int)(from - p0), rows = (int)(to - from);   // new rows of the page
    uint8_t* codes = a.codes[which] + ((size_t)page * a.Hk + h) * kPage * D;
    float* scale = a.scales[which] + (size_t)page * a.Hk + h;
    const float old = row0 > 0 ? *scale : 0.0f;                   // of the tokens that stay

    const uint16_t* x = a.x[which] + b * a.sb + h * a.sh + (from - start) * a.sl;
    u32x4 v[CH];
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        const int c = i * TEAM + t, row = c / pieces;
        v[i] = u32x4{0u, 0u, 0u, 0u};
        if (row < rows) v[i] = *(const u32x4*)(x + row * a.sl + (c - row * pieces) * 8);
    }
#pragma unroll
    for (int i = 0; i < CH; ++i) top = max(top, top8<ET>(v[i]));
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o, 64));
    if constexpr (TEAM > 64) {
        if (threadIdx.x % 64 == 0) tops[threadIdx.x / 64] = top;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kCacheThreads / 64; ++w) top = max(top, tops[w]);
    }
    constexpr uint32_t kMost = ET == kF16 ? 0x7b80 : 0x7f70;
    const float need = pow2(scale_exponent(to_float<ET>((uint16_t)min(top, kMost))));
    const float s = fmaxf(old, need);
    const float inv = 1.0f / s;
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        const int c = i * TEAM + t;
        if (c < rows * pieces) *(u32x2*)(codes + (size_t)row0 * D + c * 8) = encode8<ET>(v[i], inv);
    }
    if (row0 > 0 && s != old) {
        const float r = old * inv;
        for (int c = t; c < row0 * pieces; c += TEAM) {
            u32x2 w = *(const u32x2*)(codes + c * 8);
            *(u32x2*)(codes + c * 8) = u32x2{recode4(w[0], r), recode4(w[1], r)};
        }
    }
    // (every wave has read the old scale: the barrier above, or there is one wave)
    if (t == 0) *scale = s;
}

// 64 tokens of a sequence, one key head of K or V: the codes' values in 16 bits; zeros for
// positions without a page.
template <int ET, int TEAM, int CH>
__global__ __launch_bounds__(kCacheThreads) void cache_read_kernel(const CacheKernel a) {
    const int D = a.D, pieces = D / 8, t = threadIdx.x % TEAM;
    const long long item = (long long)blockIdx.x * (kCacheThreads / TEAM) + (TEAM == 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x / TEAM) : 0);
    if (TEAM == 64 && item >= 2LL * a.B * a.blocks * a.Hk) return;
    const int h = (int)(item % a.Hk);
    long long rest = item / a.Hk;
    const int block = (int)(rest % a.blocks);
    rest /= a.blocks;
    const int b = (int)(rest % a.B), which = (int)(rest / a.B);
    const long long start = a.starts[b];
    const int count = a.counts ? min(max(a.counts[b], 0), a.L) : a.L;
    const int l0 = block * kPage, rows = min(kPage, count - l0);
    if (rows <= 0) return;
    // the two pages that the run may lie in
    const long long p0 = start + l0;
    const long long slot0 = p0 >= 0 ? p0 / kPage : (p0 - kPage + 1) / kPage;
    const int split = (int)((slot0 + 1) * kPage - p0);   // rows of the first one
    const uint8_t* codes[2];
    float scale[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const long long slot = slot0 + i;
        int page = -1;
        if (slot >= 0 && slot < a.slots && (i == 0 || split < rows)) page = a.table[(long long)b * a.slots + slot];
        const bool there = page >= 0 && page < a.pages;
        const size_t at = (size_t)(there ? page : 0) * a.Hk + h;
        codes[i] = a.codes[which] + at * kPage * D;
        scale[i] = there ? a.scales[which][at] : -1.0f;
    }
    uint16_t* y = a.y[which] + b * a.sb + h * a.sh + (long long)l0 * a.sl;
    u32x2 w[CH];
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        const int c = i * TEAM + t, row = c / pieces, d = (c - row * pieces) * 8;
        const bool second = row >= split;
        w[i] = u32x2{0u, 0u};
        if (row < rows && (second ? scale[1] : scale[0]) >= 0.0f)
            w[i] = *(const u32x2*)((second ? codes[1] + (size_t)(row - split) * D : codes[0] + (size_t)(kPage - split + row) * D) + d);
    }
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        const int c = i * TEAM + t, row = c / pieces, d = (c - row * pieces) * 8;
        if (row >= rows) continue;
        const float s = row >= split ? scale[1] : scale[0];
        u32x4 o = {0u, 0u, 0u, 0u};
        if (s >= 0.0f) {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                o[2 * j] = pack2<ET>(__builtin_amdgcn_cvt_f32_fp8((int)w[i][j], 0) * s, __builtin_amdgcn_cvt_f32_fp8((int)w[i][j], 1) * s);
                o[2 * j + 1] = pack2<ET>(__builtin_amdgcn_cvt_f32_fp8((int)w[i][j], 2) * s, __builtin_amdgcn_cvt_f32_fp8((int)w[i][j], 3) * s);
            }
        }
        *(u32x4*)(y + row * a.sl + d) = o;
    }
}

CacheKernel kernel_args(const CacheArgs& c) {
    CacheKernel a{};
    a.codes[0] = (uint8_t*)c.k_pages, a.codes[1] = (uint8_t*)c.v_pages;
    a.scales[0] = c.k_scales, a.scales[1] = c.v_scales;
    a.table = c.table, a.starts = c.starts, a.counts = c.counts;
    a.B = c.B, a.Hk = c.Hk, a.L = c.L, a.D = c.D, a.pages = c.pages, a.slots = c.slots;
    a.sl = c.heads ? c.D : (long long)c.Hk * c.D;
    a.sh = c.heads ? (long long)c.L * c.D : c.D;
    a.sb = (long long)c.Hk * c.L * c.D;
    return a;
}

// Whether a wave takes a page's head, rather than four, which leave threads idle at D = 40 and 80 and wait for each other:
// up to D = 80 (reading: 64), with enough heads of pages (16 sequences of 8523 tokens, 5 heads of 40, written 56 -> 39 us and read 41 -> 31; 8 of
// 4096, 8 heads of 64 27.9 -> 25 and 18.8 -> 16.4, 80 32 -> 29 and, from HBM, 20.3 -> 20.8, 96 34.2 -> 39.6; 96 heads of pages of 64
// 4.8 -> 6.2, 1664 8.4 -> 8.6, 2080 of 40 8.5 -> 6.6).
bool by_wave(long long items, int D, int most) { return items >= 2048 && D <= most; }

template <int ET>
hipError_t write_e(const CacheArgs& c) {
    CacheKernel a = kernel_args(c);
    a.x[0] = (const uint16_t*)c.k, a.x[1] = (const uint16_t*)c.v;
    a.blocks = (int)min((long long)c.slots, ((long long)c.L + 2 * kPage - 2) / kPage);   // L tokens may begin at a page's last
    const long long items = 2LL * c.B * a.blocks * c.Hk;
    const bool one = c.L == 1, wave = one || by_wave(items, c.D, 80);
    const long long wgs = wave ? (items + 3) / 4 : items;
    if (!grid_fits(wgs, kCacheThreads)) return kGridTooLarge;
    const int ch = (8 * c.D + kCacheThreads - 1) / kCacheThreads;   // 64 D values, 8 a piece
    auto k = one ? cache_write_kernel<ET, 64, 1>
           : wave ? (c.D <= 40 ? cache_write_kernel<ET, 64, 5> : c.D <= 64 ? cache_write_kernel<ET, 64, 8> : cache_write_kernel<ET, 64, 10>)
           : ch <= 2 ? cache_write_kernel<ET, 256, 2> : ch <= 3 ? cache_write_kernel<ET, 256, 3> : ch <= 4 ? cache_write_kernel<ET, 256, 4>
           : ch <= 5 ? cache_write_kernel<ET, 256, 5> : cache_write_kernel<ET, 256, 8>;
    hipLaunchKernelGGL(k, dim3((unsigned)wgs), dim3(kCacheThreads), 0, (hipStream_t)c.stream, a);
    return hipGetLastError();
}

template <int ET>
hipError_t read_e(const CacheKernel& a, void* stream) {
    const int ch = (8 * a.D + kCacheThreads - 1) / kCacheThreads;
    const long long items = 2LL * a.B * a.blocks * a.Hk;
    const bool wave = by_wave(items, a.D, 64);
    const long long wgs = wave ? (items + 3) / 4 : items;
    if (!grid_fits(wgs, kCacheThreads)) return kGridTooLarge;
    auto k = wave ? (a.D <= 40 ? cache_read_kernel<ET, 64, 5> : cache_read_kernel<ET, 64, 8>)
           : ch <= 2 ? cache_read_kernel<ET, 256, 2> : ch <= 3 ? cache_read_kernel<ET, 256, 3>
           : ch <= 4 ? cache_read_kernel<ET, 256, 4> : ch <= 5 ? cache_read_kernel<ET, 256, 5> : cache_read_kernel<ET, 256, 8>;
    hipLaunchKernelGGL(k, dim3((unsigned)wgs), dim3(kCacheThreads), 0, (hipStream_t)stream, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_cache_write(const CacheArgs& c) { return c.dtype == kF16 ? write_e<kF16>(c) : write_e<kBF16>(c); }

hipError_t launch_cache_read(const CacheArgs& c) {
    CacheKernel a = kernel_args(c);
    a.y[0] = (uint16_t*)c.k, a.y[1] = (uint16_t*)c.v;
    a.blocks = (c.L + kPage - 1) / kPage;
    return c.dtype == kF16 ? read_e<kF16>(a, c.stream) : read_e<kBF16>(a, c.stream);
}

}  // namespace sdattn
