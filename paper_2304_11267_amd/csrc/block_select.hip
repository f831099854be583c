// block_select.hip -- which blocks of keys each block of queries attends to, by a
// cheap score: the product of the blocks' mean query and mean key.
//
//   means   m_j = (sum of the rows of block j) / (their number), 64 rows a block, fp32
//   score   s_ij = sum_d mq_i[d] mk_j[d],  mq_i the mean of query block i
//   mask    bit j of row i: s_ij is among the `keep` largest of row i (of equal
//           scores the lower j first)
//
// A choice between two scores is a choice between two blocks, so sums and scores are
// held in 64 bits: the sum of 64 fp16 values is exact there, the products of two
// fp32 means are too, and their sum is off by at most D 2^-53 sum_d |mq_i[d] mk_j[d]|: only
// scores that are closer than twice that could fall otherwise than the formula says.
#include "device.h"
#include "launch.h"

namespace sdattn {

namespace {

constexpr int kBsThreads = 256;
constexpr int kBsLoads = 8;               // rows of a thread in flight

// Sums of rows [r0, r1) of x, D / 8 chunks of 8 values a row, over the `size` threads of
// a team, of which this is `id`: thread (g, c) takes chunk c of rows r0 + g, + groups, ...
// and leaves its sums in row g of part [groups][D].  Returns the number of groups.  AHEAD: the
// next rows are fetched beside the sums of these (a wave with many rows).
template <int ET, bool AHEAD>
__device__ __forceinline__ int bs_sums(const uint16_t* __restrict__ x, int r0, int r1, int D, int id, int size,
                                       double* part) {
    const int cols = D / 8;
    const int groups = min(min(size / cols, 16), r1 - r0);   // (more of them only add up longer)
    const int g = id / cols, c = id - g * cols;
    if (g < groups) {
        double s[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) s[e] = 0.0;
        u32x4 v[kBsLoads], next[kBsLoads];
        auto load = [&](int r, u32x4 (&to)[kBsLoads]) __attribute__((always_inline)) {
#pragma unroll
            for (int u = 0; u < kBsLoads; ++u) {
                to[u] = u32x4{0u, 0u, 0u, 0u};
                if (r + u * groups < r1) to[u] = *(const u32x4*)(x + (size_t)(r + u * groups) * D + 8 * c);
            }
        };
        if (AHEAD) load(r0 + g, v);
        for (int r = r0 + g; r < r1; r += groups * kBsLoads) {
            if (AHEAD) load(r + groups * kBsLoads, next);
            else load(r, v);
#pragma unroll
            for (int u = 0; u < kBsLoads; ++u) {
#pragma unroll
                for (int e = 0; e < 8; ++e) s[e] += (double)to_float<ET>((uint16_t)(v[u][e >> 1] >> (16 * (e & 1))));
                if (AHEAD) v[u] = next[u];
            }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) part[g * D + 8 * c + e] = s[e];
    }
    return groups;
}

template <int ET>
__global__ __launch_bounds__(kBsThreads) void block_means_kernel(const uint16_t* __restrict__ X, float* __restrict__ Mn,
                                                                 int L, int D, int nb) {
    __shared__ double part[kBsThreads * 8];
    const int bh = blockIdx.x / nb, j = blockIdx.x - bh * nb;
    const int r0 = j * kSparseBlock, r1 = min(L, r0 + kSparseBlock);
    const int groups = bs_sums<ET, false>(X + (size_t)bh * L * D, r0, r1, D, threadIdx.x, kBsThreads, part);
    __syncthreads();
    for (int d = threadIdx.x; d < D; d += kBsThreads) {
        double s = 0.0;
        for (int g = 0; g < groups; ++g) s += part[g * D + d];
        Mn[((size_t)bh * nb + j) * D + d] = (float)(s / (double)(r1 - r0));
    }
}

// Scores as 64-bit integers of the same order (-0 as 0; no number, of either sign, past all).
__device__ __forceinline__ uint64_t bs_key(double s) {
    if (s != s) return ~0ull;
    const uint64_t u = (uint64_t)__double_as_longlong(s + 0.0);
    return u >> 63 ? ~u : u | (1ull << 63);
}

// The sum of v over a row of 16 lanes, in every lane of it: four rotations.
template <int ROR>
__device__ __forceinline__ double bs_rotated(double v) {
    const uint64_t u = (uint64_t)__double_as_longlong(v);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)u, 0x120 + ROR, 0xf, 0xf, true);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(u >> 32), 0x120 + ROR, 0xf, 0xf, true);
    return __longlong_as_double((long long)((uint64_t)hi << 32 | lo));
}
__device__ __forceinline__ double bs_row_sum(double v) {
    v += bs_rotated<8>(v);
    v += bs_rotated<4>(v);
    v += bs_rotated<2>(v);
    return v + bs_rotated<1>(v);
}

// The choice of one wave: the mask row of the `keep` largest of nb keys.  NC > 0: the
// keys (at most 64 NC) in registers; NC = 0: in LDS.  The keep-th largest is found bit by
// bit, first among the upper halves, until some value parts exactly `keep` off: some
// twenty steps where the scores are a hundredth apart, and the lower halves' steps are
// taken only where upper halves are equal.
template <int NC>
__device__ __forceinline__ void bs_choose(const uint64_t* kq, int nb, int keep, unsigned long long* row) {
    const int lane = lane_id();
    const int nw = (nb + 63) / 64;
    uint32_t hi[NC > 0 ? NC : 1], lo[NC > 0 ? NC : 1];
#pragma unroll
    for (int c = 0; c < NC; ++c) {   // no key: 0, which no step counts
        const uint64_t k = 64 * c + lane < nb ? kq[min(64 * c + lane, nb - 1)] : 0;
        hi[c] = (uint32_t)(k >> 32);
        lo[c] = (uint32_t)k;
    }
    // how many keys pass f(upper, lower half)
    auto count = [&](auto f) __attribute__((always_inline)) {
        int n = 0;
        if constexpr (NC > 0) {
#pragma unroll
            for (int c = 0; c < NC; ++c) n += __popcll(__ballot(f(hi[c], lo[c])));
        } else {
            for (int w = 0; w < nw; ++w) {
                const uint64_t k = 64 * w + lane < nb ? kq[min(64 * w + lane, nb - 1)] : 0;
                n += __popcll(__ballot(f((uint32_t)(k >> 32), (uint32_t)k)));
            }
        }
        return n;
    };
    uint32_t top = 0, low = 0;
    int n = nb;   // keys >= (top, low)
    for (int bit = 31; bit >= 0 && n != keep; --bit) {
        const uint32_t cand = top | (1u << bit);
        const int c = count([&](uint32_t h, uint32_t) { return h >= cand; });
        if (c >= keep) {
            top = cand;
            n = c;
        }
    }
    int equal = nb;   // of the keys that are (top, low) themselves, how many are taken
    if (n != keep) {
        const int above = count([&](uint32_t h, uint32_t) { return h > top; });
        for (int bit = 31; bit >= 0 && n != keep; --bit) {
            const uint32_t cand = low | (1u << bit);
            const int c = above + count([&](uint32_t h, uint32_t l) { return h == top && l >= cand; });
            if (c >= keep) {
                low = cand;
                n = c;
            }
        }
        if (n != keep) equal = keep - above - count([&](uint32_t h, uint32_t l) { return h == top && l > low; });
    }
    auto word = [&](int w, uint32_t h, uint32_t l) __attribute__((always_inline)) {
        const bool in = 64 * w + lane < nb;
        const uint64_t over = __ballot(in && (h > top || (h == top && l > low))), same = __ballot(in && h == top && l == low);
        const bool take = (over >> lane & 1) || ((same >> lane & 1) && __popcll(same & ((1ull << lane) - 1)) < equal);
        const uint64_t bits = __ballot(take);
        equal -= min(equal, (int)__popcll(same));
        if (lane == 0) row[w] = bits;
    };
    if constexpr (NC > 0) {
#pragma unroll
        for (int c = 0; c < NC; ++c)
            if (c < nw) word(c, hi[c], lo[c]);
    } else {
        for (int w = 0; w < nw; ++w) {
            const uint64_t k = kq[min(64 * w + lane, nb - 1)];
            word(w, (uint32_t)(k >> 32), (uint32_t)k);
        }
    }
}
__device__ __forceinline__ void bs_choose_any(const uint64_t* kq, int nb, int keep, unsigned long long* row) {
    if (nb <= 256) bs_choose<4>(kq, nb, keep, row);
    else if (nb <= 512) bs_choose<8>(kq, nb, keep, row);
    else if (nb <= 1024) bs_choose<16>(kq, nb, keep, row);
    else bs_choose<0>(kq, nb, keep, row);
}

// The mean of query block i as doubles at mean[0 .. D), by one wave (zeros where it is
// past the last one); part: 512 doubles of the wave's own.
template <int ET>
__device__ __forceinline__ void bs_query_mean(const uint16_t* __restrict__ q, int i, int nq, int qblock, int Lq, int D,
                                              double* mean, double* part) {
    const int lane = lane_id();
    const int r0 = i * qblock, r1 = min(Lq, r0 + qblock);
    const int groups = i < nq ? bs_sums<ET, true>(q, r0, r1, D, lane, 64, part) : 0;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");   // this wave's LDS writes before its reads
    for (int d = lane; d < D; d += 64) {
        double s = 0.0;
        for (int g = 0; g < groups; ++g) s += part[g * D + d];
        mean[d] = groups > 0 ? (double)(float)(s / (double)(r1 - r0)) : 0.0;
    }
}

// `queries` query blocks (4 to 16) a workgroup of as many waves: each wave one block's
// mean, the scores of 16 query blocks (zeros past the workgroup's own) and 16 key blocks at
// a time on 16x16x4 fp64 MFMAs (lane l brings 4 consecutive values of key l % 16, a step of
// 16 values for all lanes; on the vector unit, with sums over lanes, the products took
// four times as long), then one block's choice.  Bound by its three parts one after the
// other: with one workgroup a CU nothing runs beside any of them (17550 queries of 16 heads, 128
// a block, D = 128, bf16: 28.9 us, where block_means_kernel reads and widens as many values in 13.7).
constexpr int kTileSteps = 8;   // steps of 16 values in flight
constexpr size_t select_tile_lds(int queries, int D, int nb) {
    return (size_t)queries * 8 * ((D + 2) + (nb > 512 ? nb : 512));
}
template <int ET>
__global__ __launch_bounds__(1024) void select_tile_kernel(const uint16_t* __restrict__ Q, const float* __restrict__ Km,
                                                           unsigned long long* __restrict__ Mask, int Lq, int D,
                                                           int qblock, int nq, int nb, int keep) {
    typedef double f64x4 __attribute__((ext_vector_type(4)));
    typedef double f64x2 __attribute__((ext_vector_type(2)));
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const int stride = D + 2;                        // of a mean: rows 16 bytes apart in the LDS banks
    double* mean = (double*)smem;                    // [16][stride]
    const int queries = blockDim.x >> 6;
    double* part = mean + queries * stride;          // [queries][512], then
    uint64_t* key = (uint64_t*)part;                 // [queries][nb]
    const int lane = lane_id();
    const int l16 = lane & 15, quad = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int ng = (nq + queries - 1) / queries;
    const int bh = blockIdx.x / ng, i = (blockIdx.x - bh * ng) * queries + wave;

    bs_query_mean<ET>(Q + (size_t)bh * Lq * D, i, nq, qblock, Lq, D, mean + wave * stride, part + wave * 512);
    __syncthreads();

    const float* km = Km + (size_t)bh * nb * D;
    for (int t = wave; t < (nb + 15) / 16; t += queries) {
        const float* row = km + (size_t)min(16 * t + l16, nb - 1) * D;
        f64x4 acc = {0.0, 0.0, 0.0, 0.0};
        for (int d0 = 0; d0 < D; d0 += 16 * kTileSteps) {
            f32x4 v[kTileSteps];
#pragma unroll
            for (int u = 0; u < kTileSteps; ++u) {
                const int d = d0 + 16 * u + 4 * quad;
                v[u] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
                if (d < D) v[u] = *(const f32x4*)(row + d);
            }
#pragma unroll
            for (int u = 0; u < kTileSteps; ++u) {
                const int d = d0 + 16 * u + 4 * quad;
                if (d0 + 16 * u >= D) break;
                f64x2 m[2] = {{0.0, 0.0}, {0.0, 0.0}};
                if (d < D && l16 < queries) {
                    m[0] = *(const f64x2*)(mean + l16 * stride + d);
                    m[1] = *(const f64x2*)(mean + l16 * stride + d + 2);
                }
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    acc = __builtin_amdgcn_mfma_f64_16x16x4f64(m[e >> 1][e & 1], (double)v[u][e], acc, 0, 0, 0);
            }
        }
        // lane l has column (key) l % 16 of rows (queries) l / 16 + 4 r
        if (16 * t + l16 < nb) {
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (quad + 4 * r < queries) key[(size_t)(quad + 4 * r) * nb + 16 * t + l16] = bs_key(acc[r]);
        }
    }
    __syncthreads();
    if (i < nq) bs_choose_any(key + (size_t)wave * nb, nb, keep, Mask + ((size_t)bh * nq + i) * ((nb + 63) / 64));
}

// One query block a workgroup of 16 waves: its mean by the first; the scores by all, a row
// of 16 lanes for each key block, the lanes dealt over its values, 4 NK each; the choice by
// the first.  Bound by the latency of the three, and by reading the means, 8 KB in flight a
// wave (8 query blocks of one token, 512 key blocks each, D = 128: 10.6 us; four query blocks
// a workgroup of four waves, a thread a key block, 41).
template <int ET, int NK>
__global__ __launch_bounds__(1024) void select_one_kernel(const uint16_t* __restrict__ Q, const float* __restrict__ Km,
                                                          unsigned long long* __restrict__ Mask, int Lq, int D,
                                                          int qblock, int nq, int nb, int keep) {
    constexpr int WV = 16;
    constexpr int kFlight = 8 / NK;               // key rows of a lane in flight
    extern __shared__ __attribute__((aligned(16))) char smem[];
    double* mean = (double*)smem;                 // [D]
    double* part = mean + D;                      // [512], then
    uint64_t* key = (uint64_t*)part;              // [nb]
    const int lane = lane_id();
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int bh = blockIdx.x / nq, i = blockIdx.x - bh * nq;

    if (wave == 0) bs_query_mean<ET>(Q + (size_t)bh * Lq * D, i, nq, qblock, Lq, D, mean, part);
    __syncthreads();

    const int l16 = lane & 15;
    double qv[NK][4];
#pragma unroll
    for (int k = 0; k < NK; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int d = 64 * k + 4 * l16 + e;
            qv[k][e] = d < D ? mean[d] : 0.0;
        }
    const float* km = Km + (size_t)bh * nb * D;
    for (int j0 = 4 * wave + (lane >> 4); j0 < nb; j0 += 4 * WV * kFlight) {
        f32x4 v[kFlight][NK];
#pragma unroll
        for (int u = 0; u < kFlight; ++u)
#pragma unroll
            for (int k = 0; k < NK; ++k) {
                const int j = j0 + 4 * WV * u, d = 64 * k + 4 * l16;
                v[u][k] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
                if (j < nb && d < D) v[u][k] = *(const f32x4*)(km + (size_t)j * D + d);
            }
#pragma unroll
        for (int u = 0; u < kFlight; ++u) {
            const int j = j0 + 4 * WV * u;
            double s = 0.0;
#pragma unroll
            for (int k = 0; k < NK; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e) s = fma((double)v[u][k][e], qv[k][e], s);
            s = bs_row_sum(s);
            if (l16 == 0 && j < nb) key[j] = bs_key(s);
        }
    }
    __syncthreads();
    if (wave == 0) bs_choose_any(key, nb, keep, Mask + (size_t)blockIdx.x * ((nb + 63) / 64));
}

template <typename K>
hipError_t launch_select_with(K k, const SelectArgs& a, int nq, long long grid, int threads, size_t lds) {
    if (!grid_fits(grid, threads)) return kGridTooLarge;
    const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(k),
                                                hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024);
    if (attr != hipSuccess) return attr;
    hipLaunchKernelGGL(k, dim3((unsigned)grid), dim3(threads), lds, (hipStream_t)a.stream, (const uint16_t*)a.q, a.means,
                       (unsigned long long*)a.mask, a.Lq, a.D, a.qblock, nq, a.NB, a.keep < a.NB ? a.keep : a.NB);
    return hipGetLastError();
}

template <int ET>
hipError_t launch_select_e(const SelectArgs& a) {
    const int nq = (a.Lq + a.qblock - 1) / a.qblock;
    const long long heads = (long long)a.B * a.H;
    // A workgroup of 16 waves for each query block where those are at most two for each CU
    // (single tokens), or where the LDS does not hold four rows of scores.
    if (heads * nq <= 512 || select_tile_lds(4, a.D, a.NB) > 160 * 1024) {
        const size_t lds = 8 * ((size_t)a.D + (a.NB > 512 ? a.NB : 512));
        auto k = a.D <= 64 ? select_one_kernel<ET, 1> : a.D <= 128 ? select_one_kernel<ET, 2> : select_one_kernel<ET, 4>;
        return launch_select_with(k, a, nq, heads * nq, 1024, lds);
    }
    // Else as many query blocks a workgroup as leave the fullest CU the fewest, of two
    // such numbers the larger.  The rule's number / 4 / 5 / 8 / 9 / 12 / 16, us (bf16): 16 heads, 138 query
    // blocks, 275 key blocks, D = 128 (9) 28.9 / 40.7 / 36.2 / 37.1 / 28.8 / 27.1 / 28.5; 16, 64, 64,
    // D = 40 (4) 6.6 / 6.6 / 7.0 / 7.4 / 8.2 / 8.6 / 9.5; 8, 256, 256, D = 64 (8) 12.4 / 15.4 / 16.0 / 12.3 / 13.1
    // / 12.6 / 13.2; 64, 64, 64, D = 128 (16) 20.1 / 21.5 / 25.2 / 20.3 / 26.6 / 25.7 / 20.1; 48, 64, 128,
    // D = 64 (12) 18.2 / 18.1 / 19.2 / 17.1 / 23.5 / 24.1 / 17.3.
    int best = 4;
    long long load = 0;
    for (int n = 4; n <= 16 && select_tile_lds(n, a.D, a.NB) <= 160 * 1024; ++n) {
        const long long fullest = (heads * ((nq + n - 1) / n) + 255) / 256 * n;
        if (load == 0 || fullest <= load) {
            best = n;
            load = fullest;
        }
    }
    return launch_select_with(select_tile_kernel<ET>, a, nq, heads * ((nq + best - 1) / best), 64 * best,
                              select_tile_lds(best, a.D, a.NB));
}

}  // namespace

hipError_t launch_block_means(const BlockMeansArgs& a) {
    const int nb = (a.L + kSparseBlock - 1) / kSparseBlock;
    const long long grid = (long long)a.B * a.H * nb;
    if (!grid_fits(grid, kBsThreads)) return kGridTooLarge;
    auto k = a.dtype == kF16 ? block_means_kernel<kF16> : block_means_kernel<kBF16>;
    hipLaunchKernelGGL(k, dim3((unsigned)grid), dim3(kBsThreads), 0, (hipStream_t)a.stream, (const uint16_t*)a.x,
                       a.means, a.L, a.D, nb);
    return hipGetLastError();
}

hipError_t launch_select_blocks(const SelectArgs& a) {
    return a.dtype == kF16 ? launch_select_e<kF16>(a) : launch_select_e<kBF16>(a);
}

}  // namespace sdattn
