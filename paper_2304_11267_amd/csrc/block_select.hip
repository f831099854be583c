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
// fp32 means are too, and only scores that agree to 50 bits could fall otherwise than
// the formula says.
#include "device.h"
#include "launch.h"

namespace sdattn {

namespace {

constexpr int kBsThreads = 256;
constexpr int kBsQueries = 4;             // query blocks of a workgroup, one a wave

// Sums of rows [r0, r1) of x, D / 8 chunks of 8 values a row, over the lanes of a
// team of `size` threads of which this is `id`; part holds teams' rows of D doubles.
// Returns the number of partial rows.
template <int ET>
__device__ __forceinline__ int bs_sums(const uint16_t* x, int r0, int r1, int D, int id, int size, double* part) {
    const int cols = D / 8;
    const int groups = min(size / cols, r1 - r0);
    const int g = id / cols, c = id - g * cols;
    if (g < groups) {
        double s[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) s[e] = 0.0;
        for (int r = r0 + g; r < r1; r += groups) {
            const u32x4 v = *(const u32x4*)(x + (size_t)r * D + 8 * c);
#pragma unroll
            for (int e = 0; e < 8; ++e) s[e] += (double)to_float<ET>((uint16_t)(v[e >> 1] >> (16 * (e & 1))));
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
    const int groups = bs_sums<ET>(X + (size_t)bh * L * D, r0, r1, D, threadIdx.x, kBsThreads, part);
    __syncthreads();
    for (int d = threadIdx.x; d < D; d += kBsThreads) {
        double s = 0.0;
        for (int g = 0; g < groups; ++g) s += part[g * D + d];
        Mn[((size_t)bh * nb + j) * D + d] = (float)(s / (double)(r1 - r0));
    }
}

// Scores as 64-bit integers of the same order (-0 as 0).
__device__ __forceinline__ uint64_t bs_key(double s) {
    const uint64_t u = (uint64_t)__double_as_longlong(s + 0.0);
    return u >> 63 ? ~u : u | (1ull << 63);
}

// QG query blocks a workgroup: their means, the scores against every key block, then
// a wave for each one's choice.
template <int ET, int QG>
__global__ __launch_bounds__(kBsThreads) void select_kernel(const uint16_t* __restrict__ Q, const float* __restrict__ Km,
                                                            unsigned long long* __restrict__ Mask, int Lq, int D,
                                                            int qblock, int nq, int nb, int keep) {
    extern __shared__ __attribute__((aligned(16))) char smem[];
    double* mean = (double*)smem;                 // [QG][D]
    double* part = mean + QG * D;                 // [4 waves][512], then
    uint64_t* key = (uint64_t*)part;              // [QG][nb]
    const int lane = lane_id();
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int ng = (nq + QG - 1) / QG;
    const int bh = blockIdx.x / ng, i0 = (blockIdx.x - bh * ng) * QG;
    const int count = min(QG, nq - i0);

    for (int base = 0; base < QG; base += 4) {
        const int q = base + wave;
        int groups = 0;
        double rows = 1.0;
        if (q < count) {
            const int r0 = (i0 + q) * qblock, r1 = min(Lq, r0 + qblock);
            groups = bs_sums<ET>(Q + (size_t)bh * Lq * D, r0, r1, D, lane, 64, part + wave * 512);
            rows = (double)(r1 - r0);
        }
        __syncthreads();
        if (q < count) {
            for (int d = lane; d < D; d += 64) {
                double s = 0.0;
                for (int g = 0; g < groups; ++g) s += part[wave * 512 + g * D + d];
                mean[q * D + d] = (double)(float)(s / rows);
            }
        } else if (q < QG) {
            for (int d = lane; d < D; d += 64) mean[q * D + d] = 0.0;
        }
        __syncthreads();
    }

    for (int j = threadIdx.x; j < nb; j += kBsThreads) {
        const float* km = Km + ((size_t)bh * nb + j) * D;
        double s[QG];
#pragma unroll
        for (int q = 0; q < QG; ++q) s[q] = 0.0;
        for (int d = 0; d < D; d += 4) {
            const f32x4 k = *(const f32x4*)(km + d);
#pragma unroll
            for (int q = 0; q < QG; ++q)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[q] = fma((double)k[e], mean[q * D + d + e], s[q]);
        }
#pragma unroll
        for (int q = 0; q < QG; ++q) key[(size_t)q * nb + j] = bs_key(s[q]);
    }
    __syncthreads();

    const int nw = (nb + 63) / 64;
    for (int q = wave; q < count; q += 4) {
        const uint64_t* kq = key + (size_t)q * nb;
        // the keep-th largest key, bit by bit, until some value parts exactly `keep` off
        uint64_t at = 0;
        int n = nb;
        for (int bit = 63; bit >= 0 && n != keep; --bit) {
            const uint64_t cand = at | (1ull << bit);
            int c = 0;
            for (int j = lane; j < nw * 64; j += 64) c += __popcll(__ballot(j < nb && kq[min(j, nb - 1)] >= cand));
            if (c >= keep) {
                at = cand;
                n = c;
            }
        }
        // n keys are >= at; where they are too many, `at` is the keep-th largest and
        // the last of its equals are left out
        int equal = nb;
        if (n != keep) {
            int above = 0;
            for (int j = lane; j < nw * 64; j += 64) above += __popcll(__ballot(j < nb && kq[min(j, nb - 1)] > at));
            equal = keep - above;
        }
        unsigned long long* row = Mask + ((size_t)bh * nq + i0 + q) * nw;
        for (int w = 0; w < nw; ++w) {
            const int j = 64 * w + lane;
            const uint64_t k = kq[min(j, nb - 1)];
            const uint64_t over = __ballot(j < nb && k > at), same = __ballot(j < nb && k == at);
            const bool take = (over >> lane & 1) || ((same >> lane & 1) && __popcll(same & ((1ull << lane) - 1)) < equal);
            const uint64_t word = __ballot(take);
            equal -= min(equal, (int)__popcll(same));
            if (lane == 0) row[w] = word;
        }
    }
}

template <int ET, int QG>
hipError_t launch_select_q(const SelectArgs& a, int nq, int nb) {
    const long long grid = (long long)a.B * a.H * ((nq + QG - 1) / QG);
    if (grid > 0x7fffffff) return hipErrorInvalidValue;
    const size_t scores = (size_t)QG * nb * 8, parts = 4 * 512 * 8;
    const size_t lds = (size_t)QG * a.D * 8 + (scores > parts ? scores : parts);
    auto k = select_kernel<ET, QG>;
    static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(k),
                                                       hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024);
    if (attr != hipSuccess) return attr;
    hipLaunchKernelGGL(k, dim3((unsigned)grid), dim3(kBsThreads), lds, (hipStream_t)a.stream, (const uint16_t*)a.q,
                       a.means, (unsigned long long*)a.mask, a.Lq, a.D, a.qblock, nq, nb, a.keep < nb ? a.keep : nb);
    return hipGetLastError();
}

template <int ET>
hipError_t launch_select_e(const SelectArgs& a) {
    const int nq = (a.Lq + a.qblock - 1) / a.qblock, nb = a.NB;
    // the scores of a workgroup's query blocks lie in LDS: 4 rows of 4096, or one of kSelectMaxBlocks
    return nb <= kSelectMaxBlocks / kBsQueries ? launch_select_q<ET, kBsQueries>(a, nq, nb) : launch_select_q<ET, 1>(a, nq, nb);
}

}  // namespace

hipError_t launch_block_means(const BlockMeansArgs& a) {
    const int nb = (a.L + kSparseBlock - 1) / kSparseBlock;
    const long long grid = (long long)a.B * a.H * nb;
    if (grid > 0x7fffffff) return hipErrorInvalidValue;
    auto k = a.dtype == kF16 ? block_means_kernel<kF16> : block_means_kernel<kBF16>;
    hipLaunchKernelGGL(k, dim3((unsigned)grid), dim3(kBsThreads), 0, (hipStream_t)a.stream, (const uint16_t*)a.x,
                       a.means, a.L, a.D, nb);
    return hipGetLastError();
}

hipError_t launch_select_blocks(const SelectArgs& a) {
    return a.dtype == kF16 ? launch_select_e<kF16>(a) : launch_select_e<kBF16>(a);
}

}  // namespace sdattn
