// attn_sparse_row.hip -- attention of one query for each head over selected key blocks
// (a single new token against a long sequence).
//
// What counts is reading the named blocks' K and V once, with enough of it in flight on
// every CU.  A workgroup of 16 waves takes one (batch, head), or where those are fewer than
// the CUs one half or quarter of its columns of V: all of the scores, then its part of O,
// with the parts of a head next to each other on one XCD, whose L2 gives K to the later
// ones.  (The keys are not split over workgroups: those parts would have to be joined through
// memory.  What that costs, and what it would give where few heads leave CUs empty, is not
// measured.)  Nothing is staged in
// LDS: a row of D values lies over a team of T lanes, 16 bytes each, and a wave takes 32
// keys at a time (16 where T = 32; 64 where a lane holds a whole row of V's part, so that a load
// of V never leaves its block), K of the next ones asked for when these scores are
// done and V when their sums are.  A key's score is its team's sum of products (v_dot2,
// fp32) over DPP moves; the scores pass through LDS to the lanes that hold V, whose rows lie
// over T / N lanes.  Each wave keeps its own running maximum, sum and O in fp32 (the weights
// too: no matrix core asks for 16 bits), and the waves are joined by the block-merge rule.
//   8 heads of 8 sequences, 32 of 512 blocks, D = 128, bf16 (67 MB): 16.0 us (4.2 TB/s, from
// memory in pieces of 16 KB); the tiled kernel takes 30.4 for two queries a head.
#include "device.h"
#include "launch.h"

namespace sdattn {

namespace {

constexpr int kRowWaves = 16;

template <int CTRL>
__device__ __forceinline__ float row_moved(float v) {
    return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), CTRL, 0xf, 0xf, true));
}
// The sum of v over a team of T lanes, in each of them (as in norm_rotate.hip).
template <int T>
__device__ __forceinline__ float team_sum(float v) {
    v += row_moved<0xb1>(v);
    v += row_moved<0x4e>(v);
    if constexpr (T >= 8) v += row_moved<0x141>(v);
    if constexpr (T >= 16) v += row_moved<0x140>(v);
    if constexpr (T >= 32) v += __shfl_xor(v, 16, 64);
    return v;
}

template <int ET, int T, int N>
__global__ __launch_bounds__(kRowWaves * 64) void sparse_row_kernel(
    const uint16_t* __restrict__ Q, const uint16_t* __restrict__ K, const uint16_t* __restrict__ V,
    const unsigned long long* __restrict__ Mask, uint16_t* __restrict__ O, int heads, int Lk, int D, int nblocks, int nw,
    float c) {
    constexpr int kTeams = 64 / T;                  // keys of one load of K
    constexpr int TV = T / N;                       // lanes of a row of V
    constexpr int kKeys = T == 32 ? 16 : TV == 1 ? 64 : 32;   // of a step: whole loads of V
    constexpr int kLoads = kKeys / kTeams;
    constexpr int kSteps = kSparseBlock / kKeys;    // of a block
    constexpr int kLoadsV = kKeys * TV / 64;
    static_assert(kLoads <= T, "a lane of each team for every load");
    static_assert(kLoadsV * 64 == kKeys * TV, "a load of V ends with the step: what follows may be a block that is not named");
    __shared__ uint16_t blocks[64 * 64];            // the named blocks among 64 words'
    __shared__ int named;
    __shared__ float score[kRowWaves][kKeys];
    __shared__ float part[kRowWaves][8 * TV], pm[kRowWaves], pl[kRowWaves];
    const int lane = lane_id();
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // a head's N parts lie 8 workgroups apart: on one XCD
    const int bh = blockIdx.x / (8 * N) * 8 + blockIdx.x % 8;
    const int col0 = blockIdx.x / 8 % N * 8 * TV;
    if (bh >= heads || col0 >= D) return;
    const int team = lane / T, tl = lane % T;
    const int vkey = lane / TV, vcol = col0 + 8 * (lane % TV);   // this lane's key and columns of a load of V
    const bool in_row = 8 * tl < D;

    u32x4 q = {0u, 0u, 0u, 0u};
    if (in_row) q = *(const u32x4*)(Q + (size_t)bh * D + 8 * tl);
    const uint16_t* Kh = K + (size_t)bh * Lk * D + (in_row ? 8 * tl : 0);
    const uint16_t* Vh = V + (size_t)bh * Lk * D + (vcol < D ? vcol : 0);

    float m = -__builtin_inff(), l = 0.0f, acc[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] = 0.0f;

    bool any = false;   // block named
    for (int w0 = 0; w0 < nw; w0 += 64) {
        if (w0 > 0) __syncthreads();   // every wave is done with the last words' blocks
        if (wave == 0) {
            const int w = w0 + lane;
            uint64_t bits = w < nw ? Mask[(size_t)bh * nw + w] : 0;
            if (w == nw - 1 && nblocks % 64 != 0) bits &= (1ull << nblocks % 64) - 1;   // no blocks past Lk
            int upto = __popcll(bits);
            for (int o = 1; o < 64; o <<= 1) {
                const int below = __shfl_up(upto, o, 64);
                upto += lane >= o ? below : 0;
            }
            for (int at = upto - __popcll(bits); bits; bits &= bits - 1) blocks[at++] = (uint16_t)(64 * lane + __builtin_ctzll(bits));
            if (lane == 63) named = upto;
        }
        __syncthreads();
        const int steps = named * kSteps;
        any = any || steps > 0;
        auto first_key = [&](int s) __attribute__((always_inline)) {
            const int j = 64 * w0 + __builtin_amdgcn_readfirstlane(blocks[s / kSteps]);
            return j * kSparseBlock + s % kSteps * kKeys;
        };
        u32x4 kv[kLoads], vv[kLoadsV];
        auto load_k = [&](int key0) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) kv[i] = *(const u32x4*)(Kh + (size_t)min(key0 + kTeams * i + team, Lk - 1) * D);
            __builtin_amdgcn_sched_barrier(0);   // none of them waits for what comes next
        };
        auto load_v = [&](int key0) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < kLoadsV; ++i) vv[i] = *(const u32x4*)(Vh + (size_t)min(key0 + 64 / TV * i + vkey, Lk - 1) * D);
            __builtin_amdgcn_sched_barrier(0);
        };
        int key0 = 0;
        if (wave < steps) {
            key0 = first_key(wave);
            load_k(key0);
            load_v(key0);
        }
        for (int s = wave; s < steps; s += kRowWaves) {
            float mine = 0.0f, top = -__builtin_inff();
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                // (lanes past D have q = 0; what they read is in the row)
                float p = team_sum<T>(in_row ? dot8<ET>(kv[i], q, 0.0f) : 0.0f) * c;
                if (key0 + kTeams * i + team >= Lk) p = -__builtin_inff();   // weight 0
                top = fmaxf(top, p);
                mine = tl == i ? p : mine;
            }
            const bool more = s + kRowWaves < steps;
            if (more) {
                key0 = first_key(s + kRowWaves);
                load_k(key0);
            }
            // the scores, key by key, to the lanes that hold V (a wave's own: no barrier)
            if (tl < kLoads) score[wave][kTeams * tl + team] = mine;
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int o = T; o < 64; o <<= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
            const float m_new = fmaxf(m, top);
            if (m_new != -__builtin_inff()) {   // (no key yet: a step past Lk, or infinite products)
                const float alpha = fast_exp2(m - m_new);
                m = m_new;
                l *= alpha;
#pragma unroll
                for (int e = 0; e < 8; ++e) acc[e] *= alpha;
#pragma unroll
                for (int i = 0; i < kLoadsV; ++i) {
                    const float p = fast_exp2(score[wave][64 / TV * i + vkey] - m_new);
                    l += p;
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        acc[e] = fmaf(p, to_float<ET>((uint16_t)(vv[i][e >> 1] >> (16 * (e & 1)))), acc[e]);
                }
            } else if (__any(mine != mine)) {   // products that are no number are no weight 0
                l = __builtin_nanf("");
            }
            __builtin_amdgcn_wave_barrier();
            if (more) load_v(key0);
        }
    }

    // the rows of a wave, then the waves
#pragma unroll
    for (int o = TV; o < 64; o <<= 1) {
        l += __shfl_xor(l, o, 64);
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] += __shfl_xor(acc[e], o, 64);
    }
    if (vkey == 0) {
        *(f32x4*)&part[wave][8 * lane] = f32x4{acc[0], acc[1], acc[2], acc[3]};
        *(f32x4*)&part[wave][8 * lane + 4] = f32x4{acc[4], acc[5], acc[6], acc[7]};
    }
    if (lane == 0) {
        pm[wave] = m;
        pl[wave] = l;
    }
    __syncthreads();
    const int d = threadIdx.x;
    if (d >= 8 * TV || col0 + d >= D) return;
    float top = -__builtin_inff(), sum = 0.0f, o = 0.0f;
#pragma unroll
    for (int w = 0; w < kRowWaves; ++w) top = fmaxf(top, pm[w]);
    if (top != -__builtin_inff()) {
#pragma unroll
        for (int w = 0; w < kRowWaves; ++w) {
            const float a = fast_exp2(pm[w] - top);
            sum = fmaf(pl[w], a, sum);
            o = fmaf(part[w][d], a, o);
        }
        o /= sum;
    } else if (any) {
        o = __builtin_nanf("");   // no product of a named block is a number, or all are minus infinity
    }
    O[(size_t)bh * D + col0 + d] = from_float<ET>(o);   // 0 where no block is named
}

template <int ET, int N>
hipError_t launch_row_n(const SparseArgs& s) {
    const int nb = (s.Lk + kSparseBlock - 1) / kSparseBlock, nw = (nb + 63) / 64;
    const int heads = s.B * s.H;   // (check_attention has seen that these fit)
    if (!grid_fits(((long long)heads + 7) / 8 * 8 * N, kRowWaves * 64)) return kGridTooLarge;
    auto k = s.D <= 32 ? sparse_row_kernel<ET, 4, N> : s.D <= 64 ? sparse_row_kernel<ET, 8, N>
           : s.D <= 128 ? sparse_row_kernel<ET, 16, N> : sparse_row_kernel<ET, 32, N>;
    hipLaunchKernelGGL(k, dim3((unsigned)((heads + 7) / 8 * 8 * N)), dim3(kRowWaves * 64), 0, (hipStream_t)s.stream,
                       (const uint16_t*)s.q, (const uint16_t*)s.k, (const uint16_t*)s.v, (const unsigned long long*)s.mask,
                       (uint16_t*)s.out, heads, s.Lk, s.D, nb, nw, s.scale * kLog2e);
    return hipGetLastError();
}

template <int ET>
hipError_t launch_row_e(const SparseArgs& s) {
    // Parts of a head, whole / halves / quarters, us: 1 head, 32 blocks, D = 128 14.9 / 12.7 / 11.4; 8 heads
    // 15.9 / 13.3 / 12.2; 64 20.8 / 17.1 / 16.0; 128 29.3 / 26.4 / 38.3, D = 80 19.8 / 17.9 / 29.4; 320 heads,
    // 16 blocks, D = 128 40.7 / 42.4 / 58.8.
    const long long heads = (long long)s.B * s.H;
    return heads <= 64 ? launch_row_n<ET, 4>(s) : heads <= 128 ? launch_row_n<ET, 2>(s) : launch_row_n<ET, 1>(s);
}

}  // namespace

hipError_t launch_attn_sparse_row(const SparseArgs& a) {
    return a.dtype == kF16 ? launch_row_e<kF16>(a) : launch_row_e<kBF16>(a);
}

}  // namespace sdattn
