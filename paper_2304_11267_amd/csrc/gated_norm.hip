// gated_norm.hip -- the steps between two blocks of a transformer in one pass:
//   h = skip x + gate * post(r)                      the residual, with the block's output r
//   y = pre(h) * (1 + scale) + shift                 the next block's input
// post and pre: nothing, x / sqrt(mean x^2 + eps) * gamma, or (x - mean) / sqrt(var + eps) *
// gamma + beta (population variance), over a token's C channels; gate, scale and shift one
// vector for each group of tokens.
//
// Its bound is memory: x and r read once, h and y written once.  A token belongs to one wave,
// or to a workgroup of four where tokens are few or wide, and stays in registers
// from the reads to the writes; sums are fp32, of deviations from the mean where there is one,
// and each output is rounded once.
#include "device.h"
#include "launch.h"

namespace sdattn {

namespace {

constexpr int kGnThreads = 256;

struct GatedKernel {
    const void* x;
    const uint16_t* r;
    const uint16_t* gate;
    const uint16_t* scale;
    const uint16_t* shift;
    const uint16_t* gamma_r;
    const uint16_t* gamma;
    const uint16_t* beta;
    void* h;
    uint16_t* y;
    int L, C, M;
    int per_group;         // tokens of a modulation group
    int groups;            // of a batch item; 0 rows apart for batch items that share them
    int mod_batch;         // modulation rows from one batch item to the next
    long long sg, ss, st;  // elements from one modulation row to the next: gate, scale, shift
    int post, pre;
    float skip, eps, inv_c;
};

template <int CTRL>
__device__ __forceinline__ float gn_moved(float v) {
    return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), CTRL, 0xf, 0xf, true));
}
// sum over a wave, in every lane
__device__ __forceinline__ float gn_wave_sum(float v) {
    v += gn_moved<0xb1>(v);
    v += gn_moved<0x4e>(v);
    v += gn_moved<0x141>(v);
    v += gn_moved<0x140>(v);
    v += __shfl_xor(v, 16, 64);
    return half_sum(v);
}

template <int ET>
__device__ __forceinline__ void gn_widen(u32x4 w, float* f) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = to_float<ET>((uint16_t)(w[i] & 0xffffu));
        f[2 * i + 1] = to_float<ET>((uint16_t)(w[i] >> 16));
    }
}

// TEAM threads a token, CH pieces of 8 channels a thread; WIDE: x and h are fp32.
template <int ET, bool WIDE, int TEAM, int CH>
__global__ __launch_bounds__(kGnThreads) void gated_norm_kernel(const GatedKernel a) {
    constexpr int kTeams = kGnThreads / TEAM;
    __shared__ float sums[2][kGnThreads / 64];
    const int t = threadIdx.x % TEAM;
    const int m = blockIdx.x * kTeams + (TEAM == 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x / TEAM) : 0);
    if (m >= a.M) return;   // (teams of four waves: never)
    const int C = a.C, pieces = C / 8;
    const int b = m / a.L, g = (m - b * a.L) / a.per_group;
    const long long mod = (long long)b * a.mod_batch + g;

    int turn = 0;
    auto team_sum = [&](float v) __attribute__((always_inline)) {
        v = gn_wave_sum(v);
        if constexpr (TEAM > 64) {
            if (threadIdx.x % 64 == 0) sums[turn][threadIdx.x / 64] = v;
            __syncthreads();
            v = 0.0f;
#pragma unroll
            for (int w = 0; w < kGnThreads / 64; ++w) v += sums[turn][w];
            turn ^= 1;   // (a wave may be a sum ahead of another, never two)
        }
        return v;
    };
    // f = norm(f) without its gamma; `how` is the same for all threads
    auto normed = [&](float (&f)[CH][8], int how) __attribute__((always_inline)) {
        if (how == kNormNone) return;
        float s = 0.0f;
        if (how == kNormLayer) {
#pragma unroll
            for (int i = 0; i < CH; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) s += f[i][e];
            const float mean = team_sum(s) * a.inv_c;
#pragma unroll
            for (int i = 0; i < CH; ++i) {
                const bool in = i * TEAM + t < pieces;
#pragma unroll
                for (int e = 0; e < 8; ++e) f[i][e] = in ? f[i][e] - mean : 0.0f;
            }
            s = 0.0f;
        }
#pragma unroll
        for (int i = 0; i < CH; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) s = fmaf(f[i][e], f[i][e], s);
        const float rstd = 1.0f / sqrtf(fmaf(team_sum(s), a.inv_c, a.eps));
#pragma unroll
        for (int i = 0; i < CH; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) f[i][e] *= rstd;
    };
    // f = op(f, v) for a vector v of channels, in every piece of this thread
    auto with = [&](float (&f)[CH][8], const uint16_t* v, auto op) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const int c = i * TEAM + t;
            if (c >= pieces) continue;
            float w[8];
            gn_widen<ET>(*(const u32x4*)(v + c * 8), w);
#pragma unroll
            for (int e = 0; e < 8; ++e) f[i][e] = op(f[i][e], w[e]);
        }
    };

    float f[CH][8];
    const size_t row = (size_t)m * C;
    if (a.r) {
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const int c = i * TEAM + t;
            u32x4 w = {0u, 0u, 0u, 0u};
            if (c < pieces) w = *(const u32x4*)(a.r + row + c * 8);
            gn_widen<ET>(w, f[i]);
        }
        normed(f, a.post);
        if (a.post != kNormNone && a.gamma_r) with(f, a.gamma_r, [](float v, float g) { return v * g; });
        if (a.gate) with(f, a.gate + mod * a.sg, [](float v, float g) { return v * g; });
    }
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        const int c = i * TEAM + t;
        float w[8];
        if (c >= pieces) {
#pragma unroll
            for (int e = 0; e < 8; ++e) f[i][e] = 0.0f;
            continue;
        }
        if constexpr (WIDE) {
            const f32x4 lo = *(const f32x4*)((const float*)a.x + row + c * 8), hi = *(const f32x4*)((const float*)a.x + row + c * 8 + 4);
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = lo[e], w[4 + e] = hi[e];
        } else {
            gn_widen<ET>(*(const u32x4*)((const uint16_t*)a.x + row + c * 8), w);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) f[i][e] = a.r ? fmaf(a.skip, w[e], f[i][e]) : a.skip * w[e];
        if (a.h) {
            if constexpr (WIDE) {
                *(f32x4*)((float*)a.h + row + c * 8) = f32x4{f[i][0], f[i][1], f[i][2], f[i][3]};
                *(f32x4*)((float*)a.h + row + c * 8 + 4) = f32x4{f[i][4], f[i][5], f[i][6], f[i][7]};
            } else {
                *(u32x4*)((uint16_t*)a.h + row + c * 8) = u32x4{pack2<ET>(f[i][0], f[i][1]), pack2<ET>(f[i][2], f[i][3]),
                                                                pack2<ET>(f[i][4], f[i][5]), pack2<ET>(f[i][6], f[i][7])};
            }
        }
    }
    if (!a.y) return;
    normed(f, a.pre);
    if (a.pre != kNormNone) {
        if (a.gamma) with(f, a.gamma, [](float v, float g) { return v * g; });
        if (a.beta) with(f, a.beta, [](float v, float g) { return v + g; });
    }
    if (a.scale) with(f, a.scale + mod * a.ss, [](float v, float g) { return fmaf(v, g, v); });
    if (a.shift) with(f, a.shift + mod * a.st, [](float v, float g) { return v + g; });
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        const int c = i * TEAM + t;
        if (c < pieces)
            *(u32x4*)(a.y + row + c * 8) = u32x4{pack2<ET>(f[i][0], f[i][1]), pack2<ET>(f[i][2], f[i][3]),
                                                 pack2<ET>(f[i][4], f[i][5]), pack2<ET>(f[i][6], f[i][7])};
    }
}

template <int ET, bool WIDE, int TEAM, int CH>
hipError_t gated_launch(const GatedKernel& a, void* stream) {
    const long long wgs = ((long long)a.M + kGnThreads / TEAM - 1) / (kGnThreads / TEAM);
    if (!grid_fits(wgs, kGnThreads)) return kGridTooLarge;
    hipLaunchKernelGGL((gated_norm_kernel<ET, WIDE, TEAM, CH>), dim3((unsigned)wgs), dim3(kGnThreads), 0, (hipStream_t)stream, a);
    return hipGetLastError();
}

template <int ET, bool WIDE>
hipError_t gated_pick(const GatedKernel& a, void* stream) {
    // Many tokens: a wave each; few or wide ones: a workgroup each.
    const int pieces = a.C / 8;
    if (pieces <= 64) return gated_launch<ET, WIDE, 64, 1>(a, stream);
    if (a.M >= 1024) {
        if (pieces <= 128) return gated_launch<ET, WIDE, 64, 2>(a, stream);
        if (pieces <= 192) return gated_launch<ET, WIDE, 64, 3>(a, stream);
        if (pieces <= 256) return gated_launch<ET, WIDE, 64, 4>(a, stream);
    }
    if (pieces <= 256) return gated_launch<ET, WIDE, 256, 1>(a, stream);
    if (pieces <= 512) return gated_launch<ET, WIDE, 256, 2>(a, stream);
    if (pieces <= 1024) return gated_launch<ET, WIDE, 256, 4>(a, stream);
    return gated_launch<ET, WIDE, 256, 8>(a, stream);
}

}  // namespace

hipError_t launch_gated_norm(const GatedNormArgs& n) {
    GatedKernel a{n.x, (const uint16_t*)n.r, (const uint16_t*)n.gate, (const uint16_t*)n.scale, (const uint16_t*)n.shift,
                  (const uint16_t*)n.gamma_r, (const uint16_t*)n.gamma, (const uint16_t*)n.beta, n.h, (uint16_t*)n.y,
                  n.L, n.C, n.B * n.L, n.L / n.groups, n.groups, n.mod_batches == 1 ? 0 : n.groups,
                  n.gate_stride, n.scale_stride, n.shift_stride, n.norm_r, n.norm, n.skip, n.eps, 1.0f / (float)n.C};
    if (n.dtype == kF16) return n.wide ? gated_pick<kF16, true>(a, n.stream) : gated_pick<kF16, false>(a, n.stream);
    return n.wide ? gated_pick<kBF16, true>(a, n.stream) : gated_pick<kBF16, false>(a, n.stream);
}

}  // namespace sdattn
