// gated_norm.hip -- the steps between two blocks of a transformer in one pass:
//   h = skip x + gate * post(r)                      the residual, with the block's output r
//   y = pre(h) * (1 + scale) + shift                 the next block's input
// post and pre: nothing, x / sqrt(mean x^2 + eps) * gamma, or (x - mean) / sqrt(var + eps) *
// gamma + beta (population variance), over a token's C channels; gate, scale and shift one
// vector for each group of tokens.
//
// Its bound is memory: x and r read once, h and y written once.  A token belongs to a run
// of 8 to 64 lanes, or to a workgroup of four waves where tokens are few or wide, and stays in registers
// from the reads to the writes; sums are fp32, of deviations from the mean where there is one,
// and each output is rounded once.  17550 tokens of 2048 channels, x and h in fp32, both norms and all vectors:
// 90.5 us, 4.77 TB/s where a copy reaches 5.14; two latents of 4096 tokens of 320 channels 7.3 us, of which the
// bytes are 4.1 and the rest is the launch and one round trip; 16 tokens of 1280 3.8.
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
    int mod_batch;         // modulation rows from one batch item to the next; 0 where all share them
    long long sg, ss, st;  // elements from one modulation row to the next: gate, scale, shift
    int post, pre;
    float skip, eps, inv_c;
};

template <int CTRL>
__device__ __forceinline__ float gn_moved(float v) {
    return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), CTRL, 0xf, 0xf, true));
}
// sum over each run of LANES (8 to 64), in every lane of it
template <int LANES>
__device__ __forceinline__ float gn_lane_sum(float v) {
    v += gn_moved<0xb1>(v);
    v += gn_moved<0x4e>(v);
    v += gn_moved<0x141>(v);
    if constexpr (LANES > 8) v += gn_moved<0x140>(v);
    if constexpr (LANES > 16) v += __shfl_xor(v, 16, 64);
    if constexpr (LANES > 32) v = half_sum(v);
    return v;
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
    constexpr bool kEarly = CH <= 2;   // the vectors have registers of their own from the start
    __shared__ float sums[2][kGnThreads / 64];
    const int t = threadIdx.x % TEAM;
    int m = blockIdx.x * kTeams + threadIdx.x / TEAM;
    if (TEAM >= 64) m = __builtin_amdgcn_readfirstlane(m);
    if (m >= a.M) return;   // (teams of four waves: never)
    const int C = a.C, pieces = C / 8;
    const int b = m / a.L, g = (m - b * a.L) / a.per_group;
    const long long mod = (long long)b * a.mod_batch + g;
    const size_t row = (size_t)m * C;

    int turn = 0;
    auto team_sum = [&](float v) __attribute__((always_inline)) {
        v = gn_lane_sum<(TEAM > 64 ? 64 : TEAM)>(v);
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
    // this thread's pieces of 16-bit values at v
    auto fetch = [&](u32x4 (&w)[CH], const uint16_t* v) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const int c = i * TEAM + t;
            w[i] = u32x4{0u, 0u, 0u, 0u};
            if (c < pieces) w[i] = *(const u32x4*)(v + c * 8);
        }
    };
    // the vectors of channels that this call has
    enum { kGammaR, kGate, kGamma, kBeta, kScale, kShift, kVectors };
    const bool pre = a.pre != kNormNone;
    const uint16_t* const at[kVectors] = {a.r && a.post != kNormNone ? a.gamma_r : nullptr, a.r && a.gate ? a.gate + mod * a.sg : nullptr,
                                          a.y && pre ? a.gamma : nullptr, a.y && pre ? a.beta : nullptr,
                                          a.y && a.scale ? a.scale + mod * a.ss : nullptr, a.y && a.shift ? a.shift + mod * a.st : nullptr};
    u32x4 early[kEarly ? (int)kVectors : 1][CH];
    // f = op(f, vector) in every piece of this thread
    auto with = [&](float (&f)[CH][8], int n, auto op) __attribute__((always_inline)) {
        if (!at[n]) return;
        if constexpr (!kEarly) fetch(early[0], at[n]);
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            float w[8];
            gn_widen<ET>(early[kEarly ? n : 0][i], w);
#pragma unroll
            for (int e = 0; e < 8; ++e) f[i][e] = op(f[i][e], w[e]);
        }
    };
    const auto times = [](float v, float w) { return v * w; };
    const auto plus = [](float v, float w) { return v + w; };

    // everything on its way
    u32x4 rw[CH], xw[WIDE ? 2 : 1][CH];
    if (a.r) fetch(rw, a.r + row);
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        const int c = i * TEAM + t;
#pragma unroll
        for (int k = 0; k < (WIDE ? 2 : 1); ++k) {
            xw[k][i] = u32x4{0u, 0u, 0u, 0u};
            if (c < pieces) xw[k][i] = *(const u32x4*)((const char*)a.x + (row + c * 8) * (WIDE ? 4 : 2) + 16 * k);
        }
    }
    if constexpr (kEarly) {
#pragma unroll
        for (int n = 0; n < kVectors; ++n)
            if (at[n]) fetch(early[n], at[n]);
    }

    float f[CH][8];
    if (a.r) {
#pragma unroll
        for (int i = 0; i < CH; ++i) gn_widen<ET>(rw[i], f[i]);
        normed(f, a.post);
        with(f, kGammaR, times);
        with(f, kGate, times);
    }
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        const int c = i * TEAM + t;
        float w[8];
        if constexpr (WIDE) {
#pragma unroll
            for (int e = 0; e < 8; ++e) w[e] = __uint_as_float(xw[e / 4][i][e % 4]);
        } else {
            gn_widen<ET>(xw[0][i], w);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) f[i][e] = a.r ? fmaf(a.skip, w[e], f[i][e]) : a.skip * w[e];
        if (a.h && c < pieces) {
            if constexpr (WIDE) {
                *(f32x4*)((float*)a.h + row + c * 8) = f32x4{f[i][0], f[i][1], f[i][2], f[i][3]};
                *(f32x4*)((float*)a.h + row + c * 8 + 4) = f32x4{f[i][4], f[i][5], f[i][6], f[i][7]};
            } else {
                *(u32x4*)((uint16_t*)a.h + row + c * 8) = u32x4{pack2<ET>(f[i][0], f[i][1]), pack2<ET>(f[i][2], f[i][3]),
                                                                pack2<ET>(f[i][4], f[i][5]), pack2<ET>(f[i][6], f[i][7])};
            }
        }
        if (c >= pieces) {   // (a norm without a number, times a zero)
#pragma unroll
            for (int e = 0; e < 8; ++e) f[i][e] = 0.0f;
        }
    }
    if (!a.y) return;
    normed(f, a.pre);
    with(f, kGamma, times);
    with(f, kBeta, plus);
    with(f, kScale, [](float v, float w) { return fmaf(v, w, v); });
    with(f, kShift, plus);
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
    // A piece a thread and as many threads as there are pieces, down to 8 (16000 tokens of 64 channels 9.8 us with a wave
    // each, 4.7; 16384 of 160 10.6, 7.1, 16 threads with two pieces 7.3); past 64 a wave with more
    // where tokens are many, else four waves (512 tokens of 1280 5.4 us, 4.5).
    const int pieces = a.C / 8;
    if (pieces <= 8) return gated_launch<ET, WIDE, 8, 1>(a, stream);
    if (pieces <= 16) return gated_launch<ET, WIDE, 16, 1>(a, stream);
    if (pieces <= 32) return gated_launch<ET, WIDE, 32, 1>(a, stream);
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
                  n.L, n.C, n.B * n.L, n.L / n.groups, n.mod_batches == 1 ? 0 : n.groups,
                  n.gate_stride, n.scale_stride, n.shift_stride, n.norm_r, n.norm, n.skip, n.eps, 1.0f / (float)n.C};
    if (n.dtype == kF16) return n.wide ? gated_pick<kF16, true>(a, n.stream) : gated_pick<kF16, false>(a, n.stream);
    return n.wide ? gated_pick<kBF16, true>(a, n.stream) : gated_pick<kBF16, false>(a, n.stream);
}

}  // namespace sdattn
