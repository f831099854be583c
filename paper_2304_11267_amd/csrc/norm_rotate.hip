// norm_rotate.hip -- per-head norms of queries and keys with the position
// rotation in the same pass.
//
// A head's row x of D values becomes y = x / sqrt(mean(x^2) + eps) * gamma (or y = x),
// and each of its first P pairs (a, b) of y becomes
//   (a cos t - b sin t, b cos t + a sin t),   t = pos[axis of the pair] * freq[pair].
// The pairs are (2i, 2i + 1), or (i, P + i); the values past 2P keep their y.
//
// The angles depend on the token and the pair alone, so a workgroup takes a few
// tokens with all of their heads, of q and k both, and has each angle's cosine and
// sine once, in LDS, beside the tokens' places.  t is reduced to a part of a turn in 64
// bits (at a million positions a product in 32 bits would be off by 0.06), its sine and
// cosine are taken in 32.  A row belongs to G lanes, G the power of two that holds its
// items of V pairs: the sum of squares goes through them in DPP moves, and the row stays
// in registers between its read and its write, four rows of a lane in flight.
#include "device.h"
#include "launch.h"

namespace sdattn {

namespace {

constexpr int kNrThreads = 256;
constexpr int kNrTokens = 8;     // most tokens of a workgroup (2^3)
constexpr int kNrRows = 4;       // rows in flight of a group of lanes

struct NrKernel {
    const uint16_t* x[2];
    const uint16_t* gamma[2];
    uint16_t* y[2];
    const int* pos;        // [Bp, L, A]
    const float* freqs;    // [P]
    int n;                 // tensors: q, or q and k
    int H, L, D, P, A;
    int end[3];            // pairs before the second, third and fourth axis
    int pos_batch;         // positions from one batch item to the next (0: all alike)
    int x_heads, y_heads, norm;
    int tokens, log_tokens;   // of a workgroup, a power of two
    int M;                 // tokens in all
    float eps;
};

// n / d for 0 <= n < 2^23: the fp32 quotient is within one of the true one.
__device__ __forceinline__ int nr_div(int n, int d, float inv_d) {
    int q = (int)((float)n * inv_d);
    q -= (q * d > n) ? 1 : 0;
    q += ((q + 1) * d <= n) ? 1 : 0;
    return q;
}

// The sum of v over its G lanes, in each of them.
template <int CTRL>
__device__ __forceinline__ float nr_moved(float v) {
    return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), CTRL, 0xf, 0xf, true));
}
template <int G>
__device__ __forceinline__ float nr_sum(float v) {
    if constexpr (G >= 2) v += nr_moved<0xb1>(v);    // quad_perm: lane ^ 1
    if constexpr (G >= 4) v += nr_moved<0x4e>(v);    // quad_perm: lane ^ 2
    if constexpr (G >= 8) v += nr_moved<0x141>(v);   // row_half_mirror: the other four of 8
    if constexpr (G >= 16) v += nr_moved<0x140>(v);  // row_mirror: the other eight of 16
    if constexpr (G >= 32) v += __shfl_xor(v, 16, 64);
    if constexpr (G >= 64) v += __shfl_xor(v, 32, 64);
    return v;
}

// V consecutive values at p, to fp32
template <int ET, int V>
__device__ __forceinline__ void nr_load(const uint16_t* p, float* f) {
    if constexpr (V == 1) {
        f[0] = to_float<ET>(p[0]);
    } else {
        static_assert(V == 4, "");
        const u32x2 w = *(const u32x2*)p;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            f[2 * i] = to_float<ET>((uint16_t)(w[i] & 0xffffu));
            f[2 * i + 1] = to_float<ET>((uint16_t)(w[i] >> 16));
        }
    }
}
template <int ET, int V>
__device__ __forceinline__ void nr_store(uint16_t* p, const float* f) {
    if constexpr (V == 1) p[0] = from_float<ET>(f[0]);
    else *(u32x2*)p = u32x2{pack2<ET>(f[0], f[1]), pack2<ET>(f[2], f[3])};
}

// IPL items of V pairs a lane, G lanes a row
template <int ET, int V, int IPL, int G, bool HALVES>
__global__ __launch_bounds__(kNrThreads) void norm_rotate_kernel(const NrKernel a) {
    extern __shared__ __attribute__((aligned(16))) float2 turn[];   // [tokens][D / 2]
    __shared__ size_t xplace[kNrTokens], yplace[kNrTokens];         // of a token's head 0
    const int D = a.D, H = a.H, L = a.L, pairs = D / 2;
    const int m0 = blockIdx.x << a.log_tokens;
    const int tokens = min(a.tokens, a.M - m0);

    if (threadIdx.x < tokens) {
        const int m = m0 + threadIdx.x, b = m / L, l = m - b * L;
        const size_t heads = ((size_t)b * H * L + l) * D, rows = (size_t)m * H * D;
        xplace[threadIdx.x] = a.x_heads ? heads : rows;
        yplace[threadIdx.x] = a.y_heads ? heads : rows;
    }
    const float inv_pairs = 1.0f / (float)pairs;
    for (int i = threadIdx.x; i < tokens * pairs; i += kNrThreads) {
        const int t = nr_div(i, pairs, inv_pairs), p = i - t * pairs;
        float s = 0.0f, c = 1.0f;
        if (p < a.P) {
            const int axis = (p >= a.end[0]) + (p >= a.end[1]) + (p >= a.end[2]);
            const int m = m0 + t, b = m / L, l = m - b * L;
            const int at = a.pos[((size_t)b * a.pos_batch + l) * a.A + axis];
            double r = (double)at * ((double)a.freqs[p] * 0.15915494309189535);   // turns
            r -= rint(r);
            sincospif(2.0f * (float)r, &s, &c);
        }
        turn[i] = make_float2(c, s);
    }
    __syncthreads();

    const int lane = threadIdx.x % G;
    const int nrows = H << a.log_tokens;
    const float inv_h = 1.0f / (float)H, inv_d = 1.0f / (float)D;
    const size_t xstep = a.x_heads ? (size_t)L * D : D, ystep = a.y_heads ? (size_t)L * D : D;
    // the first and second values of item i's pairs
    auto first = [&](int i) { return !HALVES ? 2 * V * i : V * i < a.P ? V * i : V * i + a.P; };
    auto second = [&](int i) { return !HALVES ? 2 * V * i + V : V * i < a.P ? V * i + a.P : V * i + pairs; };

    for (int w = 0; w < a.n; ++w) {
        const uint16_t* X = a.x[w];
        uint16_t* Y = a.y[w];
        float g[IPL][2 * V];
#pragma unroll
        for (int k = 0; k < IPL; ++k) {
            const int i = lane + G * k;
#pragma unroll
            for (int e = 0; e < 2 * V; ++e) g[k][e] = 1.0f;
            if (a.norm && a.gamma[w] && V * i < pairs) {
                nr_load<ET, V>(a.gamma[w] + first(i), g[k]);
                nr_load<ET, V>(a.gamma[w] + second(i), g[k] + V);
            }
        }
        for (int r0 = threadIdx.x / G; r0 < nrows; r0 += kNrThreads / G * kNrRows) {
            float f[kNrRows][IPL][2 * V];
            size_t out[kNrRows];
            int tok[kNrRows];
#pragma unroll
            for (int u = 0; u < kNrRows; ++u) {
                const int r = r0 + u * (kNrThreads / G);
                // neighbouring rows of x: a head's tokens, or a token's heads
                int t, h;
                if (a.x_heads) {
                    h = r >> a.log_tokens;
                    t = r & (a.tokens - 1);
                } else {
                    t = nr_div(r, H, inv_h);
                    h = r - t * H;
                }
                const bool in = r < nrows && t < tokens;
                tok[u] = in ? t : -1;
                const size_t from = in ? xplace[t] + h * xstep : 0;
                out[u] = in ? yplace[t] + h * ystep : 0;
#pragma unroll
                for (int k = 0; k < IPL; ++k) {
                    const int i = lane + G * k;
#pragma unroll
                    for (int e = 0; e < 2 * V; ++e) f[u][k][e] = 0.0f;
                    if (in && V * i < pairs) {
                        nr_load<ET, V>(X + from + first(i), f[u][k]);
                        nr_load<ET, V>(X + from + second(i), f[u][k] + V);
                    }
                }
            }
#pragma unroll
            for (int u = 0; u < kNrRows; ++u) {
                float rstd = 1.0f;
                if (a.norm) {
                    float s = 0.0f;
#pragma unroll
                    for (int k = 0; k < IPL; ++k)
#pragma unroll
                        for (int e = 0; e < 2 * V; ++e) s = fmaf(f[u][k][e], f[u][k][e], s);
                    rstd = rsqrtf(fmaf(nr_sum<G>(s), inv_d, a.eps));
                }
                if (tok[u] < 0) continue;
#pragma unroll
                for (int k = 0; k < IPL; ++k) {
                    const int i = lane + G * k;
                    if (V * i >= pairs) continue;
                    float* v = f[u][k];
                    if (a.norm) {
#pragma unroll
                        for (int e = 0; e < 2 * V; ++e) v[e] = v[e] * rstd * g[k][e];
                    }
                    const float2* tn = turn + tok[u] * pairs + V * i;
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        const float c = tn[e].x, s = tn[e].y;
                        float& p0 = HALVES ? v[e] : v[2 * e];
                        float& p1 = HALVES ? v[V + e] : v[2 * e + 1];
                        const float q0 = p0 * c - p1 * s, q1 = p1 * c + p0 * s;
                        p0 = q0;
                        p1 = q1;
                    }
                    nr_store<ET, V>(Y + out[u] + first(i), v);
                    nr_store<ET, V>(Y + out[u] + second(i), v + V);
                }
            }
        }
    }
}

template <int ET, int V, int IPL, int G>
hipError_t launch_nr_g(const NrKernel& k, bool halves, void* stream) {
    auto f = halves ? norm_rotate_kernel<ET, V, IPL, G, true> : norm_rotate_kernel<ET, V, IPL, G, false>;
    const int grid = (k.M + k.tokens - 1) / k.tokens;
    hipLaunchKernelGGL(f, dim3((unsigned)grid), dim3(kNrThreads), (size_t)k.tokens * (k.D / 2) * sizeof(float2),
                       (hipStream_t)stream, k);
    return hipGetLastError();
}

template <int ET>
hipError_t launch_nr_e(const NrKernel& k, bool halves, void* stream) {
    // Pairs whose halves do not start on 8 bytes (P not a multiple of 4) go one by one.
    if (halves && k.P % 4 != 0) return launch_nr_g<ET, 1, 2, 64>(k, halves, stream);
    const int items = k.D / 8;
    if (items <= 1) return launch_nr_g<ET, 4, 1, 1>(k, halves, stream);
    if (items <= 2) return launch_nr_g<ET, 4, 1, 2>(k, halves, stream);
    if (items <= 4) return launch_nr_g<ET, 4, 1, 4>(k, halves, stream);
    if (items <= 8) return launch_nr_g<ET, 4, 1, 8>(k, halves, stream);
    if (items <= 16) return launch_nr_g<ET, 4, 1, 16>(k, halves, stream);
    return launch_nr_g<ET, 4, 1, 32>(k, halves, stream);
}

}  // namespace

hipError_t launch_norm_rotate(const NormRotateArgs& a) {
    NrKernel k{};
    k.x[0] = (const uint16_t*)a.q;
    k.x[1] = (const uint16_t*)a.k;
    k.gamma[0] = (const uint16_t*)a.gamma_q;
    k.gamma[1] = (const uint16_t*)a.gamma_k;
    k.y[0] = (uint16_t*)a.qo;
    k.y[1] = (uint16_t*)a.ko;
    k.pos = a.pos;
    k.freqs = a.freqs;
    k.n = a.k ? 2 : 1;
    k.H = a.H;
    k.L = a.L;
    k.D = a.D;
    k.A = a.axes;
    int p = 0;
    for (int i = 0; i < 4; ++i) {
        p += i < a.axes ? a.pairs[i] : 0;
        if (i < 3) k.end[i] = p;
    }
    k.P = p;
    k.pos_batch = a.pos_batches > 1 ? a.L : 0;
    k.x_heads = a.x_heads;
    k.y_heads = a.y_heads;
    k.norm = a.norm;
    k.eps = a.eps;
    k.M = a.B * a.L;
    // a workgroup's tokens: as many as leave each CU four workgroups
    while (k.log_tokens < 3 && (1024 << (k.log_tokens + 1)) <= k.M) ++k.log_tokens;
    k.tokens = 1 << k.log_tokens;
    const bool halves = a.halves;
    return a.dtype == kF16 ? launch_nr_e<kF16>(k, halves, a.stream) : launch_nr_e<kBF16>(k, halves, a.stream);
}

}  // namespace sdattn
