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
// sine once, from LDS, times the gammas in registers of the lanes that turn with it.  t is reduced to a part of a turn in 64
// bits (at a million positions a product in 32 bits would be off by 0.06), its sine and
// cosine are taken in 32.  A row belongs to G lanes, G the power of two that holds its
// items of V pairs: the sum of squares goes through them in DPP moves, and the row stays
// in registers between its read and its write.
#include "device.h"
#include "launch.h"

namespace sdattn {

namespace {

constexpr int kNrThreads = 256;
constexpr int kNrTokens = 8;     // most tokens of a workgroup (2^3)
constexpr int kNrRows = 2;       // rows of 4 pairs a lane in flight (of 8 pairs: half as many)

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

// V consecutive values as they lie in memory
template <int V>
using NrRaw = typename std::conditional<V == 1, uint16_t, typename std::conditional<V == 4, u32x2, u32x4>::type>::type;
template <int ET, int V>
__device__ __forceinline__ void nr_widen(NrRaw<V> w, float* f) {
    if constexpr (V == 1) {
        f[0] = to_float<ET>(w);
    } else {
#pragma unroll
        for (int i = 0; i < V / 2; ++i) {
            f[2 * i] = to_float<ET>((uint16_t)(w[i] & 0xffffu));
            f[2 * i + 1] = to_float<ET>((uint16_t)(w[i] >> 16));
        }
    }
}
// and from an address of 8 bytes' alignment (the gammas')
template <int V>
__device__ __forceinline__ NrRaw<V> nr_read8(const uint16_t* p) {
    if constexpr (V == 8) {
        const u32x2 lo = *(const u32x2*)p, hi = *(const u32x2*)(p + 4);
        return u32x4{lo[0], lo[1], hi[0], hi[1]};
    } else {
        return *(const NrRaw<V>*)p;
    }
}
template <int ET, int V>
__device__ __forceinline__ void nr_store(uint16_t* p, const float* f) {
    if constexpr (V == 1) {
        p[0] = from_float<ET>(f[0]);
    } else {
        NrRaw<V> w;
#pragma unroll
        for (int i = 0; i < V / 2; ++i) w[i] = pack2<ET>(f[2 * i], f[2 * i + 1]);
        *(NrRaw<V>*)p = w;
    }
}

// IPL items of V pairs a lane, G lanes a row, IDX the type of places in the tensors.  With
// q and k, two waves each: what differs between them is the same for a whole wave.
template <int ET, int V, int IPL, int G, bool HALVES, typename IDX>
__global__ __launch_bounds__(kNrThreads) void norm_rotate_kernel(const NrKernel a) {
    using Raw = NrRaw<V>;
    constexpr int kRows = V == 8 ? kNrRows / 2 : kNrRows;
    extern __shared__ __attribute__((aligned(16))) float2 turn[];   // [tokens][D / 2]
    __shared__ IDX xplace[kNrTokens], yplace[kNrTokens];            // of a token's head 0
    const int D = a.D, H = a.H, L = a.L, pairs = D / 2;
    const int m0 = blockIdx.x << a.log_tokens;
    const int tokens = min(a.tokens, a.M - m0);

    if (threadIdx.x < tokens) {
        const int m = m0 + threadIdx.x, b = m / L, l = m - b * L;
        const IDX heads = ((IDX)b * H * L + l) * D, rows = (IDX)m * H * D;
        xplace[threadIdx.x] = a.x_heads ? heads : rows;
        yplace[threadIdx.x] = a.y_heads ? heads : rows;
    }
    // an angle's position and frequency (its pair among the turned ones)
    const float inv_pairs = 1.0f / (float)pairs;
    auto place_of = [&](int i, int* at, float* freq) __attribute__((always_inline)) {
        const int t = nr_div(i, pairs, inv_pairs), p = i - t * pairs;
        *at = 0;
        *freq = 0.0f;   // an angle of 0 for the pairs that are not turned
        if (i < tokens * pairs && p < a.P) {
            const int axis = (p >= a.end[0]) + (p >= a.end[1]) + (p >= a.end[2]);
            const int m = m0 + t, b = m / L, l = m - b * L;
            *at = a.pos[((size_t)b * a.pos_batch + l) * a.A + axis];
            *freq = a.freqs[p];
        }
    };
    int at;
    float freq;
    place_of(threadIdx.x, &at, &freq);
    __syncthreads();

    const int lane = threadIdx.x % G;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int w = a.n > 1 ? wave >> 1 : 0;                       // this wave's tensor
    const int team = (threadIdx.x - (w << 7)) / G, teams = (a.n > 1 ? 128 : 256) / G;
    // this team's token, and its heads h0, h0 + hstep, ...
    const int t = team & (a.tokens - 1), h0 = team >> a.log_tokens, hstep = teams >> a.log_tokens;
    const bool in = t < tokens;
    const IDX xstep = a.x_heads ? (IDX)L * D : D, ystep = a.y_heads ? (IDX)L * D : D;
    const uint16_t* X = a.x[w];
    uint16_t* Y = a.y[w];
    const IDX from = in ? xplace[t] : 0, to = in ? yplace[t] : 0;
    const float inv_d = 1.0f / (float)D;
    // the first and second values of item i's pairs
    auto first = [&](int i) { return !HALVES ? 2 * V * i : V * i < a.P ? V * i : V * i + a.P; };
    auto second = [&](int i) { return !HALVES ? 2 * V * i + V : V * i < a.P ? V * i + a.P : V * i + pairs; };
    Raw raw[kRows][IPL][2];
    auto load = [&](int h) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < kRows; ++u)
#pragma unroll
            for (int k = 0; k < IPL; ++k) {
                const int i = lane + G * k;
                raw[u][k][0] = raw[u][k][1] = Raw{};
                if (in && h + u * hstep < H && V * i < pairs) {
                    const IDX row = from + (h + u * hstep) * xstep;
                    raw[u][k][0] = *(const Raw*)(X + (IDX)(row + first(i)));
                    raw[u][k][1] = *(const Raw*)(X + (IDX)(row + second(i)));
                }
            }
    };
    load(h0);   // on its way beside the angles
    float g[IPL][2 * V];
    const uint16_t* Gamma = a.norm ? a.gamma[w] : nullptr;
#pragma unroll
    for (int k = 0; k < IPL; ++k) {
        const int i = lane + G * k;
#pragma unroll
        for (int e = 0; e < 2 * V; ++e) g[k][e] = 1.0f;
        if (Gamma && V * i < pairs) {
            nr_widen<ET, V>(nr_read8<V>(Gamma + first(i)), g[k]);
            nr_widen<ET, V>(nr_read8<V>(Gamma + second(i)), g[k] + V);
        }
    }

    for (int i = threadIdx.x; i < tokens * pairs; i += kNrThreads) {
        if (i != threadIdx.x) place_of(i, &at, &freq);
        double r = (double)at * ((double)freq * 0.15915494309189535);   // turns
        r -= rint(r);
        float s, c;
        sincospif(2.0f * (float)r, &s, &c);
        turn[i] = make_float2(c, s);
    }
    __syncthreads();

    // pair e of item k: (p0, p1) -> (p0 own[0] - p1 other[1], p1 own[1] + p0 other[0]), the
    // gammas in the sine and cosine
    float own[IPL][V][2], other[IPL][V][2];
#pragma unroll
    for (int k = 0; k < IPL; ++k)
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const int p = V * (lane + G * k) + e;
            float2 cs = make_float2(1.0f, 0.0f);
            if (in && p < pairs) cs = turn[t * pairs + p];
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const float ga = g[k][HALVES ? V * q + e : 2 * e + q];
                own[k][e][q] = ga * cs.x;
                other[k][e][q] = ga * cs.y;
            }
        }

    for (int h = h0; h < H; h += hstep * kRows) {
        if (h != h0) load(h);
#pragma unroll
        for (int u = 0; u < kRows; ++u) {
            float f[IPL][2 * V];
#pragma unroll
            for (int k = 0; k < IPL; ++k) {
                nr_widen<ET, V>(raw[u][k][0], f[k]);
                nr_widen<ET, V>(raw[u][k][1], f[k] + V);
            }
            float rstd = 1.0f;
            if (a.norm) {
                float s = 0.0f;
#pragma unroll
                for (int k = 0; k < IPL; ++k)
#pragma unroll
                    for (int e = 0; e < 2 * V; ++e) s = fmaf(f[k][e], f[k][e], s);
                rstd = rsqrtf(fmaf(nr_sum<G>(s), inv_d, a.eps));
            }
            if (!in || h + u * hstep >= H) continue;
            const IDX row = to + (h + u * hstep) * ystep;
            auto turned = [&](auto all) __attribute__((always_inline)) {
#pragma unroll
                for (int k = 0; k < IPL; ++k) {
                    const int i = lane + G * k;
                    if (V * i >= pairs) continue;
                    float* v = f[k];
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        float& p0 = HALVES ? v[e] : v[2 * e];
                        float& p1 = HALVES ? v[V + e] : v[2 * e + 1];
                        // (a value that is not turned never meets its neighbour, which may be no number)
                        const bool turns = decltype(all)::value || V * i + e < a.P;
                        const float q0 = turns ? p0 * own[k][e][0] - p1 * other[k][e][1] : p0 * own[k][e][0];
                        const float q1 = turns ? p1 * own[k][e][1] + p0 * other[k][e][0] : p1 * own[k][e][1];
                        p0 = q0 * rstd;
                        p1 = q1 * rstd;
                    }
                    nr_store<ET, V>(Y + (IDX)(row + first(i)), v);
                    nr_store<ET, V>(Y + (IDX)(row + second(i)), v + V);
                }
            };
            if (a.P == pairs) turned(std::true_type{});
            else turned(std::false_type{});
        }
    }
}

template <int ET, int V, int IPL, int G>
hipError_t launch_nr_g(NrKernel k, bool halves, void* stream) {
    // places in 32 bits where the tensors have fewer than 2^32 bytes
    const bool far = (long long)k.M * k.H * k.D * 2 >= (1LL << 32);
    auto f = halves ? (far ? norm_rotate_kernel<ET, V, IPL, G, true, size_t> : norm_rotate_kernel<ET, V, IPL, G, true, uint32_t>)
                    : (far ? norm_rotate_kernel<ET, V, IPL, G, false, size_t> : norm_rotate_kernel<ET, V, IPL, G, false, uint32_t>);
    // Tokens of a workgroup: at most a team each (a team's heads then share its angles) and 8;
    // more of them while teams would have no head, or while that leaves each CU four workgroups and
    // a team fewer than four rounds of heads.  8 tokens / 4, us: 2 x 4096 tokens, 8 heads, D = 64
    // (2 rounds / 1) 9.1 / 10.9; 17550, 16 heads, D = 128 (8 / 4) 60.8 / 58.7.
    const int teams = (k.n > 1 ? 128 : 256) / G, rows = V == 8 ? kNrRows / 2 : kNrRows;
    while ((1 << k.log_tokens) < kNrTokens && (1 << k.log_tokens) < teams &&
           ((teams >> k.log_tokens) > k.H ||
            ((1024 << (k.log_tokens + 1)) <= k.M && ((long long)k.H << k.log_tokens) < 4LL * teams * rows)))
        ++k.log_tokens;
    k.tokens = 1 << k.log_tokens;
    const int grid = (k.M + k.tokens - 1) / k.tokens;
    if (!grid_fits(grid, kNrThreads)) return kGridTooLarge;
    hipLaunchKernelGGL(f, dim3((unsigned)grid), dim3(kNrThreads), (size_t)k.tokens * (k.D / 2) * sizeof(float2),
                       (hipStream_t)stream, k);
    return hipGetLastError();
}

template <int ET>
hipError_t launch_nr_e(const NrKernel& k, bool halves, void* stream) {
    // Pairs whose halves do not start on 8 bytes (P not a multiple of 4) go one by one: 2 x 4096 tokens, 8
    // heads, D = 40, P = 20 / 19 6.8 / 19.8 us; 17550, 16 heads, D = 128, P = 64 / 62 55.4 / 89.7.
    if (halves && k.P % 4 != 0) return launch_nr_g<ET, 1, 2, 64>(k, halves, stream);
    // Eight pairs a lane where both halves and their rest are whole 16-byte chunks, else four
    // (the work for a row beside its values' own is then twice as much).
    if (k.D % 16 == 0 && (!halves || k.P % 8 == 0)) {
        const int items = k.D / 16;
        if (items <= 2) return launch_nr_g<ET, 8, 1, 2>(k, halves, stream);
        if (items <= 4) return launch_nr_g<ET, 8, 1, 4>(k, halves, stream);
        if (items <= 8) return launch_nr_g<ET, 8, 1, 8>(k, halves, stream);
        return launch_nr_g<ET, 8, 1, 16>(k, halves, stream);
    }
    const int items = k.D / 8;
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
    const bool halves = a.halves;
    return a.dtype == kF16 ? launch_nr_e<kF16>(k, halves, a.stream) : launch_nr_e<kBF16>(k, halves, a.stream);
}

}  // namespace sdattn
