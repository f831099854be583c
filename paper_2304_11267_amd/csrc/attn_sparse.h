// attn_sparse.h -- attention over the blocks of 64 keys that a bit mask names for
// each block of 64 or 128 queries: the tiled kernel of attn_fwd_kernel.h, whose tiles
// are those blocks, in the geometries whose workgroup is one query block.
//
//   out_i = sum over the keys j of the blocks in the mask of i's query block of
//           softmax_j(scale q_i . k_j) v_j;  0 where the mask is empty
//
// Its work is 4 D operations for every (query, key) pair of those blocks; each block
// is read once per query block that names it, from the XCD's L2 mostly.
#pragma once

#include "attn_fwd_kernel.h"

namespace sdattn {

namespace {

// 64 queries: kGeoNarrow, four waves of 32 of them and half of the blocks (16384 tokens, 32 blocks, 8
// heads, bf16, D = 64: 103 us; two waves of all 64 leave two of a CU's SIMDs without work, 178); for D > 80
// and more than one round over the CUs kGeoNarrowSolo (kGeoNarrow / kGeoNarrowSolo, us: those tokens
// D = 80 129 / 169, D = 96 181 / 160, D = 128 236 / 195, D = 160 272 / 242; 1024 tokens, 4 blocks, 16 heads
// D = 128 9.9 / 10.5).  At D = 40 the call costs 6 us and one for each block (a 64x64 latent, 1 / 2 / 4 / 8 / 16
// / 32 of 64 blocks: 6.8 / 7.3 / 10.0 / 14.7 / 22.2 / 38.0 us); at 16 blocks the vector unit is busy for 72 %
// of the waves' life, the matrix core for 39 %: 16 exponentials, multiplies, 8 conversions and 8 sums per 32 x 32
// pairs.
// 128 queries: kGeoNormal, or past one round over the CUs kGeoPair (D = 56, 64) or kGeoSolo (D > 64).
// kGeoNormal / the other, us: 16384 tokens, 32 blocks, 8 heads, bf16 D = 64 99 / 79, D = 80 112 / 100, D = 128
// 174 / 150, D = 160 221 / 187; 17550 tokens, 40 blocks, 16 heads, D = 128 458 / 403; 1024 tokens, 4 blocks,
// 8 heads D = 80 7.6 / 7.7.
template <int ET, int D>
hipError_t launch_sparse_d(const SparseArgs& s) {
    const AttnArgs a{s.q, s.k, s.v, s.out, nullptr, s.B, s.H, s.Lq, s.Lk, D, s.scale, s.dtype, s.stream};
    const int nw = ((s.Lk + kSparseBlock - 1) / kSparseBlock + 63) / 64;
    const BlockMask mask{(const unsigned long long*)s.mask, nw};
    // (of the geometries with as many rows the one with the most waves: eight)
    if (!grid_fits((long long)s.B * s.H * ((s.Lq + s.qblock - 1) / s.qblock), 512)) return kGridTooLarge;
    if (s.qblock == 64) {
        if constexpr (D > 80) {
            if ((long long)s.B * s.H * ((s.Lq + 63) / 64) > kCus)
                return launch_kernel<ET, D, false, false, kGeoNarrowSolo>(a, mask);
        }
        return launch_kernel<ET, D, false, false, kGeoNarrow>(a, mask);
    }
    [[maybe_unused]] const bool rounds = (long long)s.B * s.H * ((s.Lq + 127) / 128) > kCus;   // more than one
    if constexpr (Geom<D, kGeoPair>::kFits) {
        if (rounds) return launch_kernel<ET, D, false, false, kGeoPair>(a, mask);
    }
    if constexpr (D > 64) {
        if (rounds) return launch_kernel<ET, D, false, false, kGeoSolo>(a, mask);
    }
    return launch_kernel<ET, D, false, false, kGeoNormal>(a, mask);
}

// The widths whose tiles fit the LDS in both geometries: D = 32, 40, ..., 160, but 152
// (whose tiles and block of ones together do not).
template <int ET, int... I>
hipError_t dispatch_sparse(const SparseArgs& s, std::integer_sequence<int, I...>) {
    hipError_t r = hipErrorInvalidValue;
    auto one = [&](auto i_c) {
        constexpr int D = kSparseMinD + 8 * decltype(i_c)::value;
        static_assert(sparse_width(D) == (Geom<D, kGeoNormal>::kFits && Geom<D, kGeoNarrow>::kFits), "");
        if constexpr (sparse_width(D)) {
            if (s.D == D) r = launch_sparse_d<ET, D>(s);
        }
    };
    (one(std::integral_constant<int, I>{}), ...);
    return r;
}
using SparseWidths = std::make_integer_sequence<int, (kSparseMaxD - kSparseMinD) / 8 + 1>;

}  // namespace

}  // namespace sdattn
