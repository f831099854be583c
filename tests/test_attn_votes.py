"""Where the tiled attention kernel's overflow votes lie in LDS (csrc/attn_geom.h, plain
C++, compiled here with g++).  A ragged last tile is read after its workgroup's last barrier,
by some waves while others vote already: no vote may lie in that tile's buffer."""
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2304_11267_amd", "csrc")

PROGRAM = r"""
#include <cstdio>
#include <utility>
#include "attn_geom.h"
using namespace sdattn;
template <int D, int G> void print() {
    using T = Geom<D, G>;
    if (!T::kFits || (T::kNarrow && D > 160)) return;
    printf("%d %d %d %d %d %d %d %d", D, G, (int)T::kStream, T::kKS, T::kWaves, T::kBufBytes, T::kHalfBytes, T::kLdsBytes);
    for (int n = 1; n <= 24; ++n) printf(" %d", T::vote_at(n));
    printf("\n");
}
template <int... Ds> void print_all(std::integer_sequence<int, Ds...>) {
    ((print<32 + 8 * Ds, 0>(), print<32 + 8 * Ds, 1>(), print<32 + 8 * Ds, 2>(), print<32 + 8 * Ds, 3>(),
      print<32 + 8 * Ds, 4>(), print<32 + 8 * Ds, 5>(), print<32 + 8 * Ds, 6>(), print<32 + 8 * Ds, 7>()), ...);
}
int main() { print_all(std::make_integer_sequence<int, 17>{}); }
"""


@pytest.fixture(scope="module")
def geometries(tmp_path_factory):
    d = tmp_path_factory.mktemp("votes")
    (d / "votes.cpp").write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-I", CSRC, str(d / "votes.cpp"), "-o", str(d / "votes")], check=True)
    out = subprocess.run([str(d / "votes")], capture_output=True, text=True, check=True).stdout.splitlines()
    rows = [tuple(int(x) for x in line.split()) for line in out]
    assert len({(r[0], r[1]) for r in rows}) == len(rows) > 80
    assert {r[1] for r in rows} == set(range(8))
    return rows


def late_reads(stream, splits, buf, half, tiles):
    """[start, end) in LDS of what run_tiles reads after its last barrier: a split's ragged last
    tile, when it is not the split's first."""
    if stream:
        return [(s * half, (s + 1) * half) for s in range(splits)]   # (the ring: any of its buffers)
    steps = -(-tiles // splits)
    last = (tiles - 1) // steps                                      # the split with the last tile
    i = tiles - 1 - last * steps
    return [] if i == 0 else [(last * half + (i & 1) * buf, last * half + ((i & 1) + 1) * buf)]


def test_votes_lie_clear_of_the_tile_that_is_read_last(geometries):
    for D, geo, stream, splits, waves, buf, half, lds, *votes in geometries:
        for tiles in range(1, 24 * splits + 1):
            vote = votes[-(-tiles // splits) - 1]
            assert 0 <= vote and vote + 4 * waves <= lds and vote % 4 == 0
            for start, end in late_reads(stream, splits, buf, half, tiles):
                assert vote + 4 * waves <= start or vote >= end, (D, geo, tiles)
