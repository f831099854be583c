"""Which kernel the sizes of the GPU tests of the attention over what a place sees get (no GPU: the launches are noted, not
made).  A rule that moves a size to another kernel has to bring the tests of the one it leaves along."""
import os
import re

import pytest

import launch_names
import span_sizes
from paper_2304_11267_amd import binding

KERNEL = re.compile(r"span_(tile|row)_kernelILi(\d)ELi(\d+)E(?:Li(\d)E)?Lb([01])E")
JOIN = re.compile(r"span_join_(wide_)?kernelILi(\d)E")


@pytest.fixture(scope="module")
def launched(tmp_path_factory):
    if not os.path.exists(binding.library_path()):
        pytest.skip("libsdattn.so not built")
    return lambda calls: launch_names.launches(calls, binding.library_path(), tmp_path_factory.mktemp("stub"))


def call(kind, size, rule, D, dtype=0):
    B, H, Hk, Lq, far = size
    if kind == "d":
        return launch_names.window_call(B, H, Hk, Lq, Lq + far, D, *rule, dtype=dtype)
    return launch_names.cache_call(B, H, Hk, Lq, D, -(-(Lq + far) // 64), *rule, dtype=dtype)


def test_tiled_sizes_are_tiled(launched):
    all_ = [(kind, size, rule, D) for size, rule, widths, kinds in span_sizes.cases() for D in widths for kind in kinds]
    variants, joins = set(), set()
    for what, (status, kernels) in zip(all_, launched([call(*c) for c in all_])):
        assert status == 0, what
        k = KERNEL.search(kernels[0][0])
        assert k and k.group(1) == "tile", (what, kernels)
        assert (k.group(5) == "1") == (what[0] == "p")
        variants.add((int(k.group(3)), int(k.group(4)), k.group(5)))
        if what[1] + (what[2],) in span_sizes.PARTS:
            assert len(kernels) == 2, what
        joins |= {j.group(1) for j in map(JOIN.search, (n for n, *_ in kernels[1:])) if j}
    # every instantiation that there is of a type, both joins
    assert len(variants) == 18 and joins == {None, "wide_"}


def test_few_rows_are_not(launched):
    calls = [call(kind, size, (1, 0, 0), D) for kind in "dp" for D in (40, 128, 160)
             for size in ((1, 2, 1, 150, 110), (2, 2, 2, 1, 299), (1, 1, 1, 33, 0), (2, 8, 2, 200, 100), (40, 16, 8, 1, 100))]
    for status, kernels in launched(calls):
        assert status == 0 and KERNEL.search(kernels[0][0]).group(1) == "row"
