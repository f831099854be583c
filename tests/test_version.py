"""The library's version tells a build with the adapters, the norms with rotation and the
selected blocks from one without them."""
import os

import pytest

from paper_2304_11267_amd import binding


def test_version():
    if not os.path.exists(binding.library_path()):
        pytest.skip("libsdattn.so not built")
    lib = binding.load_library()
    name, number, arch = lib.sdattn_version().decode().split()
    assert (name, arch) == ("sdattn", "(gfx950)")
    assert tuple(int(n) for n in number.split(".")) >= (0, 2, 0)
    assert hasattr(lib, "sdattn_sparse_forward")
