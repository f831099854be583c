"""The tests' own forms of e4m3 and of the cache's scales against torch's conversion and
direct search, on the CPU."""
import numpy as np
import pytest

import stream_ref as ref


def test_codes_are_torchs():
    import torch
    codes = np.arange(256, dtype=np.uint8)
    t = torch.from_numpy(codes).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(ref.decode(codes), t, equal_nan=True)
    rng = np.random.default_rng(1)
    x = np.concatenate([rng.normal(size=4000) * 10.0 ** rng.uniform(-5, 2, 4000), t[~np.isnan(t)]])
    mid = np.sort(t[~np.isnan(t)])
    x = np.concatenate([x, (mid[1:] + mid[:-1]) / 2])          # halves: to even
    x = x[np.abs(x) <= 448].astype(np.float32)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(ref.encode(x.astype(np.float64)), want)


@pytest.mark.parametrize("top,e", [(0.0, -100), (448.0, 0), (448.1, 1), (447.0, 0), (224.0, -1), (224.1, 0), (1.0, -8), (1.75, -8),
                                   (1.76, -7), (2.0 ** -24, -32), (61440.0, 8), (2.0 ** -130, -100), (1.875 * 2.0 ** 127, 120)])
def test_scales(top, e):
    assert ref.exponent(top) == e


def test_a_page_that_grows_is_coded_anew():
    codes, scales = np.zeros((2, 1, 64, 8), np.uint8), np.ones((2, 1))
    table = np.array([[1]])
    x = np.ones((1, 1, 3, 8))
    ref.write(x, codes, scales, table, [0], [3], "f16")
    assert scales[1, 0] == 2.0 ** -8 and (ref.decode(codes[1, 0, :3]) == 256).all()
    ref.write(x[:, :, :1] * 100, codes, scales, table, [3], [1], "f16")
    assert scales[1, 0] == 2.0 ** -2 and (ref.decode(codes[1, 0, :3]) == 4).all()
    # 100 / 2^-2 = 400 lies halfway between the codes of 384 and 416: to the even one
    assert np.allclose(ref.read(codes, scales, table, [0], [4], 4)[0, 0, :, 0], [1, 1, 1, 96])
    assert not codes[0].any() and scales[0, 0] == 1


def test_what_is_seen():
    see = ref.seen([5], [3], 4, 10, 1, 2, 1)[0]
    assert [list(np.flatnonzero(r)) for r in see] == [[0, 4, 5], [0, 5, 6], [0, 6, 7], []]
    see = ref.seen([5], [3], 3, 10, 3, 0, 0)[0]
    assert [int(r.sum()) for r in see] == [6, 8, 8]
    see = ref.seen([-2], [3], 3, 10, 1, 0, 4)[0]
    assert [int(r.sum()) for r in see] == [0, 0, 1]
    assert ref.seen([2], [3], 3, 10, 0, 2, 0)[0].sum(1).tolist() == [2, 2, 2]
