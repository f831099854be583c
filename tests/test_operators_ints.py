"""Whole numbers past 32 bits at the Python functions of the adapters, the norms with rotation,
the block selection and the attention over selected blocks: C's int would cut them silently to
others.  The entry points are replaced by recorders of the same C signatures, so no GPU."""
import ctypes
import types

import pytest

import paper_2304_11267_amd as sd
from paper_2304_11267_amd import binding

vp, i32, i64, f32 = ctypes.c_void_p, ctypes.c_int, ctypes.c_longlong, ctypes.c_float
SIGNATURES = {"sdattn_block_means": [vp, vp] + [i32] * 5 + [vp],
              "sdattn_linear_adapters_workspace": [i32] * 3,
              "sdattn_linear_adapters": [vp] * 9 + [i64] + [i32] * 10 + [vp],
              "sdattn_norm_rotate": [vp] * 8 + [i32] * 5 + [vp, i32, i32, f32, i32, i32, i32, i32, vp],
              "sdattn_select_blocks": [vp] * 3 + [i32] * 8 + [vp],
              "sdattn_sparse_forward": [vp] * 5 + [i32] * 6 + [f32, i32, vp]}
FAR = 1 << 32


@pytest.fixture
def calls(monkeypatch):
    """The arguments that arrive at the entry points."""
    seen = []
    lib = types.SimpleNamespace()
    keep = []
    for name, types_ in SIGNATURES.items():
        keep.append(ctypes.CFUNCTYPE(i32, *types_)(lambda *a: seen.append(a) or 0))
        setattr(lib, name, keep[-1])
    monkeypatch.setattr(binding, "load_library", lambda: lib)
    monkeypatch.setattr(binding, "_native", None)
    monkeypatch.setattr(binding, "_here", lambda t, name: 1 << 28)
    monkeypatch.setattr(binding, "_stream", lambda s: None)
    monkeypatch.setattr(binding, "_check", lambda name, status: None)
    return seen


def z(*shape, dt="float16"):
    import torch
    return torch.empty(*shape, dtype=getattr(torch, dt), device="meta")


@pytest.mark.parametrize("keep,arrives", [(2, 2), (3, 3), (7, 3), ((1 << 31) - 1, 3), (1 << 31, 3), (FAR + 1, 3), (1 << 70, 3),
                                          (0, 0), (-1, 0), (-FAR + 2, 0), (-(1 << 31) - 1, 0)])
def test_keep_past_the_blocks_means_all_and_none_is_refused(calls, keep, arrives):
    """NB = 3: more than that is all of them; 0 and less is left to the library's refusal."""
    sd.select_blocks(z(1, 2, 5, 16), z(1, 2, 3, 16, dt="float32"), z(1, 2, 1, 1, dt="int64"), keep)
    got = calls[0][9]
    assert min(got, 3) == arrives if arrives else got < 1


@pytest.mark.parametrize("change", [dict(norm=FAR + 1), dict(norm=-FAR), dict(pairing=FAR), dict(x_layout=FAR), dict(y_layout=FAR),
                                    dict(pairs=(FAR + 3, 3 - FAR)), dict(pairs=(FAR + 3, 3))])
def test_norm_rotate(calls, change):
    q = z(2, 5, 64)
    kw = dict(pos=z(2, 5, 2, dt="int32"), freqs=z(6, dt="float32"), pairs=(3, 3), x_layout=0, y_layout=0)
    sd.norm_rotate(q, q, 4, **kw)
    with pytest.raises(ValueError):
        sd.norm_rotate(q, q, 4, **dict(kw, **change))
    assert len(calls) == 1


@pytest.mark.parametrize("change", [dict(heads=FAR + 4), dict(heads=FAR), dict(x_layout=FAR), dict(y_layout=FAR)])
def test_linear_adapters(calls, change):
    args = (z(2, 5, 16), z(24, 16), z(2, 5, 24), z(3, 4, 16), z(3, 24, 4), z(2, dt="int32"), z(64, dt="uint8"))
    sd.linear_adapters(*args)
    with pytest.raises(ValueError):
        sd.linear_adapters(*args, **change)
    assert len(calls) == 1


def test_query_blocks(calls):
    q = z(1, 2, 5, 32)
    mask = z(1, 2, 1, 1, dt="int64")
    sd.sparse_forward(q, q, q, mask, q, 0.1)
    with pytest.raises(ValueError):
        sd.sparse_forward(q, q, q, mask, q, 0.1, qblock=FAR + 64)
    with pytest.raises(ValueError):
        sd.select_blocks(q, z(1, 2, 3, 32, dt="float32"), mask, 2, qblock=FAR + 64)
    assert len(calls) == 1


def test_sizes(calls):
    """Tensors of more rows than a C int counts (a card holds them): refused, not cut to a few rows."""
    far = FAR + 4
    for refused in (lambda: sd.linear_adapters(z(1, far, 8), z(8, 8), z(1, far, 8), z(1, 8, 8), z(1, 8, 8), z(1, dt="int32"),
                                               z(64, dt="uint8")),
                    lambda: sd.linear_adapters_workspace(far, 1, 1), lambda: sd.linear_adapters_workspace(1, far, 1),
                    lambda: sd.linear_adapters_workspace(1, 1, far),
                    lambda: sd.norm_rotate(z(1, 1, far, 8), z(1, 1, far, 8), 1),
                    lambda: sd.norm_rotate(z(far, 1, 1, 8), z(far, 1, 1, 8), 1),
                    lambda: sd.block_means(z(1, 1, far, 8), z(1, 1, far // 64 + 1, 8, dt="float32")),
                    lambda: sd.select_blocks(z(far, 1, 1, 8), z(far, 1, 1, 8, dt="float32"), z(far, 1, 1, 1, dt="int64"), 1),
                    lambda: sd.sparse_forward(*[z(1, far, 1, 32)] * 3, z(1, far, 1, 1, dt="int64"), z(1, far, 1, 32), 0.1)):
        with pytest.raises(ValueError, match="past 32 bits"):
            refused()
    assert not calls
