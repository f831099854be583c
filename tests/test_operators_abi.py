"""What the adapters, the norms with rotation, the block selection and the attention over
selected blocks refuse, before any HIP call (no GPU: the pointers are never followed), and
what their Python functions refuse."""
import ctypes
import os

import pytest

import paper_2304_11267_amd as sd
from paper_2304_11267_amd import binding

OK, INVALID, UNSUPPORTED, MISALIGNED = 0, 1, 2, 3
F16, BF16, F32 = 0, 1, 2
ROWS, HEADS = 0, 1


def at(x):
    return ctypes.c_void_p(x)


def f32(x):
    return ctypes.c_float(x)


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.library_path()):
        pytest.skip("libsdattn.so not built")
    return binding.load_library()


def refused(fn, good, cases, lib):
    """Each case changes some of the good call's arguments; none of them may reach the GPU."""
    for status, change in cases:
        assert set(change) <= set(good), change
        args = dict(good, **change)
        assert fn(*args.values(), None) == status, (change, status)
    assert lib.sdattn_last_hip_error() == 0


X, W, BIAS, DOWN, UP, IDS, SCALES, Y, WS = (0x10000000 * i for i in range(1, 10))


def test_adapters(lib):
    need = lib.sdattn_linear_adapters_workspace(4, 70, 20)
    assert need >= 2 * 4 * 70 * 32 and need % 256 == 0
    assert lib.sdattn_linear_adapters_workspace(1, 1, 1) >= 32
    for bad in ((0, 1, 1), (1, 0, 1), (1, 1, 0), (1, 1, 65537), (-1, 1, 1)):
        assert lib.sdattn_linear_adapters_workspace(*bad) == -1
    good = dict(x=at(X), w=at(W), bias=at(BIAS), down=at(DOWN), up=at(UP), ids=at(IDS), scales=at(SCALES), y=at(Y),
                ws=at(WS), wsb=need, B=4, L=70, K=320, N=640, R=20, A=3, H=8, xl=ROWS, yl=HEADS, dtype=F16)
    cases = [(INVALID, {n: None}) for n in ("x", "w", "down", "up", "ids", "y", "ws")]
    cases += [(INVALID, {n: v}) for n in ("B", "L", "K", "N", "R", "A", "H") for v in (0, -1)]
    cases += [(INVALID, dict(wsb=need - 1)), (INVALID, dict(xl=2)), (INVALID, dict(dtype=9)),
              (UNSUPPORTED, dict(dtype=F32)), (UNSUPPORTED, dict(K=324)), (UNSUPPORTED, dict(N=648, H=7)),
              (UNSUPPORTED, dict(R=65537, wsb=1 << 60)), (UNSUPPORTED, dict(A=1 << 30, R=65536, K=65536, wsb=1 << 60)),
              (UNSUPPORTED, dict(B=1 << 20, L=1 << 12, wsb=1 << 60))]
    cases += [(MISALIGNED, {n: at(good[n].value + 8)}) for n in ("x", "w", "down", "up", "y", "ws")]
    cases += [(MISALIGNED, dict(bias=at(BIAS + 4))), (MISALIGNED, dict(ids=at(IDS + 2))),
              (MISALIGNED, dict(scales=at(SCALES + 2)))]
    inside_y, inside_ws = Y + 4096, WS + 4096
    cases += [(INVALID, {n: at(inside_y)}) for n in ("x", "w", "bias", "down", "up", "ids", "scales", "ws")]
    cases += [(INVALID, {n: at(inside_ws)}) for n in ("x", "w", "bias", "down", "up", "ids", "scales")]
    # the ends: the last adapter's up runs into y, y's tail into the ids
    cases += [(INVALID, dict(up=at(Y - 2 * 3 * 640 * 20 + 16))), (INVALID, dict(ids=at(Y + 2 * 4 * 70 * 640 - 4)))]
    refused(lib.sdattn_linear_adapters, good, cases, lib)


def test_norm_rotate(lib):
    pairs = (ctypes.c_int * 4)(8, 8, 4, 0)
    good = dict(q=at(X), k=at(W), gq=at(BIAS), gk=at(DOWN), pos=at(UP), freqs=at(IDS), qo=at(SCALES), ko=at(Y), B=2, H=8,
                L=100, D=40, axes=3, pairs=pairs, batches=2, norm=1, eps=f32(1e-6), pairing=0, xl=ROWS, yl=HEADS,
                dtype=BF16)
    cases = [(INVALID, {n: None}) for n in ("q", "qo", "k", "ko", "pos", "freqs", "pairs")]
    cases += [(INVALID, {n: v}) for n in ("B", "H", "L", "D") for v in (0, -5)]
    cases += [(INVALID, dict(axes=-1)), (UNSUPPORTED, dict(axes=5)), (INVALID, dict(axes=4)),
              (INVALID, dict(batches=3)), (INVALID, dict(batches=0)), (INVALID, dict(norm=2)), (INVALID, dict(pairing=2)),
              (INVALID, dict(xl=2)), (INVALID, dict(yl=-1)), (INVALID, dict(eps=f32(-1.0))),
              (INVALID, dict(eps=f32(float("nan")))), (INVALID, dict(eps=f32(float("inf")))),
              (UNSUPPORTED, dict(dtype=F32)), (INVALID, dict(dtype=4)), (UNSUPPORTED, dict(D=44)),
              (UNSUPPORTED, dict(D=264)), (INVALID, dict(D=32)),       # 20 pairs do not fit 16
              (INVALID, dict(pairs=(ctypes.c_int * 3)(8, -1, 4))), (INVALID, dict(pairs=(ctypes.c_int * 3)(8, 8, 5))),
              (UNSUPPORTED, dict(B=1 << 20, L=1 << 12, batches=1)), (UNSUPPORTED, dict(H=1 << 30))]
    cases += [(MISALIGNED, {n: at(good[n].value + 8)}) for n in ("q", "k", "qo", "ko")]
    cases += [(MISALIGNED, {n: at(good[n].value + 4)}) for n in ("gq", "gk")]
    cases += [(MISALIGNED, {n: at(good[n].value + 2)}) for n in ("pos", "freqs")]
    nbytes = 2 * 2 * 8 * 100 * 40
    for o in ("qo", "ko"):
        cases += [(INVALID, {n: at(good[o].value + 1024)}) for n in ("q", "k", "gq", "gk", "pos", "freqs")]
    cases += [(INVALID, dict(ko=at(SCALES + nbytes - 16))),
              (INVALID, dict(qo=at(X))),                               # in place with another layout
              (INVALID, dict(qo=at(X + 16), yl=ROWS)),                 # nearly in place
              (INVALID, dict(qo=at(W), ko=at(X), yl=ROWS))]            # each in the other's place
    refused(lib.sdattn_norm_rotate, good, cases, lib)


def test_block_means(lib):
    good = dict(x=at(X), means=at(Y), B=2, H=8, L=1000, D=40, dtype=F16)
    cases = [(INVALID, dict(x=None)), (INVALID, dict(means=None)), (UNSUPPORTED, dict(dtype=F32)), (INVALID, dict(dtype=3)),
             (UNSUPPORTED, dict(D=36)), (UNSUPPORTED, dict(D=264)), (UNSUPPORTED, dict(L=(1 << 30) + 1)),
             (UNSUPPORTED, dict(B=1 << 20, H=1 << 12)), (MISALIGNED, dict(x=at(X + 8))), (MISALIGNED, dict(means=at(Y + 8))),
             (INVALID, dict(means=at(X + 2 * 2 * 8 * 1000 * 40 - 16)))]
    cases += [(INVALID, {n: 0}) for n in ("B", "H", "L", "D")]
    refused(lib.sdattn_block_means, good, cases, lib)


def test_select_blocks(lib):
    good = dict(q=at(X), means=at(W), mask=at(Y), B=2, H=8, Lq=1000, NB=70, D=40, qblock=64, keep=9, dtype=F16)
    cases = [(INVALID, {n: None}) for n in ("q", "means", "mask")]
    cases += [(INVALID, {n: v}) for n in ("B", "H", "Lq", "NB", "D", "keep") for v in (0, -1)]
    cases += [(INVALID, dict(qblock=n)) for n in (0, 32, 65, 256)]
    cases += [(UNSUPPORTED, dict(dtype=F32)), (INVALID, dict(dtype=3)), (UNSUPPORTED, dict(D=42)), (UNSUPPORTED, dict(D=512)),
              (UNSUPPORTED, dict(NB=16385)), (UNSUPPORTED, dict(Lq=(1 << 30) + 1)), (UNSUPPORTED, dict(B=1 << 20, H=1 << 12)),
              (MISALIGNED, dict(q=at(X + 8))), (MISALIGNED, dict(means=at(W + 4))), (MISALIGNED, dict(mask=at(Y + 4))),
              (INVALID, dict(mask=at(X + 64))), (INVALID, dict(mask=at(W + 4 * 2 * 8 * 70 * 40 - 8)))]
    refused(lib.sdattn_select_blocks, good, cases, lib)


def test_sparse_forward(lib):
    good = dict(q=at(X), k=at(W), v=at(BIAS), mask=at(DOWN), out=at(Y), B=2, H=8, Lq=1000, Lk=900, D=64, qblock=64,
                scale=f32(0.125), dtype=F16)
    cases = [(INVALID, {n: None}) for n in ("q", "k", "v", "mask", "out")]
    cases += [(INVALID, {n: v}) for n in ("B", "H", "Lq", "Lk", "D") for v in (0, -1)]
    cases += [(INVALID, dict(qblock=n)) for n in (0, 32, 96, 256)]
    cases += [(UNSUPPORTED, dict(D=d)) for d in (8, 24, 44, 152, 168, 256, 264)]
    cases += [(INVALID, dict(scale=f32(float("inf")))), (UNSUPPORTED, dict(dtype=F32)), (INVALID, dict(dtype=7)),
              (UNSUPPORTED, dict(Lk=(1 << 30) + 1)), (UNSUPPORTED, dict(Lq=(1 << 30) + 1)),
              (UNSUPPORTED, dict(B=1 << 20, H=1 << 12)), (MISALIGNED, dict(mask=at(DOWN + 4)))]
    cases += [(MISALIGNED, {n: at(good[n].value + 8)}) for n in ("q", "k", "v", "out")]
    cases += [(INVALID, {n: at(Y + 4096)}) for n in ("q", "k", "v", "mask")]
    cases += [(INVALID, dict(mask=at(Y + 2 * 2 * 8 * 1000 * 64 - 8)))]
    refused(lib.sdattn_sparse_forward, good, cases, lib)


def test_launches_of_more_threads_than_32_bits(lib):
    far = [at(i << 42) for i in range(1, 10)]
    names = "x w bias down up ids scales y ws".split()
    adapters = dict(zip(names, far), wsb=1 << 40, B=4, L=70, K=520, N=640, R=20, A=3, H=1, xl=ROWS, yl=ROWS, dtype=F16)
    refused(lib.sdattn_linear_adapters, adapters, [
        (UNSUPPORTED, dict(B=1 << 24, L=1, K=8, N=8)), (UNSUPPORTED, dict(B=1 << 18, L=33, N=65536)),
        (UNSUPPORTED, dict(B=1 << 18, L=65, N=65536)), (UNSUPPORTED, dict(B=1 << 20, L=16, N=65536, R=40))], lib)
    rotate = dict(q=far[0], k=None, gq=None, gk=None, pos=None, freqs=None, qo=far[1], ko=None, B=1, H=1, L=1 << 28, D=8,
                  axes=0, pairs=None, batches=1, norm=1, eps=f32(1e-6), pairing=0, xl=ROWS, yl=HEADS, dtype=BF16)
    refused(lib.sdattn_norm_rotate, rotate, [(UNSUPPORTED, {})], lib)
    means = dict(x=far[0], means=far[1], B=1 << 12, H=1 << 12, L=1, D=8, dtype=F16)
    refused(lib.sdattn_block_means, means, [(UNSUPPORTED, {})], lib)
    select = dict(q=far[0], means=far[1], mask=far[2], B=1 << 12, H=1 << 12, Lq=1, NB=1, D=8, qblock=64, keep=1, dtype=F16)
    refused(lib.sdattn_select_blocks, select, [(UNSUPPORTED, {}), (UNSUPPORTED, dict(B=1 << 10, NB=16384))], lib)
    sparse = dict(zip("q k v mask out".split(), far), B=1 << 12, H=1 << 10, Lq=1, Lk=1, D=32, qblock=64, scale=f32(0.125),
                  dtype=F16)
    refused(lib.sdattn_sparse_forward, sparse, [(UNSUPPORTED, {}), (UNSUPPORTED, dict(B=1 << 13, Lq=2))], lib)


def test_python_refuses_shapes_types_and_places(lib):
    import torch
    h, f, i32, i64 = torch.float16, torch.float32, torch.int32, torch.int64

    def z(*shape, dt=h):
        return torch.zeros(*shape, dtype=dt)

    x, w, y, down, up, ids, ws = z(2, 5, 16), z(24, 16), z(2, 5, 24), z(3, 4, 16), z(3, 24, 4), z(2, dt=i32), z(64, dt=torch.uint8)
    for args, kw, err, words in (
            ((x, w, y, down, up, ids, ws), {}, ValueError, "GPU tensor"),
            ((x, z(24, 8), y, down, up, ids, ws), {}, ValueError, "w has shape"),
            ((x, w, y, z(3, 4, 8), up, ids, ws), {}, ValueError, "down has shape"),
            ((x, w, y, down, z(3, 24, 8), ids, ws), {}, ValueError, "up has shape"),
            ((x, w, y, down, up, z(3, dt=i32), ws), {}, ValueError, "ids has shape"),
            ((x, w, y, down, up, z(2, dt=i64), ws), {}, TypeError, "ids is"),
            ((x, w, y, down, up, ids, ws), dict(scales=z(2, dt=f)), ValueError, "scales has shape"),
            ((x, w, y, down, up, ids, ws), dict(scales=z(3)), TypeError, "scales is"),
            ((x, w, y.bfloat16(), down, up, ids, ws), {}, TypeError, "y is"),
            ((x, w, y, down, up, ids, ws), dict(heads=5, y_layout=1), ValueError, "divide"),
            ((z(2, 4, 5, 4), w, y, down, up, ids, ws), dict(heads=2, x_layout=1), ValueError, "head count")):
        with pytest.raises(err, match=words):
            sd.linear_adapters(*args, **kw)
    q, pos, freqs = z(2, 4, 5, 16), z(2, 5, 2, dt=i32), z(6, dt=f)
    turn = dict(pos=pos, freqs=freqs, pairs=(3, 3))
    for args, kw, err, words in (
            ((q, q, 4), turn, ValueError, "GPU tensor"),
            ((q, q, 3), turn, ValueError, "head count"),
            ((q, z(2, 4, 5, 8), 4), turn, ValueError, "qo has shape"),
            ((q, q, 4), dict(turn, k=q), ValueError, "go together"),
            ((q, q, 4), dict(turn, k=q, ko=z(2, 5, 64)), ValueError, "ko has shape"),
            ((q, q, 4), dict(pairs=(3, 3)), ValueError, "need pos"),
            ((q, q, 4), dict(turn, pairs=(3, 2)), ValueError, "freqs has shape"),
            ((q, q, 4), dict(turn, pairs=(6,)), ValueError, "pos has shape"),
            ((q, q, 4), dict(turn, pos=z(3, 5, 2, dt=i32)), ValueError, "pos has shape"),
            ((q, q, 4), dict(turn, pos=pos.long()), TypeError, "pos is"),
            ((q, q, 4), dict(turn, freqs=freqs.double()), TypeError, "freqs is"),
            ((q, q, 4), dict(turn, gamma_q=z(8)), ValueError, "gamma_q has shape"),
            ((z(2, 5, 63), z(2, 5, 63), 4), dict(x_layout=0, y_layout=0), ValueError, "divide")):
        with pytest.raises(err, match=words):
            sd.norm_rotate(*args, **kw)
    for fn, args, err, words in (
            (sd.block_means, (q, z(2, 4, 1, 16, dt=f)), ValueError, "GPU tensor"),
            (sd.block_means, (q, z(2, 4, 2, 16, dt=f)), ValueError, "means has shape"),
            (sd.block_means, (q, z(2, 4, 1, 16)), TypeError, "means is"),
            (sd.select_blocks, (q, z(2, 4, 3, 16, dt=f), z(2, 4, 1, 1, dt=i64), 2), ValueError, "GPU tensor"),
            (sd.select_blocks, (q, z(2, 4, 3, 8, dt=f), z(2, 4, 1, 1, dt=i64), 2), ValueError, "means has shape"),
            (sd.select_blocks, (q, z(2, 4, 65, 16, dt=f), z(2, 4, 1, 1, dt=i64), 2), ValueError, "mask has shape"),
            (sd.select_blocks, (q, z(2, 4, 3, 16, dt=f), z(2, 4, 1, 1, dt=i32), 2), TypeError, "mask is"),
            (sd.select_blocks, (q, z(2, 4, 3, 16, dt=f), z(2, 4, 1, 1, dt=i64), 2, 0), ValueError, "qblock"),
            (sd.sparse_forward, (q, q, q, z(2, 4, 1, 1, dt=i64), q, 0.1), ValueError, "GPU tensor"),
            (sd.sparse_forward, (q, q, z(2, 4, 6, 16), z(2, 4, 1, 1, dt=i64), q, 0.1), ValueError, "v has shape"),
            (sd.sparse_forward, (q, q, q, z(2, 4, 2, 1, dt=i64), q, 0.1), ValueError, "mask has shape"),
            (sd.sparse_forward, (q, q, q, z(2, 4, 1, 1, dt=f), q, 0.1), TypeError, "mask is"),
            (sd.sparse_forward, (q, q.bfloat16(), q, z(2, 4, 1, 1, dt=i64), q, 0.1), TypeError, "k is")):
        with pytest.raises(err, match=words):
            fn(*args)


def test_native_marshalling_leaves_cpu_tensors_and_odd_arguments_to_python(lib):
    import torch
    native = binding._native
    assert native is not None, "the extension module is not built"
    t = torch.zeros(1, 1, 8, 32, dtype=torch.float16)
    fn = binding._fn["sdattn_forward"]
    for name in ("linear_adapters", "norm_rotate", "block_means", "select_blocks", "sparse_forward"):
        call = getattr(native, name)
        assert call() is None and call(fn) is None and call(fn, None, 3, "x") is None
        assert call(fn, *[t] * 10, (1,), 1, 0.1, 0, 0, 0, None) is None
