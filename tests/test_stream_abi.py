"""What the gated norms, the cache and the attention over it refuse, before any HIP call (no GPU: the
pointers are never followed), what their Python functions refuse, whole numbers past 32 bits, and what a launch that
HIP refuses comes back as."""
import ctypes
import os
import subprocess
import sys
import textwrap
import types

import pytest

import paper_2304_11267_amd as sd
from paper_2304_11267_amd import binding
from test_operators_abi import BF16, F16, F32, HEADS, INVALID, MISALIGNED, ROWS, UNSUPPORTED, at, f32, lib, refused  # noqa: F401
from test_operators_launch_errors import INVALID_CONFIGURATION, ROOT, STUB

P = [0x10000000 * i for i in range(1, 15)]


def big(n):
    return ctypes.c_longlong(n)


def test_gated_norm(lib):  # noqa: F811
    names = ("x", "r", "gate", "scale", "shift", "gamma_r", "gamma", "beta", "h", "y")
    good = dict(zip(names, map(at, P)), B=2, L=60, C=320, batches=2, groups=3, sg=big(1920), ss=big(1920), st=big(320),
                skip=f32(1.0), norm_r=1, norm=2, eps=f32(1e-6), x_dtype=F32, dtype=BF16)
    cases = [(INVALID, dict(x=None)), (INVALID, dict(h=None, y=None)), (INVALID, dict(r=None))]   # (a gate without what it gates)
    cases += [(INVALID, {n: v}) for n in ("B", "L", "C", "groups") for v in (0, -1)]
    cases += [(INVALID, dict(groups=7)), (INVALID, dict(batches=3)), (INVALID, dict(batches=0)), (INVALID, dict(norm=3)),
              (INVALID, dict(norm_r=-1)), (INVALID, dict(eps=f32(-1))), (INVALID, dict(eps=f32(float("nan")))),
              (INVALID, dict(skip=f32(float("inf")))), (INVALID, dict(sg=big(-8))), (MISALIGNED, dict(ss=big(1924))),
              (UNSUPPORTED, dict(st=big(1 << 60))),
              (UNSUPPORTED, dict(dtype=F32)), (INVALID, dict(dtype=5)), (UNSUPPORTED, dict(x_dtype=F16)), (INVALID, dict(x_dtype=4)),
              (UNSUPPORTED, dict(C=324)), (UNSUPPORTED, dict(C=16392)), (UNSUPPORTED, dict(B=1 << 20, L=3 << 12, batches=1))]
    cases += [(MISALIGNED, {n: at(good[n].value + 8)}) for n in names]
    n = 2 * 60 * 320
    for o in ("h", "y"):
        cases += [(INVALID, {m: at(good[o].value + 1600)}) for m in names if m != o]
    cases += [(INVALID, dict(h=at(P[0] + 4 * n - 16))), (INVALID, dict(y=at(P[0]))), (INVALID, dict(y=at(P[1]))),
              # the last modulation row's end: ((2 * 3 - 1) * 1920 + 320) values
              (INVALID, dict(gate=at(P[9] - 2 * (5 * 1920 + 320) + 16))),
              (INVALID, dict(h=at(P[0]), x_dtype=F32, x=at(P[0] + 16)))]
    refused(lib.sdattn_gated_norm, good, cases, lib)


CACHE = dict(B=2, Hk=4, L=100, D=80, pages=9, slots=4)


def cache_cases(good, out, into):
    cases = [(INVALID, {n: None}) for n in ("k", "v", "kp", "vp", "ks", "vs", "table", "starts")]
    cases += [(INVALID, {n: v}) for n in ("B", "Hk", "L", "D", "pages", "slots") for v in (0, -1)]
    cases += [(INVALID, dict(layout=2)), (INVALID, dict(dtype=3)), (UNSUPPORTED, dict(dtype=F32)), (UNSUPPORTED, dict(D=84)),
              (UNSUPPORTED, dict(D=264)), (UNSUPPORTED, dict(Hk=65537)), (UNSUPPORTED, dict(L=(1 << 30) + 1)),
              (UNSUPPORTED, dict(slots=(1 << 24) + 1))]
    cases += [(MISALIGNED, {n: at(good[n].value + 8)}) for n in ("k", "v", "kp", "vp")]
    cases += [(MISALIGNED, {n: at(good[n].value + 2)}) for n in ("ks", "vs", "table", "starts", "counts")]
    for o in out:
        for n in ("k", "v", "kp", "vp", "ks", "vs", "table", "starts", "counts"):
            if n != o and (n in out or n in into or n in ("table", "starts", "counts")):
                cases.append((INVALID, {n: at(good[o].value)}))
    return cases


def test_cache_write_and_read(lib):  # noqa: F811
    w = dict(zip(("k", "v", "kp", "vp", "ks", "vs", "table", "starts", "counts"), map(at, P)), **CACHE, layout=ROWS, dtype=F16)
    pages, tokens = ("kp", "vp", "ks", "vs"), ("k", "v")
    cases = cache_cases(w, pages, tokens)
    cases += [(INVALID, dict(vp=at(P[2] + 9 * 4 * 64 * 80 - 16))), (INVALID, dict(k=at(P[2] - 2 * 2 * 4 * 100 * 80 + 16)))]
    refused(lib.sdattn_cache_write, w, cases, lib)
    r = {n: w[n] for n in ("kp", "vp", "ks", "vs", "table", "starts", "counts", "k", "v")}
    r.update(**CACHE, layout=HEADS, dtype=BF16)
    refused(lib.sdattn_cache_read, r, cache_cases(r, tokens, pages), lib)


SPAN = dict(frame=1, window=100, sinks=4)


def test_cache_forward(lib):  # noqa: F811
    space = lib.sdattn_cache_forward_workspace
    assert space(2, 8, 4, 1, 64, 8, 1, 0, 0) >= 0
    far = space(1, 8, 4, 1, 64, 4096, 1, 0, 0)
    assert far > 0
    good = dict(zip(("q", "kp", "vp", "ks", "vs", "table", "starts", "counts", "out", "ws"), map(at, P)), wsb=big(far), B=1, H=8, Hk=4,
                Lq=1, D=64, pages=9, slots=4096, frame=1, window=0, sinks=0, scale=f32(0.125), xl=HEADS, yl=ROWS, dtype=F16)
    sizes = ("B", "H", "Hk", "Lq", "D", "slots")
    for bad in [{n: v} for n in sizes for v in (0, -1)] + [dict(frame=-1), dict(window=-1), dict(sinks=-1), dict(Hk=3), dict(D=24),
                                                            dict(D=168), dict(D=68), dict(slots=(1 << 24) + 1), dict(H=1 << 17)]:
        a = dict(good, **bad)
        assert space(*(a[n] for n in ("B", "H", "Hk", "Lq", "D", "slots", "frame", "window", "sinks"))) == -1, bad
    cases = [(INVALID, {n: None}) for n in ("q", "kp", "vp", "ks", "vs", "table", "starts", "out", "ws")]
    cases += [(INVALID, {n: v}) for n in sizes + ("pages",) for v in (0, -1)]
    cases += [(INVALID, {n: -1}) for n in ("frame", "window", "sinks")]
    cases += [(INVALID, dict(Hk=3)), (INVALID, dict(wsb=big(far - 1))), (INVALID, dict(wsb=big(0))), (INVALID, dict(xl=2)),
              (INVALID, dict(yl=-1)), (INVALID, dict(scale=f32(float("nan")))), (INVALID, dict(dtype=3)), (UNSUPPORTED, dict(dtype=F32)),
              (UNSUPPORTED, dict(D=24)), (UNSUPPORTED, dict(D=168)), (UNSUPPORTED, dict(D=68)), (UNSUPPORTED, dict(slots=(1 << 24) + 1)),
              (UNSUPPORTED, dict(H=1 << 17)), (UNSUPPORTED, dict(Lq=(1 << 30) + 1)), (UNSUPPORTED, dict(H=32, Lq=1 << 28))]
    cases += [(MISALIGNED, {n: at(good[n].value + 8)}) for n in ("q", "kp", "vp", "out", "ws")]
    cases += [(MISALIGNED, {n: at(good[n].value + 2)}) for n in ("ks", "vs", "table", "starts", "counts")]
    ins = ("q", "kp", "vp", "ks", "vs", "table", "starts", "counts")
    cases += [(INVALID, {n: good[o]}) for o in ("out", "ws") for n in ins] + [(INVALID, dict(ws=good["out"]))]
    cases += [(INVALID, dict(table=at(P[8] - 4 * 4096 + 16)))]
    refused(lib.sdattn_cache_forward, good, cases, lib)


def test_window_forward(lib):  # noqa: F811
    space = lib.sdattn_window_forward_workspace
    need = space(2, 8, 4, 1, 20000, 64, 1, 0, 0)
    assert need > 0 and space(2, 8, 4, 5000, 5000, 64, 1, 0, 0) >= 0 and space(1, 1, 1, 1, 1, 32, 0, 0, 0) == 0
    good = dict(zip(("q", "k", "v", "starts", "counts", "out", "ws"), map(at, P)), wsb=big(need), B=2, H=8, Hk=4, Lq=1, Lk=20000, D=64,
                frame=1, window=0, sinks=0, scale=f32(0.125), xl=HEADS, yl=ROWS, dtype=BF16)
    cases = [(INVALID, {n: None}) for n in ("q", "k", "v", "out", "ws")]
    cases += [(INVALID, {n: v}) for n in ("B", "H", "Hk", "Lq", "Lk", "D") for v in (0, -1)]
    cases += [(INVALID, {n: -1}) for n in ("frame", "window", "sinks")]
    cases += [(INVALID, dict(Hk=5)), (INVALID, dict(wsb=big(need - 1))), (INVALID, dict(xl=3)), (INVALID, dict(scale=f32(float("inf")))),
              (UNSUPPORTED, dict(D=176)), (UNSUPPORTED, dict(D=36)), (UNSUPPORTED, dict(Lk=(1 << 30) + 1)), (UNSUPPORTED, dict(dtype=F32))]
    cases += [(MISALIGNED, {n: at(good[n].value + 8)}) for n in ("q", "k", "v", "out", "ws")]
    cases += [(MISALIGNED, {n: at(good[n].value + 2)}) for n in ("starts", "counts")]
    cases += [(INVALID, {n: good[o]}) for o in ("out", "ws") for n in ("q", "k", "v", "starts", "counts")]
    cases += [(INVALID, dict(k=at(P[5] - 2 * 2 * 4 * 20000 * 64 + 16)))]
    refused(lib.sdattn_window_forward, good, cases, lib)
    for bad in (dict(B=0), dict(Hk=3), dict(D=33), dict(frame=-2)):
        a = dict(good, **bad)
        assert space(*(a[n] for n in ("B", "H", "Hk", "Lq", "Lk", "D", "frame", "window", "sinks"))) == -1


def test_launches_of_more_threads_than_32_bits(lib):  # noqa: F811
    far = [at(i << 44) for i in range(1, 12)]
    gated = dict(zip(("x", "r", "gate", "scale", "shift", "gamma_r", "gamma", "beta", "h", "y"), [far[0]] + [None] * 7 + [None, far[1]]),
                 B=1, L=1 << 27, C=1024, batches=1, groups=1, sg=big(0), ss=big(0), st=big(0), skip=f32(1), norm_r=0, norm=1,
                 eps=f32(0), x_dtype=F16, dtype=F16)
    refused(lib.sdattn_gated_norm, gated, [(UNSUPPORTED, {})], lib)
    cache = dict(zip(("k", "v", "kp", "vp", "ks", "vs", "table", "starts", "counts"), far), B=1 << 14, Hk=1 << 10, L=1, D=88, pages=4,
                 slots=1, layout=ROWS, dtype=F16)
    refused(lib.sdattn_cache_write, cache, [(UNSUPPORTED, dict(Hk=1 << 12)), (UNSUPPORTED, dict(L=2, Hk=1 << 10)),
                                            (UNSUPPORTED, dict(L=2, Hk=1 << 12, D=8))], lib)
    read = {n: cache[n] for n in ("kp", "vp", "ks", "vs", "table", "starts", "counts", "k", "v")}
    read.update({n: cache[n] for n in ("B", "Hk", "L", "D", "pages", "slots", "layout", "dtype")})
    refused(lib.sdattn_cache_read, read, [(UNSUPPORTED, {}), (UNSUPPORTED, dict(Hk=1 << 12, D=8))], lib)
    window = dict(zip(("q", "k", "v", "starts", "counts", "out", "ws"), far), wsb=big(1 << 50), B=1 << 12, H=1 << 12, Hk=1 << 12, Lq=200,
                  Lk=1, D=32, frame=1, window=0, sinks=0, scale=f32(1), xl=HEADS, yl=HEADS, dtype=F16)
    refused(lib.sdattn_window_forward, window, [(UNSUPPORTED, {}), (UNSUPPORTED, dict(Lq=1, B=1 << 13))], lib)


def z(*shape, dt="float16", device="cpu"):
    import torch
    return torch.zeros(*shape, dtype=getattr(torch, dt), device=device)


def cache_of(P=5, Hk=2, D=16, B=3, slots=4, **kw):
    c = dict(k_pages=z(P, Hk, 64, D, dt="uint8"), v_pages=z(P, Hk, 64, D, dt="uint8"), k_scales=z(P, Hk, dt="float32"),
             v_scales=z(P, Hk, dt="float32"), table=z(B, slots, dt="int32"), starts=z(B, dt="int32"))
    c.update(kw)
    return c


def test_python_refuses_shapes_types_and_places(lib):  # noqa: F811
    x, g = z(2, 6, 16), z(2, 3, 16)
    for kw, err, words in (
            (dict(y=x), ValueError, "GPU tensor"), (dict(), ValueError, "neither"), (dict(y=z(2, 6, 8)), ValueError, "y has shape"),
            (dict(y=x, r=x.bfloat16()), TypeError, "r is"), (dict(y=x.bfloat16()), TypeError, "x is"),
            (dict(h=x.float()), TypeError, "h is"), (dict(y=x, gate=z(3, 3, 16), r=x), ValueError, "gate has shape"),
            (dict(y=x, scale=g, shift=z(2, 2, 16)), ValueError, "shift has shape"), (dict(y=x, scale=z(2, 3, 32)[..., ::2]), ValueError, "side by side"),
            (dict(y=x, scale=z(4, 3, 16)[::2]), ValueError, "evenly"), (dict(y=x, gamma=z(8)), ValueError, "gamma has shape"),
            (dict(y=x, beta=z(16, dt="float32")), TypeError, "beta is")):
        with pytest.raises(err, match=words):
            sd.gated_norm(x, **kw)
    k = z(3, 2, 7, 16)
    for fn in (sd.cache_write, sd.cache_read):
        for change, err, words in (
                ({}, ValueError, "GPU tensor"), (dict(v=z(3, 2, 8, 16)), ValueError, "v has shape"),
                (dict(v_pages=z(4, 2, 64, 16, dt="uint8")), ValueError, "v_pages has shape"),
                (dict(k_pages=z(5, 2, 64, 16)), TypeError, "k_pages is"), (dict(k_scales=z(5, 3, dt="float32")), ValueError, "k_scales has"),
                (dict(v_scales=z(5, 2)), TypeError, "v_scales is"), (dict(table=z(3, 4, dt="int64")), TypeError, "table is"),
                (dict(table=z(2, 4, dt="int32")), ValueError, "table has"), (dict(starts=z(4, dt="int32")), ValueError, "starts has"),
                (dict(counts=z(3, dt="int64")), TypeError, "counts is"), (dict(layout=sd.LAYOUT_ROWS, k=z(3, 7, 33), v=z(3, 7, 33)), ValueError, "divide"),
                (dict(k=z(3, 4, 7, 16), v=z(3, 4, 7, 16)), ValueError, "head count")):
            with pytest.raises(err, match=words):
                fn(**{**dict(k=k, v=k), **cache_of(), **change})
    q = z(3, 4, 7, 32)
    good = dict(q=q, **cache_of(D=32), out=q, scale=0.1, heads=4)
    for change, err, words in (
            ({}, ValueError, "GPU tensor"), (dict(heads=2), ValueError, "head count"), (dict(out=z(3, 4, 7, 40)), ValueError, "out has"),
            (dict(out=q.bfloat16()), TypeError, "out is"), (dict(out=q, y_layout=sd.LAYOUT_ROWS), ValueError, "out has"),
            (dict(k_pages=z(5, 2, 32, 32, dt="uint8")), ValueError, "k_pages has"), (dict(counts=z(2, dt="int32")), ValueError, "counts has")):
        with pytest.raises(err, match=words):
            sd.cache_forward(**{**good, **change})
    kv = z(3, 2, 9, 32)
    good = dict(q=q, k=kv, v=kv, out=q, scale=0.1, heads=4, kv_heads=2)
    for change, err, words in (
            ({}, ValueError, "GPU tensor"), (dict(kv_heads=1), ValueError, "k has"), (dict(v=z(3, 2, 8, 32)), ValueError, "v has"),
            (dict(k=kv.bfloat16()), TypeError, "k is"), (dict(kv_heads=None), ValueError, "k has"), (dict(starts=z(2, dt="int32")), ValueError, "starts has"),
            (dict(counts=z(3, dt="int64")), TypeError, "counts is")):
        with pytest.raises(err, match=words):
            sd.window_forward(**{**good, **change})


def test_native_marshalling_leaves_cpu_tensors_and_odd_arguments_to_python(lib):  # noqa: F811
    native = binding._native
    assert native is not None, "the extension module is not built"
    t = z(1, 1, 8, 32)
    fn = binding._fn["sdattn_forward"]
    for name in ("gated_norm", "cache_write", "cache_read", "cache_forward", "window_forward"):
        call = getattr(native, name)
        assert call() is None and call(fn) is None and call(fn, None, 3, "x") is None
        assert call(fn, *[t] * 10, (1,), 1, 0.1, 0, 0, 0, None) is None
        assert call(fn, *[None] * 20) is None


FAR = 1 << 32
vp, ci, cl, cf = ctypes.c_void_p, ctypes.c_int, ctypes.c_longlong, ctypes.c_float
SIGNATURES = {"sdattn_gated_norm": [vp] * 10 + [ci] * 5 + [cl] * 3 + [cf, ci, ci, cf, ci, ci, vp],
              "sdattn_cache_write": [vp] * 9 + [ci] * 8 + [vp], "sdattn_cache_read": [vp] * 9 + [ci] * 8 + [vp],
              "sdattn_cache_forward_workspace": [ci] * 9, "sdattn_window_forward_workspace": [ci] * 9,
              "sdattn_cache_forward": [vp] * 10 + [cl] + [ci] * 10 + [cf, ci, ci, ci, vp],
              "sdattn_window_forward": [vp] * 7 + [cl] + [ci] * 9 + [cf, ci, ci, ci, vp]}


def test_whole_numbers_past_32_bits(monkeypatch):
    seen, lib, keep = [], types.SimpleNamespace(), []   # noqa: F811
    for name, types_ in SIGNATURES.items():
        keep.append(ctypes.CFUNCTYPE(ci, *types_)(lambda *a: seen.append(a) or 0))
        setattr(lib, name, keep[-1])
    monkeypatch.setattr(binding, "load_library", lambda: lib)
    monkeypatch.setattr(binding, "_native", None)
    monkeypatch.setattr(binding, "_here", lambda t, name: 1 << 28)
    monkeypatch.setattr(binding, "_stream", lambda s: None)
    monkeypatch.setattr(binding, "_check", lambda name, status: None)

    def m(*shape, dt="float16"):
        return z(*shape, dt=dt, device="meta")

    cache = {n: m(*t.shape, dt=str(t.dtype).split(".")[1]) for n, t in cache_of(D=32).items()}
    q, k = m(3, 4, 7, 32), m(3, 2, 7, 32)
    x = m(2, 6, 16)
    ok = [lambda: sd.gated_norm(x, x), lambda: sd.cache_write(k, k, **cache), lambda: sd.cache_read(k, k, **cache),
          lambda: sd.cache_forward(q, **cache, out=q, scale=0.1, heads=4), lambda: sd.window_forward(q, k, k, q, 0.1, 4, 2)]
    for f in ok:
        f()
    assert len(seen) == len(ok)
    for f in [lambda: sd.gated_norm(x, x, norm=FAR + 1), lambda: sd.gated_norm(x, x, norm_r=FAR), lambda: sd.gated_norm(m(1, FAR, 8), m(1, FAR, 8)),
              lambda: sd.cache_write(k, k, **cache, layout=FAR + 1), lambda: sd.cache_read(k, k, **cache, layout=FAR + 1),
              lambda: sd.cache_forward_workspace(1, 1, 1, FAR + 1, 64, 1), lambda: sd.window_forward_workspace(1, 1, 1, 1, FAR + 1, 64)] + \
            [lambda n=n: sd.cache_forward(q, **cache, out=q, scale=0.1, heads=4, **{n: FAR + 1}) for n in ("frame", "window", "sinks", "x_layout", "y_layout")] + \
            [lambda n=n: sd.window_forward(q, k, k, q, 0.1, 4, 2, **{n: FAR + 1}) for n in ("frame", "window", "sinks", "x_layout", "y_layout")]:
        with pytest.raises(ValueError, match="past 32 bits"):
            f()
    assert len(seen) == len(ok)


CALLS = textwrap.dedent("""
    import ctypes, sys
    stub = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
    lib = ctypes.CDLL(sys.argv[2])
    p = [ctypes.c_void_p(0x10000000 * i) for i in range(1, 15)]
    f, n = ctypes.c_float, ctypes.c_longlong
    for name, args in (
            ("sdattn_gated_norm", (*p[:10], 2, 60, 320, 2, 3, n(320), n(320), n(320), f(1), 1, 2, f(0), 2, 0)),
            ("sdattn_gated_norm", (*p[:10], 2, 6000, 320, 2, 3, n(320), n(320), n(320), f(1), 1, 2, f(0), 1, 1)),
            ("sdattn_cache_write", (*p[:9], 2, 4, 100, 80, 9, 4, 0, 0)),
            ("sdattn_cache_write", (*p[:9], 2, 4, 1, 80, 9, 4, 0, 1)),
            ("sdattn_cache_read", (*p[:9], 2, 4, 100, 80, 9, 4, 0, 0)),
            ("sdattn_cache_forward", (*p[:10], n(1 << 27), 1, 8, 4, 1, 64, 9, 500, 1, 0, 0, f(0.1), 0, 0, 0)),
            ("sdattn_cache_forward", (*p[:10], n(1 << 27), 1, 8, 4, 200, 64, 9, 500, 1, 0, 0, f(0.1), 0, 0, 1)),
            ("sdattn_window_forward", (*p[:7], n(1 << 27), 1, 8, 4, 1, 9000, 64, 1, 0, 0, f(0.1), 0, 0, 0)),
            ("sdattn_window_forward", (*p[:7], n(1 << 27), 1, 8, 4, 200, 9000, 128, 1, 64, 0, f(0.1), 1, 0, 1))):
        status = getattr(lib, name)(*args, None)
        print(name, status, lib.sdattn_last_hip_error(), stub.launched(), flush=True)
""")


def test_a_refused_launch_is_an_error_of_hip(tmp_path):
    if not os.path.exists(binding.library_path()):
        pytest.skip("libsdattn.so not built")
    (tmp_path / "stub.c").write_text(STUB)
    (tmp_path / "calls.py").write_text(CALLS)
    subprocess.run(["gcc", "-shared", "-fPIC", "-w", str(tmp_path / "stub.c"), "-o", str(tmp_path / "stub.so")], check=True)
    r = subprocess.run([sys.executable, str(tmp_path / "calls.py"), str(tmp_path / "stub.so"), binding.library_path()],
                       cwd=ROOT, capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stderr
    lines = [line.split() for line in r.stdout.splitlines()]
    assert len(lines) == 9
    for name, status, error, launched in lines:
        assert int(launched) == 1, name   # the first refused launch ends the call
        assert (int(status), int(error)) == (binding.STATUS_HIP, INVALID_CONFIGURATION), name


def test_version():
    if not os.path.exists(binding.library_path()):
        pytest.skip("libsdattn.so not built")
    number = binding.load_library().sdattn_version().decode().split()[1]
    assert tuple(int(n) for n in number.split(".")) >= (0, 3, 0)
