"""sdattn_gated_norm against its 64-bit form: both norms on either side, residual streams of 16
and 32 bits, modulation from slices of a wider tensor, per batch item, per group and shared, missing
parts, in place, one channel piece to the widest rows, one token to many."""
import numpy as np
import pytest

import operators_ref as op
import paper_2304_11267_amd as sd
import stream_ref as ref

pytestmark = pytest.mark.gpu
NORMS = {"none": sd.NORM_NONE, "rms": sd.NORM_RMS, "layer": sd.NORM_LAYER}


@pytest.fixture(scope="module", autouse=True)
def _needs_gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    sd.load_library()


def inputs(B, L, C, groups=1, dtype="f16", wide=False, batches=None, seed=0, spread=6):
    import torch
    g = op.generator(seed + C + L)
    x = torch.randn(B, L, C, device="cuda", generator=g) * 2 + 0.5
    t = dict(x=x if wide else x.to(op.t_type(dtype)), r=op.randn(g, B, L, C, dtype=dtype, sigma=1.5))
    mods = op.randn(g, batches or B, groups, spread * C, dtype=dtype, sigma=0.4).chunk(spread, dim=-1)
    t.update(gate=mods[0], scale=mods[1 % spread], shift=mods[-1])
    t.update(gamma_r=1 + op.randn(g, C, dtype=dtype, sigma=0.2), gamma=1 + op.randn(g, C, dtype=dtype, sigma=0.2),
             beta=op.randn(g, C, dtype=dtype, sigma=0.2))
    return t


def each(m, B, L, C, default):
    if m is None:
        return default
    m = op.host(m)
    return np.broadcast_to(np.repeat(m, L // m.shape[1], axis=1), (B, L, C))


def check(t, norm_r, norm, skip, dtype, eps=1e-6, in_place=False, h=True, y=True, stream=None):
    import torch
    B, L, C = t["x"].shape
    wide = t["x"].dtype == torch.float32
    like = op.t_type(dtype)
    guard = 64
    want = ref.gated(op.host(t["x"]), None if t["r"] is None else op.host(t["r"]), each(t["gate"], B, L, C, 1.0),
                     each(t["scale"], B, L, C, 0.0), each(t["shift"], B, L, C, 0.0),
                     *(None if t[n] is None else op.host(t[n]) for n in ("gamma_r", "gamma", "beta")), skip, norm_r, norm, eps)
    hb = torch.full((t["x"].numel() + guard,), 7.0, dtype=t["x"].dtype, device="cuda")
    yb = torch.full((t["x"].numel() + guard,), 7.0, dtype=like, device="cuda")
    x = t["x"]
    ho, yo = hb[:-guard].view(B, L, C), yb[:-guard].view(B, L, C)
    if in_place:
        ho.copy_(x)
        x = ho
    got = sd.gated_norm(x, yo if y else None, r=t["r"], h=ho if h else None, gate=t["gate"], scale=t["scale"], shift=t["shift"],
                        gamma_r=t["gamma_r"], gamma=t["gamma"], beta=t["beta"], skip=skip, norm_r=NORMS[norm_r], norm=NORMS[norm],
                        eps=eps, stream=stream)
    torch.cuda.synchronize()
    assert got[0] is (ho if h else None) and got[1] is (yo if y else None)
    assert (hb[-guard:] == 7).all() and (yb[-guard:] == 7).all()
    if h:
        g = op.host(ho)
        last = 2.0 ** -24 * np.abs(want[0]) if wide else op.half_step(g, want[0], dtype)
        assert (np.abs(g - want[0]) <= last + want[1] + 1e-30).all()
    else:
        assert (hb == 7).all()
    if y:
        g = op.host(yo)
        assert (np.abs(g - want[2]) <= op.half_step(g, want[2], dtype) + want[3]).all(), np.max(np.abs(g - want[2]) / (op.half_step(g, want[2], dtype) + want[3]))
    else:
        assert (yb == 7).all()
    return ho, yo


@pytest.mark.parametrize("norm", ["none", "rms", "layer"])
@pytest.mark.parametrize("norm_r", ["none", "rms", "layer"])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("wide", [False, True])
def test_norms_and_types(norm, norm_r, dtype, wide):
    for B, L, C, groups in ((2, 6, 320, 3), (1, 5, 1288, 1)):
        check(inputs(B, L, C, groups, dtype, wide), norm_r, norm, 0.75, dtype)


@pytest.mark.parametrize("C", [8, 16, 504, 512, 520, 640, 1024, 1032, 1536, 1544, 2048, 2056, 4096, 4104, 8192, 8200, 16384])
@pytest.mark.parametrize("M", [(1, 1), (3, 7), (1, 1100)])
def test_widths(C, M):
    if M[1] > 100 and C > 2056:
        pytest.skip("the same kernel as with few tokens")
    check(inputs(*M, C, dtype="bf16", wide=C % 16 == 0), "rms", "layer", 1.0, "bf16")


@pytest.mark.parametrize("C", [24, 64, 72, 128, 136, 160, 256, 264, 320])
@pytest.mark.parametrize("M,groups", [((1, 1), 1), ((3, 21), 7), ((2, 1100), 2)])
def test_narrow_tokens(C, M, groups):
    """Several tokens a wave, of different groups and batch items."""
    for dtype, wide, norm_r in (("f16", False, "layer"), ("bf16", True, "rms")):
        t = inputs(*M, C, groups=groups, dtype=dtype, wide=wide)
        check(t, norm_r, "layer", 0.75, dtype)


@pytest.mark.parametrize("missing", ["r", "gate", "scale", "shift", "gamma_r", "gamma", "beta", "all"])
def test_missing_parts(missing):
    t = inputs(2, 4, 320, 2)
    for n in ("gate", "scale", "shift", "gamma_r", "gamma", "beta") if missing == "all" else (missing,):
        t[n] = None
    if missing == "r":
        t["gate"] = None
    check(t, "layer", "rms", -1.5, "f16")


@pytest.mark.parametrize("wide", [False, True])
def test_in_place_and_one_output(wide):
    t = inputs(2, 9, 640, dtype="bf16", wide=wide)
    a = check(t, "none", "layer", 0.5, "bf16")
    b = check(t, "none", "layer", 0.5, "bf16", in_place=True)
    assert all((p == q).all() for p, q in zip(a, b))
    check(t, "none", "layer", 0.5, "bf16", h=False)
    check(t, "none", "layer", 0.5, "bf16", y=False)


@pytest.mark.parametrize("B,L,groups,batches,spread", [(3, 4, 1, 3, 6), (3, 4, 2, 3, 6), (3, 4, 4, 1, 6), (3, 4, 1, 1, 1), (1, 26, 13, 1, 2)])
def test_modulation_rows(B, L, groups, batches, spread):
    check(inputs(B, L, 72, groups, "f16", batches=batches, spread=spread), "rms", "rms", 1.0, "f16")


def test_rows_far_from_zero_and_constant_rows():
    """A layer norm is of deviations: a mean of 1000 costs the sum's error of it, no cancelled squares."""
    import torch
    t = inputs(1, 3, 1024, wide=True)
    t["x"] += 1000.0
    t["r"] = None
    t["gate"] = None
    check(t, "none", "layer", 1.0, "f16")
    t["x"] = torch.full_like(t["x"], 3.0)
    check(t, "none", "layer", 1.0, "f16")
    t["x"].zero_()
    check(t, "none", "rms", 1.0, "f16")


def test_more_values_than_32_bits_count():
    import torch
    M, C = 140000, 16384
    x = torch.zeros(1, M, C, dtype=torch.bfloat16, device="cuda")
    x[0, -1] = torch.randn(C, device="cuda").to(torch.bfloat16)
    y = torch.empty_like(x)
    sd.gated_norm(x, y, norm=sd.NORM_RMS)
    torch.cuda.synchronize()
    last = op.host(x[0, -1])
    want = last / np.sqrt((last ** 2).mean() + 1e-6)
    assert not y[0, :-1].any() and (np.abs(op.host(y[0, -1]) - want) <= 2.0 ** -7 * np.abs(want)).all()


def test_another_stream_and_native_marshalling(monkeypatch):
    import torch
    from paper_2304_11267_amd import binding
    t = inputs(2, 6, 320, 3, wide=True)
    a = check(t, "rms", "layer", 0.75, "f16")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    b = check(t, "rms", "layer", 0.75, "f16", stream=side)
    monkeypatch.setattr(binding, "_native", None)
    c = check(t, "rms", "layer", 0.75, "f16")
    assert all((p == q).all() and (p == r).all() for p, q, r in zip(a, b, c))
