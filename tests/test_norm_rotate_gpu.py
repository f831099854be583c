"""Per-head norms with the position rotation against the 64-bit form: every head width,
one to four axes, adjacent and halved pairs, part of a head turned, both layouts on both
sides, in place, far and negative positions, shared positions, one token."""
import numpy as np
import pytest

import operators_ref as ref
import paper_2304_11267_amd as sd

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _needs_gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    sd.load_library()


def split(P, n):
    return tuple(P // n + (i < P % n) for i in range(n))


def run(B, H, L, D, pairs, dtype="f16", halves=False, xl=1, yl=1, norm=True, eps=1e-6, k=True, gammas=True, far=100,
        batches=None, in_place=False, seed=3):
    import torch
    g = ref.generator(seed)
    P = sum(pairs)
    shape, into = ((B, H, L, D) if h else (B, L, H * D) for h in (xl, yl))
    q, kt = ref.randn(g, *shape, dtype=dtype, sigma=3.0), ref.randn(g, *shape, dtype=dtype) if k else None
    qh, kh = ref.host(q), ref.host(kt) if k else None
    gq, gk = (ref.randn(g, D, dtype=dtype) if gammas else None for _ in range(2))
    batches = B if batches is None else batches
    pos = freqs = None
    if P:
        pos = torch.randint(-far, far, (batches, L, len(pairs)), device="cuda", generator=g, dtype=torch.int32)
        freqs = (10000.0 ** (-torch.arange(P, dtype=torch.float64) / P)).float().cuda()
    full = [torch.full((int(np.prod(into)) + 64,), 7.0, dtype=ref.t_type(dtype), device="cuda") for _ in range(2)]
    qo, ko = (q, kt) if in_place else (t[:-64].view(into) for t in full)
    sd.norm_rotate(q, qo, H, k=kt, ko=ko if k else None, gamma_q=gq, gamma_k=gk if k else None, pos=pos, freqs=freqs,
                   pairs=pairs, norm=sd.NORM_RMS if norm else sd.NORM_NONE, eps=eps,
                   pairing=sd.PAIR_HALVES if halves else sd.PAIR_ADJACENT, x_layout=xl, y_layout=yl)
    torch.cuda.synchronize()
    assert (full[0][-64:] == 7).all() and (full[1][-64:] == 7).all()
    for x, gamma, y in ((qh, gq, qo), (kh, gk, ko))[:2 if k else 1]:
        x = x if xl else ref.rows_to_heads(x, H)
        out = ref.host(y) if yl else ref.rows_to_heads(ref.host(y), H)
        r, off = ref.norm_rotate(x, None if gamma is None else ref.host(gamma), None if pos is None else pos.cpu().numpy().astype(float),
                                 None if freqs is None else ref.host(freqs), pairs, norm, eps, halves)
        bound = off + ref.half_step(out, r, dtype) * (1 + 2.0 ** -10)
        assert np.all(np.abs(out - r) <= bound), float(np.max(np.abs(out - r) / bound))


@pytest.mark.parametrize("halves", [False, True], ids=["adjacent", "halves"])
@pytest.mark.parametrize("D", list(range(8, 257, 8)))
def test_every_width(D, halves):
    run(2, 3, 11, D, split(D // 2, 2), halves=halves, dtype="bf16" if D % 16 else "f16")


@pytest.mark.parametrize("halves", [False, True], ids=["adjacent", "halves"])
@pytest.mark.parametrize("P,n", [(1, 1), (2, 1), (3, 3), (4, 2), (7, 4), (10, 2), (16, 3), (19, 4), (20, 4), (0, 0)])
def test_part_of_a_head(P, n, halves):
    run(2, 2, 9, 40, split(P, n) if n else (), halves=halves)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("xl,yl", [(0, 0), (0, 1), (1, 0), (1, 1)], ids=["rr", "rh", "hr", "hh"])
@pytest.mark.parametrize("B,H,L,D", [(1, 1, 1, 64), (16, 8, 1, 160), (3, 5, 700, 40), (1, 7, 2100, 128)],
                         ids=lambda v: str(v))
def test_layouts(B, H, L, D, xl, yl, dtype):
    run(B, H, L, D, split(D // 2, 3), dtype=dtype, xl=xl, yl=yl, halves=D == 128)


@pytest.mark.parametrize("layout", [0, 1], ids=["rows", "heads"])
@pytest.mark.parametrize("P", [20, 7])
def test_in_place(layout, P):
    run(2, 8, 300, 40, (P,), xl=layout, yl=layout, in_place=True, halves=True)


@pytest.mark.parametrize("kw", [dict(norm=False), dict(gammas=False), dict(k=False), dict(batches=1),
                                dict(far=1 << 20), dict(far=(1 << 31) - 1), dict(eps=0.0), dict(eps=10.0),
                                dict(norm=False, gammas=False, k=False)],
                         ids=lambda k: "_".join("%s" % n for n in k))
def test_options(kw):
    run(3, 4, 50, 64, (10, 22), **kw)
    run(3, 4, 50, 64, (10, 22), halves=True, dtype="bf16", **kw)


def test_a_row_of_zeros_stays_zero():
    import torch
    q = torch.zeros(1, 2, 5, 64, dtype=torch.float16, device="cuda")
    q[0, 1, 3] = 1.0
    out = torch.empty_like(q)
    sd.norm_rotate(q, out, 2)
    torch.cuda.synchronize()
    want = q.clone()
    want[0, 1, 3] = 1.0
    assert torch.equal(out, want)   # mean of ones 1, eps 1e-6: rounds to 1


def test_not_a_number_stays_in_its_row():
    import torch
    q = ref.randn(ref.generator(1), 1, 3, 40, 80, dtype="f16")
    q[0, 1, 7, 3] = float("nan")
    out = torch.empty_like(q)
    sd.norm_rotate(q, out, 3)
    torch.cuda.synchronize()
    bad = torch.isnan(out).any(-1)
    assert bad[0, 1, 7] and int(bad.sum()) == 1


@pytest.mark.parametrize("halves", [False, True], ids=["adjacent", "halves"])
@pytest.mark.parametrize("D,P", [(64, 16), (64, 6), (40, 12), (128, 40), (128, 0)])
def test_values_that_are_not_turned_never_meet_their_neighbours(D, P, halves):
    import torch
    g = ref.generator(6)
    q = ref.randn(g, 1, 2, 9, D, dtype="bf16")
    q[0, 1, 4, 2 * P] = float("inf")
    q[0, 0, 2, D - 1] = float("nan")
    q[0, 0, 5, 2 * P:] = -0.0
    pos = torch.arange(9, device="cuda", dtype=torch.int32).view(1, 9, 1) if P else None
    freqs = torch.ones(P, device="cuda") if P else None
    out = torch.empty_like(q)
    sd.norm_rotate(q, out, 2, pos=pos, freqs=freqs, pairs=(P,) if P else (), norm=sd.NORM_NONE,
                   pairing=sd.PAIR_HALVES if halves else sd.PAIR_ADJACENT)
    torch.cuda.synchronize()
    assert torch.equal(out[..., 2 * P:].view(torch.int16), q[..., 2 * P:].view(torch.int16))
    assert torch.isfinite(out[..., :2 * P].float()).all()
