"""Infinities and no numbers in keys that are seen: the score is what the product of query and key is, at every width alike (the
columns that fill the matrix core's last step at D = 8 (mod 16) are no key's).  A score of minus infinity has no weight; one
of plus infinity, or that is no number, makes the row one of no numbers; zeros where no score is above minus infinity."""
import numpy as np
import pytest

import operators_ref as op
import paper_2304_11267_amd as sd
import span_sizes as sizes
import stream_ref as ref
from test_span_gpu import window

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module", autouse=True)
def _needs_gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    sd.load_library()


def expected(q, k, v, see, scale):
    """[H, Lq, D] in 64 bits for q [H, Lq, D], k and v [Hk, keys, D], see [Lq, keys], with dev of ref.bound and the rows that
    are no numbers."""
    import torch
    H, Hk = q.shape[0], k.shape[0]
    kk, vv = (t.repeat_interleave(H // Hk, 0) for t in (k, v))
    a = (q[:, :, None] * kk[:, None]).sum(-1) * scale      # (a sum of infinities, not a matrix product's order)
    on = see[None].expand_as(a)
    bad = (on & (torch.isnan(a) | (a == INF))).any(-1)
    on = on & torch.isfinite(a)
    p = torch.softmax(a.masked_fill(~on, -INF), -1)
    p = torch.where(on, p, torch.zeros_like(p))            # (rows of none: softmax gives no numbers)
    o = torch.bmm(p, vv.contiguous())
    dev = torch.stack([(p[:, i, :, None] * (vv - o[:, i, None]).abs()).sum(1) for i in range(q.shape[1])], 1)
    top = a.abs().masked_fill(~on, 0.0).amax(-1)
    return o, dev, top, bad


def run(B, H, Hk, Lq, far, D, rule, dtype, odd, at_end=False):
    import torch
    kept = {}
    Lk = Lq + far

    def own(q, k, v):
        for key, col, x in odd:
            k[:, :, key, col] = x
        if at_end:
            q[:, :, :, 0] = q[:, :, :, 0].abs() + 0.5      # all keys from here on: minus infinity
            k[:, :, :, 0] = -INF
        kept.update(q=q.clone(), k=k.clone(), v=v.clone())
    got = op.host(window(B, H, Hk, Lq, Lk, D, *rule, dtype=dtype, tweak=own, check=False))
    see = ref.seen([far] * B, [Lq] * B, Lq, Lk, *rule)
    for b in range(B):
        o, dev, top, bad = (op.host(t) if t.dtype != torch.bool else t.cpu().numpy() for t in expected(
            *(kept[n][b].double() for n in "qkv"), torch.from_numpy(see[b]).cuda(), float(np.float32(D ** -0.5))))
        assert np.isnan(got[b][bad]).all(), (D, rule)
        g = np.where(bad[..., None], o, got[b])
        off = np.abs(g - o) / ref.bound(g, o, dev, top, Lk, D, float(kept["v"].abs().max()), dtype)
        assert off.max() <= 1.0, (D, rule, float(off.max()))
        if not at_end:
            assert bad.any() and not bad.all()


def places(D):
    """Keys of one infinity each, in the first columns, the last ones and between them."""
    return [(key, col % D, x) for key, (col, x) in zip((3, 40, 41, 97, 130, 150, 199),
                                                       ((0, INF), (D - 1, INF), (1, -INF), (D - 8, INF), (D - 7, -INF), (17, INF), (0, -INF)))]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("D", [32, 40, 56, 64, 72, 104, 120, 128, 136, 152, 160])
def test_few_rows(D, dtype):
    for place in places(D):
        run(2, 24, 12, 1, 199, D, (1, 0, 0), dtype, [place])
        run(2, 4, 2, 5, 200, D, (1, 0, 0), dtype, [place])
    run(2, 4, 4, 70, 140, D, (1, 60, 4), dtype, places(D))
    run(2, 4, 4, 70, 140, D, (0, 0, 0), dtype, places(D)[-1:])


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("D", [32, 40, 56, 64, 72, 104, 120, 128, 136, 152, 160])
def test_many_rows(D, dtype):
    B, H, Hk, L, far = sizes.LARGE
    for rule in ((1, 0, 0), (1, 90, 20)):
        run(B, H, Hk, L, far, D, rule, dtype, places(D) if rule[1] else places(D)[4:5])


@pytest.mark.parametrize("D", [40, 64, 136])
def test_rows_of_minus_infinity(D):
    for size in ((2, 4, 2, 1, 100), (2, 4, 2, 40, 60), sizes.LARGE):
        run(*size, D, (1, 0, 0), "bf16", [], at_end=True)
