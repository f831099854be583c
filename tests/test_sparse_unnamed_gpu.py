"""Attention over selected blocks: what lies in blocks that nobody names reaches no output,
for single queries in every form (head widths by the lanes of a row, one, two and four parts
of a head) and for many queries in every geometry; and single queries of many heads against
their 64-bit form."""
import numpy as np
import pytest

import operators_ref as ref
import paper_2304_11267_amd as sd
from parity_util import assert_close

pytestmark = pytest.mark.gpu

WIDTHS = [d for d in range(32, 161, 8) if d != 152]


@pytest.fixture(scope="module", autouse=True)
def _needs_gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    sd.load_library()


def spoilt_call(heads, Lq, Lk, D, qblock, dtype, seed):
    """Every head names its own half of the blocks, at least one; the others' keys and values are
    NaN or infinite in the second call."""
    import torch
    g = ref.generator(seed)
    q, k, v = (ref.randn(g, 1, heads, n, D, dtype=dtype) for n in (Lq, Lk, Lk))
    nb, nq = -(-Lk // 64), -(-Lq // qblock)
    rng = np.random.default_rng(seed)
    named = rng.random((1, heads, 1, nb)) < 0.5
    named[0, np.arange(heads), 0, rng.integers(0, nb, heads)] = True
    sel = np.repeat(named, nq, 2)
    mask = torch.from_numpy(ref.pack(sel)).cuda()
    clean, out = torch.empty_like(q), torch.empty_like(q)
    sd.sparse_forward(q, k, v, mask, clean, 0.125, qblock=qblock)
    other = torch.from_numpy(~named[0, :, 0]).cuda().repeat_interleave(64, 1)[:, :Lk]
    odd = (torch.arange(Lk, device="cuda") // 64) % 2 == 1
    for t in (k, v):
        t[0][other & odd] = float("nan")
        t[0][other & ~odd] = float("inf")
    sd.sparse_forward(q, k, v, mask, out, 0.125, qblock=qblock)
    torch.cuda.synchronize()
    assert torch.isfinite(clean.float()).all()
    assert torch.equal(out, clean)


@pytest.mark.parametrize("Lk", [1000, 1024, 1057])
@pytest.mark.parametrize("heads", [3, 65, 129])
@pytest.mark.parametrize("D", WIDTHS)
def test_single_queries(D, heads, Lk):
    spoilt_call(heads, 1, Lk, D, 64, "bf16" if D % 16 else "f16", D + heads)


@pytest.mark.parametrize("qblock", [64, 128])
@pytest.mark.parametrize("heads", [2, 140])    # at most, and more than, one round over the CUs
@pytest.mark.parametrize("D", WIDTHS)
def test_many_queries(D, heads, qblock):
    spoilt_call(heads, 250, 620, D, qblock, "f16" if D % 16 else "bf16", D + heads)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("heads", [64, 65, 128, 129, 300])
@pytest.mark.parametrize("D", [32, 40, 64, 104, 128, 136, 160])
def test_single_queries_of_many_heads(D, heads, dtype):
    import torch
    g = ref.generator(D + heads)
    Lk = 777
    q, k, v = (ref.randn(g, 1, heads, n, D, dtype=dtype) for n in (1, Lk, Lk))
    rng = np.random.default_rng(heads)
    sel = rng.random((1, heads, 1, 13)) < (np.arange(heads) % 5 / 4)[None, :, None, None]   # from none to all
    out = torch.full_like(q, 7.0)
    scale = float(np.float32(D ** -0.5))
    sd.sparse_forward(q, k, v, torch.from_numpy(ref.pack(sel)).cuda(), out, scale)
    torch.cuda.synchronize()
    got = ref.host(out)
    assert not got[~sel.any(-1)[..., 0]].any()
    r, dev = ref.sparse(ref.host(q), ref.host(k), ref.host(v), sel, scale, 64)
    assert_close(got, r, dtype=dtype, what=f"single {heads}x{Lk}x{D}", dev=dev)
