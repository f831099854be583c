"""Attention over selected blocks in full grids whose last key block is ragged: odd and even
numbers of named blocks with that block among them, in the geometries without a key split
and their neighbours, with and without the second pass of late dominant keys."""
import numpy as np
import pytest

import operators_ref as ref
import paper_2304_11267_amd as sd
from parity_util import assert_close

pytestmark = pytest.mark.gpu

WIDTHS = [d for d in range(32, 161, 8) if d != 152]
HEADS, LQ = 264, 65      # 264 blocks of 128 queries, 528 of 64
LK, NB = 401, 7


@pytest.fixture(scope="module", autouse=True)
def _needs_gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    sd.load_library()


def some_blocks(nq, seed):
    """1 to NB named blocks, another number for each block of queries in turn, the ragged last
    one among them (but in every ninth)."""
    rng = np.random.default_rng(seed)
    sel = np.zeros((1, HEADS, nq, NB), bool)
    for n, at in enumerate(np.ndindex(1, HEADS, nq)):
        last = n % 9 != 8
        count = n % NB + (not last)
        sel[at][rng.permutation(NB - 1)[:count]] = True
        sel[at][NB - 1] = last
    return sel


def reference(q, k, v, sel, scale, qblock):
    """operators_ref.sparse in torch's 64 bits on the GPU: out, and what rounding the weights may move."""
    import torch
    q, k, v = (t[0].double() for t in (q, k, v))
    on = torch.from_numpy(sel[0]).cuda().repeat_interleave(64, 2)[:, :, :LK].repeat_interleave(qblock, 1)[:, :LQ]
    s = torch.matmul(q, k.transpose(1, 2).contiguous()) * scale
    p = torch.softmax(s.masked_fill(~on, -float("inf")), -1)
    out = torch.matmul(p, v)
    dev = torch.stack([(p[h, :, :, None] * (v[h, None] - out[h, :, None]).abs()).sum(1) for h in range(HEADS)])
    return ref.host(out)[None], ref.host(dev)[None]


def check(D, qblock, dtype, grow, seed):
    import torch
    g = ref.generator(seed)
    q, k, v = (ref.randn(g, 1, HEADS, n, D, dtype=dtype) for n in (LQ, LK, LK))
    if grow:
        k *= torch.linspace(0.2, 6.0, LK, device="cuda").to(k.dtype)[:, None]
    sel = some_blocks(-(-LQ // qblock), seed)
    mask = torch.from_numpy(ref.pack(sel)).cuda()
    scale = float(np.float32(D ** -0.5))
    out, again = torch.empty_like(q), torch.empty_like(q)
    sd.sparse_forward(q, k, v, mask, out, scale, qblock=qblock)
    sd.sparse_forward(q, k, v, mask, again, scale, qblock=qblock)
    torch.cuda.synchronize()
    assert torch.equal(out, again)
    r, dev = reference(q, k, v, sel, scale, qblock)
    assert_close(ref.host(out), r, dtype=dtype, what=f"ragged {D} {qblock}", dev=dev)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("qblock", [64, 128])
@pytest.mark.parametrize("D", WIDTHS)
def test_odd_and_even_numbers_of_blocks(D, qblock, dtype):
    check(D, qblock, dtype, False, 100 + D)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("D,qblock", [(40, 64), (64, 128), (72, 128), (88, 64), (128, 64), (128, 128), (160, 128)])
def test_late_dominant_keys(D, qblock, dtype):
    check(D, qblock, dtype, True, 200 + D)
