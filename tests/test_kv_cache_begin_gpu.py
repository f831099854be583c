"""A sequence whose first token lies inside of a page: a scale of 0 is that of a page without tokens, whatever its codes."""
import pytest

import operators_ref as op
import paper_2304_11267_amd as sd
import stream_ref as ref
from test_kv_cache_gpu import Cache

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _needs_gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    sd.load_library()


@pytest.mark.parametrize("L", [1, 30, 100])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_a_page_without_tokens(L, dtype):
    import numpy as np
    import torch
    B, Hk, D = 2, 2, 40
    c = Cache(B, Hk, D, 4)
    for s, d in zip(c.scales, c.dev_scales):
        s[:] = 0.0
        d.zero_()
    g = op.generator(L)
    k, v = (op.randn(g, B, Hk, L, D, dtype=dtype) for _ in range(2))
    starts = [10, 100]
    sd.cache_write(k, v, *c.dev(), torch.tensor(starts, dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    back = [torch.empty_like(t) for t in (k, v)]
    sd.cache_read(*back, *c.dev(), torch.tensor(starts, dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    for x, y, scale in zip((k, v), back, c.dev_scales):
        x, y = op.host(x), op.host(y)
        for b in range(B):
            for slot in range(starts[b] // 64, -(-(starts[b] + L) // 64)):
                i, j = max(starts[b], 64 * slot) - starts[b], min(starts[b] + L, 64 * slot + 64) - starts[b]
                for h in range(Hk):
                    new, s = x[b, h, i:j], float(scale[c.table[b, slot], h])
                    assert s == 2.0 ** ref.exponent(np.abs(new).max())
                    assert (np.abs(y[b, h, i:j] - new) <= 2.0 ** -4 * np.abs(new) + 2.0 ** -10 * s).all()
    # and a window that begins with them
    q, o = op.randn(g, B, 4, L, D, dtype=dtype), torch.empty(B, 4, L, D, dtype=op.t_type(dtype), device="cuda")
    ws = torch.empty(max(16, sd.cache_forward_workspace(B, 4, Hk, L, D, 4, 1, 1, 0)), dtype=torch.uint8, device="cuda")
    sd.cache_forward(q, *c.dev(), torch.tensor(starts, dtype=torch.int32, device="cuda"), o, 0.1, 4, workspace=ws, window=1)
    torch.cuda.synchronize()
    assert torch.equal(o, back[1].repeat_interleave(2, 1))   # (a token that sees itself alone)
