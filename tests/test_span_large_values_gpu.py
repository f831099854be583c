"""Values of V at the ends of bf16 in the attention over what a place sees: an average of finite values is finite, however many
keys there are, and small ones keep their steps."""
import pytest

import paper_2304_11267_amd as sd
import span_sizes as sizes
from test_span_gpu import cached, window

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _needs_gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    sd.load_library()


CALLS = [(2, 4, 2, 1, 300), (1, 4, 1, 1, 5000), (1, 2, 1, 1, 40000), (2, 4, 2, 33, 200), sizes.LARGE, sizes.CAUSAL, sizes.PARTS[0][:5]]


@pytest.mark.parametrize("call", CALLS, ids=lambda c: "{}-{}-{}-{}-{}".format(*c))
@pytest.mark.parametrize("D", [40, 64, 128, 136])
def test_dense(call, D):
    B, H, Hk, Lq, far = call
    for what in ("largest", "large", "small"):
        def own(q, k, v):
            import torch
            if what == "largest":
                v.fill_(torch.finfo(v.dtype).max)
                v[:, :, ::3] *= -1
                v[..., 0] = torch.finfo(v.dtype).max
            elif what == "large":
                v.clamp_(-7.0, 7.0)
                v *= 2.0 ** 124
            else:
                v *= 2.0 ** -90
        window(B, H, Hk, Lq, Lq + far, D, 1, 0, 0, dtype="bf16", tweak=own)


@pytest.mark.parametrize("call", CALLS, ids=lambda c: "{}-{}-{}-{}-{}".format(*c))
@pytest.mark.parametrize("D", [40, 64, 128, 136])
def test_pages(call, D):
    """As above, by the pages' scales (the keys' are as large, and so the call's scale is as small)."""
    B, H, Hk, Lq, far = call
    for e in (124, -90):
        # (sizes are powers of two, of both K and V)
        cached(B, H, Hk, Lq, D, far, dtype="bf16", sizes=[2.0 ** (e - 1), 2.0 ** (e - 2)], scale=D ** -0.5 * 2.0 ** -e)
