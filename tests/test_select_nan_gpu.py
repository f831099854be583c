"""Block selection where scores are no numbers: a NaN score, of either sign, counts as larger
than any number, and of several the lower blocks come first, in both kernels."""
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


NAN, MINUS_NAN, ALL_ONES = 0x7fc00000, 0xffc00000 - (1 << 32), -1


@pytest.mark.parametrize("bits", [NAN, MINUS_NAN, ALL_ONES], ids=["nan", "minus_nan", "all_ones"])
@pytest.mark.parametrize("H,nb", [(2, 130), (2, 600), (2, 1500), (300, 130), (300, 1500)])   # few and many query blocks
def test_a_score_that_is_no_number_is_the_largest(H, nb, bits):
    import torch
    g = ref.generator(nb + H)
    D, Lq = 40, 150
    q = ref.randn(g, 1, H, Lq, D, dtype="f16")
    means = torch.randn(1, H, nb, D, device="cuda", generator=g)
    at = sorted({0, 3, 63, 64, 100, nb - 1})
    words = means.view(torch.int32)
    for j, d in zip(at, (0, 39, 5, 8, 17, 31)):
        words[:, :, j, d] = bits
    means[:, :, 7, ::2], means[:, :, 7, 1::2] = float("inf"), -float("inf")   # infinities of both signs, or one
    means[:, :, 9, 11] = float("inf")
    with np.errstate(invalid="ignore"):
        scores = np.matmul(ref.block_means(ref.host(q), 64).astype(np.float32).astype(np.float64),
                           np.ascontiguousarray(ref.host(means).swapaxes(2, 3)))
    missing = np.isnan(scores)
    best = np.lexsort((np.broadcast_to(np.arange(nb), scores.shape), -np.where(missing, 0, scores), ~missing), axis=-1)
    for keep in (1, 4, len(at) + 1, len(at) + 20):
        mask = torch.empty(1, H, 3, -(-nb // 64), dtype=torch.int64, device="cuda")
        sd.select_blocks(q, means, mask, keep)
        torch.cuda.synchronize()
        sel = ref.unpack(mask.cpu().numpy(), nb)
        want = np.zeros(scores.shape, bool)
        np.put_along_axis(want, best[..., :keep], True, -1)
        assert np.array_equal(sel, want), keep
