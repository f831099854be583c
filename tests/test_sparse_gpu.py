"""Block means, the choice of key blocks, and the attention over chosen blocks against
their 64-bit forms: every head width, ragged last blocks, masks with everything, one block,
the last block alone or nothing, more blocks than a wave holds words for, ties, keys that
send a workgroup through its second pass, and values in blocks that nobody names."""
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


def nblocks(n, block=64):
    return -(-n // block)


def masks(B, H, nq, nb, how, seed):
    rng = np.random.default_rng(seed)
    sel = np.zeros((B, H, nq, nb), bool)
    if how == "all":
        sel[:] = True
    elif how == "last":
        sel[..., -1] = True
    elif how == "first":
        sel[..., 0] = True
    elif how == "mixed":   # from none to all, row by row
        for i in range(nq):
            sel[:, :, i] = rng.random((B, H, nb)) < (i % 5) / 4
    elif how == "few":
        sel = rng.random(sel.shape) < 3 / nb
    return sel


def run(B, H, Lq, Lk, D, qblock, how, dtype="f16", seed=11, tweak=None, scale=None, n_keys=None):
    import torch
    g = ref.generator(seed)
    q, k, v = (ref.randn(g, B, H, n, D, dtype=dtype) for n in (Lq, Lk, Lk))
    if tweak:
        tweak(q, k, v)
    sel = masks(B, H, nblocks(Lq, qblock), nblocks(Lk), how, seed) if isinstance(how, str) else how
    words = ref.pack(sel)
    if nblocks(Lk) % 64:   # bits past the last block are ignored
        words[..., -1] |= np.int64(-1) << np.int64(nblocks(Lk) % 64)
    mask = torch.from_numpy(words).cuda()
    buf = torch.full((q.numel() + 64,), 7.0, dtype=q.dtype, device="cuda")
    out = buf[:q.numel()].view_as(q)
    scale = float(np.float32(D ** -0.5)) if scale is None else scale
    sd.sparse_forward(q, k, v, mask, out, scale, qblock=qblock)
    torch.cuda.synchronize()
    assert (buf[q.numel():] == 7).all()
    r, dev = ref.sparse(ref.host(q), ref.host(k), ref.host(v), sel, scale, qblock)
    got = ref.host(out)
    empty = ~sel.any(-1)
    for b, h, i in np.argwhere(empty):
        assert not got[b, h, i * qblock:(i + 1) * qblock].any()
    if not empty.all():   # (nothing named at all: the zeros above are the whole answer)
        assert_close(got, r, dtype=dtype, what=f"sparse {B}x{H}x{Lq}x{Lk}x{D} {qblock}", dev=dev, n_keys=n_keys)
    return out


@pytest.mark.parametrize("qblock", [64, 128])
@pytest.mark.parametrize("D", WIDTHS)
def test_every_width(D, qblock):
    run(1, 2, 200, 333, D, qblock, "mixed", dtype="bf16" if D % 16 else "f16", seed=D)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("qblock", [64, 128])
@pytest.mark.parametrize("how", ["all", "first", "last", "mixed", "few"])
@pytest.mark.parametrize("D", [40, 64, 80, 160])
def test_masks(D, how, qblock, dtype):
    run(2, 2, 300, 1000, D, qblock, how, dtype=dtype)


@pytest.mark.parametrize("Lq,Lk", [(1, 1), (1, 63), (1, 64), (1, 65), (1, 5000), (64, 64), (65, 127), (129, 31), (700, 2049)],
                         ids=lambda v: str(v))
@pytest.mark.parametrize("D,qblock", [(40, 64), (64, 128), (128, 64), (128, 128)])
def test_lengths(Lq, Lk, D, qblock):
    run(2, 3, Lq, Lk, D, qblock, "all" if Lk < 200 else "mixed")


@pytest.mark.parametrize("Lk", [64, 100, 1000, 5000, 32768])
@pytest.mark.parametrize("D", [40, 64, 128, 160])
def test_one_token_over_half_of_the_blocks(D, Lk):
    sel = np.random.default_rng(Lk + D).random((2, 3, 1, nblocks(Lk))) < 0.5
    sel[:, 0, :, -1] = True
    run(2, 3, 1, Lk, D, 64, sel, dtype="bf16")


@pytest.mark.parametrize("D,qblock", [(40, 128), (64, 64), (64, 128), (96, 64)] +
                         [(d, q) for d in WIDTHS if d > 64 for q in ((64, 128) if d > 80 else (128,)) if (d, q) != (96, 64)])
def test_full_grid(D, qblock):
    """More query blocks than CUs (the geometry of two workgroups a CU at D = 64)."""
    run(4, 8, 1300, 640, D, qblock, "few", seed=5)


@pytest.mark.parametrize("qblock", [64, 128])
def test_more_words_than_lanes(qblock):
    """4100 and 9000 key blocks: 65 and 141 words a row, bits on both sides of every 64th word."""
    for nb, on in ((4100, (3, 4095, 4096, 4099)), (9000, (0, 63, 64, 4032, 4095, 4096, 8191, 8192, 8999))):
        sel = np.zeros((1, 1, nblocks(70, qblock), nb), bool)
        sel[..., list(on)] = True
        if qblock == 64:
            sel[0, 0, 1] = False
            sel[0, 0, 1, nb - 1] = True
        run(1, 1, 70, 64 * nb - 30, 32, qblock, sel)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("D,qblock", [(40, 64), (40, 128), (64, 128), (80, 64), (128, 128)])
def test_late_dominant_keys(D, qblock, dtype):
    """Keys whose norms grow along the sequence: the fixed maximum's second pass."""
    import torch

    def grow(q, k, v):
        k *= torch.linspace(0.2, 6.0, k.shape[2], device="cuda").to(k.dtype)[:, None]

    run(1, 2, 130, 1500, D, qblock, "mixed", dtype=dtype, tweak=grow)


def test_scale_of_either_sign_and_zero():
    for scale in (-0.3, 0.0, 2.0):
        run(1, 2, 100, 400, 40, 64, "mixed", scale=scale)


def test_blocks_that_nobody_names_are_not_read():
    import torch
    sel = masks(1, 2, 2, 8, "mixed", 3)
    sel[:, :, :, 2] = sel[:, :, :, 7] = False
    sel[..., 0] = True

    def spoil(q, k, v):
        for t in (k, v):
            t[:, :, 128:192] = float("nan")
            t[:, :, 448:] = float("inf")

    import torch
    g = ref.generator(4)
    q, k, v = (ref.randn(g, 1, 2, n, 64, dtype="f16") for n in (128, 500, 500))
    out, clean = torch.empty_like(q), torch.empty_like(q)
    mask = torch.from_numpy(ref.pack(sel)).cuda()
    sd.sparse_forward(q, k, v, mask, clean, 0.125)
    spoil(q, k, v)
    sd.sparse_forward(q, k, v, mask, out, 0.125)
    torch.cuda.synchronize()
    assert torch.equal(out, clean) and torch.isfinite(out).all()


def test_everything_named_is_the_plain_attention():
    """All blocks: the same sums as sdattn_forward's, in the same geometry the same bits."""
    import torch
    g = ref.generator(8)
    q, k, v = (ref.randn(g, 2, 8, 1024, 64, dtype="f16") for _ in range(3))
    out, plain = torch.empty_like(q), torch.empty_like(q)
    mask = torch.full((2, 8, 8, 1), -1, dtype=torch.int64, device="cuda")
    sd.sparse_forward(q, k, v, mask, out, 0.125, qblock=128)
    sd.forward(q, k, v, plain, 0.125)
    torch.cuda.synchronize()
    assert (out.float() - plain.float()).abs().max() <= 2e-3


# ---------------------------------------------------------------- means and choice

@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("L", [1, 63, 64, 65, 1000])
@pytest.mark.parametrize("D", [8, 40, 64, 136, 256])
def test_means(D, L, dtype):
    import torch
    x = ref.randn(ref.generator(D + L), 2, 3, L, D, dtype=dtype, sigma=2.0)
    buf = torch.full((2 * 3 * nblocks(L) * D + 32,), 7.0, device="cuda")
    sd.block_means(x, buf[:-32].view(2, 3, nblocks(L), D))
    torch.cuda.synchronize()
    g, r = ref.host(buf[:-32]).reshape(2, 3, nblocks(L), D), ref.block_means(ref.host(x), 64)
    # the sum is held in 64 bits (exact, or within 64 2^-53 of the values' sizes), one rounding to 32
    size = ref.block_means(np.abs(ref.host(x)), 64)
    assert np.all(np.abs(g - r) <= 2.0 ** -24 * np.abs(r) * (1 + 2.0 ** -10) + 2.0 ** -46 * size)
    assert (buf[-32:] == 7).all()


def choose(q, means, keep, qblock):
    import torch
    B, H, Lq, _ = q.shape
    nb = means.shape[2]
    words = nblocks(nb)
    buf = torch.full((B * H * nblocks(Lq, qblock) * words + 8,), 7, dtype=torch.int64, device="cuda")
    mask = buf[:-8].view(B, H, nblocks(Lq, qblock), words)
    sd.select_blocks(q, means, mask, keep, qblock=qblock)
    torch.cuda.synchronize()
    assert (buf[-8:] == 7).all()
    w = mask.cpu().numpy()
    sel = ref.unpack(w, nb)
    assert np.array_equal(ref.pack(sel), w)   # no bits past the last block
    return sel


def f32(a):
    return a.astype(np.float32).astype(np.float64)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("qblock", [64, 128])
@pytest.mark.parametrize("Lq,nb,D,keep", [(1, 1, 64, 1), (1, 512, 128, 32), (1000, 16, 40, 4), (333, 65, 80, 64),
                                          (700, 300, 8, 1), (129, 129, 256, 128), (200, 64, 160, 63), (300, 100, 64, 1000),
                                          (64, 1025, 64, 400)], ids=lambda v: str(v))
def test_choice(Lq, nb, D, keep, qblock, dtype):
    import torch
    g = ref.generator(Lq + nb)
    q = ref.randn(g, 2, 3, Lq, D, dtype=dtype)
    means = torch.randn(2, 3, nb, D, device="cuda", generator=g)
    sel = choose(q, means, keep, qblock)
    want = ref.select(f32(ref.block_means(ref.host(q), qblock)), ref.host(means), keep)
    assert np.array_equal(sel, want)


@pytest.mark.parametrize("qblock", [64, 128])
@pytest.mark.parametrize("nb,D,keep,dtype", [(19, 40, 5, "f16"), (100, 8, 30, "bf16"), (257, 256, 100, "f16"),
                                             (600, 160, 77, "bf16"), (1100, 72, 300, "f16"), (4000, 64, 64, "bf16")],
                         ids=lambda v: str(v))
def test_choice_for_many_queries(nb, D, keep, dtype, qblock):
    """More query blocks than two for each CU: several of them a workgroup."""
    import torch
    g = ref.generator(nb + D)
    B, H, Lq = 7, 8, 10 * qblock + 3
    q = ref.randn(g, B, H, Lq, D, dtype=dtype)
    means = torch.randn(B, H, nb, D, device="cuda", generator=g)
    sel = choose(q, means, keep, qblock)
    assert np.array_equal(sel, ref.select(f32(ref.block_means(ref.host(q), qblock)), ref.host(means), keep))


@pytest.mark.parametrize("nb,keep", [(4096, 100), (4097, 37), (16384, 4000)])
def test_choice_among_many(nb, keep):
    import torch
    g = ref.generator(nb)
    q = ref.randn(g, 1, 2, 300, 32, dtype="f16")
    means = torch.randn(1, 2, nb, 32, device="cuda", generator=g)
    assert np.array_equal(choose(q, means, keep, 64),
                          ref.select(f32(ref.block_means(ref.host(q), 64)), ref.host(means), keep))


def test_ties_go_to_the_lower_block():
    """Whole-number queries and means of a few values: many equal scores, zeros of both signs."""
    import torch
    g = ref.generator(2)
    q = torch.randint(-1, 2, (1, 4, 640, 16), device="cuda", generator=g).repeat_interleave(64, 2)[:, :, :640].half()
    means = torch.randint(-1, 2, (1, 4, 200, 16), device="cuda", generator=g).float()
    means[:, 0] = 0.0
    means[:, 1, ::2] = -0.0
    for keep in (1, 7, 64, 150):
        assert np.array_equal(choose(q, means, keep, 64),
                              ref.select(f32(ref.block_means(ref.host(q), 64)), ref.host(means), keep)), keep


def test_scores_next_to_each_other():
    """Means one step of fp32 apart: a score in 32 bits would not tell them from each other."""
    import torch
    g = ref.generator(6)
    q = ref.randn(g, 1, 1, 64, 64, dtype="f16")
    row = torch.randn(64, device="cuda", generator=g)
    means = row.repeat(1, 1, 128, 1).clone()
    for j in range(128):   # the first j % 64 values one step up
        means[0, 0, j, :j % 64] = torch.nextafter(row[:j % 64], torch.full_like(row[:j % 64], 10.0))
    for keep in (1, 5, 64):
        assert np.array_equal(choose(q, means, keep, 64),
                              ref.select(f32(ref.block_means(ref.host(q), 64)), ref.host(means), keep)), keep


def test_infinite_and_missing_scores_end():
    """NaN and infinite means: as many bits as asked for, whatever they are."""
    import torch
    g = ref.generator(7)
    q = ref.randn(g, 1, 1, 64, 64, dtype="f16")
    means = torch.randn(1, 1, 200, 64, device="cuda", generator=g)
    means[0, 0, 5] = float("nan")
    means[0, 0, 9, 3] = float("inf")
    means[0, 0, 11, 3] = -float("inf")
    assert int(choose(q, means, 20, 64).sum()) == 20
    means[:] = float("nan")
    assert int(choose(q, means, 20, 64).sum()) == 20


@pytest.mark.parametrize("Lq,qblock", [(1, 64), (130, 64), (130, 128)])
@pytest.mark.parametrize("D", [32, 64, 128, 160])
def test_a_named_block_without_numbers_shows(D, Lq, qblock):
    """Keys that are NaN all over one named block, or over all of them: no finite output of
    their head, and the other head's as before."""
    import torch
    g = ref.generator(21)
    q, k, v = (ref.randn(g, 1, 2, n, D, dtype="bf16") for n in (Lq, 700, 700))
    sel = np.ones((1, 2, -(-Lq // qblock), 11), bool)
    mask = torch.from_numpy(ref.pack(sel)).cuda()
    clean, out = torch.empty_like(q), torch.empty_like(q)
    sd.sparse_forward(q, k, v, mask, clean, 0.125, qblock=qblock)
    for spoilt in (slice(128, 192), slice(640, 700), slice(None)):
        bad = k.clone()
        bad[:, 1, spoilt] = float("nan")
        sd.sparse_forward(q, bad, v, mask, out, 0.125, qblock=qblock)
        torch.cuda.synchronize()
        assert torch.equal(out[:, 0], clean[:, 0])
        assert not torch.isfinite(out[:, 1].float()).any(), spoilt
