"""Scores far from zero in the attention over what a place sees: below every ordinary bound, and so large that a rounding
of one is many octaves of a weight.  Queries are powers of two and keys small whole numbers times one, so that products and
sums are exact in 32 bits: equal scores have equal weights, others lie far apart, and the softmax is as well known as of small ones."""
import numpy as np
import pytest

import operators_ref as op
import paper_2304_11267_amd as sd
import span_sizes as sizes
import stream_ref as ref
from test_span_gpu import compare, i32

pytestmark = pytest.mark.gpu

SIGNS = {"below": [-1], "above": [1], "mixed": [1, -1, -1], "rising": [-1]}
# exponents of queries and keys: sums of D products of at most 13 2^(q + k) stay within 32 bits
SPAN = {"f16": (14, 11), "bf16": (61, 45)}


@pytest.fixture(scope="module", autouse=True)
def _needs_gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    sd.load_library()


def inputs(B, H, Hk, Lq, Lk, D, sign, dtype, far=None):
    """Queries of 2^0 to 2^(the type's), or all of 2^far."""
    import torch
    qe, ke = SPAN[dtype]
    i, j = torch.arange(Lq, device="cuda"), torch.arange(Lk, device="cuda")
    e = (i * 5 % (qe + 1)).double() if far is None else torch.full((Lq,), float(far), device="cuda", dtype=torch.double)
    s = torch.tensor(SIGNS[sign], device="cuda", dtype=torch.double)[j % len(SIGNS[sign])]
    # (rising: far below zero at first, near it in the end)
    c = s * (1 + j * 7 % 13) * 2.0 ** torch.where((j < Lk // 2) | (sign != "rising"), ke, -qe - 1)
    t = op.t_type(dtype)
    q = (2.0 ** e).to(t)[None, None, :, None].expand(B, H, Lq, D).contiguous()
    k = c.to(t)[None, None, :, None].expand(B, Hk, Lk, D).contiguous()
    assert (k[0, 0, :, 0].double() == c).all() and torch.isfinite(q).all()
    return q, k, op.randn(op.generator(Lq + Lk), B, Hk, Lk, D, dtype=dtype)


def check(out, q, k, v, starts, rule, scale, dtype, what):
    import torch
    torch.cuda.synchronize()
    B, H, Lq, D = q.shape
    see = ref.seen(starts, [Lq] * B, Lq, k.shape[2], *rule)
    r, dev, top = ref.attention(q.double(), k.double(), v.double(), torch.from_numpy(see).cuda(), float(np.float32(scale)))
    # a score that is off by 2^-22 of its distance from the largest: nothing where that is more than 64
    top = top.clamp(max=64.0)
    compare(*(op.host(t) for t in (out, r, dev, top)), see, np.ones((B, Lq), bool), D, float(v.abs().max()), dtype, what)


def dense(B, H, Hk, Lq, far, D, sign, dtype, rule=(1, 0, 0), scale=None, q_exp=None, tweak=None):
    import torch
    q, k, v = inputs(B, H, Hk, Lq, Lq + far, D, sign, dtype, q_exp)
    if tweak:
        tweak(q, k)
    scale = D ** -0.5 if scale is None else scale
    ws = torch.full((max(16, sd.window_forward_workspace(B, H, Hk, Lq, Lq + far, D, *rule)),), 0x7f, dtype=torch.uint8, device="cuda")
    out = sd.window_forward(q, k, v, torch.empty_like(q), scale, H, Hk, workspace=ws, frame=rule[0], window=rule[1], sinks=rule[2])
    check(out, q, k, v, [far] * B, rule, scale, dtype, f"{sign} {dtype} {Lq} after {far}, {D}, {rule}")


def paged(B, H, Hk, Lq, far, D, sign, dtype, rule=(1, 0, 0), scale=None, q_exp=None, tweak=None):
    import torch
    q, k, v = inputs(B, H, Hk, Lq, Lq + far, D, sign, dtype, q_exp)
    if tweak:
        tweak(q, k)
    scale = D ** -0.5 if scale is None else scale
    slots = -(-(Lq + far) // 64)
    c = [torch.zeros(B * slots, Hk, 64, D, dtype=torch.uint8, device="cuda") for _ in range(2)]
    c += [torch.ones(B * slots, Hk, device="cuda") for _ in range(2)]
    table = torch.arange(B * slots, dtype=torch.int32, device="cuda").flip(0).view(B, slots).contiguous()
    sd.cache_write(k, v, *c, table, i32([0] * B))
    k2, v2 = sd.cache_read(torch.empty_like(k), torch.empty_like(v), *c, table, i32([0] * B))
    assert sign == "rising" or torch.equal(k, k2)   # (rising: the page with both sizes has one scale)
    ws = torch.full((max(16, sd.cache_forward_workspace(B, H, Hk, Lq, D, slots, *rule)),), 0x7f, dtype=torch.uint8, device="cuda")
    out = sd.cache_forward(q, *c, table, i32([far] * B), torch.empty_like(q), scale, H, workspace=ws, frame=rule[0], window=rule[1],
                           sinks=rule[2])
    check(out, q, k2, v2, [far] * B, rule, scale, dtype, f"pages {sign} {dtype} {Lq} after {far}, {D}, {rule}")


FORMS = {"dense": dense, "paged": paged}


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("sign", SIGNS)
@pytest.mark.parametrize("D", [40, 64, 128, 136])
def test_few_rows(D, sign, dtype, form):
    run = FORMS[form]
    for far in SPAN[dtype][0], 3:
        run(2, 4, 2, 1, 300, D, sign, dtype, q_exp=far)
        run(1, 4, 1, 1, 5000, D, sign, dtype, q_exp=far)          # in parts
    for rule in ((1, 0, 0), (1, 90, 20), (0, 100, 0)):
        run(2, 4, 2, 33, 200, D, sign, dtype, rule)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("sign", SIGNS)
@pytest.mark.parametrize("D", [40, 64, 128, 136])
def test_many_rows(D, sign, dtype, form):
    run = FORMS[form]
    B, H, Hk, L, far = sizes.LARGE
    for rule in ((1, 0, 0), (1, 90, 20)):
        run(B, H, Hk, L, far, D, sign, dtype, rule)
    if D in (64, 128):
        B, H, Hk, L, far = sizes.CAUSAL                           # in parts
        run(B, H, Hk, L, far, D, sign, dtype)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("Lq", [1, 40, 250])
def test_large_scales(Lq, form):
    """A scale of any finite size: of products that it makes huge, and of products that are zero."""
    B, H, Hk = sizes.LARGE[:3] if Lq == 250 else (2, 4, 2)
    for scale in (1e30, -1e30):
        FORMS[form](B, H, Hk, Lq, 60 if Lq < 250 else 0, 64, "mixed", "bf16", scale=scale, q_exp=-50)

    def zero(q, k):
        q.zero_()
    for scale in (3e38, -3e38, 1e20):
        FORMS[form](B, H, Hk, Lq, 60 if Lq < 250 else 0, 64, "mixed", "bf16", scale=scale, tweak=zero)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("Lq", [1, 40, 250])
def test_small_scales(Lq, form):
    """A scale among the subnormals, of products of up to 2^127."""
    B, H, Hk = sizes.LARGE[:3] if Lq == 250 else (2, 4, 2)
    for D in (40, 128):
        for scale in (2.0 ** -127.5, -2.0 ** -127.5):
            FORMS[form](B, H, Hk, Lq, 60 if Lq < 250 else 0, D, "mixed", "bf16", scale=scale, q_exp=72 if D == 40 else 70)
