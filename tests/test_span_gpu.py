"""sdattn_window_forward and sdattn_cache_forward against their 64-bit form: every head width, one
token to many, frames, windows and first tokens, groups of heads, both layouts, ragged batches, rows
that see nothing, values that are no numbers where they are not seen, keys split over
workgroups, pages that are not there, scales of either sign, large logits, caches past 32 bits."""
import numpy as np
import pytest

import operators_ref as op
import paper_2304_11267_amd as sd
import stream_ref as ref

pytestmark = pytest.mark.gpu
WIDTHS = list(range(32, 161, 8))


@pytest.fixture(scope="module", autouse=True)
def _needs_gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    sd.load_library()


def i32(v):
    import torch
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def rows(t):
    return t.transpose(1, 2).flatten(2).contiguous()


def finish(out, buf, see, q, k, v, scale, dtype, what):
    """`out` [B, H, Lq, D] against the 64-bit form; rows that are no queries hold the 7s they held."""
    import torch
    torch.cuda.synchronize()
    assert (buf[-64:] == 7).all()
    see_t = torch.from_numpy(see).cuda()
    r, dev, top = ref.attention(q.double(), k, v, see_t, scale)
    g, r, dev, top = (op.host(t) for t in (out, r, dev, top))
    return g, r, dev, top


def compare(g, r, dev, top, see, live, D, vmax, dtype, what):
    live = np.broadcast_to(live[:, None, :, None], g.shape)
    assert (g[~live] == 7).all(), what
    assert np.isfinite(g[live]).all(), what
    off = np.abs(g - r) / ref.bound(g, r, dev, top, max(1, see.sum(-1).max()), D, vmax, dtype)
    worst = float(off[live].max()) if live.any() else 0.0
    assert worst <= 1.0, f"{what}: {worst}"
    empty = live & ~np.broadcast_to(see.any(-1)[:, None, :, None], g.shape)
    assert not g[empty].any(), what


def window(B, H, Hk, Lq, Lk, D, frame=1, window=0, sinks=0, dtype="f16", starts=None, counts=None, x_rows=False, y_rows=False,
           scale=None, tweak=None, seed=3, workspace=True, stream=None, check=True):
    import torch
    g = op.generator(seed + Lq + Lk)
    q, k, v = op.randn(g, B, H, Lq, D, dtype=dtype), op.randn(g, B, Hk, Lk, D, dtype=dtype), op.randn(g, B, Hk, Lk, D, dtype=dtype)
    if tweak:
        tweak(q, k, v)
    scale = float(np.float32(D ** -0.5)) if scale is None else scale
    buf = torch.full((q.numel() + 64,), 7.0, dtype=q.dtype, device="cuda")
    o = buf[:-64].view(B, Lq, H * D) if y_rows else buf[:-64].view(B, H, Lq, D)
    n = sd.window_forward_workspace(B, H, Hk, Lq, Lk, D, frame, window, sinks)
    ws = torch.full((n,), 0x7f, dtype=torch.uint8, device="cuda") if n else None
    a = [rows(t) if x_rows else t for t in (q, k, v)]
    sd.window_forward(*a, o, scale, H, Hk, workspace=ws, starts=None if starts is None else i32(starts),
                      counts=None if counts is None else i32(counts), frame=frame, window=window, sinks=sinks,
                      x_layout=sd.LAYOUT_ROWS if x_rows else sd.LAYOUT_HEADS, y_layout=sd.LAYOUT_ROWS if y_rows else sd.LAYOUT_HEADS,
                      stream=stream)
    torch.cuda.synchronize()
    assert (buf[-64:] == 7).all()
    out = o.unflatten(2, (H, D)).transpose(1, 2) if y_rows else o
    if check:
        starts = [Lk - Lq] * B if starts is None else starts
        counts = [Lq] * B if counts is None else counts
        see = ref.seen(starts, counts, Lq, Lk, frame, window, sinks)
        live = np.arange(Lq) < np.clip(counts, 0, Lq)[:, None]
        r, dev, top = ref.attention(q.double(), k.double(), v.double(), torch.from_numpy(see).cuda(), scale)
        fine = torch.where(torch.isfinite(v), v, torch.zeros_like(v))
        compare(*(op.host(t) for t in (out, r, dev, top)), see, live, D, float(fine.abs().max()), dtype,
                f"window {B}x{H}/{Hk}x{Lq}x{Lk}x{D} frame {frame} window {window} sinks {sinks} {dtype}")
    return out


def cached(B, H, Hk, Lq, D, far, frame=1, window=0, sinks=0, dtype="f16", starts=None, counts=None, x_rows=False, y_rows=False,
           scale=None, missing=(), spoil=True, seed=5, slots=None, sizes=None):
    """Far tokens and Lq new ones through cache_write; what nobody has written holds no numbers."""
    import torch
    g = op.generator(seed + Lq + far)
    starts = [far] * B if starts is None else starts
    counts = [Lq] * B if counts is None else counts
    slots = slots or -(-(far + Lq) // 64)
    total = 64 * slots
    P = B * slots + 1
    table = np.random.default_rng(seed).permutation(P)[:B * slots].reshape(B, slots).astype(np.int32)
    codes = [torch.full((P, Hk, 64, D), 0x7f if spoil else 0x7e, dtype=torch.uint8, device="cuda") for _ in range(2)]
    scales = [torch.full((P, Hk), 2.0 ** 40, device="cuda") for _ in range(2)]
    k, v = (op.randn(g, B, Hk, total, D, dtype=dtype) for _ in range(2))
    if sizes is not None:
        k, v = (t * torch.tensor(sizes, device="cuda").to(t.dtype)[torch.arange(total, device="cuda") // 64 % len(sizes)][:, None] for t in (k, v))
    n = [min(max(s + min(max(c, 0), Lq), 0), 64 * slots) for s, c in zip(starts, counts)]
    dev = lambda: (*codes, *scales, torch.from_numpy(table).cuda())   # noqa: E731
    sd.cache_write(k, v, *dev(), i32([0] * B), counts=i32(n))
    back = sd.cache_read(torch.zeros_like(k), torch.zeros_like(v), *dev(), i32([0] * B), counts=i32(n))
    gone = np.zeros((B, slots), bool)
    for b, s in missing:
        table[b, s] = -1 if (b + s) % 2 else P + s
        gone[b, s] = True
    q = op.randn(g, B, H, Lq, D, dtype=dtype)
    scale = float(np.float32(D ** -0.5)) if scale is None else scale
    buf = torch.full((q.numel() + 64,), 7.0, dtype=q.dtype, device="cuda")
    o = buf[:-64].view(B, Lq, H * D) if y_rows else buf[:-64].view(B, H, Lq, D)
    nw = sd.cache_forward_workspace(B, H, Hk, Lq, D, slots, frame, window, sinks)
    ws = torch.full((nw,), 0x7f, dtype=torch.uint8, device="cuda") if nw else None
    sd.cache_forward(rows(q) if x_rows else q, *dev(), i32(starts), o, scale, H, workspace=ws, counts=i32(counts), frame=frame,
                     window=window, sinks=sinks, x_layout=sd.LAYOUT_ROWS if x_rows else sd.LAYOUT_HEADS,
                     y_layout=sd.LAYOUT_ROWS if y_rows else sd.LAYOUT_HEADS)
    torch.cuda.synchronize()
    assert (buf[-64:] == 7).all()
    out = o.unflatten(2, (H, D)).transpose(1, 2) if y_rows else o
    see = ref.seen(starts, counts, Lq, 64 * slots, frame, window, sinks)
    see &= ~np.repeat(gone, 64, axis=1)[:, None]
    see = see[:, :, :total]
    live = np.arange(Lq) < np.clip(counts, 0, Lq)[:, None]
    r, d, top = ref.attention(q.double(), *(t.double() for t in back), torch.from_numpy(see).cuda(), scale)
    compare(*(op.host(t) for t in (out, r, d, top)), see, live, D, float(back[1].abs().max()), dtype,
            f"cached {B}x{H}/{Hk}x{Lq}x{D} after {far} frame {frame} window {window} sinks {sinks} {dtype}")
    return out


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("D", WIDTHS)
def test_widths(D, dtype):
    window(1, 2, 1, 150, 260, D, window=100, sinks=5, dtype=dtype, x_rows=D % 16 == 0)
    cached(1, 2, 1, 150, D, 110, window=100, sinks=5, dtype=dtype, y_rows=D % 16 == 0)
    window(2, 2, 2, 1, 300, D, window=200, sinks=3, dtype=dtype, y_rows=D % 16 == 0)
    cached(2, 2, 2, 1, D, 300, window=200, sinks=3, dtype=dtype, x_rows=D % 16 == 0)


RULES = [(1, 0, 0), (1, 1, 0), (1, 64, 0), (1, 65, 1), (1, 200, 64), (1, 1000, 100), (0, 0, 0), (0, 130, 0), (0, 50, 70), (7, 0, 0),
         (7, 20, 3), (64, 128, 65), (90, 180, 90), (1 << 30, 0, 0), (2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1)]


@pytest.mark.parametrize("rule", RULES, ids=lambda r: "{}-{}-{}".format(*r))
def test_rules(rule):
    for Lq, Lk in ((300, 300), (129, 640), (1, 500), (5, 77)):
        window(1, 2, 2, Lq, Lk, 64, *rule)
        cached(1, 2, 2, Lq, 64, Lk - Lq, *rule, dtype="bf16")


@pytest.mark.parametrize("Lq,Lk", [(1, 1), (1, 2), (1, 63), (1, 64), (1, 65), (2, 64), (2, 65), (31, 32), (32, 33), (33, 33), (64, 64), (65, 65),
                                   (127, 128), (128, 129), (129, 129), (257, 1000)])
@pytest.mark.parametrize("D", [40, 128])
def test_lengths(Lq, Lk, D):
    window(2, 3, 3, Lq, Lk, D)
    cached(2, 3, 3, Lq, D, Lk - Lq)
    window(2, 3, 1, Lq, Lk, D, frame=0, window=40, sinks=2, dtype="bf16")


@pytest.mark.parametrize("H,Hk", [(1, 1), (2, 1), (5, 1), (6, 2), (7, 1), (8, 2), (32, 2), (33, 3), (40, 1), (64, 1), (130, 1)])
@pytest.mark.parametrize("Lq", [1, 2, 3, 9, 70])
def test_groups_of_heads(H, Hk, Lq):
    window(2, H, Hk, Lq, 200, 40, window=90, sinks=4)
    cached(2, H, Hk, Lq, 40, 200 - Lq, window=90, sinks=4, dtype="bf16")


@pytest.mark.parametrize("x_rows", [False, True])
@pytest.mark.parametrize("y_rows", [False, True])
def test_layouts(x_rows, y_rows):
    for Lq in (1, 70):
        window(2, 6, 3, Lq, 150, 48, x_rows=x_rows, y_rows=y_rows)
        cached(2, 6, 3, Lq, 48, 150, x_rows=x_rows, y_rows=y_rows)


@pytest.mark.parametrize("Lq", [1, 4, 40, 200])
def test_ragged_batches(Lq):
    far = 260
    starts = [far, 0, 100, 63, 64, -3, far, 17]
    counts = [Lq, Lq, Lq - 1, 1, 0, Lq, -5, 10 * Lq]
    for rule in ((1, 0, 0), (1, 70, 9), (0, 0, 0), (5, 64, 64)):
        window(8, 4, 2, Lq, far + Lq, 64, *rule, starts=starts, counts=counts)
        cached(8, 4, 2, Lq, 64, far, *rule, starts=starts, counts=counts)


def test_places_out_of_bounds():
    """Whatever the integers on the device say, what is read and written lies within the tensors."""
    for s in (2 ** 31 - 1, -2 ** 31, 2 ** 31 - 40, -39, 500, 270):
        for Lq in (1, 40):
            window(2, 2, 2, Lq, 300, 40, 1, 64, 3, starts=[s, 5], counts=[Lq, Lq])
            cached(2, 2, 2, Lq, 40, 260, 1, 64, 3, starts=[s, 5], counts=[Lq, Lq])
            window(2, 2, 2, Lq, 300, 40, 0, 0, 0, starts=[s, 5], counts=[Lq, Lq])


def test_more_queries_than_keys():
    """Without starts the first queries lie before the sequence: they see nothing, or with no order everything."""
    for rule in ((1, 0, 0), (1, 8, 2), (0, 0, 0), (6, 0, 0)):
        window(2, 2, 1, 90, 30, 40, *rule)
        window(2, 2, 1, 3, 1, 40, *rule)


@pytest.mark.parametrize("what", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("Lq", [1, 3, 150])
def test_no_numbers_where_nothing_is_seen(what, Lq):
    """Keys past the end, before the window, and after each query's own place (those rows aside that see them)."""
    import torch
    for rule in ((1, 60, 5), (0, 100, 5), (8, 64, 0)):
        def spoil(q, k, v):
            for t in (k, v):
                t[:, :, 250:] = what          # past the sequences' ends
                t[:, :, 5:20] = what          # before every window
        window(2, 4, 2, Lq, 300, 64, *rule, starts=[250 - Lq, 240 - Lq] if Lq < 150 else [100, 90], counts=[Lq, Lq], tweak=spoil)
    # within a tile that other queries see: rows before it as without it, rows that see it without a number
    if Lq > 1:
        for dtype in ("f16", "bf16"):
            at = 200 - Lq // 2

            def own(q, k, v):
                v[:, :, at, 3] = what
                k[:, :, at] = what if what != what else k[:, :, at]
            a = window(1, 2, 2, Lq, 200, 64, dtype=dtype, tweak=own, check=False)
            b = window(1, 2, 2, Lq, 200, 64, dtype=dtype, check=False)
            first = at - (200 - Lq)   # the first row that sees it
            assert torch.equal(a[:, :, :first], b[:, :, :first])
            assert not torch.isfinite(a[:, :, first:, 3]).any()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("D", [40, 64, 128, 136])
@pytest.mark.parametrize("Lq", [1, 7, 150, 260])
def test_infinite_values_and_no_numbers_reach_their_columns(Lq, D, dtype):
    """A value of V that is no number, or infinite, makes that of its column for the queries that see it: what else
    they give, and what the others give, is as with a zero there."""
    import torch
    Lk, H = 260, 2
    inf, nan = float("inf"), float("nan")
    # (key, column, value): two infinities of one column meet at key 258
    odd = [(30, 3, inf), (130, 3, inf), (131, 8, -inf), (200, 8, -inf), (129, 17, nan), (210, D - 1, inf), (255, 9, inf), (258, 9, -inf)]
    for rule in ((1, 0, 0), (1, 64, 0), (1, 40, 31), (0, 100, 33)):
        def own(q, k, v):
            for key, col, x in odd:
                v[:, :, key, col] = x

        def none(q, k, v):
            for key, col, x in odd:
                v[:, :, key, col] = 0
        got = window(1, H, 1, Lq, Lk, D, *rule, dtype=dtype, tweak=own, check=False).float()
        want = window(1, H, 1, Lq, Lk, D, *rule, dtype=dtype, tweak=none, check=False).float()
        see = torch.from_numpy(ref.seen([Lk - Lq], [Lq], Lq, Lk, *rule)[0]).cuda()
        for key, col, x in odd:
            want[:, :, see[:, key], col] += x
        assert torch.equal(torch.nan_to_num(got, 1e5, 2e5, -2e5), torch.nan_to_num(want, 1e5, 2e5, -2e5)), rule


@pytest.mark.parametrize("Lq", [1, 7, 150])
def test_codes_of_no_numbers_reach_their_columns(Lq):
    """As above, for a cache, in which infinities are no numbers."""
    import torch
    n, H, D, dtype = 260, 2, 64, "bf16"
    odd = [(30, 3), (130, 3), (131, 8), (200, 8), (129, 17), (210, 63), (258, 9)]
    g = op.generator(4)
    k, v, q = (op.randn(g, 1, h, l, D, dtype=dtype) for h, l in ((1, n), (1, n), (H, Lq)))
    k[:], table = 0.5 * k, i32([[2, 0, 3, 1, 4]])
    for rule in ((1, 0, 0), (1, 64, 0), (1, 40, 31), (0, 100, 33)):
        outs = []
        for x in (0.0, float("nan")):
            for key, col in odd:
                v[:, :, key, col] = x
            c = [torch.zeros(5, 1, 64, D, dtype=torch.uint8, device="cuda") for _ in range(2)]
            c += [torch.ones(5, 1, device="cuda") for _ in range(2)]
            sd.cache_write(k, v, *c, table, i32([0]))
            ws = torch.empty(max(16, sd.cache_forward_workspace(1, H, 1, Lq, D, 5, *rule)), dtype=torch.uint8, device="cuda")
            outs.append(sd.cache_forward(q, *c, table, i32([n - Lq]), torch.empty_like(q), 0.125, H, workspace=ws, frame=rule[0],
                                         window=rule[1], sinks=rule[2]).float())
        see = torch.from_numpy(ref.seen([n - Lq], [Lq], Lq, n, *rule)[0]).cuda()
        for key, col in odd:
            outs[0][:, :, see[:, key], col] = float("nan")
        assert torch.equal(torch.nan_to_num(outs[1], 1e5), torch.nan_to_num(outs[0], 1e5)), rule


def test_no_numbers_in_the_cache():
    """A token of no numbers in the cache: rows before it as without it, and a window leaves it behind."""
    import torch
    B, H, D, n = 1, 2, 64, 200
    g = op.generator(2)
    k, v, q = (op.randn(g, B, H, n, D) for _ in range(3))
    codes = [torch.zeros(4, H, 64, D, dtype=torch.uint8, device="cuda") for _ in range(2)]
    scales = [torch.ones(4, H, device="cuda") for _ in range(2)]
    table, zero = i32([[2, 0, 3, 1]]), i32([0])
    outs = []
    for bad in (False, True):
        if bad:
            k[:, :, 70], v[:, :, 70] = float("nan"), float("nan")
        sd.cache_write(k, v, *codes, *scales, table, zero)
        outs.append([torch.empty_like(q) for _ in range(2)])
        for o, w in zip(outs[-1], (0, 50)):
            ws = torch.empty(max(16, sd.cache_forward_workspace(B, H, H, n, D, 4, 1, w, 0)), dtype=torch.uint8, device="cuda")
            sd.cache_forward(q, *codes, *scales, table, zero, o, 0.125, H, workspace=ws, window=w)
    torch.cuda.synchronize()
    for w, a, b in zip((0, 50), *outs):
        see = [p for p in range(n) if p >= 70 and (w == 0 or p < 120)]
        rest = [p for p in range(n) if p not in see]
        # (the page's scale may go by the token that is no number now: a step of its codes)
        assert torch.isfinite(b[:, :, rest]).all() and (a - b)[:, :, rest].abs().max() < 0.25
        assert not torch.isfinite(b[:, :, see]).any()
        assert torch.equal(a[:, :, :64], b[:, :, :64])


@pytest.mark.parametrize("Lq", [1, 2, 40, 130])
def test_pages_that_are_not_there(Lq):
    for rule in ((1, 0, 0), (1, 130, 70)):
        cached(2, 4, 2, Lq, 64, 700, *rule, missing=[(0, 0), (0, 3), (0, 4), (1, 9), (1, 10)])
        cached(2, 4, 2, Lq, 64, 100, *rule, missing=[(b, s) for b in range(2) for s in range(4) if s * 64 < 100 + Lq])


@pytest.mark.parametrize("Lk", [2000, 5000, 20000])
@pytest.mark.parametrize("Lq", [1, 3, 33, 130])
def test_keys_split_over_workgroups(Lq, Lk):
    """Few rows and many keys; windows leave some of the parts without a key."""
    for dtype, rule in (("f16", (1, 0, 0)), ("bf16", (1, 1500, 300)), ("f16", (0, 70, 1))):
        window(1, 2, 1, Lq, Lk, 128, *rule, dtype=dtype)
        cached(2, 2, 1, Lq, 128, Lk - Lq, *rule, dtype=dtype, starts=[Lk - Lq, 10], counts=[Lq, Lq])


@pytest.mark.parametrize("scale", [0.0, -0.0, -0.2, 3.0])
def test_scales(scale):
    for Lq in (1, 140):
        window(1, 2, 2, Lq, 300, 40, 1, 150, 3, scale=scale)
        cached(1, 2, 2, Lq, 40, 300 - Lq, 1, 150, 3, scale=scale, dtype="bf16")


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_late_dominant_keys(dtype):
    """Keys whose norms grow along the sequence: the maximum moves from tile to tile."""
    import torch

    def grow(q, k, v):
        k *= torch.linspace(0.2, 6.0, k.shape[2], device="cuda").to(k.dtype)[:, None]
    for Lq in (1, 5, 200):
        window(1, 2, 2, Lq, 900, 64, dtype=dtype, tweak=grow)
        cached(1, 2, 2, Lq, 64, 900, dtype=dtype, sizes=[0.25, 4.0, 1.0, 8.0, 0.125, 8.0])


def test_splits_share_nothing_between_calls():
    """Another call's leavings in the workspace, and ragged counts that leave rows of it unwritten."""
    import torch
    B, H, Hk, Lq, Lk, D = 2, 4, 2, 3, 4000, 64
    n = sd.window_forward_workspace(B, H, Hk, Lq, Lk, D)
    assert n > 0
    g = op.generator(1)
    q, k, v = op.randn(g, B, H, Lq, D), op.randn(g, B, Hk, Lk, D), op.randn(g, B, Hk, Lk, D)
    outs = []
    for fill in (0, 0xff, 0x7f):
        ws = torch.full((n,), fill, dtype=torch.uint8, device="cuda")
        o = torch.zeros_like(q)
        sd.window_forward(q, k, v, o, 0.1, H, Hk, workspace=ws, starts=i32([3000, 2]), counts=i32([3, 2]))
        outs.append(o)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


def test_long_tensors():
    """Keys past 2^31 values of one tensor, pages past 2^32 bytes."""
    import torch
    Lk, D = (1 << 24) + 200, 128
    k = torch.zeros(1, 1, Lk, D, dtype=torch.float16, device="cuda")
    v = torch.zeros(1, 1, Lk, D, dtype=torch.float16, device="cuda")
    g = op.generator(1)
    tail = [op.randn(g, 1, 1, 300, D) for _ in range(2)]
    k[:, :, -300:], v[:, :, -300:] = tail
    for Lq in (1, 100):
        q, o = op.randn(g, 1, 2, Lq, D), torch.empty(1, 2, Lq, D, dtype=torch.float16, device="cuda")
        small = torch.empty_like(o)
        ws = torch.empty(max(16, sd.window_forward_workspace(1, 2, 1, Lq, Lk, D, 1, 150, 0)), dtype=torch.uint8, device="cuda")
        sd.window_forward(q, k, v, o, 0.1, 2, 1, workspace=ws, window=150)
        ws2 = torch.empty(max(16, sd.window_forward_workspace(1, 2, 1, Lq, 300, D, 1, 150, 0)), dtype=torch.uint8, device="cuda")
        sd.window_forward(q, *tail, small, 0.1, 2, 1, workspace=ws2, window=150)
        torch.cuda.synchronize()
        assert (o.float() - small.float()).abs().max() <= 2e-3
    del k, v
    P, Hk = 140000, 4
    codes = [torch.zeros(P, Hk, 64, D, dtype=torch.uint8, device="cuda") for _ in range(2)]
    scales = [torch.ones(P, Hk, device="cuda") for _ in range(2)]
    near = [torch.zeros(3, Hk, 64, D, dtype=torch.uint8, device="cuda") for _ in range(2)]
    near_scales = [torch.ones(3, Hk, device="cuda") for _ in range(2)]
    x, y = (op.randn(g, 1, Hk, 170, D) for _ in range(2))
    far_t, near_t = i32([[P - 1, P - 2, 139999 - 7]]), i32([[0, 1, 2]])
    sd.cache_write(x, y, *codes, *scales, far_t, i32([0]))
    sd.cache_write(x, y, *near, *near_scales, near_t, i32([0]))
    for Lq in (1, 100):
        q = op.randn(g, 1, 8, Lq, D)
        outs = [torch.empty_like(q) for _ in range(2)]
        for o, c, s, t in ((outs[0], codes, scales, far_t), (outs[1], near, near_scales, near_t)):
            ws = torch.empty(max(16, sd.cache_forward_workspace(1, 8, Hk, Lq, D, 3)), dtype=torch.uint8, device="cuda")
            sd.cache_forward(q, *c, *s, t, i32([170 - Lq]), o, 0.1, 8, workspace=ws)
        torch.cuda.synchronize()
        assert torch.equal(*outs)


def test_another_stream_and_native_marshalling(monkeypatch):
    import torch
    from paper_2304_11267_amd import binding
    a = [window(2, 4, 2, Lq, 3000, 64, 1, 2000, 7) for Lq in (1, 90)]
    side = torch.cuda.Stream()
    b = [window(2, 4, 2, Lq, 3000, 64, 1, 2000, 7, stream=side) for Lq in (1, 90)]
    c0 = [cached(2, 4, 2, Lq, 64, 2900, 1, 2000, 7) for Lq in (1, 90)]
    monkeypatch.setattr(binding, "_native", None)
    c = [window(2, 4, 2, Lq, 3000, 64, 1, 2000, 7) for Lq in (1, 90)]
    c1 = [cached(2, 4, 2, Lq, 64, 2900, 1, 2000, 7) for Lq in (1, 90)]
    assert all(torch.equal(p, q) and torch.equal(p, r) for p, q, r in zip(a, b, c)) and all(torch.equal(p, q) for p, q in zip(c0, c1))


@pytest.mark.parametrize("D", [40, 64, 128, 160])
def test_few_tiles_in_parts(D):
    """Few blocks of rows over few tiles, in parts of two or three; one token over wide heads, whose parts are short."""
    for dtype, rule in (("f16", (1, 0, 0)), ("bf16", (1, 150, 70)), ("f16", (0, 0, 0)), ("bf16", (100, 300, 0))):
        window(1, 2, 1, 310, 863, D, *rule, dtype=dtype)
        cached(1, 2, 1, 310, D, 553, *rule, dtype=dtype)
        window(1, 4, 1, 1, 1389, D, *rule, dtype=dtype)
        cached(2, 4, 1, 1, D, 1388, *rule, dtype=dtype, starts=[1388, 3])


def test_what_a_page_holds_behind_the_sequence():
    """Codes that are no numbers, or large ones, behind the last token: the same bits."""
    import torch
    for Lq in (1, 9, 70):
        for D in (40, 128):
            a, b = (cached(2, 8, 2, Lq, D, 3, spoil=s) for s in (True, False))
            assert torch.equal(a, b)


@pytest.mark.parametrize("D", [40, 72, 128, 160])
@pytest.mark.parametrize("H,Hk", [(1, 1), (6, 2), (5, 1)])
def test_blocks_of_32_rows(H, Hk, D):
    """More rows than one block of 32 and few blocks: tokens whose heads lie in two blocks, ragged counts, parts of keys."""
    for Lq in (12, 33, 70, 201):
        for rule in ((1, 0, 0), (1, 45, 9), (0, 0, 0), (16, 64, 40)):
            window(2, H, Hk, Lq, Lq + 90, D, *rule, starts=[90, 17], counts=[Lq, Lq - 5], x_rows=D == 72, y_rows=D != 72)
            cached(2, H, Hk, Lq, D, 90, *rule, dtype="bf16", starts=[90, 64], counts=[Lq - 9, Lq], x_rows=D != 72, missing=[(0, 0)])
        cached(1, H, Hk, Lq, D, 9000, 1, 0, 0)
        window(1, H, Hk, Lq, 9000, D, 1, 8000, 100, dtype="bf16")


@pytest.mark.parametrize("D", [40, 64, 128, 160])
def test_many_short_sequences(D):
    """More blocks than CUs, of one tile or a few: workgroups of fewer waves."""
    for Lq, keys in ((1, 1), (1, 20), (1, 64), (1, 130), (4, 40), (8, 8), (5, 97)):
        counts = [Lq - b % 2 if Lq > 1 else 1 - b % 3 // 2 for b in range(40)]
        window(40, 16, 8, Lq, max(keys, Lq), D, counts=counts, starts=[max(keys, Lq) - Lq - b % 3 for b in range(40)])
        cached(40, 16, 8, Lq, D, max(keys - Lq, 0), dtype="bf16", counts=counts, starts=[max(keys - Lq - b % 5, 0) for b in range(40)])
