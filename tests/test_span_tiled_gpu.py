"""The tiled kernel of the attention over what a query's place lets it see, against the 64-bit form: sizes of more than 256 blocks of
32 rows (span_sizes.py, which test_span_plan.py holds to that kernel), over every width, rule, edge of a tile, group of heads and
layout, ragged batches, values that are no numbers, pages that are not there, parts of keys and their joins, tensors
past 32 bits, other streams and graphs."""
import numpy as np
import pytest

import operators_ref as op
import paper_2304_11267_amd as sd
import span_sizes as sizes
import stream_ref as ref
from test_span_gpu import cached, i32, window

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _needs_gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    sd.load_library()


def both(size, D, rule, dtype="f16", **kw):
    B, H, Hk, Lq, far = size
    window(B, H, Hk, Lq, Lq + far, D, *rule, dtype=dtype, **kw)
    cached(B, H, Hk, Lq, D, far, *rule, dtype="bf16" if dtype == "f16" else "f16", **kw)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("D", sizes.WIDTHS)
def test_widths(D, dtype):
    both(sizes.USUAL, D, (1, 100, 5), dtype, x_rows=D % 16 == 0, y_rows=D % 24 == 0)


@pytest.mark.parametrize("rule", sizes.RULES, ids=lambda r: "{}-{}-{}".format(*r))
def test_rules(rule):
    both(sizes.USUAL, 64, rule)


@pytest.mark.parametrize("length", sizes.LENGTHS, ids=lambda n: "{}-{}".format(*n))
@pytest.mark.parametrize("D", [40, 128])
def test_lengths(length, D):
    both(sizes.MANY + length, D, (1, 0, 0))
    both(sizes.MANY + length, D, (0, 40, 2), "bf16")


@pytest.mark.parametrize("group", sizes.GROUPS, ids=lambda g: "{}-{}".format(*g[1:3]))
@pytest.mark.parametrize("D", [40, 128])
def test_groups_of_heads(group, D):
    both(group, D, (1, 90, 4), x_rows=D == 40, y_rows=D == 128)


@pytest.mark.parametrize("D", [64, 128])
def test_ragged_batches(D):
    B, H, Hk, Lq, far = sizes.RAGGED
    starts = [far, 0, 100, 63, 64, -3, far, 17]
    counts = [Lq, Lq, Lq - 1, 1, 0, Lq, -5, 10 * Lq]
    for rule in ((1, 0, 0), (1, 70, 9), (0, 0, 0), (5, 64, 64)):
        both(sizes.RAGGED, D, rule, starts=starts, counts=counts)
    starts = [2 ** 31 - 1, -2 ** 31, 2 ** 31 - 40, -39, 500, 270, 0, 5]   # what is read and written lies within the tensors
    both(sizes.RAGGED, D, (1, 70, 9), starts=starts, counts=[Lq] * B)
    both(sizes.RAGGED, D, (0, 0, 0), starts=starts, counts=[Lq] * B)


@pytest.mark.parametrize("what", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("D", [40, 64, 128, 136])
def test_no_numbers_where_nothing_is_seen(what, D):
    B, H, Hk, Lq, _ = sizes.USUAL
    for rule in ((1, 60, 5), (0, 100, 5), (8, 64, 0)):
        def spoil(q, k, v):
            for t in (k, v):
                t[:, :, 320:] = what          # past the sequences' ends
                t[:, :, 5:20] = what          # before every window
        window(B, H, Hk, Lq, 360, D, *rule, starts=[120 - b for b in range(B)], counts=[Lq] * B, tweak=spoil)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("D", [40, 64, 128, 136])
def test_infinite_values_and_no_numbers_reach_their_columns(D, dtype):
    import torch
    B, H, Hk, L, _ = sizes.INFINITE
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
        got = window(B, H, Hk, L, L, D, *rule, dtype=dtype, tweak=own, check=False).float()
        want = window(B, H, Hk, L, L, D, *rule, dtype=dtype, tweak=none, check=False).float()
        see = torch.from_numpy(ref.seen([0], [L], L, L, *rule)[0]).cuda()
        for key, col, x in odd:
            want[:, :, see[:, key], col] += x
        assert torch.equal(torch.nan_to_num(got, 1e5, 2e5, -2e5), torch.nan_to_num(want, 1e5, 2e5, -2e5)), rule


@pytest.mark.parametrize("D", [40, 64, 128, 136])
def test_codes_of_no_numbers_reach_their_columns(D):
    import torch
    B, H, Hk, L, _ = sizes.INFINITE
    odd = [(30, 3), (130, 3), (131, 8), (200, 8), (129, 17), (210, D - 1), (258, 9)]
    g = op.generator(4)
    k, v, q = (op.randn(g, 1, h, L, D, dtype="bf16") for h in (Hk, Hk, H))
    table, zero = i32([[2, 0, 3, 1, 4]]), i32([0])
    for rule in ((1, 0, 0), (1, 64, 0), (1, 40, 31), (0, 100, 33)):
        outs = []
        for x in (0.0, float("nan")):
            for key, col in odd:
                v[:, :, key, col] = x
            c = [torch.zeros(5, Hk, 64, D, dtype=torch.uint8, device="cuda") for _ in range(2)]
            c += [torch.ones(5, Hk, device="cuda") for _ in range(2)]
            sd.cache_write(k, v, *c, table, zero)
            ws = torch.empty(max(16, sd.cache_forward_workspace(1, H, Hk, L, D, 5, *rule)), dtype=torch.uint8, device="cuda")
            outs.append(sd.cache_forward(q, *c, table, zero, torch.empty_like(q), 0.125, H, workspace=ws, frame=rule[0],
                                         window=rule[1], sinks=rule[2]).float())
        see = torch.from_numpy(ref.seen([0], [L], L, L, *rule)[0]).cuda()
        for key, col in odd:
            outs[0][:, :, see[:, key], col] = float("nan")
        assert torch.equal(torch.nan_to_num(outs[1], 1e5), torch.nan_to_num(outs[0], 1e5)), rule


@pytest.mark.parametrize("D", [64, 128])
def test_keys_of_no_numbers(D):
    """A key that is no number: rows before it as without it, rows that see it without a number, those past it as without it."""
    import torch
    B, H, Hk, L, _ = sizes.INFINITE
    rule = (1, 64, 0)

    def own(q, k, v):
        k[:, :, 100, D - 1] = float("nan")
    got = window(B, H, Hk, L, L, D, *rule, tweak=own, check=False)
    want = window(B, H, Hk, L, L, D, *rule, check=False)
    assert torch.equal(got[:, :, :100], want[:, :, :100]) and torch.equal(got[:, :, 164:], want[:, :, 164:])
    assert torch.isnan(got[:, :, 100:164]).all()


@pytest.mark.parametrize("D", [64, 128])
def test_pages_that_are_not_there(D):
    B, H, Hk, Lq, far = sizes.PAGES
    for rule in ((1, 0, 0), (1, 130, 70)):
        cached(B, H, Hk, Lq, D, far, *rule, missing=[(0, 0), (0, 3), (0, 4), (1, 9), (1, 10)])
        cached(B, H, Hk, Lq, D, far, *rule, missing=[(b, s) for b in range(2) for s in range(14)])


@pytest.mark.parametrize("D", [40, 64, 128, 160])
def test_keys_in_parts(D):
    """Parts of two and more, some of them without a key: ragged sequences, windows that leave parts behind."""
    for size in sizes.PARTS:
        B, H, Hk, Lq, far = size[:5]
        both(size[:5], D, size[5], starts=[far] + [10] * (B - 1), counts=[Lq - 3 * b for b in range(B)])


@pytest.mark.parametrize("scale", [0.0, -0.2, 3.0])
def test_scales(scale):
    both(sizes.LARGE, 40, (1, 90, 20), scale=scale)
    both(sizes.LARGE, 128, (1, 0, 0), scale=scale)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
def test_late_dominant_keys(D, dtype):
    """Keys whose norms grow along the sequence: the maximum moves from tile to tile."""
    import torch
    B, H, Hk, L, _ = sizes.LARGE

    def grow(q, k, v):
        k *= torch.linspace(0.2, 6.0, k.shape[2], device="cuda").to(k.dtype)[:, None]
    window(B, H, Hk, L, L, D, dtype=dtype, tweak=grow)
    cached(B, H, Hk, L, D, 0, dtype=dtype, sizes=[0.25, 4.0, 1.0, 8.0, 0.125, 8.0])


def test_what_a_page_holds_behind_the_sequence():
    import torch
    B, H, Hk, Lq, far = sizes.RAGGED
    for D in (64, 128):
        a, b = (cached(B, H, Hk, Lq, D, far, spoil=s) for s in (True, False))
        assert torch.equal(a, b)


def test_long_tensors():
    """Keys past 2^31 values of one tensor, pages past 2^32 bytes."""
    import torch
    B, H, Hk, Lq, far = sizes.FAR_DENSE
    Lk, D, n = far + Lq, 128, Lq + 200
    g = op.generator(1)
    k, v = (torch.zeros(1, 1, Lk, D, dtype=torch.float16, device="cuda") for _ in range(2))
    tail = [op.randn(g, 1, 1, n, D) for _ in range(2)]
    k[:, :, -n:], v[:, :, -n:] = tail
    q = op.randn(g, 1, H, Lq, D)
    outs = []
    for kk, vv in ((k, v), tail):
        ws = torch.empty(max(16, sd.window_forward_workspace(1, H, 1, Lq, kk.shape[2], D, 1, 150, 0)), dtype=torch.uint8, device="cuda")
        outs.append(sd.window_forward(q, kk, vv, torch.empty_like(q), 0.1, H, 1, workspace=ws, window=150))
    torch.cuda.synchronize()
    # (tiles begin at other keys: weights are rounded relative to another maximum)
    assert (outs[0].float() - outs[1].float()).abs().max() <= 4e-3
    del k, v, kk, vv
    B, H, Hk, Lq, far = sizes.FAR
    P, slots = 140000, -(-(Lq + far) // 64)
    codes = [torch.zeros(P, Hk, 64, D, dtype=torch.uint8, device="cuda") for _ in range(2)]
    scales = [torch.ones(P, Hk, device="cuda") for _ in range(2)]
    near = [torch.zeros(slots, Hk, 64, D, dtype=torch.uint8, device="cuda") for _ in range(2)]
    near_scales = [torch.ones(slots, Hk, device="cuda") for _ in range(2)]
    x, y = (op.randn(g, 1, Hk, Lq + far, D) for _ in range(2))
    far_t, near_t = i32([[P - 1 - 3 * s for s in range(slots)]]), i32([list(range(slots))])
    q = op.randn(g, 1, H, Lq, D)
    outs = []
    for c, s, t in ((codes, scales, far_t), (near, near_scales, near_t)):
        sd.cache_write(x, y, *c, *s, t, i32([0]))
        ws = torch.empty(max(16, sd.cache_forward_workspace(1, H, Hk, Lq, D, slots)), dtype=torch.uint8, device="cuda")
        outs.append(sd.cache_forward(q, *c, *s, t, i32([far]), torch.empty_like(q), 0.1, H, workspace=ws))
    torch.cuda.synchronize()
    assert torch.equal(*outs)


@pytest.mark.parametrize("D", [64, 128])
def test_another_stream_and_replays(D):
    """One workspace for both calls of a graph, as its calls come one after another: every replay as the eager call."""
    import torch
    B, H, Hk, L, _ = sizes.CAUSAL
    g = op.generator(6)
    q, k, v = (op.randn(g, B, h, L, D) for h in (H, Hk, Hk))
    n = sd.window_forward_workspace(B, H, Hk, L, L, D)
    assert n > 0
    slots = -(-L // 64)
    c = [torch.zeros(B * slots, Hk, 64, D, dtype=torch.uint8, device="cuda") for _ in range(2)]
    c += [torch.ones(B * slots, Hk, device="cuda") for _ in range(2)]
    table = torch.randperm(B * slots, device="cuda", generator=g).to(torch.int32).view(B, slots)
    zero = i32([0] * B)
    ws2 = torch.full((max(n, sd.cache_forward_workspace(B, H, Hk, L, D, slots)),), 0x7f, dtype=torch.uint8, device="cuda")
    out = [torch.empty_like(q) for _ in range(2)]

    def step(w):
        sd.window_forward(q, k, v, out[0], D ** -0.5, H, workspace=w)
        sd.cache_write(k, v, *c, table, zero)
        sd.cache_forward(q, *c, table, zero, out[1], D ** -0.5, H, workspace=w)

    step(ws2)
    torch.cuda.synchronize()
    want = [t.clone() for t in out]
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        side.wait_stream(torch.cuda.default_stream())
        for t in out:
            t.zero_()
        step(ws2)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(ws2)
    for i in range(3):
        q.copy_(op.randn(g, B, H, L, D))
        for t in out:
            t.fill_(i)
        ws2.fill_(0xff)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        step(ws2)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, got)) and not torch.equal(got[0], want[0])


@pytest.mark.parametrize("Lq", [1, 90])
def test_calls_on_a_stream_that_waits(Lq):
    """Of few rows: a stream given to a call, which waits for the inputs."""
    import torch
    B, H, Hk, Lk, D = 2, 4, 2, 3000, 64
    g = op.generator(8)
    q, k, v = op.randn(g, B, H, Lq, D), op.randn(g, B, Hk, Lk, D), op.randn(g, B, Hk, Lk, D)
    n = sd.window_forward_workspace(B, H, Hk, Lq, Lk, D, 1, 2000, 7)
    outs = [torch.zeros_like(q) for _ in range(2)]
    works = [torch.full((max(n, 16),), 0x7f, dtype=torch.uint8, device="cuda") for _ in range(2)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for o, w, s in zip(outs, works, (None, side)):
        sd.window_forward(q, k, v, o, 0.125, H, Hk, workspace=w, window=2000, sinks=7, stream=s)
    torch.cuda.synchronize()
    assert torch.equal(*outs) and outs[0].any()
