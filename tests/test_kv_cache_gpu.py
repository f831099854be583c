"""sdattn_cache_write and sdattn_cache_read against their plain form, code by code: every width,
both layouts, tokens that begin and end inside a page, pages that grow, ragged counts, positions and pages that are not
there, values at the types' ends and no numbers, caches past 32 bits."""
import numpy as np
import pytest

import operators_ref as op
import paper_2304_11267_amd as sd
import stream_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _needs_gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    sd.load_library()


class Cache:
    """A cache on the GPU beside its plain form; `fill` is what nobody has written."""

    def __init__(self, B, Hk, D, slots, spare=2, seed=0, fill=0x7f):
        import torch
        P = B * slots + spare
        rng = np.random.default_rng(seed)
        self.table = rng.permutation(P)[:B * slots].reshape(B, slots).astype(np.int32)
        self.shape = (P, Hk, 64, D)
        self.codes = [np.full(self.shape, fill, np.uint8) for _ in range(2)]
        self.scales = [np.full((P, Hk), 3.0) for _ in range(2)]
        self.dev_codes = [torch.from_numpy(c.copy()).cuda() for c in self.codes]
        self.dev_scales = [torch.from_numpy(s.astype(np.float32)).cuda() for s in self.scales]

    def dev(self):
        import torch
        return (*self.dev_codes, *self.dev_scales, torch.from_numpy(self.table).cuda())

    def write(self, k, v, starts, counts, dtype, layout=sd.LAYOUT_HEADS, none=False, stream=None):
        import torch
        i32 = dict(dtype=torch.int32, device="cuda")
        a, b = k, v
        if layout == sd.LAYOUT_ROWS:
            a, b = (t.transpose(1, 2).flatten(2).contiguous() for t in (k, v))
        sd.cache_write(a, b, *self.dev(), torch.tensor(starts, **i32), counts=None if none else torch.tensor(counts, **i32),
                       layout=layout, stream=stream)
        torch.cuda.synchronize()
        for x, c, s in ((k, self.codes[0], self.scales[0]), (v, self.codes[1], self.scales[1])):
            ref.write(op.host(x), c, s, self.table, starts, counts, dtype)
        self.check()

    def check(self):
        for i in range(2):
            assert ref.same_codes(self.dev_codes[i].cpu().numpy(), self.codes[i])
            assert np.array_equal(self.dev_scales[i].cpu().numpy().astype(np.float64), self.scales[i])

    def read(self, starts, counts, L, dtype, layout=sd.LAYOUT_HEADS, none=False):
        import torch
        B, Hk, D = len(starts), self.shape[1], self.shape[3]
        shape = (B, Hk, L, D) if layout == sd.LAYOUT_HEADS else (B, L, Hk * D)
        out = [torch.full(shape, 7.0, dtype=op.t_type(dtype), device="cuda") for _ in range(2)]
        i32 = dict(dtype=torch.int32, device="cuda")
        assert sd.cache_read(*out, *self.dev(), torch.tensor(starts, **i32), counts=None if none else torch.tensor(counts, **i32),
                             layout=layout) == tuple(out)
        torch.cuda.synchronize()
        for o, c, s in zip(out, self.codes, self.scales):
            want = ref.read(c, s, self.table, starts, counts, L)
            behind = (np.arange(L) >= np.minimum(np.array(counts), L)[:, None])[:, None, :, None]
            want = np.where(behind, 7.0, want)
            want = torch.from_numpy(want).to(op.t_type(dtype))   # (codes times a power of two: one rounding, of fp16's subnormals)
            if layout == sd.LAYOUT_ROWS:
                o = o.unflatten(2, (Hk, D)).transpose(1, 2)
            assert torch.equal(torch.nan_to_num(o.cpu(), nan=-1.0), torch.nan_to_num(want, nan=-1.0))
        return out


def tokens(B, Hk, L, D, dtype, seed, sigma=1.0):
    g = op.generator(seed)
    return tuple(op.randn(g, B, Hk, L, D, dtype=dtype, sigma=s) for s in (sigma, 0.3 * sigma))


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("layout", [sd.LAYOUT_ROWS, sd.LAYOUT_HEADS])
@pytest.mark.parametrize("D", [8, 24, 32, 40, 64, 72, 80, 128, 136, 160, 200, 256])
def test_widths(D, layout, dtype):
    c = Cache(2, 3, D, 4, seed=D)
    c.write(*tokens(2, 3, 150, D, dtype, D), [0, 37], [150, 150], dtype, layout, none=True)
    c.write(*tokens(2, 3, 1, D, dtype, D + 1, 4.0), [150, 187], [1, 1], dtype, layout)
    c.read([0, 3], [151, 100], 151, dtype, layout)


@pytest.mark.parametrize("start", [0, 1, 62, 63, 64, 65, 100])
@pytest.mark.parametrize("L", [1, 2, 63, 64, 65, 66, 128, 129])
def test_places_in_a_page(start, L):
    c = Cache(1, 2, 40, 5, seed=L)
    if start:
        c.write(*tokens(1, 2, start, 40, "f16", start, 0.1), [0], [start], "f16")
    c.write(*tokens(1, 2, L, 40, "f16", L), [start], [L], "f16", none=True)
    c.read([0], [start + L], start + L, "f16", none=True)


def test_token_by_token_over_two_pages():
    c = Cache(2, 2, 64, 3)
    k, v = tokens(2, 2, 130, 64, "bf16", 9)
    for i in range(130):   # sizes that grow and shrink
        f = 2.0 ** ((i * 7) % 11 - 5)
        c.write(k[:, :, i:i + 1].contiguous() * f, v[:, :, i:i + 1].contiguous() * f, [i, i], [1, 1], "bf16")
    c.read([0, 0], [130, 130], 130, "bf16")


def test_rewriting_the_last_tokens():
    """A chunk that is written again and again (a frame that is denoised): its pages' scales go by what is there now."""
    c = Cache(1, 2, 64, 6)
    c.write(*tokens(1, 2, 100, 64, "f16", 1), [0], [100], "f16")
    for s in (30.0, 0.01, 1.0):
        c.write(*tokens(1, 2, 200, 64, "f16", 2, s), [100], [200], "f16")
    c.read([0], [300], 300, "f16")


def test_ragged_counts_and_what_is_not_there():
    c = Cache(6, 2, 32, 3, seed=4)
    c.table[1, 1] = -1
    c.table[2, 0] = c.shape[0]
    c.table[2, 1] = 1 << 30
    starts, counts = [0, 10, 5, 150, -20, 190], [0, 100, 130, 70, 90, 500]
    k, v = tokens(6, 2, 130, 32, "f16", 5)
    c.write(k, v, starts, counts, "f16")
    c.write(k, v, [3] * 6, [-7, 1, 64, 65, 0, 130], "f16", sd.LAYOUT_ROWS)
    c.read([-5, 0, 0, 100, -200, 191], [60, 130, 130, 100, 100, -1], 130, "f16")
    c.read([0] * 6, [200] * 6, 130, "f16", sd.LAYOUT_ROWS, none=True)
    for far in (2 ** 31 - 1, -2 ** 31, 2 ** 31 - 130):
        c.write(k, v, [far] * 6, [130] * 6, "f16")
        c.read([far] * 6, [130] * 6, 130, "f16")


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_values_at_the_ends(dtype):
    import torch
    t = op.t_type(dtype)
    big, tiny = torch.finfo(t).max, torch.finfo(t).smallest_normal
    c = Cache(1, 1, 8, 12)
    rows = [[big, -big, 1.0, 0.0, -0.0, big / 2, 63488.0, 61440.0], [tiny, -tiny, tiny / 2, 0, 0, 0, 0, 0], [0.0] * 8,
            [448.0, 447.0, -448.0, 1, 2, 3, 4, 5], [449.0] * 8, [float("nan"), float("inf"), -float("inf"), 1, 2, 3, -4, 5],
            [float("nan")] * 8, [1e-3] * 8, [16.5, 17.5, 18.5, 19.5, 20.5, 21.5, 448.0, 240.0]]
    for i, r in enumerate(rows):
        x = torch.tensor(r, device="cuda").to(t).view(1, 1, 1, 8)
        c.write(x, -x, [64 * i], [1], dtype)
        c.write(x, x, [64 * i + 1], [1], dtype)
        k, _ = c.read([64 * i], [2], 2, dtype)
        if i != 5 and i != 6:
            assert torch.isfinite(k).all()
    c.write(torch.full((1, 1, 1, 8), float("nan"), device="cuda").to(t), x, [2], [1], dtype)   # joins a page of numbers
    assert torch.isfinite(c.read([0], [2], 2, dtype)[0]).all()


def test_float8_pages_and_python_path(monkeypatch):
    import torch
    from paper_2304_11267_amd import binding
    k, v = tokens(1, 2, 70, 40, "f16", 6)
    a, b = Cache(1, 2, 40, 2), Cache(1, 2, 40, 2)
    a.write(k, v, [0], [70], "f16")
    b.dev_codes = [t.view(torch.float8_e4m3fn) for t in b.dev_codes]
    monkeypatch.setattr(binding, "_native", None)
    starts = torch.zeros(1, dtype=torch.int32, device="cuda")
    sd.cache_write(k, v, *b.dev(), starts)
    torch.cuda.synchronize()
    assert all(torch.equal(p, q.view(torch.uint8)) for p, q in zip(a.dev_codes, b.dev_codes))
    o = sd.cache_read(torch.empty_like(k), torch.empty_like(v), *b.dev(), starts)
    monkeypatch.undo()
    o2 = sd.cache_read(torch.empty_like(k), torch.empty_like(v), *b.dev(), starts)
    assert all(torch.equal(p, q) for p, q in zip(o, o2))


def test_pages_past_32_bits():
    """Pages of 32 KB, the last of 140000 more than 2^32 bytes in."""
    import torch
    P, Hk, D = 140000, 4, 128
    codes = [torch.zeros(P, Hk, 64, D, dtype=torch.uint8, device="cuda") for _ in range(2)]
    scales = [torch.zeros(P, Hk, device="cuda") for _ in range(2)]
    table = torch.tensor([[P - 1, 3]], dtype=torch.int32, device="cuda")
    at = torch.tensor([10], dtype=torch.int32, device="cuda")
    k, v = tokens(1, Hk, 60, D, "f16", 3)
    sd.cache_write(k, v, *codes, *scales, table, at)
    back = sd.cache_read(torch.empty_like(k), torch.empty_like(v), *codes, *scales, table, at)
    torch.cuda.synchronize()
    for x, y, c in zip((k, v), back, codes):
        assert ((x - y).abs() <= 2.0 ** -4 * x.abs() + 2.0 ** -9).all()
        assert c[P - 1, :, 10:].any() and c[3, :, :6].any() and not c[4:P - 1].any() and not c[:3].any()


def test_replays():
    import torch
    c = Cache(2, 2, 64, 4)
    k, v = tokens(2, 2, 100, 64, "f16", 7)
    starts = torch.tensor([5, 60], dtype=torch.int32, device="cuda")
    args = c.dev()
    out = [torch.empty_like(k) for _ in range(2)]

    def step():
        sd.cache_write(k, v, *args, starts)
        sd.cache_read(*out, *args, starts)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(3):
        for t in out:
            t.fill_(3)
        for t in args[:2]:
            t.fill_(i)   # (the tokens before 5 and 60 as well: the same codes at each replay)
        args[2].fill_(0.25)
        args[3].fill_(0.25)
        graph.replay()
        torch.cuda.synchronize()
        fresh = [t.clone() for t in (*args, *out)]
        for t in args[:2]:
            t.fill_(i)
        args[2].fill_(0.25)
        args[3].fill_(0.25)
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(fresh, (*args, *out)))


@pytest.mark.parametrize("layout", ["heads", "rows"])
@pytest.mark.parametrize("D", [8, 40, 48, 64, 72, 80, 88, 160])
def test_many_pages_are_as_few(D, layout):
    """A call over many sequences gives what calls over some of them give, bit for bit, and back."""
    import torch
    B, Hk, L, slots = 64, 8, 70, 3
    P = B * slots
    g = op.generator(D)
    lay = sd.LAYOUT_ROWS if layout == "rows" else sd.LAYOUT_HEADS
    shape = (B, L, Hk * D) if layout == "rows" else (B, Hk, L, D)
    k, v = (op.randn(g, *shape, dtype="bf16", sigma=s) for s in (1.0, 9.0))
    table = torch.randperm(P, device="cuda", generator=g).to(torch.int32).view(B, slots)
    starts = (torch.arange(B, device="cuda") * 7 % 100).to(torch.int32)
    counts = (L - torch.arange(B, device="cuda") * 5 % 80).to(torch.int32)
    caches, backs = [], []
    for parts in (1, 16):
        c = [torch.full((P, Hk, 64, D), 0x30, dtype=torch.uint8, device="cuda") for _ in range(2)]
        c += [torch.full((P, Hk), 2.0 ** -4, device="cuda") for _ in range(2)]
        back = [torch.full(shape, 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        n = B // parts
        for i in range(0, B, n):
            s = slice(i, i + n)
            sd.cache_write(k[s], v[s], *c, table[s], starts[s], counts=counts[s], layout=lay)
        for i in range(0, B, n):
            s = slice(i, i + n)
            sd.cache_read(back[0][s], back[1][s], *c, table[s], starts[s], counts=counts[s], layout=lay)
        caches.append(c)
        backs.append(back)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(*caches)) and all(torch.equal(a, b) for a, b in zip(*backs))
    rows = backs[0][0].unflatten(2, (Hk, D)).transpose(1, 2) if layout == "rows" else backs[0][0]
    x = k.unflatten(2, (Hk, D)).transpose(1, 2) if layout == "rows" else k
    for b in (0, 1, 17, 63):
        n = max(int(counts[b]), 0)
        assert (rows[b, :, n:] == 7).all()
        top = float(x[b].abs().max())
        assert ((rows[b, :, :n].float() - x[b, :, :n].float()).abs() <= x[b, :, :n].float().abs() * 2.0 ** -4 + top * 2.0 ** -17 * 2).all()
