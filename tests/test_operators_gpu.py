"""The adapters, the norms with rotation, the block selection and the attention over the
selected blocks as they are used together, on other streams, captured into graphs, and
through ctypes beside the native marshalling."""
import numpy as np
import pytest

import operators_ref as ref
import paper_2304_11267_amd as sd
from paper_2304_11267_amd import binding
from parity_util import assert_close

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _needs_gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    sd.load_library()


class Block:
    """An attention block of a latent: projections with adapters, norms and rotation, the
    choice of key blocks, attention over them, and the output projection with adapters."""

    def __init__(self, B, H, side, D, R, keep, dtype, seed, qblock=64):
        import torch
        g = ref.generator(seed)
        self.B, self.H, self.L, self.D, self.keep, self.qblock, self.dtype = B, H, side * (side + 1), D, keep, qblock, dtype
        C = H * D

        def rnd(*shape, sigma=1.0):
            return ref.randn(g, *shape, dtype=dtype, sigma=sigma)

        def empty(*shape, dt=None):
            return torch.empty(*shape, dtype=dt or ref.t_type(dtype), device="cuda")

        self.x = rnd(B, self.L, C)
        self.w = [rnd(C, C, sigma=C ** -0.5) for _ in range(4)]
        self.down = [rnd(3, R, C, sigma=C ** -0.5) for _ in range(4)]
        self.up = [rnd(3, C, R, sigma=0.5 * R ** -0.5) for _ in range(4)]
        self.bias = rnd(C, sigma=0.1)
        self.scales = 0.5 + torch.rand(3, device="cuda", generator=g)
        self.ids = (torch.arange(B, dtype=torch.int32) % 4 - 1).cuda()
        self.gq, self.gk = (1 + rnd(D, sigma=0.2).float()).to(ref.t_type(dtype)), (1 + rnd(D, sigma=0.2).float()).to(ref.t_type(dtype))
        l = torch.arange(self.L)
        self.pos = torch.stack([l // (side + 1), l % (side + 1)], 1)[None].int().cuda()   # height and width
        self.pairs = (D // 4, D // 2 - D // 4)
        self.freqs = (100.0 ** (-torch.arange(D // 2, dtype=torch.float64) / (D // 2))).float().cuda()
        nb = -(-self.L // 64)
        self.qkv = [empty(B, H, self.L, D) for _ in range(3)]
        self.raw = [empty(B, H, self.L, D) for _ in range(2)]
        self.means = empty(B, H, nb, D, dt=torch.float32)
        self.mask = empty(B, H, -(-self.L // qblock), -(-nb // 64), dt=torch.int64)
        self.o, self.out = empty(B, H, self.L, D), empty(B, self.L, C)
        self.ws = empty(sd.linear_adapters_workspace(B, self.L, R), dt=torch.uint8)
        self.scale = float(np.float32(D ** -0.5))

    def adapters(self, i, x, y, stream, bias=None, **kw):
        sd.linear_adapters(x, self.w[i], y, self.down[i], self.up[i], self.ids, self.ws, scales=self.scales, bias=bias,
                           heads=self.H, stream=stream, **kw)

    def run(self, stream=None):
        q, k, v = self.qkv
        for i, y in enumerate((self.raw[0], self.raw[1], v)):
            self.adapters(i, self.x, y, stream, y_layout=sd.LAYOUT_HEADS)
        sd.norm_rotate(self.raw[0], q, self.H, k=self.raw[1], ko=k, gamma_q=self.gq, gamma_k=self.gk, pos=self.pos,
                       freqs=self.freqs, pairs=self.pairs, pairing=sd.PAIR_HALVES, stream=stream)
        sd.block_means(k, self.means, stream=stream)
        sd.select_blocks(q, self.means, self.mask, self.keep, qblock=self.qblock, stream=stream)
        sd.sparse_forward(q, k, v, self.mask, self.o, self.scale, qblock=self.qblock, stream=stream)
        self.adapters(3, self.o, self.out, stream, bias=self.bias, x_layout=sd.LAYOUT_HEADS)
        return [self.raw[0], self.raw[1], q, k, v, self.means, self.mask, self.o, self.out]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("B,H,side,D,R,keep,qblock", [(4, 4, 16, 40, 4, 2, 64), (2, 3, 25, 64, 16, 5, 128)],
                         ids=lambda v: str(v))
def test_a_block_of_them(B, H, side, D, R, keep, qblock, dtype):
    """Every step against the 64-bit form of the step, on what the step before left."""
    import torch
    b = Block(B, H, side, D, R, keep, dtype, 40 + side, qblock)
    raw_q, raw_k, q, k, v, means, mask, o, out = (t.cpu().numpy() if t.dtype == torch.int64 else ref.host(t) for t in b.run())
    ids, scales = b.ids.cpu().numpy(), ref.host(b.scales)

    def near(g, r, off):
        bound = off + ref.half_step(g, r, dtype) * (1 + 2.0 ** -10)
        assert np.all(np.abs(g - r) <= bound), float(np.max(np.abs(g - r) / bound))

    for i, (x, y, bias) in enumerate(((b.x, raw_q, None), (b.x, raw_k, None), (b.x, v, None), (b.o, out, b.bias))):
        x = ref.host(x)
        r, off = ref.adapters(ref.heads_to_rows(x) if x.ndim == 4 else x, ref.host(b.w[i]),
                              None if bias is None else ref.host(bias), ref.host(b.down[i]), ref.host(b.up[i]), ids, scales, dtype)
        near(ref.heads_to_rows(y) if y.ndim == 4 else y, r, off)
    pos, freqs = b.pos.cpu().numpy().astype(float), ref.host(b.freqs)
    for x, gamma, y in ((raw_q, b.gq, q), (raw_k, b.gk, k)):
        near(y, *ref.norm_rotate(x, ref.host(gamma), pos, freqs, b.pairs, True, 1e-6, True))
    r = ref.block_means(k, 64)
    assert np.all(np.abs(means - r) <= 2.0 ** -23 * np.abs(r) + 2.0 ** -46 * ref.block_means(np.abs(k), 64))
    sel = ref.select(ref.block_means(q, qblock).astype(np.float32).astype(np.float64), means, keep)
    assert np.array_equal(ref.unpack(mask, sel.shape[-1]), sel)
    r, dev = ref.sparse(q, k, v, sel, b.scale, qblock)
    assert_close(o, r, dtype=dtype, what="sparse in a block", dev=dev)


def test_captured_blocks_replay_beside_eager_work():
    """Two blocks with workspaces of their own captured into two graphs, replayed in turn with
    eager work between, each replay against the eager outputs bit for bit; then on new inputs."""
    import torch
    blocks = [Block(2, 4, 20, 40, 16, 3, "f16", 1), Block(3, 2, 9, 64, 4, 2, "bf16", 2, qblock=128)]
    want = [[t.clone() for t in b.run()] for b in blocks]
    torch.cuda.synchronize()
    graphs, side = [], torch.cuda.Stream()
    for b in blocks:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=side):
            b.run()
    for turn in range(3):
        for b, graph, w in zip(blocks, graphs, want):
            for t in b.run():
                t.zero_()
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(t, r) for t, r in zip([b.raw[0], b.raw[1], *b.qkv, b.means, b.mask, b.o, b.out], w)), turn
    b, graph = blocks[0], graphs[0]
    b.x.copy_(b.x.flip(1).contiguous())
    b.ids.copy_(b.ids.flip(0).contiguous())
    graph.replay()
    torch.cuda.synchronize()
    got = b.out.clone()
    assert not torch.equal(got, want[0][-1])
    b.run()
    torch.cuda.synchronize()
    assert torch.equal(b.out, got)


def test_streams():
    """On a stream of its own, given or current, and two blocks on two streams at once."""
    import torch
    blocks = [Block(2, 4, 20, 40, 16, 3, "f16", 1), Block(2, 2, 16, 64, 8, 3, "bf16", 2)]
    want = [[t.clone() for t in b.run()] for b in blocks]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in blocks]
    for how in ("given", "current"):
        for b, s in zip(blocks, streams):
            old, new = b.x.clone(), b.x.clone()
            b.x.zero_()
            torch.cuda.synchronize()
            with torch.cuda.stream(s):
                torch.cuda._sleep(10_000_000)   # some milliseconds
                b.x.copy_(new)                  # seen only by calls queued behind it
                if how == "current":
                    b.run()
            if how == "given":
                b.run(s)
        torch.cuda.synchronize()
        for b, w in zip(blocks, want):
            assert torch.equal(b.out, w[-1]) and torch.equal(b.mask, w[6]), how


def test_ctypes_gives_the_native_calls_bits(monkeypatch):
    import torch
    b = Block(2, 4, 12, 64, 16, 2, "f16", 5)
    fast = [t.clone() for t in b.run()]
    monkeypatch.setattr(binding, "_native", None)
    slow = b.run()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(fast, slow))


@pytest.mark.parametrize("native", [True, False], ids=["native", "ctypes"])
def test_refusals_leave_the_outputs(native, monkeypatch):
    import torch
    if not native:
        monkeypatch.setattr(binding, "_native", None)
    b = Block(2, 4, 12, 64, 16, 2, "f16", 5)
    b.out.fill_(7.0)
    with pytest.raises(sd.SdattnError) as e:
        b.ws = b.ws[:-256]
        b.adapters(3, b.o, b.out, None, x_layout=sd.LAYOUT_HEADS)
    assert e.value.status == sd.STATUS_INVALID_ARG
    with pytest.raises(ValueError, match="contiguous"):
        b.adapters(0, b.x.transpose(0, 1).contiguous().transpose(0, 1), b.out, None)
    q = torch.full((1, 1, 8, 24), 7.0, dtype=torch.float16, device="cuda")
    o = q.clone()
    with pytest.raises(sd.SdattnError) as e:
        sd.sparse_forward(q, q, q, torch.zeros(1, 1, 1, 1, dtype=torch.int64, device="cuda"), o, 0.1)
    assert e.value.status == sd.STATUS_UNSUPPORTED
    with pytest.raises(sd.SdattnError) as e:
        sd.norm_rotate(q, o, 1, pos=torch.zeros(1, 8, 1, dtype=torch.int32, device="cuda"),
                       freqs=torch.zeros(13, device="cuda"), pairs=(13,))
    assert e.value.status == sd.STATUS_INVALID_ARG
    torch.cuda.synchronize()
    assert (b.out == 7).all() and (o == 7).all()


@pytest.mark.parametrize("halves", [0, 1])
@pytest.mark.parametrize("D", [40, 128, 256])
def test_small_arguments_at_their_smallest_alignment(D, halves):
    """Gammas and biases on 8 bytes, positions, frequencies, adapter numbers and scales on 4:
    the bits of the aligned call."""
    import torch
    g = ref.generator(31)

    def moved(t, bytes_):
        room = torch.empty(t.numel() * t.element_size() + 16, dtype=torch.uint8, device="cuda")
        at = room[bytes_:bytes_ + t.numel() * t.element_size()].view(t.dtype).view(t.shape)
        at.copy_(t)
        assert at.data_ptr() % 16 == bytes_
        return at

    q = ref.randn(g, 2, 3, 50, D, dtype="bf16")
    gamma, pos = ref.randn(g, D, dtype="bf16"), torch.randint(0, 99, (2, 50, 1), generator=g, device="cuda", dtype=torch.int32)
    freqs = torch.rand(16, generator=g, device="cuda")
    a, b = torch.empty_like(q), torch.empty_like(q)
    sd.norm_rotate(q, a, 3, gamma_q=gamma, pos=pos, freqs=freqs, pairs=(16,), pairing=halves)
    sd.norm_rotate(q, b, 3, gamma_q=moved(gamma, 8), pos=moved(pos, 4), freqs=moved(freqs, 12), pairs=(16,), pairing=halves)
    torch.cuda.synchronize()
    assert torch.equal(a, b)
    for L, R in ((40, 16), (3, 24)):
        x, w = ref.randn(g, 2, L, D, dtype="bf16"), ref.randn(g, 64, D, dtype="bf16")
        down, up, bias = (ref.randn(g, *s, dtype="bf16") for s in ((3, R, D), (3, 64, R), (64,)))
        ids = torch.tensor([2, 0], dtype=torch.int32, device="cuda")
        scales = torch.tensor([0.5, 1.0, 2.0], device="cuda")
        ws = torch.empty(sd.linear_adapters_workspace(2, L, R), dtype=torch.uint8, device="cuda")
        y, z = (torch.empty(2, L, 64, dtype=x.dtype, device="cuda") for _ in range(2))
        sd.linear_adapters(x, w, y, down, up, ids, ws, scales=scales, bias=bias)
        sd.linear_adapters(x, w, z, down, up, moved(ids, 4), ws, scales=moved(scales, 12), bias=moved(bias, 8))
        torch.cuda.synchronize()
        assert torch.equal(y, z)
