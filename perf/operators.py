"""Cases of four operators on the path from hidden states to attention.

  adapt   a projection with low-rank adapters of many requests beside it
  rotate  per-head norms of queries and keys with a position rotation over
          several axes
  select  means of 64-key blocks, and for every block of queries the key blocks
          with the largest scores, as a bit mask
  sparse  attention over the key blocks that a mask names

The sizes are those of the SD1.4 UNet (latent side 64, 320 to 1280 channels, head
widths 40, 80, 160, a 77-token text), of video latents of a few dozen frames, and
of single tokens against long key sequences.
"""
import math

import numpy as np
import torch

own = False

BLOCK = 64       # keys of a block
EPS = 1e-6
TEXT = 77
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}


def listed():
    return [
        # sixteen requests of one token each, an adapter of its own for every one
        _adapt("adapt_tokens", 16, 1, 1280, 1280, 8, 16, "f16", none=False, heads=0),
        # the text's keys of eight prompts, rank 4, some prompts without an adapter
        _adapt("adapt_text", 8, TEXT, 768, 640, 4, 5, "bf16", none=True, heads=8),
        # eight 64x64 latents through a projection of the first level, three adapters
        _adapt("adapt_latents", 8, 4096, 320, 320, 16, 3, "f16", none=True, heads=0),
        # one new token for each of sixteen sequences, far along them
        _rotate("rotate_tokens", 16, 8, 1, 160, (80,), 1 << 20, "bf16", halves=True, rows=False, norm=True),
        # a 64x64 latent's queries and keys, height and width, straight from the projection
        _rotate("rotate_latent", 2, 8, 4096, 40, (10, 10), 64, "f16", halves=False, rows=True, norm=True),
        # 13 frames of 30 x 45: time, height and width
        _rotate("rotate_video", 1, 16, 17550, 128, (16, 24, 24), 64, "bf16", halves=True, rows=False, norm=True),
        # one token against 32768 keys whose means are at hand
        _select("select_tokens", 8, 8, 1, 32768, 128, 32, 64, "bf16", cached=True),
        # a quarter of a 64x64 latent's blocks
        _select("select_latent", 2, 8, 4096, 4096, 40, 16, 64, "f16", cached=False),
        # the video's, a query block of 128 each
        _select("select_video", 1, 16, 17550, 17550, 128, 40, 128, "bf16", cached=False),
        # one token over 32 of 512 blocks
        _sparse("sparse_tokens", 8, 8, 1, 32768, 128, 32, 64, "bf16", holes=False),
        # the latent's, some blocks of queries with nothing to read
        _sparse("sparse_latent", 2, 8, 4096, 4096, 40, 16, 64, "f16", holes=True),
        # the video's: a seventh of all pairs
        _sparse("sparse_video", 1, 16, 17550, 17550, 128, 40, 128, "bf16", holes=False),
    ]


def _named(name, case):
    return dict(case, name=name) if name else case


def _adapt(name, B, L, K, N, R, A, dtype, none, heads):
    return _named(name, dict(kind="adapt", B=B, L=L, K=K, N=N, R=R, A=A, dtype=dtype, none=none, heads=heads))


def _rotate(name, B, H, L, D, pairs, far, dtype, halves, rows, norm):
    pairs = tuple(pairs) + (0, 0, 0)
    return _named(name, dict(kind="rotate", B=B, H=H, L=L, D=D, p0=pairs[0], p1=pairs[1], p2=pairs[2], far=far,
                             dtype=dtype, halves=halves, rows=rows, norm=norm))


def _select(name, B, H, Lq, Lk, D, keep, qblock, dtype, cached):
    return _named(name, dict(kind="select", B=B, H=H, Lq=Lq, Lk=Lk, D=D, keep=keep, qblock=qblock, dtype=dtype,
                             cached=cached))


def _sparse(name, B, H, Lq, Lk, D, keep, qblock, dtype, holes):
    return _named(name, dict(kind="sparse", B=B, H=H, Lq=Lq, Lk=Lk, D=D, keep=keep, qblock=qblock, dtype=dtype,
                             holes=holes))


def draw(rng):
    """One more case: other requests, lengths, widths, ranks and shares of blocks."""
    while True:
        case = _draw(rng)
        w = work(case)
        most = [work(c) for c in listed() if c["kind"] == case["kind"]]
        if w["flops"] <= max(m["flops"] for m in most) and w["bytes"] <= max(m["bytes"] for m in most):
            return case


def _log(rng, lo, hi):
    """A whole number spread over the logarithm of [lo, hi]."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw(rng):
    kind = rng.choice(["adapt", "rotate", "select", "sparse"])
    dtype = rng.choice(["f16", "bf16"])
    if kind == "adapt":
        B = _log(rng, 1, 64)
        K, N = (rng.choice([320, 640, 768, 1280]) for _ in range(2))
        return _adapt(None, B, rng.choice([1, TEXT, _log(rng, 2, 4096)]), K, N, rng.choice([4, 8, 16, 20, 32, 64, 128]),
                      _log(rng, 1, 32), dtype, none=rng.random() < 0.5, heads=rng.choice([0, 0, 8]))
    D = rng.choice([40, 64, 80, 128, 160])
    H = rng.choice([1, 5, 8, 8, 16])
    if kind == "rotate":
        n = rng.choice([1, 2, 3])
        p = D // 2 if rng.random() < 0.7 else D // 4   # a part of each head is left as it is
        pairs = tuple(p // n + (i < p % n) for i in range(n))
        return _rotate(None, rng.choice([1, 2, 16]), H, rng.choice([1, _log(rng, 2, 17550), _log(rng, 64, 17550)]), D,
                       pairs, rng.choice([64, 4096, 1 << 20]), dtype, halves=rng.random() < 0.5,
                       rows=rng.random() < 0.5, norm=rng.random() < 0.8)
    B = rng.choice([1, 2, 8])
    Lk = _log(rng, 64, 32768)
    Lq = rng.choice([1, Lk, Lk])
    nb = (Lk + BLOCK - 1) // BLOCK
    keep = rng.randint(1, max(1, min(nb, 64)))
    qblock = rng.choice([64, 128])
    if kind == "select":
        return _select(None, B, H, Lq, Lk, D, keep, qblock, dtype, cached=rng.random() < 0.3)
    return _sparse(None, B, H, Lq, Lk, D, keep, qblock, dtype, holes=rng.random() < 0.3)


# ---------------------------------------------------------------- inputs

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _ids(case, seed):
    """The adapter of each request; every third has none where the case says so."""
    B, A = case["B"], case["A"]
    ids = np.arange(B) % A
    if case["none"]:
        ids[::3] = -1
    return np.random.default_rng(seed).permutation(ids).astype(np.int32)


def _keep_of(case):
    """How many blocks each block of queries reads."""
    nq, nb = -(-case["Lq"] // case["qblock"]), -(-case["Lk"] // BLOCK)
    rows = np.full(nq, min(case["keep"], nb))
    if case["holes"]:
        rows[5::16] = 0
    return rows


def _frequencies(case, dtype=torch.float32):
    """10000^(-i / n) for pair i of the n pairs of each axis."""
    parts = [10000.0 ** (-np.arange(n) / n) for n in (case["p0"], case["p1"], case["p2"]) if n]
    return torch.from_numpy(np.concatenate(parts)).to(dtype)


def _tokens(g, B, H, L, D, dt):
    """Queries or keys of an image: neighbours are alike, blocks differ."""
    near = torch.randn(B, H, -(-L // 16), D, device="cuda", generator=g).repeat_interleave(16, dim=2)[:, :, :L]
    return (0.7 * near + 0.7 * torch.randn(B, H, L, D, device="cuda", generator=g)).to(dt)


def _pack(sel):
    """Booleans [..., NB] as the bits of 64-bit words [..., ceil(NB / 64)]."""
    n = sel.shape[-1]
    sel = torch.nn.functional.pad(sel, (0, -n % 64)).unflatten(-1, (-1, 64)).to(torch.int64)
    return (sel << torch.arange(64, device=sel.device)).sum(-1)


def prepare(case, seed):
    g, dt, kind, B = _generator(seed), TYPES[case["dtype"]], case["kind"], case["B"]

    def randn(*shape, sigma=1.0):
        return (torch.randn(*shape, device="cuda", generator=g) * sigma).to(dt)

    st = dict(case=case)
    if kind == "adapt":
        L, K, N, R, A = (case[n] for n in ("L", "K", "N", "R", "A"))
        st.update(x=randn(B, L, K), w=randn(N, K, sigma=K ** -0.5), bias=randn(N, sigma=0.1),
                  down=randn(A, R, K, sigma=K ** -0.5), up=randn(A, N, R, sigma=R ** -0.5),
                  ids=torch.from_numpy(_ids(case, seed)).cuda(),
                  scales=0.25 + torch.rand(A, device="cuda", generator=g))
        st["y"] = torch.empty((B, case["heads"], L, N // case["heads"]) if case["heads"] else (B, L, N), dtype=dt,
                              device="cuda")
    elif kind == "rotate":
        H, L, D = case["H"], case["L"], case["D"]
        shape = (B, L, H * D) if case["rows"] else (B, H, L, D)
        st.update(q=randn(*shape, sigma=3.0), k=randn(*shape, sigma=2.0),
                  gq=(1 + randn(D, sigma=0.2).float()).to(dt), gk=(1 + randn(D, sigma=0.2).float()).to(dt),
                  freqs=_frequencies(case).cuda())
        axes = sum(case[n] > 0 for n in ("p0", "p1", "p2"))
        st["pos"] = torch.randint(0, case["far"], (B, L, axes), device="cuda", generator=g, dtype=torch.int32)
        st.update(qo=torch.empty(B, H, L, D, dtype=dt, device="cuda"), ko=torch.empty(B, H, L, D, dtype=dt, device="cuda"))
    else:
        H, Lq, Lk, D = (case[n] for n in ("H", "Lq", "Lk", "D"))
        nq, nb = -(-Lq // case["qblock"]), -(-Lk // BLOCK)
        st.update(q=_tokens(g, B, H, Lq, D, dt), k=_tokens(g, B, H, Lk, D, dt))
        if kind == "select":
            st.update(means=torch.empty(B, H, nb, D, device="cuda"),
                      mask=torch.empty(B, H, nq, -(-nb // 64), dtype=torch.int64, device="cuda"))
            if case["cached"]:
                st["means"] = torch.randn(B, H, nb, D, device="cuda", generator=g)
        else:
            order = torch.rand(B, H, nq, nb, device="cuda", generator=g).argsort(-1).argsort(-1)
            st.update(v=randn(B, H, Lk, D), out=torch.empty_like(st["q"]),
                      mask=_pack(order < torch.from_numpy(_keep_of(case)).cuda()[:, None]))
    return st


def run(st):
    return globals()[("_own_" if own else "_plain_") + st["case"]["kind"]](st, st["case"])


# ---------------------------------------------------------------- the framework's calls

def _own_adapt(st, case):
    import paper_2304_11267_amd as sd
    if "workspace" not in st:   # kept with the weights, as a server does
        n = sd.linear_adapters_workspace(case["B"], case["L"], case["R"])
        st["workspace"] = torch.empty(n, dtype=torch.uint8, device="cuda")
    return sd.linear_adapters(st["x"], st["w"], st["y"], st["down"], st["up"], st["ids"], st["workspace"],
                              scales=st["scales"], bias=st["bias"], heads=case["heads"] or 1,
                              y_layout=sd.LAYOUT_HEADS if case["heads"] else sd.LAYOUT_ROWS)


def _own_rotate(st, case):
    import paper_2304_11267_amd as sd
    return sd.norm_rotate(st["q"], st["qo"], case["H"], k=st["k"], ko=st["ko"], gamma_q=st["gq"], gamma_k=st["gk"],
                          pos=st["pos"], freqs=st["freqs"],
                          pairs=tuple(case[n] for n in ("p0", "p1", "p2") if case[n]),
                          norm=sd.NORM_RMS if case["norm"] else sd.NORM_NONE, eps=EPS,
                          pairing=sd.PAIR_HALVES if case["halves"] else sd.PAIR_ADJACENT,
                          x_layout=sd.LAYOUT_ROWS if case["rows"] else sd.LAYOUT_HEADS, y_layout=sd.LAYOUT_HEADS)


def _own_select(st, case):
    import paper_2304_11267_amd as sd
    if not case["cached"]:
        sd.block_means(st["k"], st["means"])
    mask = sd.select_blocks(st["q"], st["means"], st["mask"], case["keep"], qblock=case["qblock"])
    return mask if case["cached"] else (st["means"], mask)


def _own_sparse(st, case):
    import paper_2304_11267_amd as sd
    return sd.sparse_forward(st["q"], st["k"], st["v"], st["mask"], st["out"], _scale(case["D"]), qblock=case["qblock"])


def _scale(D):
    return float(np.float32(1.0 / math.sqrt(D)))


# ---------------------------------------------------------------- plain forms

def _plain_adapt(st, case):
    x, ids = st["x"].float(), st["ids"].long()
    at = ids.clamp(min=0)
    s = torch.where(ids >= 0, st["scales"][at], torch.zeros_like(st["scales"][at]))
    t = torch.bmm(x, st["down"].float()[at].transpose(1, 2).contiguous()) * s[:, None, None]
    y = torch.matmul(x, st["w"].float().t()) + st["bias"].float()
    y = (y + torch.bmm(t, st["up"].float()[at].transpose(1, 2).contiguous())).to(st["x"].dtype)
    return y.unflatten(2, (case["heads"], -1)).transpose(1, 2).contiguous() if case["heads"] else y


def _plain_rotate(st, case):
    return _plain_rotated(st["q"], st["gq"], st, case), _plain_rotated(st["k"], st["gk"], st, case)


def _plain_rotated(x, gamma, st, case):
    p = case["p0"] + case["p1"] + case["p2"]
    axis = [a for a, n in enumerate(case[n] for n in ("p0", "p1", "p2")) for _ in range(n)]
    # far positions lose the angle in 32 bits
    angle = st["pos"][:, :, axis].double() * st["freqs"].double()
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    y = x.float().unflatten(2, (case["H"], -1)).transpose(1, 2) if case["rows"] else x.float()
    if case["norm"]:
        y = y / (y.square().mean(-1, keepdim=True) + EPS).sqrt() * gamma.float()
    r, rest = y[..., :2 * p], y[..., 2 * p:]
    if case["halves"]:
        a, b = r[..., :p], r[..., p:]
        r = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    else:
        a, b = r[..., 0::2], r[..., 1::2]
        r = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    return torch.cat([r, rest], -1).to(x.dtype)


def _plain_means(x, block):
    """Means of `block` rows at a time, the last of fewer; 64 bits, rounded to 32."""
    n = x.shape[2]
    rows = torch.nn.functional.pad(x.double(), (0, 0, 0, -n % block)).unflatten(2, (-1, block)).sum(3)
    count = torch.full((rows.shape[2], 1), float(block), dtype=torch.float64, device=x.device)
    count[-1] = n - block * (rows.shape[2] - 1)
    return (rows / count).float()


def _plain_select(st, case):
    means = st["means"] if case["cached"] else _plain_means(st["k"], BLOCK)
    # two scores next to each other decide which block is read: 64 bits
    scores = torch.matmul(_plain_means(st["q"], case["qblock"]).double(), means.double().transpose(2, 3).contiguous())
    best = scores.sort(dim=-1, descending=True, stable=True)[1][..., :case["keep"]]
    mask = _pack(torch.zeros_like(scores, dtype=torch.bool).scatter(-1, best, True))
    return mask if case["cached"] else (means, mask)


def _plain_sparse(st, case):
    q, D, Lk = st["q"], case["D"], case["Lk"]
    B, H, Lq, _ = q.shape
    nq, nb = -(-Lq // case["qblock"]), -(-Lk // BLOCK)
    bits = (st["mask"][..., None] >> torch.arange(64, device=q.device) & 1).flatten(-2)[..., :nb].bool()
    most = min(case["keep"], nb)
    at = torch.arange(nb, device=q.device).where(bits, torch.tensor(nb, device=q.device)).sort(-1)[0][..., :most]
    # each block of queries beside the keys that it reads, in blocks past the last one nothing
    rows = torch.nn.functional.pad(q.float(), (0, 0, 0, -Lq % case["qblock"])).view(B, H, nq, -1, D)
    at, pad = at.reshape(B, H, -1), (0, 0, 0, (nb + 1) * BLOCK - Lk)
    keys = (at[..., None] * BLOCK + torch.arange(BLOCK, device=q.device)).view(B, H, -1, 1)
    k, v = (torch.nn.functional.pad(t.float(), pad).gather(2, keys.expand(-1, -1, -1, D)).view(B, H, nq, -1, D)
            for t in (st["k"], st["v"]))
    a = torch.matmul(rows, k.transpose(3, 4).contiguous()) * _scale(D)
    a.masked_fill_(keys.view(B, H, nq, 1, -1) >= Lk, -math.inf)
    top = a.amax(-1, keepdim=True)
    a = a.sub_(top.masked_fill(top == -math.inf, 0.0)).exp_()
    o = torch.matmul(a, v) / a.sum(-1, keepdim=True).clamp(min=1e-30)
    return o.view(B, H, -1, D)[:, :, :Lq].contiguous().to(q.dtype)


# ---------------------------------------------------------------- work

def work(case):
    """Inputs read once and outputs written once; multiply-adds of the definition."""
    kind, B = case["kind"], case["B"]
    if kind == "adapt":
        L, K, N, R = (case[n] for n in ("L", "K", "N", "R"))
        ids = _ids(case, 0)
        ids = ids[ids >= 0]
        used, rows = len(set(ids.tolist())), L * len(ids)
        return dict(bytes=2 * (B * L * (K + N) + N * K + N + used * R * (K + N)) + 4 * (B + case["A"]),
                    flops=2 * B * L * K * N + 2 * rows * R * (K + N))
    H, D = case["H"], case["D"]
    if kind == "rotate":
        n = B * H * case["L"] * D
        axes = sum(case[p] > 0 for p in ("p0", "p1", "p2"))
        # the norm's sum, root and scaling, and the rotation: about ten a value
        return dict(bytes=2 * 2 * 2 * n + 4 * B * case["L"] * axes, flops=20 * n)
    Lq, Lk = case["Lq"], case["Lk"]
    nq, nb = -(-Lq // case["qblock"]), -(-Lk // BLOCK)
    if kind == "select":
        keys = 0 if case["cached"] else Lk
        return dict(bytes=B * H * (2 * D * (Lq + keys) + 4 * nb * D + 8 * nq * -(-nb // 64)),
                    flops=B * H * D * (Lq + keys + 2 * nq * nb))
    rows = _keep_of(case)
    size = np.full(nq, case["qblock"])
    size[-1] = Lq - case["qblock"] * (nq - 1)
    pairs = int((rows * size).sum()) * min(BLOCK, Lk)
    keys = min(Lk, int(rows.sum()) * BLOCK)
    return dict(bytes=B * H * (4 * D * (Lq + keys) + 8 * nq * -(-nb // 64)), flops=4 * B * H * D * pairs)


# ---------------------------------------------------------------- 64 bits, by the definitions

def exact(case, seed):
    st = prepare(case, seed)
    return globals()["_exact_" + case["kind"]](st, case)


def _exact_adapt(st, case):
    w, bias, N = st["w"].double(), st["bias"].double(), case["N"]
    y = torch.empty(case["B"], case["L"], N, dtype=torch.float64, device="cuda")
    for b, i in enumerate(st["ids"].tolist()):
        x = st["x"][b].double()
        y[b] = x @ w.t().contiguous() + bias
        if i >= 0:
            y[b] += float(st["scales"][i]) * (x @ (st["up"][i].double() @ st["down"][i].double()).t().contiguous())
    return y.view(case["B"], case["L"], case["heads"], -1).permute(0, 2, 1, 3).contiguous() if case["heads"] else y


def _exact_rotate(st, case):
    H, D, B, L = case["H"], case["D"], case["B"], case["L"]
    counts = [case[n] for n in ("p0", "p1", "p2") if case[n]]
    p, out = sum(counts), []
    for x, gamma in ((st["q"], st["gq"]), (st["k"], st["gk"])):
        x = x.double()
        if case["rows"]:
            x = x.view(B, L, H, D).permute(0, 2, 1, 3)
        y = x.contiguous().clone()
        if case["norm"]:
            y *= (y.pow(2).sum(-1, keepdim=True) / D + EPS).rsqrt() * gamma.double()
        z, i = y.clone(), 0
        for axis, n in enumerate(counts):
            for _ in range(n):
                t = (st["pos"][:, :, axis].double() * float(st["freqs"][i]))[:, None]
                a, b = (i, i + p) if case["halves"] else (2 * i, 2 * i + 1)
                z[..., a] = y[..., a] * t.cos() - y[..., b] * t.sin()
                z[..., b] = y[..., b] * t.cos() + y[..., a] * t.sin()
                i += 1
        out.append(z)
    return tuple(out)


def _exact_select(st, case):
    if case["cached"]:
        return None
    parts = [t.double().mean(2) for t in st["k"].split(BLOCK, dim=2)]
    return torch.stack(parts, 2), None


def _exact_sparse(st, case):
    B, H, Lq, Lk, D = (case[n] for n in ("B", "H", "Lq", "Lk", "D"))
    out = torch.zeros(B, H, Lq, D, dtype=torch.float64, device="cuda")
    word = torch.arange(-(-Lk // BLOCK), device="cuda")
    for b in range(B):
        for h in range(H):
            on = (st["mask"][b, h][:, word // 64] >> (word % 64)) & 1
            for i in range(0, on.shape[0], 64):   # 64 blocks of queries at a time
                sel = on[i:i + 64].repeat_interleave(BLOCK, 1)[:, :Lk].bool()
                sel = sel.repeat_interleave(case["qblock"], 0)
                r = slice(i * case["qblock"], min(Lq, (i + 64) * case["qblock"]))
                sel = sel[:r.stop - r.start]
                a = (st["q"][b, h, r].double() @ st["k"][b, h].double().t().contiguous()) * _scale(D)
                a[~sel] = -math.inf
                p = (a - a.amax(1, keepdim=True)).exp().nan_to_num(0.0)
                out[b, h, r] = (p @ st["v"][b, h].double()) / p.sum(1, keepdim=True).clamp(min=1e-300)
    return out
