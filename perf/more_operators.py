"""Cases of a transformer block over a stream: tokens or video frames that come one after another.

  gated   norms before and after a block with its gate, its residual scale and its modulation
  cache   keys and values quantised to 8 bits as they are written into pages of 64 tokens
          (a scale for each page and head), and read back
  cached  attention of new tokens over that cache
  window  attention over 16-bit keys and values with a sliding window and first tokens that
          stay visible

A query at position p sees key j < hi with j >= hi - window or j < sinks, where hi is the end of p's
frame (the query itself, with frames of one token), or of all keys (frame 0); window 0 is no limit.

The sizes are those of the SD1.4 UNet (latent side 64, 320 to 1280 channels, head widths 40, 80,
160, a 77-token text), of video latents of a few dozen frames of 30 x 45, and of single tokens
against long key sequences.
"""
import math

import numpy as np
import torch

own = False

PAGE = 64        # tokens of a page
EPS = 1e-6
TEXT = 77
SKIP = 0.75      # the residual's scale
MOST = 448.0     # the largest e4m3 value
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
# the largest value of each type that e4m3 holds without rounding past the type
HELD = {"f16": 1.875 * 2.0 ** 15, "bf16": 1.875 * 2.0 ** 127}


def listed():
    return [
        # one token of each of sixteen requests between two blocks of 1280 channels
        _gated("gated_tokens", 16, 1, 1280, 1, "f16", f32=False, post="none", pre="layer", affine=False),
        # two 64x64 latents at the first level
        _gated("gated_latent", 2, 4096, 320, 1, "bf16", f32=False, post="none", pre="layer", affine=True),
        # 13 frames of 30 x 45, each with a modulation of its own, a 32-bit residual stream, norms on both sides
        _gated("gated_video", 1, 17550, 2048, 13, "bf16", f32=True, post="rms", pre="rms", affine=True),
        # a new token for each of 64 sequences, somewhere in a page
        _cache("cache_tokens", "write", 64, 8, 1, 128, 1000, "bf16", ragged=False, rows=True),
        # the whole video behind a text
        _cache("cache_video", "write", 1, 16, 17550, 128, TEXT, "bf16", ragged=False, rows=False),
        # eight sequences of different lengths back in 16 bits
        _cache("cache_back", "read", 8, 8, 4096, 80, 0, "f16", ragged=True, rows=False),
        # one token of two prompts over a text of 77
        _cached("cached_text", 2, 8, 8, 1, 40, 76, 1, 0, 0, "f16", ragged=False, rows=False),
        # one token of eight sequences of up to 32768, four query heads to a key head
        _cached("cached_tokens", 8, 32, 8, 1, 128, 32767, 1, 0, 0, "bf16", ragged=True, rows=True),
        # the thirteenth frame over the four last ones and the first
        _cached("cached_frame", 1, 16, 16, 1350, 128, 16200, 1350, 5400, 1350, "bf16", ragged=False, rows=False),
        # one token of sixteen sequences, the last thousand and the first 64
        _window("window_tokens", 16, 16, 4, 1, 8192, 64, 1, 1024, 64, "bf16", ragged=True, rows=False),
        # the rows of a 64x64 latent one after another
        _window("window_latent", 2, 8, 8, 4096, 4096, 40, 64, 1024, TEXT, "f16", ragged=False, rows=True),
        # the video, each frame over the three before it and the first
        _window("window_video", 1, 16, 16, 17550, 17550, 128, 1350, 5400, 1350, "bf16", ragged=False, rows=False),
    ]


def _named(name, case):
    return dict(case, name=name) if name else case


def _gated(name, B, L, C, groups, dtype, f32, post, pre, affine):
    return _named(name, dict(kind="gated", B=B, L=L, C=C, groups=groups, dtype=dtype, f32=f32, post=post, pre=pre,
                             affine=affine))


def _cache(name, way, B, Hk, L, D, far, dtype, ragged, rows):
    return _named(name, dict(kind="cache", way=way, B=B, Hk=Hk, L=L, D=D, far=far, dtype=dtype, ragged=ragged, rows=rows))


def _cached(name, B, H, Hk, Lq, D, far, frame, window, sinks, dtype, ragged, rows):
    return _named(name, dict(kind="cached", B=B, H=H, Hk=Hk, Lq=Lq, D=D, far=far, frame=frame, window=window, sinks=sinks,
                             dtype=dtype, ragged=ragged, rows=rows))


def _window(name, B, H, Hk, Lq, Lk, D, frame, window, sinks, dtype, ragged, rows):
    return _named(name, dict(kind="window", B=B, H=H, Hk=Hk, Lq=Lq, Lk=Lk, D=D, frame=frame, window=window, sinks=sinks,
                             dtype=dtype, ragged=ragged, rows=rows))


def draw(rng):
    """One more case: other widths, lengths, groups of heads, windows and places in a page."""
    while True:
        case = _draw(rng)
        w = work(case)
        most = [work(c) for c in listed() if c["kind"] == case["kind"]]
        scores = case["B"] * case["H"] * case["Lq"] * _keys(case) if case["kind"] in ("cached", "window") else 0
        if (w["flops"] <= max(m["flops"] for m in most) and w["bytes"] <= max(m["bytes"] for m in most) and
                scores <= 16 * 17550 ** 2):
            return case


def _log(rng, lo, hi):
    """A whole number spread over the logarithm of [lo, hi]."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw(rng):
    kind = rng.choice(["gated", "cache", "cached", "window"])
    dtype = rng.choice(["f16", "bf16"])
    if kind == "gated":
        groups = rng.choice([1, 1, 2, 13])
        L = groups * rng.choice([1, _log(rng, 1, 1350), _log(rng, 1, 1350)])
        return _gated(None, rng.choice([1, 2, 16, 64]), L, rng.choice([320, 640, 1280, 2048, 8 * _log(rng, 8, 512)]), groups,
                      dtype, rng.random() < 0.4, rng.choice(["none", "rms", "layer"]), rng.choice(["rms", "layer"]),
                      rng.random() < 0.5)
    D = rng.choice([40, 64, 80, 128, 160])
    Hk = rng.choice([1, 2, 5, 8, 16])
    B = rng.choice([1, 2, 8, 16, 64])
    ragged, rows = rng.random() < 0.5, rng.random() < 0.5
    if kind == "cache":
        return _cache(None, rng.choice(["write", "write", "read"]), B, Hk, rng.choice([1, _log(rng, 2, 17550), _log(rng, 2, 17550)]),
                      D, _log(rng, 1, 4096), dtype, ragged, rows)
    H = Hk * rng.choice([1, 1, 2, 4, 7, 8])
    Lq = rng.choice([1, 1, _log(rng, 2, 64), _log(rng, 64, 4096)])
    frame = rng.choice([1, 1, 0, _log(rng, 2, 1350)])
    window = rng.choice([0, _log(rng, 16, 8192), _log(rng, 16, 8192)])
    sinks = rng.choice([0, 4, _log(rng, 1, 1350)])
    far = rng.choice([0, _log(rng, 1, 32767), _log(rng, 1, 32767)])
    if kind == "cached":
        return _cached(None, B, H, Hk, Lq, D, far, frame, window, sinks, dtype, ragged, rows)
    return _window(None, B, H, Hk, Lq, Lq + far, D, frame, window, sinks, dtype, ragged, rows)


# ---------------------------------------------------------------- lengths

def _spread(n, B, ragged, seed):
    """n for each of B sequences, or down to a third of it, in an order by the seed; at least 1."""
    v = np.full(B, n)
    if ragged:
        v = n - (np.arange(B) * 2 * n) // (3 * B)
    return np.random.default_rng(seed).permutation(np.maximum(v, 1)).astype(np.int32)


def _plan(case, seed):
    """Position of each sequence's first new token, and how many it has."""
    B, ragged, kind = case["B"], case["ragged"], case["kind"]
    if kind == "cache" and case["way"] == "read":
        return np.zeros(B, np.int32), _spread(case["L"], B, ragged, seed)
    L = case["L"] if kind == "cache" else case["Lq"]
    far = case["Lk"] - L if kind == "window" else case["far"]
    counts = _spread(L, B, ragged and L > 1, seed)
    starts = _spread(far, B, ragged, seed + 1) if far else np.zeros(B, np.int32)
    return starts, counts


def _keys(case):
    """How many positions the cache's table or the keys' tensor has."""
    if case["kind"] == "window":
        return case["Lk"]
    return _slots(case) * PAGE


def _slots(case):
    n = case["far"] + (case["L"] if case["kind"] == "cache" else case["Lq"])
    return -(-n // PAGE)


def _visible(case, starts, counts, dev):
    """Booleans [B, Lq, keys]."""
    p = starts[:, None] + torch.arange(case["Lq"], device=dev)
    n = (starts + counts)[:, None]
    hi = n.expand_as(p)
    if case["frame"]:
        hi = torch.minimum(hi, (p // case["frame"] + 1) * case["frame"])
    hi = hi[:, :, None]
    j = torch.arange(_keys(case), device=dev)
    near = j >= hi - case["window"] if case["window"] else j >= 0
    return (j < hi) & (near | (j < case["sinks"]))


# ---------------------------------------------------------------- inputs

def _scale(D):
    return float(np.float32(1.0 / math.sqrt(D)))


def _exponents(top):
    """The least e with top <= 448 * 2^e."""
    m, x = torch.frexp(top)   # top = m 2^x, 0.5 <= m < 1
    e = x - 9 + (m > 0.875).to(x.dtype)
    return torch.where(top > 0, e, torch.full_like(e, -100)).clamp(-100, 120)


def _e4m3(x):
    return x.to(torch.float8_e4m3fn)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt, kind, B = TYPES[case["dtype"]], case["kind"], case["B"]

    def randn(*shape, sigma=1.0, to=dt):
        return (torch.randn(*shape, device="cuda", generator=g) * sigma).to(to)

    st = dict(case=case)
    if kind == "gated":
        L, C, G = case["L"], case["C"], case["groups"]
        sd = torch.float32 if case["f32"] else dt
        six = randn(B, G, 6 * C, sigma=0.3).chunk(6, dim=-1)   # as one projection of the time step gives them
        st.update(x=randn(B, L, C, sigma=2.0, to=sd) + 0.5, r=randn(B, L, C, sigma=1.5), gate=six[2], scale=six[4],
                  shift=six[3], gamma_r=None, gamma=None, beta=None, h=torch.empty(B, L, C, dtype=sd, device="cuda"),
                  y=torch.empty(B, L, C, dtype=dt, device="cuda"))
        if case["post"] != "none":
            st["gamma_r"] = 1 + randn(C, sigma=0.2)
        if case["affine"]:
            st["gamma"] = 1 + randn(C, sigma=0.2)
            st["beta"] = randn(C, sigma=0.2) if case["pre"] == "layer" else None
        return st
    D, Hk = case["D"], case["Hk"]
    starts, counts = _plan(case, seed)
    st.update(starts=torch.from_numpy(starts).cuda(), counts=torch.from_numpy(counts).cuda())

    def tokens(H, L, sigma=1.0):
        return randn(B, L, H * D, sigma=sigma) if case["rows"] else randn(B, H, L, D, sigma=sigma)

    if kind in ("cache", "cached"):
        slots = _slots(case)
        P = B * slots + 3
        table = torch.randperm(P, device="cuda", generator=g)[:B * slots].view(B, slots).to(torch.int32)
        st["table"] = table
        for name in ("k", "v"):
            # what earlier calls wrote; neighbouring pages differ in size
            x = torch.randn(P, Hk, PAGE, D, device="cuda", generator=g)
            x *= torch.exp2(torch.randint(-2, 3, (P, Hk, 1, 1), device="cuda", generator=g).float())
            e = _exponents(x.abs().amax((2, 3)))
            codes = _e4m3(torch.ldexp(x, -e[:, :, None, None]))
            if kind == "cached" or case["way"] == "write":
                # behind the sequences nothing is written yet: whatever the memory holds, no numbers among it
                n = st["starts"] + (0 if kind == "cache" else st["counts"])
                pos = torch.arange(slots * PAGE, device="cuda").view(slots, 1, PAGE, 1)
                stale = (pos >= n[:, None, None, None, None]).expand(B, slots, Hk, PAGE, D)
                at = table.long()
                codes = codes.view(torch.uint8)
                codes[at] = codes[at].masked_fill(stale, 0x7f)
                codes = codes.view(torch.float8_e4m3fn)
            st[name + "_pages"] = codes
            st[name + "_scales"] = torch.exp2(e.float())
        del x, codes
    if kind == "cache":
        L = case["L"]
        if case["way"] == "write":
            st.update(k=tokens(Hk, L, 1.5), v=tokens(Hk, L, 0.7))
        else:
            shape = (B, L, Hk * D) if case["rows"] else (B, Hk, L, D)
            st.update(k=torch.zeros(shape, dtype=dt, device="cuda"), v=torch.zeros(shape, dtype=dt, device="cuda"))
        return st
    H, Lq = case["H"], case["Lq"]
    st["q"] = tokens(H, Lq)
    st["out"] = torch.zeros_like(st["q"])
    if kind == "window":
        st.update(k=tokens(Hk, case["Lk"]), v=tokens(Hk, case["Lk"]))
    return st


def run(st):
    return globals()[("_own_" if own else "_plain_") + st["case"]["kind"]](st, st["case"])


# ---------------------------------------------------------------- the framework's calls

def _own_gated(st, case):
    import paper_2304_11267_amd as sd
    norms = {"none": sd.NORM_NONE, "rms": sd.NORM_RMS, "layer": sd.NORM_LAYER}
    sd.gated_norm(st["x"], st["y"], r=st["r"], h=st["h"], gate=st["gate"], scale=st["scale"], shift=st["shift"],
                  gamma_r=st["gamma_r"], gamma=st["gamma"], beta=st["beta"], skip=SKIP, norm_r=norms[case["post"]],
                  norm=norms[case["pre"]], eps=EPS)
    return st["h"], st["y"]


def _layout(case):
    import paper_2304_11267_amd as sd
    return sd.LAYOUT_ROWS if case["rows"] else sd.LAYOUT_HEADS


def _own_cache(st, case):
    import paper_2304_11267_amd as sd
    call = sd.cache_write if case["way"] == "write" else sd.cache_read
    call(st["k"], st["v"], st["k_pages"], st["v_pages"], st["k_scales"], st["v_scales"], st["table"], st["starts"],
         counts=st["counts"], layout=_layout(case))
    if case["way"] == "read":
        return st["k"], st["v"]
    return st["k_pages"], st["v_pages"], st["k_scales"], st["v_scales"]


def _own_cached(st, case):
    import paper_2304_11267_amd as sd
    if "workspace" not in st:   # kept with the cache, as a server does
        n = sd.cache_forward_workspace(case["B"], case["H"], case["Hk"], case["Lq"], case["D"], _slots(case),
                                       case["frame"], case["window"], case["sinks"])
        st["workspace"] = torch.empty(n, dtype=torch.uint8, device="cuda")
    return sd.cache_forward(st["q"], st["k_pages"], st["v_pages"], st["k_scales"], st["v_scales"], st["table"],
                            st["starts"], st["out"], _scale(case["D"]), case["H"], workspace=st["workspace"],
                            counts=st["counts"], frame=case["frame"], window=case["window"], sinks=case["sinks"],
                            x_layout=_layout(case), y_layout=_layout(case))


def _own_window(st, case):
    import paper_2304_11267_amd as sd
    if "workspace" not in st:
        n = sd.window_forward_workspace(case["B"], case["H"], case["Hk"], case["Lq"], case["Lk"], case["D"],
                                        case["frame"], case["window"], case["sinks"])
        st["workspace"] = torch.empty(n, dtype=torch.uint8, device="cuda")
    return sd.window_forward(st["q"], st["k"], st["v"], st["out"], _scale(case["D"]), case["H"], case["Hk"],
                             workspace=st["workspace"], starts=st["starts"], counts=st["counts"], frame=case["frame"],
                             window=case["window"], sinks=case["sinks"], x_layout=_layout(case), y_layout=_layout(case))


# ---------------------------------------------------------------- plain forms

def _plain_normed(x, how, gamma, beta):
    if how == "none":
        return x
    if how == "layer":
        x = x - x.mean(-1, keepdim=True)
    x = x / (x.square().mean(-1, keepdim=True) + EPS).sqrt()
    x = x if gamma is None else x * gamma.float()
    return x if beta is None else x + beta.float()


def _plain_gated(st, case):
    def each(m):   # a group's modulation for each of its tokens
        return m.float().repeat_interleave(case["L"] // case["groups"], dim=1)
    h = SKIP * st["x"].float() + each(st["gate"]) * _plain_normed(st["r"].float(), case["post"], st["gamma_r"], None)
    y = _plain_normed(h, case["pre"], st["gamma"], st["beta"]) * (1 + each(st["scale"])) + each(st["shift"])
    return h.to(st["x"].dtype), y.to(st["r"].dtype)


def _heads(x, H, rows):
    """[B, H, L, D] of either layout."""
    return x.unflatten(2, (H, -1)).transpose(1, 2) if rows else x


def _plain_cache(st, case):
    B, Hk, L, D = (case[n] for n in ("B", "Hk", "L", "D"))
    starts, counts, table = st["starts"].long(), st["counts"].long(), st["table"].long()
    if case["way"] == "read":
        pos = starts[:, None] + torch.arange(L, device="cuda")
        page = table.gather(1, (pos // PAGE).clamp(max=_slots(case) - 1))
        valid = (torch.arange(L, device="cuda") < counts[:, None])[:, None, :, None]
        return tuple(_plain_back(st[n], st[n + "_pages"], st[n + "_scales"], page, pos % PAGE, valid, case) for n in ("k", "v"))
    # the pages that new tokens fall into, from the one with the first of them
    first = starts // PAGE
    touched = min(_slots(case), (L + 2 * PAGE - 2) // PAGE)
    slot = first[:, None] + torch.arange(touched, device="cuda")
    inside = slot < _slots(case)
    at = table.gather(1, slot.clamp(max=_slots(case) - 1))
    pos = (slot[:, :, None] * PAGE + torch.arange(PAGE, device="cuda"))[:, :, None, :, None]   # [B, touched, 1, PAGE, 1]
    b, n = (v[:, None, None, None, None] for v in (starts, starts + counts))
    fresh, kept = (pos >= b) & (pos < n), pos < b
    live = (fresh.flatten(2).any(2) & inside)
    return tuple(t for n in (0, 1) for t in (
        _plain_codes(st["kv"[m]], st["kv"[m] + "_pages"], st["kv"[m] + "_scales"], at, pos - b, fresh, kept, live, case)[n]
        for m in (0, 1)))


def _plain_back(out, pages, scales, page, place, valid, case):
    x = pages.view(torch.uint8)[page, :, place].view(torch.float8_e4m3fn).float() * scales[page][..., None]   # [B, L, Hk, D]
    x = x.to(out.dtype)
    x = x.flatten(2) if case["rows"] else x.transpose(1, 2)
    return torch.where(valid[:, 0] if case["rows"] else valid, x, out)


def _plain_codes(x, pages, scales, at, token, fresh, kept, live, case):
    """Codes and scales with the pages `at` written anew."""
    new = _heads(x, case["Hk"], case["rows"]).float().clamp(-HELD[case["dtype"]], HELD[case["dtype"]])
    L = case["L"]
    token = token[:, :, 0, :, 0].clamp(0, L - 1).flatten(1)[:, None, :, None].expand(-1, case["Hk"], -1, case["D"])
    new = new.gather(2, token).unflatten(2, (-1, PAGE)).transpose(1, 2)       # [B, touched, Hk, PAGE, D]
    new = torch.where(fresh, new, torch.zeros_like(new))
    begun = kept.any(3, keepdim=True)
    old_scale = torch.where(begun, scales[at][..., None, None], torch.zeros((), device=x.device))
    old_codes = pages.view(torch.uint8)[at]
    need = torch.exp2(_exponents(new.abs().amax((3, 4), keepdim=True)).float())
    scale = torch.maximum(old_scale, need)
    old = old_codes.view(torch.float8_e4m3fn).float() * torch.where(kept, old_scale / scale, torch.ones_like(scale))
    codes = _e4m3(torch.where(fresh, new / scale, old)).view(torch.uint8)
    codes = torch.where(fresh | kept, codes, old_codes)
    w = live.flatten().nonzero()[:, 0]
    at = at.flatten()[w]
    pages, scales = pages.view(torch.uint8), scales
    pages[at] = codes.flatten(0, 1)[w]
    scales[at] = scale[..., 0, 0].flatten(0, 1)[w]
    return pages.view(torch.float8_e4m3fn), scales


def _plain_attention(st, case, k, v):
    """k, v [B, Hk, keys, D] in 32 bits."""
    H, Hk, rows = case["H"], case["Hk"], case["rows"]
    starts, counts = st["starts"].long(), st["counts"].long()
    q = _heads(st["q"], H, rows).float()
    written = torch.arange(k.shape[2], device="cuda") < (starts + counts)[:, None]
    k, v = (t.masked_fill(~written[:, None, :, None], 0.0).repeat_interleave(H // Hk, dim=1) for t in (k, v))
    seen = _visible(case, starts, counts, "cuda")[:, None]
    a = torch.matmul(q.contiguous(), k.transpose(2, 3).contiguous()).mul_(_scale(case["D"])).masked_fill_(~seen, -math.inf)
    top = a.amax(-1, keepdim=True)
    a = a.sub_(top.masked_fill(top == -math.inf, 0.0)).exp_()
    o = (torch.matmul(a, v) / a.sum(-1, keepdim=True).clamp(min=1e-30)).to(st["q"].dtype)
    valid = (torch.arange(case["Lq"], device="cuda") < counts[:, None])
    if rows:
        return torch.where(valid[:, :, None], o.transpose(1, 2).flatten(2), st["out"])
    return torch.where(valid[:, None, :, None], o, st["out"])


def _plain_cached(st, case):
    k, v = ((st[n + "_pages"].float() * st[n + "_scales"][:, :, None, None])[st["table"].long()].transpose(1, 2).flatten(2, 3)
            for n in ("k", "v"))
    return _plain_attention(st, case, k, v)


def _plain_window(st, case):
    return _plain_attention(st, case, *(_heads(st[n], case["Hk"], case["rows"]).float() for n in ("k", "v")))


# ---------------------------------------------------------------- work

def work(case):
    """Inputs read once and outputs written once; multiply-adds of the definition."""
    kind, B = case["kind"], case["B"]
    if kind == "gated":
        L, C, n = case["L"], case["C"], B * case["L"] * case["C"]
        wide = 4 if case["f32"] else 2
        return dict(bytes=n * (2 * wide + 4) + 2 * 3 * B * case["groups"] * C + 2 * 3 * C, flops=20 * n)
    starts, counts = (a.astype(np.int64) for a in _plan(case, 0))
    D, Hk = case["D"], case["Hk"]
    if kind == "cache":
        n = int(counts.sum()) * Hk * D
        pages = int(((starts + counts + PAGE - 1) // PAGE - starts // PAGE).sum())
        return dict(bytes=2 * 3 * n + 8 * pages * (Hk + 1), flops=2 * 4 * n)
    H, Lq = case["H"], case["Lq"]
    pairs = seen = 0
    for s, c in zip(starts, counts):
        p = s + np.arange(c)
        hi = np.minimum(s + c, (p // case["frame"] + 1) * case["frame"]) if case["frame"] else np.full(c, s + c)
        lo = np.maximum(hi - case["window"], 0) if case["window"] else np.zeros_like(hi)
        sinks = np.minimum(case["sinks"], hi)
        pairs += int((hi - lo + np.minimum(sinks, lo)).sum())
        seen += int(hi.max() - lo.min() + min(sinks.max(), lo.min()))
    wide = 1 if kind == "cached" else 2
    return dict(bytes=2 * wide * seen * Hk * D + 2 * 2 * int(counts.sum()) * H * D, flops=4 * H * D * pairs)


# ---------------------------------------------------------------- 64 bits, by the definitions

def exact(case, seed):
    st = prepare(case, seed)
    return globals()["_exact_" + case["kind"]](st, case)


def _exact_gated(st, case):
    def norm(x, how, gamma, beta):
        if how == "none":
            return x
        mean = x.sum(-1, keepdim=True) / case["C"] if how == "layer" else 0.0
        x = (x - mean) * (((x - mean) ** 2).sum(-1, keepdim=True) / case["C"] + EPS).rsqrt()
        x = x * (1.0 if gamma is None else gamma.double())
        return x + (0.0 if beta is None else beta.double())
    shape = (case["B"], case["groups"], case["L"] // case["groups"], case["C"])
    x, r = (st[n].double().view(shape) for n in ("x", "r"))
    gate, scale, shift = (st[n].double()[:, :, None] for n in ("gate", "scale", "shift"))
    h = SKIP * x + gate * norm(r, case["post"], st["gamma_r"], None)
    y = norm(h, case["pre"], st["gamma"], st["beta"]) * (1 + scale) + shift
    return tuple(t.view(case["B"], case["L"], case["C"]) for t in (h, y))


def _exact_cache(st, case):
    B, Hk, L, D = (case[n] for n in ("B", "Hk", "L", "D"))
    starts, counts, table = st["starts"].tolist(), st["counts"].tolist(), st["table"].tolist()
    if case["way"] == "read":
        out = []
        for n in ("k", "v"):
            x = torch.zeros(B, L, Hk, D, dtype=torch.float64, device="cuda")
            for b in range(B):
                for s in range(-(-counts[b] // PAGE)):   # (these start at a page's first token)
                    rows = min(PAGE, counts[b] - s * PAGE)
                    page = table[b][s]
                    x[b, s * PAGE:s * PAGE + rows] = (st[n + "_pages"][page, :, :rows].double() *
                                                      st[n + "_scales"][page].double()[:, None, None]).transpose(0, 1)
            out.append(x.flatten(2) if case["rows"] else x.transpose(1, 2).contiguous())
        return tuple(out)
    # codes and scales are choices of a grid: the scales alone, from the values' sizes
    if sum(counts) // PAGE + B > 3000:
        return None
    out = []
    for n in ("k", "v"):
        x = st[n].double()
        x = x.view(B, L, Hk, D) if case["rows"] else x.transpose(1, 2)
        scales = st[n + "_scales"].double().clone()
        for b in range(B):
            for s in range(starts[b] // PAGE, (starts[b] + counts[b] - 1) // PAGE + 1):
                i, j = max(0, s * PAGE - starts[b]), min(counts[b], (s + 1) * PAGE - starts[b])
                need = torch.exp2(torch.log2(x[b, i:j].abs().amax((0, 2)) / MOST).ceil())
                page = table[b][s]
                scales[page] = need if s * PAGE >= starts[b] else torch.maximum(scales[page], need)
        out.append(scales)
    return None, None, out[0], out[1]


def _exact_attention(st, case, keys):
    """keys(b, n, h): [keys, D] in 64 bits."""
    B, H, Hk, Lq, D = (case[n] for n in ("B", "H", "Hk", "Lq", "D"))
    starts, counts = st["starts"].tolist(), st["counts"].tolist()
    out = torch.zeros(B, H, Lq, D, dtype=torch.float64, device="cuda")
    q = st["q"].view(B, Lq, H, D).transpose(1, 2) if case["rows"] else st["q"]
    for b in range(B):
        n = starts[b] + counts[b]
        j = torch.arange(n, device="cuda")
        p = torch.arange(starts[b], n, device="cuda")
        hi = ((p // case["frame"] + 1) * case["frame"]).clamp(max=n) if case["frame"] else torch.full_like(p, n)
        for h in range(H):
            if h % (H // Hk) == 0:
                k, v = (keys(b, x, h // (H // Hk))[:n] for x in "kv")
            for i in range(0, counts[b], 4096):
                top = hi[i:i + 4096, None]
                off = j >= top
                if case["window"]:
                    off |= (j < top - case["window"]) & (j >= case["sinks"])
                a = q[b, h, i:min(i + 4096, counts[b])].double() @ k.t().contiguous() * _scale(D)
                w = torch.softmax(a.masked_fill(off, -math.inf), -1).nan_to_num(0.0)
                out[b, h, i:min(i + 4096, counts[b])] = w @ v
    return out.transpose(1, 2).flatten(2) if case["rows"] else out


def _exact_cached(st, case):
    def keys(b, x, h):
        at = st["table"][b].long()
        return (st[x + "_pages"].view(torch.uint8)[at, h].view(torch.float8_e4m3fn).double() *
                st[x + "_scales"][at, h].double()[:, None, None]).flatten(0, 1)
    return _exact_attention(st, case, keys)


def _exact_window(st, case):
    def keys(b, x, h):
        t = st[x].unflatten(2, (case["Hk"], -1)).transpose(1, 2) if case["rows"] else st[x]
        return t[b, h].double()
    return _exact_attention(st, case, keys)
