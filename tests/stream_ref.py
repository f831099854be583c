"""Plain 64-bit forms of the gated norms, the 8-bit cache and the attention over what a
query's place lets it see, for the tests (numpy on the host, torch's 64 bits on the GPU)."""
import numpy as np

from operators_ref import TINY, U16, half_step
from parity_util import torch_mod

PAGE = 64
HELD = {"f16": 1.875 * 2.0 ** 15, "bf16": 1.875 * 2.0 ** 127}


# ---------------------------------------------------------------- e4m3

def decode(codes):
    """Values of e4m3 codes (uint8)."""
    c = codes.astype(np.int64)
    e, m = (c >> 3) & 15, c & 7
    v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))
    v = np.where((c & 0x7f) == 0x7f, np.nan, v)
    return np.where(c & 0x80, -v, v)


def encode(x):
    """Codes of numbers of at most 448, to nearest, ties to even; what is no number: 0x7f."""
    a = np.abs(np.nan_to_num(x, nan=0.0))
    e = np.floor(np.log2(np.maximum(a, 2.0 ** -6)))
    step = 2.0 ** (e - 3)
    q = np.round(a / step)                      # (numpy rounds halves to even)
    e, q = np.where(q == 16, e + 1, e), np.where(q == 16, 8, q)
    code = np.where(q < 8, q, (e + 7) * 8 + (q - 8))   # subnormals: q of steps of 2^-9
    code = np.where(np.isnan(x), 0x7f, code).astype(np.uint8)
    return code | (np.signbit(x) & ~np.isnan(x)).astype(np.uint8) << 7


def exponent(top):
    """The least e in [-100, 120] with top <= 448 2^e."""
    if not top > 0:
        return -100
    e = int(np.floor(np.log2(top))) - 9
    while top > 448.0 * 2.0 ** e:
        e += 1
    return min(max(e, -100), 120)


def write(x, codes, scales, table, starts, counts, dtype):
    """cache_write of one of K and V in place: x [B, Hk, L, D] in 64 bits, codes uint8 [P, Hk, 64, D], scales [P, Hk]."""
    B, Hk, L, D = x.shape
    P, slots = codes.shape[0], table.shape[1]
    x = np.where(np.isfinite(x), np.clip(x, -HELD[dtype], HELD[dtype]), np.nan)
    for b in range(B):
        s, n = int(starts[b]), int(starts[b]) + min(max(int(counts[b]), 0), L)
        for slot in range(max(s, 0) // PAGE, min(slots, -(-max(n, 0) // PAGE))):
            page = table[b, slot]
            i, j = max(s, slot * PAGE, 0), min(n, (slot + 1) * PAGE)
            if not 0 <= page < P or i >= j:
                continue
            r0 = i - slot * PAGE
            for h in range(Hk):
                new = x[b, h, i - s:j - s]
                top = np.nanmax(np.abs(new)) if not np.isnan(new).all() else 0.0
                need = 2.0 ** exponent(top)
                scale = max(float(scales[page, h]), need) if r0 else need
                if r0 and scale != scales[page, h]:
                    codes[page, h, :r0] = encode(decode(codes[page, h, :r0]) * (float(scales[page, h]) / scale))
                codes[page, h, r0:r0 + j - i] = encode(new / scale)
                scales[page, h] = scale


def read(codes, scales, table, starts, counts, L):
    """[B, Hk, L, D] in 64 bits; nan behind counts, zeros where there is no page."""
    P, Hk, _, D = codes.shape
    B, slots = table.shape
    out = np.full((B, Hk, L, D), np.nan)
    val = decode(codes) * scales[:, :, None, None]
    for b in range(B):
        for l in range(min(max(int(counts[b]), 0), L)):
            p = int(starts[b]) + l
            page = table[b, p // PAGE] if 0 <= p < slots * PAGE else -1
            out[b, :, l] = val[page, :, p % PAGE] if 0 <= page < P else 0.0
    return out


def same_codes(a, b):
    """Equal codes; codes that are no numbers are all alike."""
    return ((a == b) | (((a & 0x7f) == 0x7f) & ((b & 0x7f) == 0x7f))).all()


# ---------------------------------------------------------------- attention

def seen(starts, counts, Lq, keys, frame, window, sinks):
    """Booleans [B, Lq, keys]; rows from counts on see nothing."""
    out = np.zeros((len(starts), Lq, keys), bool)
    j = np.arange(keys)
    for b, (s, c) in enumerate(zip(starts, counts)):
        c = min(max(int(c), 0), Lq)
        n = min(max(int(s) + c, 0), keys)
        for l in range(c):
            p = int(s) + l
            hi = n if frame == 0 else min(n, (p // frame + 1) * frame)
            lo = hi - window if window else 0
            out[b, l] = (j < hi) & ((j >= lo) | (j < sinks))
    return out


def attention(q, k, v, see, scale):
    """q [B, H, Lq, D], k and v [B, Hk, keys, D], see [B, Lq, keys], torch tensors in 64 bits on one
    device.  Keys that are not seen are left out, whatever they hold.  Returns out, dev = sum_j p_ij |v_jd -
    o_id|, and the largest |score| of each row."""
    torch = torch_mod()
    H, Hk = q.shape[1], k.shape[1]
    out, dev = torch.zeros_like(q), torch.zeros_like(q)
    top = torch.zeros(q.shape[:3], dtype=q.dtype, device=q.device)
    for b in range(q.shape[0]):
        on = see[b]
        for h in range(H):
            kk, vv = k[b, h // (H // Hk)], v[b, h // (H // Hk)]
            used = on.any(0)
            kk, vv = (torch.where(used[:, None], t, torch.zeros_like(t)) for t in (kk, vv))
            a = torch.matmul(q[b, h], kk.t().contiguous()) * scale
            top[b, h] = torch.where(on, a.abs(), torch.zeros_like(a)).amax(1)
            p = torch.softmax(a.masked_fill(~on, -float("inf")), 1)
            p = torch.where(on.any(1, keepdim=True), p, torch.zeros_like(p))
            o = torch.matmul(p, vv)
            out[b, h] = o
            for i in range(0, q.shape[2], 64):
                dev[b, h, i:i + 64] = (p[i:i + 64, :, None] * (vv[None] - o[i:i + 64, None]).abs()).sum(1)
    return out, dev, top


def bound(g, r, dev, top, n, D, vmax, dtype):
    """What the kernels may be off by.  Scores are sums of D products in 32 bits, so an exponent is off by at
    most (D + 8) 2^-24 of the largest score's size (twice: the score's own and the maximum's), which moves o by
    that times dev, as does rounding every weight to the type (half a step, an eighth more for the exponential); n
    keys' sums in 32 bits lose at most n 2^-24 of dev + |r|, and weights below fp16's subnormals, 2^-33 of the
    largest, are lost.  The output is rounded once."""
    size = dev + np.abs(r)
    return (half_step(g, r, dtype) + U16[dtype] * 1.125 * dev + 2 * (D + 8) * 2.0 ** -24 * (top[..., None] + 1) * 2 * dev +
            (n + 8) * 2.0 ** -24 * size + n * 2.0 ** -33 * vmax + TINY[dtype])


# ---------------------------------------------------------------- gated norms

def normed(x, how, gamma, beta, eps):
    """norm(x), and the size that errors of its sums are relative to."""
    if how == "none":
        return x, np.abs(x)
    mean = x.mean(-1, keepdims=True) if how == "layer" else 0.0
    sd = np.sqrt(((x - mean) ** 2).mean(-1, keepdims=True) + eps)
    y, size = (x - mean) / sd, (np.abs(x) + np.abs(x).mean(-1, keepdims=True)) / sd
    if gamma is not None:
        y, size = y * gamma, size * np.abs(gamma)
    if beta is not None:
        y, size = y + beta, size + np.abs(beta)
    return y, size


def gated(x, r, gate, scale, shift, gamma_r, gamma, beta, skip, norm_r, norm, eps):
    """x, r [B, L, C]; gate, scale, shift [B, L, C] or numbers.  Returns (h, its bound, y, its bound), before
    the last rounding: a norm takes two sums of C terms in 32 bits, a root and a few products, each within
    2^-24: (C + 16) 2^-24 of its size, twice over for y, whose input is h."""
    C = x.shape[-1]
    u = (C + 16) * 2.0 ** -24
    h, hoff = skip * x, 4 * 2.0 ** -24 * np.abs(skip * x)
    if r is not None:
        p, size = normed(r, norm_r, gamma_r, None, eps)
        h = h + gate * p
        hoff = hoff + np.abs(gate) * size * (u if norm_r != "none" else 2.0 ** -22)
    y, size = normed(h, norm, gamma, beta, eps)
    # an error of h moves its norm by at most that over the deviation, and the mean's and deviation's parts of it
    if norm == "none":
        yoff = hoff
    else:
        mean = h.mean(-1, keepdims=True) if norm == "layer" else 0.0
        sd = np.sqrt(((h - mean) ** 2).mean(-1, keepdims=True) + eps)
        rel = np.sqrt((hoff ** 2).mean(-1, keepdims=True)) / sd
        z = np.abs(h - mean) / sd
        yoff = (hoff / sd + rel + rel * z) * (1.0 if gamma is None else np.abs(gamma)) + u * size
    out = y * (1 + scale) + shift
    return h, hoff, out, yoff * np.abs(1 + scale) + 2.0 ** -22 * (size * np.abs(1 + scale) + np.abs(shift))
