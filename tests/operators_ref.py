"""Plain 64-bit forms of the adapters, the norms with rotation, the block selection and
the attention over selected blocks, in numpy, for the GPU tests."""
import numpy as np

from parity_util import torch_mod

U16 = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}     # half a step of the type, relative
TINY = {"f16": 2.0 ** -25, "bf16": 2.0 ** -134}  # and absolute, among its subnormals


def t_type(dtype):
    torch = torch_mod()
    return {"f16": torch.float16, "bf16": torch.bfloat16}[dtype]


def randn(g, *shape, dtype="f16", sigma=1.0):
    torch = torch_mod()
    return (torch.randn(*shape, device="cuda", generator=g) * sigma).to(t_type(dtype))


def generator(seed):
    torch = torch_mod()
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def host(t):
    return t.double().cpu().numpy()


def heads_to_rows(a):
    """[B, H, L, D] -> [B, L, H D]."""
    B, H, L, D = a.shape
    return np.ascontiguousarray(a.transpose(0, 2, 1, 3)).reshape(B, L, H * D)


def rows_to_heads(a, H):
    B, L, C = a.shape
    return np.ascontiguousarray(a.reshape(B, L, H, C // H).transpose(0, 2, 1, 3))


def step(r, dtype):
    """Spacing of the type's grid at |r|."""
    mant, low = (10, 2.0 ** -24) if dtype == "f16" else (7, 2.0 ** -133)
    a = np.maximum(np.abs(r), 1e-300)
    return np.maximum(2.0 ** (np.floor(np.log2(a)) - mant), low)


def half_step(g, r, dtype):
    """What rounding to the type may change: half a step, at the larger of the two values."""
    return step(np.maximum(np.abs(g), np.abs(r)), dtype) / 2


def adapters(x, w, bias, down, up, ids, scales, dtype):
    """y [B, L, N] and how far the kernels may be from it before the last rounding: T is
    rounded to the type once, sums of n products in 32 bits are within (n + 2) 2^-22 of
    the sum of their sizes."""
    K, R = x.shape[2], down.shape[1]
    y = x @ w.T + (0.0 if bias is None else bias)
    size = np.abs(x) @ np.abs(w).T
    off = np.zeros_like(y)
    for b, i in enumerate(ids):
        if not 0 <= i < down.shape[0]:
            continue
        s = 1.0 if scales is None else scales[i]
        t = s * (x[b] @ down[i].T)
        ts = abs(s) * (np.abs(x[b]) @ np.abs(down[i]).T)
        y[b] += t @ up[i].T
        t_off = (K + 2) * 2.0 ** -22 * ts + U16[dtype] * np.abs(t) + TINY[dtype]
        off[b] = t_off @ np.abs(up[i]).T
        size[b] += (np.abs(t) + t_off) @ np.abs(up[i]).T
    return y, off + (K + R + 2) * 2.0 ** -22 * size


def norm_rotate(x, gamma, pos, freqs, pairs, norm, eps, halves):
    """x [B, H, L, D] and the bound before the last rounding: D squares summed in 32 bits, a
    root, a quotient and two products, a sine and a cosine of 2^-22, two products and a sum."""
    D, P = x.shape[3], sum(pairs)
    y = x
    if norm:
        y = x / np.sqrt(np.mean(x * x, axis=-1, keepdims=True) + eps)
        y = y if gamma is None else y * gamma
    out, size = y.copy(), np.abs(y)
    turns = 0.0
    if P:
        axis = np.repeat(np.arange(len(pairs)), pairs)
        t = (pos[:, :, axis] * freqs)[:, None]
        turns = np.abs(t).max() / (2 * np.pi)
        a, b = (np.arange(P), P + np.arange(P)) if halves else (2 * np.arange(P), 2 * np.arange(P) + 1)
        out[..., a] = y[..., a] * np.cos(t) - y[..., b] * np.sin(t)
        out[..., b] = y[..., b] * np.cos(t) + y[..., a] * np.sin(t)
        size[..., a] = size[..., b] = np.abs(y[..., a]) + np.abs(y[..., b])
    return out, size * ((D + 20) * 2.0 ** -24 + 2.0 ** -22 + 2 * np.pi * turns * 2.0 ** -51)


def block_means(x, block):
    B, H, L, D = x.shape
    return np.stack([x[:, :, i:i + block].sum(2) / min(block, L - i) for i in range(0, L, block)], 2)


def select(q_means, k_means, keep):
    """Booleans [B, H, NQ, NB]."""
    s = np.matmul(q_means, np.ascontiguousarray(k_means.swapaxes(2, 3)))
    best = np.argsort(-s, axis=-1, kind="stable")[..., :keep]
    sel = np.zeros(s.shape, bool)
    np.put_along_axis(sel, best, True, -1)
    return sel


def pack(sel):
    """Booleans [..., NB] -> int64 words [..., ceil(NB / 64)]."""
    n = sel.shape[-1]
    sel = np.concatenate([sel, np.zeros(sel.shape[:-1] + (-n % 64,), bool)], -1).reshape(sel.shape[:-1] + (-1, 64))
    return np.bitwise_or.reduce(sel.astype(np.uint64) << np.arange(64, dtype=np.uint64), axis=-1).view(np.int64)


def unpack(words, nb):
    bits = (words.view(np.uint64)[..., None] >> np.arange(64, dtype=np.uint64)) & np.uint64(1)
    return bits.reshape(words.shape[:-1] + (-1,))[..., :nb].astype(bool)


def sparse(q, k, v, sel, scale, qblock):
    """out, and dev = sum_j p_ij |v_jd - o_id| (what rounding the weights may move)."""
    B, H, Lq, D = q.shape
    Lk = k.shape[2]
    out, dev = np.zeros_like(q), np.zeros_like(q)
    for b in range(B):
        for h in range(H):
            for i in range(sel.shape[2]):
                on = np.repeat(sel[b, h, i], 64)[:Lk]
                r = slice(i * qblock, min(Lq, (i + 1) * qblock))
                if not on.any():
                    continue
                kk, vv = k[b, h, on], v[b, h, on]
                a = scale * (q[b, h, r] @ kk.T)
                p = np.exp(a - a.max(1, keepdims=True))
                p /= p.sum(1, keepdims=True)
                out[b, h, r] = p @ vv
                for n in range(r.start, r.stop):
                    dev[b, h, n] = p[n - r.start] @ np.abs(vv - out[b, h, n])
    return out, dev
