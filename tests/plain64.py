"""Plain forms, in 64 bits and from the definitions, of what the kernels are tested against: the 4-bit cache, attention
over it, head norms with rotation, and the maps of a step."""
import math

import numpy as np
import torch

D = 128
LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
RANGE = {torch.bfloat16: (-100, 125), torch.float16: (-23, 13)}


def quantise(x):
    """Rows [..., 128] of a 16-bit type -> (codes [..., 128], scale bytes [..., 4], values in 64 bits)."""
    lo, hi = RANGE[x.dtype]
    g = x.detach().cpu().double().numpy().reshape(*x.shape[:-1], 4, 32)
    finite = np.isfinite(g).all(-1)
    top = np.where(np.isfinite(g), np.abs(g), 0.0).max(-1)
    # least e with top <= 7 * 2^e
    m, k = np.frexp(top / 7)
    e = np.where(top > 0, np.where(m == 0.5, k - 1, k), lo)
    e = np.clip(e, lo, hi).astype(np.int64)
    y = np.abs(np.where(finite[..., None], g, 0.0)) / np.exp2(e)[..., None]
    mids = (LEVELS[1:] + LEVELS[:-1]) / 2
    code = np.zeros(y.shape, np.int64)
    for i, mid in enumerate(mids, 1):  # a tie goes to the even code
        code = np.where((y > mid) | ((y == mid) & (i % 2 == 0)), i, code)
    neg = np.signbit(g) & finite[..., None]
    val = np.where(neg, -1.0, 1.0) * LEVELS[code] * np.exp2(e)[..., None]
    val = np.where(finite[..., None], val, np.nan)
    code = code | (neg << 3)
    byte = np.where(finite, e + 127, 255).astype(np.uint8)
    return (torch.from_numpy(code.reshape(x.shape)), torch.from_numpy(byte),
            torch.from_numpy(val.reshape(x.shape)))


def pack(k, v, bs):
    """Keys and values [n][hkv][bs][128] of a 16-bit type -> blocks [n][hkv * 136 * bs] of bytes, one code at a time."""
    n, h = k.shape[:2]
    kc, ks, _ = quantise(k)
    vc, vs, _ = quantise(v)
    kc, ks, vc, vs = (t.numpy() for t in (kc, ks, vc, vs))
    out = np.zeros((n, h, 136 * bs), np.uint8)
    for t in range(bs):
        for c in range(D):
            out[:, :, t * 64 + c // 2] |= (kc[:, :, t, c] << (4 * (c % 2))).astype(np.uint8)
            word = (t // 8 * 16 + c % 16) * 8 + c // 16
            out[:, :, 64 * bs + 4 * word + t % 8 // 2] |= (vc[:, :, t, c] << (4 * (t % 2))).astype(np.uint8)
        out[:, :, 128 * bs + 4 * t:128 * bs + 4 * t + 4] = ks[:, :, t]
        for g in range(4):
            out[:, :, 132 * bs + g * bs + t] = vs[:, :, t, g]
    return torch.from_numpy(out.reshape(n, -1))


def unpack(pool, hkv, bs):
    """Blocks of bytes -> keys and values [n][hkv][bs][128] in 64 bits."""
    b = pool.cpu().numpy().reshape(pool.shape[0], hkv, 136 * bs)
    sign = np.concatenate([LEVELS, -LEVELS])

    def scale(x):
        return np.where(x == 255, np.nan, np.exp2(x.astype(np.float64) - 127))

    t, c = np.meshgrid(np.arange(bs), np.arange(D), indexing="ij")
    k = sign[b[:, :, t * 64 + c // 2] >> (4 * (c % 2)) & 15] * scale(b[:, :, 128 * bs + 4 * t + c // 32])
    word = (t // 8 * 16 + c % 16) * 8 + c // 16
    v = sign[b[:, :, 64 * bs + 4 * word + t % 8 // 2] >> (4 * (t % 2)) & 15] * scale(
        b[:, :, 132 * bs + c // 32 * bs + t])
    return torch.from_numpy(k), torch.from_numpy(v)


def attention(q, k, v, scale):
    """One request: q [hq][128], k and v [hkv][n][128] -> (out, lse, sum of p |v|, largest sum of |q k| * scale)."""
    hq, hkv = q.shape[0], k.shape[0]
    G = hq // hkv
    q, k, v = q.double(), k.double(), v.double()
    out, lse = torch.zeros((hq, D), dtype=torch.float64), torch.full((hq,), -math.inf, dtype=torch.float64)
    mass, reach = torch.zeros((hq, D), dtype=torch.float64), torch.zeros(hq, dtype=torch.float64)
    if k.shape[1] == 0:
        return out, lse, mass, reach
    for h in range(hkv):
        s = slice(h * G, (h + 1) * G)
        x = q[s] @ k[h].T * scale
        p = torch.softmax(x, 1)
        out[s], lse[s], mass[s] = p @ v[h], torch.logsumexp(x, 1), p @ v[h].abs()
        reach[s] = (q[s].abs() @ k[h].abs().T * scale).amax(1)
    return out, lse, mass, reach


def norm_rope(x, weight, eps, positions, inv_freq, rot, interleaved):
    """Rows [T][heads][128] -> (result, size of what each element is a sum of) in 64 bits."""
    x = x.detach().cpu().double()
    if weight is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * weight.detach().cpu().double()
    t = positions.detach().cpu().double()[:, None] * inv_freq.detach().cpu()
    c, s = torch.cos(t)[:, None], torch.sin(t)[:, None]
    i = torch.arange(rot // 2)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
    y, size = x.clone(), x.abs()
    if rot:
        u, w = x[..., a], x[..., b]
        y[..., a], y[..., b] = u * c - w * s, u * s + w * c
        size[..., a] = size[..., b] = u.abs() + w.abs()
    return y, size


def tables(ctx, new, bs, table, free, head, max_tokens):
    """The maps of a step by loops over requests, blocks and tokens; lengths and slots are taken to be right."""
    table = [list(map(int, r)) for r in table]
    blk, tok, place, pos = [0], [0], [], []
    for r, (x, n) in enumerate(zip(ctx, new)):
        blk.append(blk[-1] + -(-x // bs))
        tok.append(tok[-1] + n)
        for p in range(x - n, x):
            if table[r][p // bs] == -1:
                table[r][p // bs] = int(free[head])
                head += 1
            place.append(table[r][p // bs] * bs + p % bs)
            pos.append(p)
    rest = [-1] * (max_tokens - len(pos))
    return blk, tok, place + rest, pos + rest, table, head
