"""The 8-bit cache in 64 bits, from its definition: codes by comparison with every value, blocks as numbers, appends by
loops over blocks, heads and tokens."""
import numpy as np
import torch

D = 128
RANGE = {torch.bfloat16: (-100, 119), torch.float16: (-15, 7)}
# what the codes 0 .. 126 stand for: 4 bits of exponent, 3 of mantissa
LEVELS = np.array([(c & 7) * 2.0**-9 if c < 8 else (8 + (c & 7)) / 8 * 2.0 ** ((c >> 3) - 7) for c in range(127)])
MIDS = (LEVELS[1:] + LEVELS[:-1]) / 2


def exponent(top, dtype):
    lo, hi = RANGE[dtype]
    m, k = np.frexp(np.asarray(top) / 448)
    return np.clip(np.where(np.asarray(top) > 0, np.where(m == 0.5, k - 1, k), lo), lo, hi).astype(np.int64)


def encode(x, e):
    """Codes of x / 2^e: nearest, the even one of two, 448 beyond it; NaN for what is not finite."""
    y = np.abs(x) / np.exp2(np.asarray(e, np.float64))
    fin = np.isfinite(x)
    y = np.where(fin, y, 0)
    up = np.searchsorted(MIDS, y, side="left")  # midpoints below y
    tie = (up < 126) & (MIDS[np.minimum(up, 125)] == y) & (up % 2 == 1)
    code = np.where(fin, np.minimum(up + tie, 126), 127)
    return (code | (np.signbit(x) & fin).astype(np.int64) << 7).astype(np.uint8)


def decode(code, e):
    c = code & 127
    v = np.where(c == 127, np.nan, LEVELS[np.minimum(c, 126)])
    return np.where(code & 128, -v, v) * np.exp2(np.asarray(e, np.float64))


class Cache:
    """Blocks [n][heads][2][bs][128] of codes and exponents [n][heads][2]; of a token not yet written nothing is known."""

    def __init__(self, n, heads, bs, dtype):
        self.n, self.heads, self.bs, self.dtype = n, heads, bs, dtype
        self.code = np.zeros((n, heads, 2, bs, D), np.uint8)
        self.exp = np.zeros((n, heads, 2), np.int64)
        self.known = np.zeros((n, bs), bool)

    def append(self, k, v, places):
        """Rows [T][heads][128] at places (None: nowhere)."""
        rows = [x.detach().cpu().double().numpy() for x in (k, v)]
        blocks = {}
        for i, p in enumerate(places):
            if p is not None and p >= 0:
                blocks.setdefault(p // self.bs, {})[p % self.bs] = i
        for b, toks in blocks.items():
            anew = 0 in toks
            if anew:
                self.known[b] = False
            ids = list(toks.values())
            for h in range(self.heads):
                for side in (0, 1):
                    x = rows[side][ids, h]
                    top = np.where(np.isfinite(x), np.abs(x), 0).max()
                    e, old = int(exponent(top, self.dtype)), int(self.exp[b, h, side])
                    if not anew:
                        e = max(e, old)
                    if e != old and not anew:
                        c = self.code[b, h, side]
                        self.code[b, h, side] = encode(decode(c, old), e)
                    self.exp[b, h, side] = e
                    self.code[b, h, side, list(toks)] = encode(x, e)
            self.known[b, list(toks)] = True

    def values(self):
        """Keys and values [n][heads][bs][128] in 64 bits."""
        v = decode(self.code, self.exp[..., None, None])
        return torch.from_numpy(v[:, :, 0]), torch.from_numpy(v[:, :, 1])

    def bytes(self):
        """The blocks as bytes; and where they are known."""
        n, h, bs = self.n, self.heads, self.bs
        U = h * 256 * bs + (2 * h + 127) // 128 * 128
        out, sure = np.zeros((n, U), np.uint8), np.zeros((n, U), bool)
        t, c = np.meshgrid(np.arange(bs), np.arange(D), indexing="ij")
        for i in range(h):
            k_at = i * 256 * bs + t * D + c
            v_at = i * 256 * bs + 128 * bs + ((t // 8 * 16 + c % 16) * 8 + c // 16) * 8 + t % 8
            for side, at in ((0, k_at), (1, v_at)):
                out[:, at] = self.code[:, i, side]
                sure[:, at] = self.known[:, :, None]
                out[:, h * 256 * bs + 2 * i + side] = self.exp[:, i, side] + 127
                sure[:, h * 256 * bs + 2 * i + side] = self.known.any(1)
        return out, sure


def pack(k, v, bs):
    """Keys and values [n][heads][bs][128] of a 16-bit type, whole blocks, as bytes."""
    n, h = k.shape[:2]
    cache = Cache(n, h, bs, k.dtype)
    x = torch.stack([k, v], 2).double().numpy()
    cache.exp = exponent(np.abs(x).max((-1, -2)), k.dtype)
    cache.code = encode(x, cache.exp[..., None, None])
    return torch.from_numpy(cache.bytes()[0]), cache
