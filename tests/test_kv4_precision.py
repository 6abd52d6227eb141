"""How exact the attention over the 4-bit cache is where little else than the cut of its probabilities can be wrong:
four tokens have a probability other than 0 (the others' logits are some hundreds lower), logits are small and exact
products, values are not negative, and every token's value groups have scales of their own."""
import numpy as np
import pytest
import torch

import plain64
from paper_2609_34555_amd import pulse as P
from parity import say
from test_kv4 import DEV, SCALE, TYPES, D, attend, dev

U = 2.0**-24


def bound(reach, steps):
    """Relative, of sums of positive terms. A logit's argument of exp2: three roundings in the scale, one of its product,
    the same of the maximum's, one of the difference; exp2 is 2 U off. A probability times a power of two is exact and
    so are its three parts of 8 bits. Three products of at most four terms, each addition at most 2 U off; three
    additions of the denominator, the division. Over several steps and waves: three times alpha (exp2, its argument,
    the product) and two merges (the same and four additions), in numerator and denominator."""
    p = 10 * reach * U + 2 * U
    one = 2 * p + 24 * U + 5 * U + U
    return one if steps == 1 else one + 2 * (3 * (3 * U + 2 * reach * U)) + 2 * 2 * (7 * U + 2 * reach * U)


def rows(n, hq, hkv, dtype, gen, rng):
    """q [hq][128], keys and values [hkv][n][128] that the cache holds as they are, and the four tokens."""
    q = torch.zeros((hq, D))
    k, v = torch.zeros((2, hkv, n, D))
    live = rng.choice(n, size=4, replace=False)
    q[:, 77] = torch.rand(hq, generator=gen) / 2 + 0.5
    level = torch.tensor([0.25, 0.375, 0.5, 0.75, 1.0, 1.5])
    k[:, :, 77] = -6144.0
    k[:, live, 77] = level[torch.randint(0, 6, (hkv, 4), generator=gen)]
    v = torch.randn((hkv, n, D), generator=gen).abs()
    v = v * torch.exp2(torch.randint(-4, 4, (hkv, n, 4), generator=gen).float()).repeat_interleave(32, -1)
    v = plain64.quantise(v.to(dtype))[2].to(dtype)
    return q.to(dtype), k.to(dtype), v, live


def model(q, k, v, live, parts):
    """The step's arithmetic with the probabilities cut into that many bf16 parts, sums in 64 bits."""
    G = q.shape[0] // k.shape[0]
    out = np.zeros((q.shape[0], D))
    for h in range(q.shape[0]):
        x = (k[h // G, live, 77].double().numpy() * q[h, 77].double().item()) * SCALE
        p = np.exp(x - x.max()).astype(np.float32)
        cut, rest = np.zeros(4, np.float32), p.copy()
        for _ in range(parts):
            part = (rest.view(np.uint32) & np.uint32(0xFFFF0000)).view(np.float32)
            cut, rest = cut + part, rest - part
        out[h] = cut.astype(np.float64) @ v[h // G, live].double().numpy() / p.astype(np.float64).sum()
    return torch.from_numpy(out)


def test_the_bound_tells_two_parts_from_three():
    gen, rng = torch.Generator().manual_seed(1), np.random.default_rng(1)
    q, k, v, live = rows(32, 16, 2, torch.bfloat16, gen, rng)
    want, _, mass, _ = plain64.attention(q, k, v, SCALE)
    reach = float((q[:, 77].double().max() * 1.5 * SCALE))
    assert torch.equal(want, mass)
    for steps in (1, 2):
        over = [((model(q, k, v, live, n) - want).abs() / want.clamp(min=1e-30) / bound(reach, steps)).max().item()
                for n in (1, 2, 3)]
        say(f"  one, two, three parts: {over} of the bound")
        assert over[0] > 100 and over[1] > 1.5 and over[2] < 0.3


# query heads, KV heads, bs, tokens of the context
CASES = [(4, 1, 16, 32), (3, 3, 32, 32), (8, 1, 16, 32), (6, 1, 32, 32), (16, 1, 16, 32), (24, 2, 32, 32), (32, 8, 16, 32),
         (4, 1, 64, 64), (16, 1, 64, 2000), (8, 2, 16, 2000), (16, 2, 32, 5000), (12, 1, 16, 2000), (32, 8, 16, 9000)]


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("hq,hkv,bs,ctx", CASES)
def test_probabilities_keep_all_their_bits(hq, hkv, bs, ctx, dt):
    dtype, _, code = TYPES[dt]
    B, n = 3, -(-ctx // bs)
    gen, rng = torch.Generator().manual_seed(hq + ctx), np.random.default_rng(hq + ctx)
    sh = P.make_shape(hq, hkv, D, bs, code)
    drawn = [rows(ctx, hq, hkv, dtype, gen, rng) for _ in range(B)]
    k, v = torch.zeros((2, B, hkv, n * bs, D), dtype=dtype)
    for r in range(B):
        k[r, :, :ctx], v[r, :, :ctx] = drawn[r][1], drawn[r][2]
    k, v = (x.view(B, hkv, n, bs, D).transpose(1, 2).reshape(B * n, hkv, bs, D) for x in (k, v))
    pool = plain64.pack(k, v, bs)
    slots = rng.permutation(B * n)
    placed = torch.empty_like(pool)
    placed[torch.from_numpy(slots)] = pool
    sel = np.tile(np.arange(n, dtype=np.int32), (B, 1))
    q = torch.stack([d[0] for d in drawn])
    out, _ = attend(sh, q.to(DEV), placed.to(DEV), dev(slots.reshape(B, n)), dev(sel), dev([n] * B), dev([ctx] * B))
    for r, (qr, kr, vr, live) in enumerate(drawn):
        want, _, mass, _ = plain64.attention(qr, kr, vr, SCALE)
        assert torch.equal(want, mass)
        reach = float(qr[:, 77].double().max() * 1.5 * SCALE)
        over = ((out[r].double().cpu() - want).abs() / (want * bound(reach, 1 if ctx <= 32 else 2) + 1e-30)).max().item()
        say(f"\n[gpu] hq={hq} hkv={hkv} bs={bs} ctx={ctx} {dt}: {over:.3f} of the bound")
        assert over <= 1
