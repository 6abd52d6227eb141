"""How exact the attention of new tokens is where little else than the rounding of its probabilities can be wrong: four
tokens have a probability other than 0 (the others' logits are some hundreds lower), logits are one exact product each,
and values are not negative.  A result is the exact one, moved by no more than the bound, rounded to the 16-bit type: the
type's own rounding leaves no slack."""
import numpy as np
import pytest
import torch

import plain64
from paper_2609_34555_amd import pulse as P
from parity import say
from test_kv4_precision import bound
from test_prompt import CODES, SCALE, TYPES, D, dev, pack

DEV = "cuda"


def drawn(ctx, new, hq, hkv, bs, dt, bits, seed):
    """Queries [T][hq][128], blocks as bytes, keys and values [request][hkv][ctx][128] as the cache holds them."""
    gen, rng = torch.Generator().manual_seed(seed), np.random.default_rng(seed)
    dtype = TYPES[dt]
    q = torch.zeros((sum(new), hq, D))
    q[..., 77] = torch.rand(q.shape[:2], generator=gen) / 2 + 0.5
    level = torch.tensor([0.25, 0.375, 0.5, 0.75, 1.0, 1.5])
    n = [-(-x // bs) for x in ctx]
    kv = torch.zeros((2, sum(n), hkv, bs, D))
    kv[0, ..., 77] = -6144.0
    at = 0
    for x, k, m in zip(ctx, new, n):
        for t in rng.choice(x - k + 1, size=4, replace=False):  # every new token attends to them
            kv[0, at + t // bs, :, t % bs, 77] = level[torch.randint(0, 6, (hkv,), generator=gen)]
        at += m
    kv[1] = torch.randn(kv[1].shape, generator=gen).abs()
    pool, k, v = pack(kv.to(dtype), bits, bs)
    assert torch.equal(k, kv[0].double())
    per, at = [], 0
    for x, m in zip(ctx, n):
        per.append([y[at:at + m].transpose(0, 1).reshape(hkv, -1, D)[:, :x] for y in (k, v)])
        at += m
    return q.to(dtype), pool, per


def between(got, want, rel, dtype):
    """Share of the results that are not between the rounded ends of want * (1 -+ rel)."""
    low, high = ((want * (1 + s * rel)).to(dtype).double() for s in (-1, 1))
    got = got.double().cpu()
    return ((got < low) | (got > high)).double().mean().item()


def rel_of(q, dt, parts):
    """`bound`, and what the last part of a probability leaves: half a step of half a step, once for each part."""
    reach = float(q[..., 77].double().max() * 1.5 * SCALE)
    return bound(reach, 2) + (torch.finfo(TYPES[dt]).eps / 2) ** parts


@pytest.mark.parametrize("dt", ["bf16", "f16"])
def test_the_bound_tells_one_part_from_two(dt):
    """The probabilities cut on the CPU, sums in 64 bits."""
    dtype = TYPES[dt]
    q, _, per = drawn([300], [1], 32, 2, 16, dt, 16, 1)
    k, v = per[0]
    want = plain64.attention(q[0], k, v, SCALE)[0]
    for parts in (1, 2):
        out = torch.zeros_like(want)
        for h in range(32):
            x = k[h // 16, :, 77] * q[0, h, 77].double() * SCALE
            p = torch.exp(x - x.max())
            cut, rest = torch.zeros_like(p), p.clone()
            for _ in range(parts):
                part = rest.float().to(dtype).double()
                cut, rest = cut + part, rest - part
            out[h] = (cut @ v[h // 16]) / p.sum()
        out = out.to(dtype)
        assert between(out, want, rel_of(q, dt, parts), dtype) == 0
        if parts == 1:
            # four roundings of a third of a half step on average move their sum by about an eighth of the result's half
            # step, so about one result in twelve is rounded to its other neighbour; two parts: none
            assert between(out, want, rel_of(q, dt, 2), dtype) > 1 / 24


# contexts, new tokens, query heads, KV heads, bs, bits, parts of a probability: two where the rows of a request are 32 (16
# bits) or 64 (8 bits) on average, or fewer
CASES = [
    ([3000, 900, 60], [5, 3, 6], 16, 4, 16, 16, 2),
    ([3000, 900, 60], [5, 3, 6], 16, 4, 16, 8, 2),
    ([9000], [1], 16, 1, 64, 16, 2),
    ([9000], [1], 16, 1, 32, 8, 2),
    ([70, 40], [1, 1], 3, 3, 32, 16, 2),
    ([2000, 2000], [8, 8], 32, 8, 16, 16, 2),        # 32 rows a request
    ([2000, 2000], [9, 8], 32, 8, 16, 16, 1),        # and more
    ([2000, 2000], [16, 16], 32, 8, 64, 8, 2),       # 64 over codes
    ([2000, 2000], [17, 16], 32, 8, 64, 8, 1),
    ([2000, 2000], [8, 8], 32, 8, 16, 4, 1),
    ([6001], [300], 32, 8, 16, 16, 1),               # tiles of 128 rows, split over the context
    ([2600], [2500], 32, 8, 16, 16, 1),              # of 256
    ([900], [64], 8, 2, 16, 8, 1),
]


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_bits_of_a_probability(case, dt):
    ctx, new, hq, hkv, bs, bits, parts = CASES[case]
    dtype = TYPES[dt]
    q, pool, per = drawn(ctx, new, hq, hkv, bs, dt, bits, case)
    n, B, T = [-(-x // bs) for x in ctx], len(ctx), sum(new)
    slots = np.random.default_rng(case).permutation(len(pool))
    placed = torch.empty_like(pool)
    placed[torch.from_numpy(slots)] = pool
    table, at = np.full((B, max(n)), -1, np.int32), 0
    for r, m in enumerate(n):
        table[r, :m] = slots[at:at + m]
        at += m
    sh = P.make_shape(hq, hkv, D, bs, CODES[dt, bits])
    nb = P.pulse_prompt_workspace_bytes(sh, B, T, max(n))
    ws = torch.full((nb,), 255, dtype=torch.uint8, device=DEV)
    out = torch.zeros((T, hq, D), dtype=dtype, device=DEV)
    status = dev([0])
    P.pulse_prompt_attn(sh, q.to(DEV), hq * D, dev(np.concatenate([[0], np.cumsum(new)])), T, dev(ctx), B, placed.to(DEV),
                        len(pool), dev(table), max(n), SCALE, out, hq * D, None, status, ws, nb)
    assert status.item() == 0
    row, off = 0, []
    for r in range(B):
        k, v = per[r]
        for i in range(new[r]):
            if i < 20 or i > new[r] - 3:
                p = ctx[r] - new[r] + i + 1
                want, _, mass, _ = plain64.attention(q[row], k[:, :p], v[:, :p], SCALE)
                assert torch.equal(want, mass)
                off.append(between(out[row], want, rel_of(q, dt, parts), dtype))
            row += 1
    say(f"\n[gpu] prompt bits={bits} rows={new} hq={hq} hkv={hkv} {dt} in {parts}: {max(off)}")
    assert max(off) == 0
