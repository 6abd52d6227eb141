"""Forms of the 8-bit cache's kernels that only large calls, or long contexts in blocks of 64, take."""
import math

import numpy as np
import pytest
import torch

import plain8
import plain64
from paper_2609_34555_amd import pulse as P
from parity import say
from test_kv4 import attend, check_attention
from test_kv8 import DEV, SCALE, TYPES, D, case_state, dev, same_bytes


def places_of(bs, window, rows, rng):
    """Slots and tokens of two calls: the tokens that requests had before, and the `rows` or more of the second call, among
    them whole blocks that begin at every place of a window of rows, blocks that begin unaligned, requests of one token,
    and rows without a place."""
    before, then, slot = [], [], 0

    def request(start, n):
        nonlocal slot
        t = np.arange(start + n)
        at = (slot + t // bs) * bs + t % bs
        before.extend(at[:start])
        then.extend(at[start:])
        slot += -(-(start + n) // bs)

    while len(then) < rows:
        for place in rng.permutation(window):
            while len(then) % window != place:
                if rng.random() < 0.8:
                    then.append(-1)
                else:
                    request(int(rng.integers(0, bs)), 1)
            request(0 if rng.random() < 0.7 else int(rng.integers(0, bs)), int(rng.integers(1, 4)) * bs)
    slots = rng.permutation(slot + 2)
    move = lambda x: np.array([p if p < 0 else slots[p // bs] * bs + p % bs for p in x], np.int64)  # noqa: E731
    return move(before), move(then), slot + 2


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("bs,hkv", [(16, 8), (32, 12), (64, 16)])
def test_rows_by_whole_blocks(bs, hkv, dt):
    """More than 65536 rows and heads: a workgroup looks at 16 rows (blocks of 16) or 32, and at a block behind them."""
    say(f"\n[gpu] kv8 rows by blocks bs={bs} hkv={hkv} {dt}")
    dtype, code = TYPES[dt]
    rng = np.random.default_rng(bs)
    before, then, n_slots = places_of(bs, min(bs, 32), 65536 // hkv + 1, rng)
    assert len(then) * hkv > 65536
    sh = P.make_shape(hkv, hkv, D, bs, code)
    cache = plain8.Cache(n_slots, hkv, bs, dtype)
    pool = torch.zeros((n_slots, P.pulse_block_bytes(sh)), dtype=torch.uint8, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    gen = torch.Generator().manual_seed(bs)
    for places in (before, then):
        T = len(places)
        x = (torch.randn((2, T, hkv, D), generator=gen) * torch.exp2(torch.randn((2, T, 1, 1), generator=gen))).to(dtype)
        xd = x.to(DEV)
        P.pulse_append_kv(sh, xd[0], hkv * D, xd[1], hkv * D, dev(places, torch.int64), T, pool, n_slots, status)
        assert status.item() == 0
        cache.append(x[0], x[1], [int(p) for p in places])
        same_bytes(pool, cache)


# contexts, selected blocks, query heads, KV heads: blocks of 64, groups of more than 8 heads, so few requests and heads
# and so many blocks that workgroups of four waves are taken
LONG = [
    ([5000], [79], 12, 1),
    ([4095], [64], 16, 1),
    ([9000], [9], 16, 1),                              # the first count beyond one workgroup's
    ([6400, 6400], [100, 100], 32, 2),                 # equal counts
    ([6000, 700, 2500, 64], [94, 11, 40, 1], 12, 1),   # counts that differ
    ([20000, 0, 3001], [300, 0, 20], 24, 2),
    ([65536], [1024], 16, 1),                          # the last that are few enough
    ([65600], [1025], 16, 1),
]


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("case", range(len(LONG)))
def test_attention_of_large_groups_over_blocks_of_64(case, dt):
    ctx, cnt, hq, hkv = LONG[case]
    say(f"\n[gpu] kv8 attention ctx={ctx} cnt={cnt} hq={hq} hkv={hkv} {dt}")
    gen = torch.Generator().manual_seed(100 + case)
    sh, q, pool, table, sel, vals = case_state(ctx, cnt, hq, hkv, 64, dt, gen)
    args = (sh, *(x.to(DEV) for x in (q, pool, table, sel)), dev(cnt), dev(ctx))
    out, lse = attend(*args)
    for r in range(len(ctx)):
        if not cnt[r]:
            assert (out[r] == 0).all() and (lse[r] == -math.inf).all()
            continue
        j = sel[r, : cnt[r]].long()
        k, v = (x[table[r, j].long()].transpose(0, 1).reshape(hkv, -1, D) for x in vals)
        n = (j[:, None] * 64 + torch.arange(64)).view(-1) < ctx[r]
        check_attention(out[r], lse[r], *plain64.attention(q[r], k[:, n], v[:, n], SCALE), int(n.sum()))
    again = attend(*args, ws_fill=0)
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])
