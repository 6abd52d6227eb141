"""Blocks whose tokens behind the end of a context hold what an earlier owner of the slot left there, infinities and NaN
among it: a 16-bit cache's results do not depend on them."""
import numpy as np
import pytest
import torch

import plain64
from paper_2609_34555_amd import pulse as P
from parity import say
from test_kv4 import DEV, SCALE, TYPES, D, attend, check_attention, dev
from test_kv4_step import Run

pytestmark = pytest.mark.gpu

# what a stale 16-bit element may be: NaN of either sign, infinities, the largest finite value
STALE = {"bf16": (0x7FC1, 0xFFFF, 0x7F80, 0xFF80, 0x7F7F), "f16": (0x7E01, 0xFFFF, 0x7C00, 0xFC00, 0x7BFF)}


def stale(shape, dt, gen):
    v = torch.tensor(np.array(STALE[dt], np.uint16).view(np.int16))
    return v[torch.randint(0, len(v), shape, generator=gen)].view(TYPES[dt][0])


# contexts, selected blocks (the last one among them), query heads, KV heads, bs
CASES = [
    ([1], [1], 4, 1, 16),
    ([1, 7, 8, 9, 15, 16, 17, 31], [1, 1, 1, 1, 1, 1, 2, 2], 8, 2, 16),
    ([33, 63, 64, 1], [2, 2, 2, 1], 16, 2, 32),                       # blocks of one step
    ([65, 100, 127, 30], [2, 2, 2, 1], 12, 1, 64),                    # of two steps: the second, or both, without a token
    ([1999, 1201], [125, 60], 32, 8, 16),                             # several workgroups per head, counts that differ
    ([4001], [251], 16, 1, 16),
    ([1000 + r for r in range(70)], [9 + r % 5 for r in range(70)], 2, 2, 32),
]


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_attention_does_not_read_behind_a_context(case, dt):
    ctx, cnt, hq, hkv, bs = CASES[case]
    say(f"\n[gpu] stale tokens ctx={ctx[:4]} hq={hq} hkv={hkv} bs={bs} {dt}")
    dtype, code, _ = TYPES[dt]
    gen = torch.Generator().manual_seed(case)
    B, n = len(ctx), [-(-x // bs) for x in ctx]
    total = sum(cnt)
    slots = np.random.default_rng(case).permutation(total + 2)
    keys, values = torch.randn((2, total + 2, hkv, bs, D), generator=gen).to(dtype)
    table, sel = np.full((B, max(n)), -1, np.int32), np.full((B, max(cnt)), -1, np.int32)
    live = torch.ones((total + 2, bs), dtype=torch.bool)
    g = 0
    for r in range(B):
        j = np.sort(np.random.default_rng(r).choice(n[r] - 1, size=cnt[r] - 1, replace=False)) if cnt[r] > 1 else []
        j = np.append(np.asarray(j, int), n[r] - 1)
        sel[r, : cnt[r]], table[r, j] = j, slots[g:g + cnt[r]]
        live[table[r, n[r] - 1]] = torch.arange(bs) < ctx[r] - (n[r] - 1) * bs
        g += cnt[r]
    sh = P.make_shape(hq, hkv, D, bs, code)
    q = torch.randn((B, hq, D), generator=gen).to(dtype)
    got = []
    for rest in (torch.zeros(keys.shape, dtype=dtype), stale(keys.shape, dt, gen)):
        k, v = (torch.where(live[:, None, :, None], x, rest) for x in (keys, values))
        pool = torch.cat([k.reshape(total + 2, -1), v.transpose(2, 3).reshape(total + 2, -1)], 1).contiguous()
        got.append(attend(sh, q.to(DEV), pool.to(DEV), dev(table), dev(sel), dev(cnt), dev(ctx)))
    for a, b in zip(*got):
        assert torch.equal(a, b) and not b.isnan().any()
    for r in range(B):
        j = torch.from_numpy(sel[r, : cnt[r]]).long()
        s = torch.from_numpy(table)[r, j].long()
        m = live[s].view(-1)
        kk, vv = (x[s].double().transpose(0, 1).reshape(hkv, -1, D)[:, m] for x in (keys, values))
        check_attention(got[1][0][r], got[1][1][r], *plain64.attention(q[r], kk, vv, SCALE), int(m.sum()))


@pytest.mark.parametrize("dt,hq,hkv,bs", [("bf16", 8, 2, 16), ("f16", 24, 3, 32), ("bf16", 12, 1, 64)])
@pytest.mark.parametrize("four", [True, False])
def test_prompt_and_tokens_in_slots_taken_again(dt, hq, hkv, bs, four):
    """Maps, rows and attention over a pool that no one has cleared; a request ends, its slots go back to the free list
    and a new request takes them."""
    say(f"\n[gpu] slots taken again {dt} hq={hq} hkv={hkv} bs={bs} four={four}")
    dtype, code16, code4 = TYPES[dt]
    prompt = [37, 1, 160, 64]
    st = Run([x + 40 for x in prompt], 20, hq, hkv, bs, code4 if four else code16, dtype, 5)
    gen = torch.Generator().manual_seed(1)
    if four:
        st.pool.fill_(255)  # every scale byte NaN
    else:
        st.pool.copy_(stale((st.pool.numel() // 2,), dt, gen).view(torch.uint8).view_as(st.pool))
    ctx, kept = list(prompt), [[] for _ in prompt]

    def step(new):
        st.ctx.copy_(dev(ctx))
        st.new.copy_(dev(new))
        x = st.rows(sum(new) + 2)
        st.buffers(x.shape[0])
        st.write(x)
        T = sum(new)
        k, v = st.k[:T].cpu(), x[:T, (hq + hkv) * D:].unflatten(1, (hkv, D)).cpu()
        k, v = (plain64.quantise(t)[2] for t in (k, v)) if four else (k.double(), v.double())
        at = 0
        for r, c in enumerate(new):
            kept[r].append((k[at:at + c], v[at:at + c]))
            at += c
        # (the first rows' queries, one a request)
        q = st.q[: len(new)]
        cnt = (st.blk[1:] - st.blk[:-1]).int()
        P.pulse_sparse_decode_attn(st.sh, q, st.pool, st.n_slots, st.table, st.mb, st.sel, cnt, st.mb, st.ctx, st.B, SCALE,
                                   st.out, st.lse, st.status, st.ws, st.ws.numel())
        assert st.status.item() == 0
        for r in range(len(new)):
            kk, vv = (torch.cat([p[i] for p in kept[r]]).transpose(0, 1) for i in (0, 1))
            assert kk.shape[1] == ctx[r]
            check_attention(st.out[r], st.lse[r], *plain64.attention(q[r].cpu(), kk, vv, SCALE), ctx[r])

    step(prompt)
    for i in range(3):
        ctx = [c + 1 for c in ctx]
        step([1] * len(prompt))
        # request 2 ends; its slots return, its place goes to a shorter prompt
        n = -(-ctx[2] // bs)
        head = st.head.item() - n
        st.free[head:head + n] = st.table[2, :n].flip(0)
        st.head.fill_(head)
        st.table[2] = -1
        ctx = [c + 1 for c in ctx]
        ctx[2], kept[2] = 21 + 9 * i, []
        step([1, 1, ctx[2], 1])
