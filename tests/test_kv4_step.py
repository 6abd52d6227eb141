"""The 4-bit cache inside the steps: digests of its blocks, their recall, the chained layer-step, and a run of a
prompt and tokens through tables, norms and rotation, cache and attention, eager and as a replayed graph."""
import math

import numpy as np
import pytest
import torch

import plain64
from paper_2609_34555_amd import harness as H
from paper_2609_34555_amd import pulse as P
from parity import say
from test_kv4 import DEV, SCALE, TYPES, D, check_attention, dev, equal

pytestmark = pytest.mark.gpu


def host_store(data):
    """Pinned memory holding the bytes of `data`."""
    store = H.PinnedStore(data.numel())
    torch.from_numpy(store.numpy(tuple(data.shape), np.uint8)).copy_(data)
    return store


# contexts, hq, hkv, bs, dtype, middle blocks: blocks of 2 to 17 KiB, of a whole number of 8 KiB chunks (bs 64, 16 heads)
LAYERS = [
    ([1000, 517], 8, 2, 16, "bf16", 9),
    ([700], 4, 1, 32, "f16", 3),
    ([999, 1, 64, 2000], 24, 3, 16, "f16", 11),
    ([1500, 1290], 32, 8, 16, "bf16", 20),
    ([2500], 16, 16, 64, "bf16", 12),
    ([3000, 100], 8, 8, 64, "f16", 13),
]


@pytest.mark.parametrize("ctx,hq,hkv,bs,dt,k_mid", LAYERS)
def test_layer_step(ctx, hq, hkv, bs, dt, k_mid):
    say(f"\n[gpu] kv4 layer-step ctx={ctx} hq={hq} hkv={hkv} bs={bs} {dt}")
    dtype, _, code = TYPES[dt]
    gen = torch.Generator().manual_seed(sum(ctx))
    B, n = len(ctx), [-(-x // bs) for x in ctx]
    off = np.concatenate([[0], np.cumsum(n)])
    total, mb, solo = int(off[-1]), max(n), hkv - 1
    kv = torch.randn((2, total, hkv, bs, D), generator=gen).to(dtype)
    data = plain64.pack(kv[0], kv[1], bs)
    for r in range(B):  # behind the last token: anything
        left = n[r] * bs - ctx[r]
        if left:
            b = data.view(total, hkv, 136 * bs)[off[r + 1] - 1]
            b[:, (bs - left) * 64:bs * 64] = 0x77
            b[:, 128 * bs + 4 * (bs - left):132 * bs] = 255
    store = host_store(data)
    sh = P.make_shape(hq, hkv, D, bs, code)
    blk_off, ctx_len = dev(off, torch.int64), dev(ctx)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    # digests from host and from device memory: extremes of the values that the codes stand for
    keys, _ = plain64.unpack(data, hkv, bs)
    got = [torch.zeros((total, 2, D), dtype=dtype, device=DEV) for _ in range(2)]
    P.pulse_build_digests(sh, store.ptr, blk_off, ctx_len, B, total, solo, got[0], status)
    P.pulse_build_digests(sh, data.to(DEV), blk_off, ctx_len, B, total, solo, got[1], status)
    assert status.item() == 0
    for r in range(B):
        for j in range(n[r]):
            k = keys[off[r] + j, solo, : min(bs, ctx[r] - j * bs)]
            for d in got:
                assert equal(d[off[r] + j, 0], k.amin(0)) and equal(d[off[r] + j, 1], k.amax(0))
    # one layer-step; the first blocks of every request are resident
    k_max = k_mid + 3
    res = [(r, j) for r in range(B) for j in range(n[r]) if j in (0, 3, n[r] - 1)]
    n_slots = len(res) + B * k_max
    table0 = torch.full((B, mb), -1, dtype=torch.int32)
    pool0 = torch.full((n_slots, data.shape[1]), 9, dtype=torch.uint8)
    for s, (r, j) in enumerate(res):
        table0[r, j], pool0[s] = s, data[off[r] + j]
    q = torch.randn((B, hq, D), generator=gen).to(dtype).to(DEV)
    free = torch.arange(len(res), n_slots, dtype=torch.int32, device=DEV).flip(0).contiguous()
    want = None
    for how in ("calls", "chain", "noalloc", "release"):
        table, pool = (table0.to(DEV), pool0.to(DEV)) if how != "release" else (table, pool)  # noqa: F821
        if how != "release":
            head = torch.zeros(1, dtype=torch.int32, device=DEV)
            stats = torch.zeros(2, dtype=torch.int64, device=DEV)
            nb = P.pulse_workspace_bytes(sh, B, k_max, total)
            ws = torch.full((nb,), 255, dtype=torch.uint8, device=DEV)
        sel = torch.full((B, k_max), -5, dtype=torch.int32, device=DEV)
        cnt = torch.zeros(B, dtype=torch.int32, device=DEV)
        out, lse = torch.zeros((B, hq, D), device=DEV), torch.zeros((B, hq), device=DEV)
        km = dev([k_mid] * B)
        if how == "calls":
            P.pulse_select_solohead(sh, q, got[0], blk_off, B, total, solo, km, 1, 2, k_max, sel, cnt, None, status,
                                    ws, nb)
            P.pulse_recall_gather(sh, store.ptr, blk_off, B, sel, cnt, k_max, table, mb, free, head, free.numel(),
                                  pool, n_slots, stats, status, ws, nb)
            P.pulse_sparse_decode_attn(sh, q, pool, n_slots, table, mb, sel, cnt, k_max, ctx_len, B, SCALE, out, lse,
                                       status, ws, nb)
        else:
            a = P.pulse_layer_args()
            a.shape, a.B, a.total_blocks, a.solo_kv_head = sh, B, total, solo
            a.n_sink_blocks, a.n_local_blocks, a.k_max, a.max_blocks = 1, 2, k_max, mb
            a.n_free, a.n_slots, a.sm_scale, a.host_kv = free.numel(), n_slots, SCALE, store.ptr
            a.release_previous = how == "release"
            for f, t in dict(ctx_len=ctx_len, blk_off=blk_off, q=q, digests=got[0], k_mid=km, sel_idx=sel, sel_cnt=cnt,
                             block_table=table, free_slots=free, free_head=head, slot_pool=pool, stats=stats, out=out,
                             lse=lse, dev_status=status).items():
                setattr(a, f, t.data_ptr())
            if how != "noalloc":
                a.ws, a.ws_bytes = ws.data_ptr(), nb
            (P.pulse_decode_layer_noalloc if how == "noalloc" else P.pulse_decode_layer)(a)
            if how == "noalloc":
                table, pool, head, stats, ws = None, None, None, None, None
        assert status.item() == 0
        if how == "calls":
            # the selection on the digests' scores is the 16-bit path's; the recalled blocks are the store's bytes
            for r in range(B):
                j = sel[r, : cnt[r]].cpu().long()
                assert len(j) == min(n[r], k_max)
                slots = table[r].cpu()[j].long()
                assert len(set(slots.tolist())) == len(j) and (slots >= 0).all()
                assert torch.equal(pool.cpu()[slots], data[off[r] + j])
                k, v = (x.transpose(0, 1).reshape(hkv, -1, D) for x in plain64.unpack(data[off[r] + j], hkv, bs))
                m = (j[:, None] * bs + torch.arange(bs)).view(-1) < ctx[r]
                check_attention(out[r], lse[r], *plain64.attention(q[r].cpu(), k[:, m], v[:, m], SCALE), int(m.sum()))
            moved = int((table0 >= 0).sum())
            moved = int((table.cpu() >= 0).sum()) - moved
            assert stats[1].item() == moved * data.shape[1] and head.item() == moved > 0
            used = torch.zeros(n_slots, dtype=torch.bool)
            used[table.cpu()[table.cpu() >= 0].long()] = True
            assert (pool.cpu()[~used] == 9).all()
            want = [x.clone() for x in (sel, cnt, out, lse, table, pool, head, stats)]
        elif how == "noalloc":
            assert all(torch.equal(x, y) for x, y in zip((sel, cnt, out, lse), want))
            # the next step releases a recall made with a workspace of its own
            table, pool, head, stats, ws = keep
        else:
            assert all(torch.equal(x, y) for x, y in zip((sel, cnt, out, lse, table, pool, head, stats), want))
        if how == "chain":
            keep = (table, pool, head, stats, ws)
    store.free()


def test_recall_of_more_than_the_streaming_store_size():
    """More than 256 MiB of 17 KiB blocks in one recall (written past the cache)."""
    bs, hkv, n = 16, 8, 16384
    sh = P.make_shape(32, hkv, D, bs, P.PULSE_BF16_KV4)
    U = P.pulse_block_bytes(sh)
    store = H.PinnedStore(n * U)
    host = torch.from_numpy(store.numpy((n, U), np.uint8))
    host.copy_(torch.randint(0, 255, (n, U), dtype=torch.uint8, device=DEV))
    k_max = n // 4 - 3  # four requests, all but three blocks of each
    blk = dev(np.arange(5) * (n // 4), torch.int64)
    sel = torch.arange(k_max, dtype=torch.int32, device=DEV).add(2).repeat(4, 1).contiguous()
    table = torch.full((4, n // 4), -1, dtype=torch.int32, device=DEV)
    free = torch.randperm(4 * k_max + 5, device=DEV).int()
    pool = torch.zeros((4 * k_max + 5, U), dtype=torch.uint8, device=DEV)
    head, status = torch.zeros((2, 1), dtype=torch.int32, device=DEV)
    stats = torch.zeros(2, dtype=torch.int64, device=DEV)
    nb = P.pulse_workspace_bytes(sh, 4, k_max, 0)
    ws = torch.zeros(nb, dtype=torch.uint8, device=DEV)
    P.pulse_recall_gather(sh, store.ptr, blk, 4, sel, dev([k_max] * 4), k_max, table, n // 4, free, head, free.numel(),
                          pool, pool.shape[0], stats, status, ws, nb)
    assert status.item() == 0 and stats[1].item() == 4 * k_max * U > 256 << 20
    for r in range(4):
        assert torch.equal(pool[table[r, 2:2 + k_max].long()].cpu(), host[r * (n // 4) + 2:r * (n // 4) + 2 + k_max])
        assert (table[r, :2] == -1).all() and (table[r, 2 + k_max:] == -1).all()
    store.free()


def test_irq_step_with_4_bit_offload_layers():
    """The layer-wise scheduler on 4-bit offload layers: the results of the chained layer-step."""
    gen = torch.Generator().manual_seed(4)
    ctx, hq, hkv, bs = 900, 8, 2, 16
    n = -(-ctx // bs)
    sh = P.make_shape(hq, hkv, D, bs, P.PULSE_BF16_KV4)
    layers = []
    for _ in range(3):
        kv = torch.randn((2, n, hkv, bs, D), generator=gen).bfloat16()
        data = plain64.pack(kv[0], kv[1], bs)
        s = dict(store=host_store(data), q=torch.randn((1, hq, D), generator=gen).bfloat16().to(DEV),
                 ctx_len=dev([ctx]), blk_off=dev([0, n], torch.int64), k_mid=dev([10]))
        s["digests"] = torch.zeros((n, 2, D), dtype=torch.bfloat16, device=DEV)
        s["status"] = torch.zeros(1, dtype=torch.int32, device=DEV)
        P.pulse_build_digests(sh, s["store"].ptr, s["blk_off"], s["ctx_len"], 1, n, 0, s["digests"], s["status"])
        layers.append(s)
    nb = P.pulse_workspace_bytes(sh, 1, 16, n)

    def args(s):
        o = s["o"] = dict(sel_idx=torch.full((1, 16), -1, dtype=torch.int32, device=DEV), sel_cnt=dev([0]),
                          block_table=torch.full((1, n), -1, dtype=torch.int32, device=DEV), free_head=dev([0]),
                          slot_pool=torch.zeros((20, P.pulse_block_bytes(sh)), dtype=torch.uint8, device=DEV),
                          stats=torch.zeros(2, dtype=torch.int64, device=DEV), out=torch.zeros((1, hq, D), device=DEV),
                          lse=torch.zeros((1, hq), device=DEV))
        s["free"], s["ws"] = dev(np.arange(20)), torch.zeros(nb, dtype=torch.uint8, device=DEV)
        a = P.pulse_layer_args()
        a.shape, a.B, a.total_blocks, a.n_sink_blocks, a.n_local_blocks, a.k_max, a.max_blocks = sh, 1, n, 1, 2, 16, n
        a.n_free, a.n_slots, a.sm_scale, a.host_kv, a.ws_bytes = 20, 20, SCALE, s["store"].ptr, nb
        for f, t in dict(o, ctx_len=s["ctx_len"], blk_off=s["blk_off"], q=s["q"], digests=s["digests"], k_mid=s["k_mid"],
                         free_slots=s["free"], dev_status=s["status"], ws=s["ws"]).items():
            setattr(a, f, t.data_ptr())
        return a

    for s in layers:
        P.pulse_decode_layer(args(s))
        s["want"] = {k: v.clone() for k, v in s["o"].items()}
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    sched = P.IrqScheduler(*streams)
    packs = [args(s) for s in layers]
    torch.cuda.synchronize()
    sched.step(packs, [])
    for s in layers:
        assert s["status"].item() == 0
        assert all(torch.equal(s["o"][k], s["want"][k]) for k in s["want"])
    sched.destroy()
    for s in layers:
        s["store"].free()


class Run:
    """A batch that a serving program carries through prompt and decode steps; rows of the projections are inputs."""

    def __init__(self, prompt, steps, hq, hkv, bs, code, dtype, seed):
        self.B, self.hq, self.hkv, self.bs, self.dtype = len(prompt), hq, hkv, bs, dtype
        self.sh = P.make_shape(hq, hkv, D, bs, code)
        gen = torch.Generator(device=DEV)
        gen.manual_seed(seed)
        self.mb = -(-(max(prompt) + steps) // bs)
        self.n_slots = sum(-(-(x + steps) // bs) for x in prompt)
        self.pool = torch.randint(0, 255, (self.n_slots, P.pulse_block_bytes(self.sh)), generator=gen, device=DEV,
                                  dtype=torch.uint8)
        self.table = torch.full((self.B, self.mb), -1, dtype=torch.int32, device=DEV)
        self.free = torch.randperm(self.n_slots, generator=gen, device=DEV).int()
        self.head, self.status = torch.zeros((2, 1), dtype=torch.int32, device=DEV)
        self.ctx, self.new = dev(prompt), dev(prompt)
        self.blk = torch.zeros(self.B + 1, dtype=torch.int64, device=DEV)
        self.tok = torch.zeros(self.B + 1, dtype=torch.int32, device=DEV)
        self.sel = torch.arange(self.mb, dtype=torch.int32, device=DEV).repeat(self.B, 1).contiguous()
        self.qw, self.kw = torch.randn((2, D), generator=gen, device=DEV).add_(1).to(dtype)
        self.inv = 10000.0 ** (-torch.arange(0, D, 2, dtype=torch.float64, device=DEV) / D)
        self.gen = gen
        self.out = torch.zeros((self.B, hq, D), device=DEV)
        self.lse = torch.zeros((self.B, hq), device=DEV)
        nb = P.pulse_workspace_bytes(self.sh, self.B, self.mb, 0)
        self.ws = torch.full((nb,), 255, dtype=torch.uint8, device=DEV)

    def rows(self, T):
        return torch.randn((T, (self.hq + 2 * self.hkv) * D), generator=self.gen, device=DEV).to(self.dtype)

    def buffers(self, T):
        self.T = T
        nb = P.pulse_tables_workspace_bytes(self.sh, self.B, T)
        self.tws = torch.full((nb,), 255, dtype=torch.uint8, device=DEV)
        self.slot_map = torch.zeros(T, dtype=torch.int64, device=DEV)
        self.pos = torch.zeros(T, dtype=torch.int32, device=DEV)
        self.q = torch.zeros((T, self.hq, D), dtype=self.dtype, device=DEV)
        self.k = torch.zeros((T, self.hkv, D), dtype=self.dtype, device=DEV)

    def write(self, x):
        """Maps, norms and rotation, rows into the cache."""
        w, hq, hkv = x.shape[1], self.hq, self.hkv
        P.pulse_build_tables(self.sh, self.ctx, self.new, self.B, self.table, self.mb, self.free, self.head,
                             self.n_slots, self.n_slots, self.blk, self.tok, self.slot_map, self.pos, self.T,
                             self.status, self.tws, self.tws.numel())
        P.pulse_qk_norm_rope(self.sh, x, w, x[:, hq * D:], w, self.T, self.pos, self.qw, self.kw, 1e-6, self.inv, D, 0,
                             self.q, hq * D, self.k, hkv * D)
        P.pulse_append_kv(self.sh, self.k, hkv * D, x[:, (hq + hkv) * D:], w, self.slot_map, self.T, self.pool,
                          self.n_slots, self.status)

    def attend(self):
        """A decode step's attention over everything; blocks per request from the maps' offsets."""
        cnt = (self.blk[1:] - self.blk[:-1]).int()
        P.pulse_sparse_decode_attn(self.sh, self.q, self.pool, self.n_slots, self.table, self.mb, self.sel, cnt, self.mb,
                                   self.ctx, self.B, SCALE, self.out, self.lse, self.status, self.ws, self.ws.numel())

    def snapshot(self):
        torch.cuda.synchronize()
        return [t.clone() for t in (self.out, self.lse, self.table, self.head, self.pool, self.slot_map, self.pos, self.q,
                                    self.k, self.blk, self.tok, self.status)]


@pytest.mark.parametrize("dt,hq,hkv,bs", [("bf16", 8, 2, 16), ("f16", 24, 3, 32)])
@pytest.mark.parametrize("four", [True, False])
def test_prompt_and_tokens(dt, hq, hkv, bs, four):
    say(f"\n[gpu] prompt and tokens {dt} hq={hq} hkv={hkv} bs={bs} four={four}")
    dtype, code16, code4 = TYPES[dt]
    prompt, steps = [37, 1, 160, 64], 18
    st = Run(prompt, steps, hq, hkv, bs, code4 if four else code16, dtype, 11)
    if not four:
        st.pool.zero_()  # a 16-bit block's tokens behind the last one must be zero
    keys = [[] for _ in prompt]  # what the cache is to hold, per request
    ctx = list(prompt)
    for step in range(steps + 1):
        new = prompt if step == 0 else [1] * len(prompt)
        if step:
            ctx = [c + 1 for c in ctx]
            st.ctx += 1
        st.new.copy_(dev(new))
        T = sum(new) + (3 if step % 2 else 0)  # some rows behind the last token
        x = st.rows(T)
        st.buffers(T)
        st.write(x)
        assert st.status.item() == 0
        # q and k of every new row, by the formula; then k and v as the cache holds them
        pos = torch.cat([torch.arange(c - n, c) for c, n in zip(ctx, new)])
        for got, part, w in ((st.q, x[:, : hq * D], st.qw), (st.k, x[:, hq * D:(hq + hkv) * D], st.kw)):
            rows = part[: len(pos)].unflatten(1, (-1, D))
            ref, size = plain64.norm_rope(rows, w, 1e-6, pos, st.inv, D, 0)
            err = (got[: len(pos)].double().cpu() - ref).abs()
            before = size * 24 * 2.0**-24
            assert (err <= (ref.abs() + before) * torch.finfo(dtype).eps / 2 + before
                    + torch.finfo(dtype).tiny * torch.finfo(dtype).eps).all()
            assert (got[len(pos):] == 0).all()
        k, v = st.k[: len(pos)].cpu(), x[: len(pos), (hq + hkv) * D:].unflatten(1, (hkv, D)).cpu()
        k, v = (plain64.quantise(t)[2] for t in (k, v)) if four else (k.double(), v.double())
        at = 0
        for r, n in enumerate(new):
            keys[r].append((k[at:at + n], v[at:at + n]))
            at += n
        if step == 0:
            continue
        st.attend()
        assert st.status.item() == 0
        for r in range(len(prompt)):
            kk, vv = (torch.cat([p[i] for p in keys[r]]).transpose(0, 1) for i in (0, 1))
            ref = plain64.attention(st.q[r].cpu(), kk, vv, SCALE)
            check_attention(st.out[r], st.lse[r], *ref, ctx[r])
    # every row back from the cache, in the order of the requests
    total = sum(ctx)
    m = torch.cat([st.table[r, torch.arange(c, device=DEV) // bs].long() * bs + torch.arange(c, device=DEV) % bs
                   for r, c in enumerate(ctx)])
    back = torch.zeros((2, total, hkv, D), dtype=dtype, device=DEV)
    P.pulse_load_kv(st.sh, st.pool, st.n_slots, m, total, back[0], hkv * D, back[1], hkv * D, st.status)
    for i in (0, 1):
        assert equal(back[i], torch.cat([p[i] for r in keys for p in r]))


def test_captured_decode_step_replays_as_eager():
    """Lengths counted up, maps, norms, rows and attention captured once and replayed over block boundaries, with the
    program's own eager work between; an eager twin does the same steps."""
    dtype, _, code = TYPES["bf16"]
    prompt, steps = [30, 5, 100], 21

    def start():
        st = Run(prompt, steps, 8, 2, 16, code, dtype, 3)
        x = st.rows(sum(prompt))
        st.buffers(sum(prompt))
        st.write(x)
        st.new.fill_(1)
        st.x = torch.zeros((5, x.shape[1]), dtype=dtype, device=DEV)  # two rows behind the last token
        st.buffers(5)
        return st

    def step(st):
        st.ctx.add_(1)
        st.write(st.x)
        st.attend()

    eager, st = start(), start()
    side = torch.cuda.Stream()
    rows = [eager.rows(5) for _ in range(steps)]
    for s in (eager, st):
        s.x.copy_(rows[0])
    torch.cuda.synchronize()
    step(eager)
    with torch.cuda.stream(side):
        step(st)
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip(eager.snapshot(), st.snapshot()):
        assert torch.equal(a, b)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        step(st)
    for i in range(1, steps):
        for s in (eager, st):
            s.x.copy_(rows[i])
        g.replay()
        step(eager)
        torch.cuda.synchronize()
        for n, (a, b) in enumerate(zip(eager.snapshot(), st.snapshot())):
            assert torch.equal(a, b), (i, n)
    assert eager.status.item() == 0 and eager.head.item() == eager.n_slots  # every slot was taken


@pytest.mark.parametrize("ctx,shared", [(40, False), (40, True), (1500, False), (1500, True)])
def test_resident_layer_of_a_4_bit_cache(ctx, shared):
    """A normal layer whose cache is held in 4 bits: the attention's output, its bf16 copy (also where it lies over the
    queries, which takes a launch of its own) and the FFN on it."""
    say(f"\n[gpu] kv4 resident layer ctx={ctx} shared={shared}")
    B, hq, hkv, bs, F = 3, 8, 2, 16, 264
    st = Run([ctx - r for r in range(B)], 0, hq, hkv, bs, P.PULSE_BF16_KV4, torch.bfloat16, 7)
    x = st.rows(sum(ctx - r for r in range(B)))
    st.buffers(x.shape[0])
    st.write(x)
    q = torch.randn((B, hq, D), device=DEV).bfloat16()
    st.q = q
    st.attend()
    want, want_lse = st.out.clone(), st.lse.clone()
    assert st.status.item() == 0
    gen = torch.Generator(device=DEV).manual_seed(1)
    wgu, wd = (torch.randn(s, generator=gen, device=DEV).mul_(0.02).bfloat16() for s in ((2 * F, hq * D), (hq * D, F)))
    bufs = {k: torch.zeros((B, n), dtype=torch.bfloat16, device=DEV) for k, n in (("x", hq * D), ("gu", 2 * F), ("h", F),
                                                                                  ("y", hq * D))}
    q2 = q.clone()
    xb = q2 if shared else bufs["x"]
    cnt = (st.blk[1:] - st.blk[:-1]).int()
    out, lse = torch.zeros_like(want), torch.zeros_like(want_lse)
    n = P.pulse_normal_layer()
    n.shape, n.B, n.n_slots, n.max_blocks, n.k_max, n.sm_scale, n.d_ff, n.ws_bytes = (
        st.sh, B, st.n_slots, st.mb, st.mb, SCALE, F, st.ws.numel())
    for f, t in dict(q=q2, slot_pool=st.pool, block_table=st.table, sel_idx=st.sel, sel_cnt=cnt, ctx_len=st.ctx, out=out,
                     lse=lse, ws=st.ws, w_gate_up=wgu, w_down=wd, x=xb, gu=bufs["gu"], h=bufs["h"], y=bufs["y"],
                     dev_status=st.status).items():
        setattr(n, f, t.data_ptr())
    # one offload layer beside it, of the same cache type
    kv = torch.randn((2, 4, hkv, bs, D)).bfloat16()
    store = host_store(plain64.pack(kv[0], kv[1], bs))
    dig = torch.zeros((4, 2, D), dtype=torch.bfloat16, device=DEV)
    o = dict(ctx_len=dev([64]), blk_off=dev([0, 4], torch.int64), q=q[:1].contiguous(), digests=dig, k_mid=dev([4]),
             sel_idx=dev([[0] * 4]), sel_cnt=dev([0]), block_table=dev([[-1] * 4]), free_slots=dev(np.arange(4)),
             free_head=dev([0]), slot_pool=torch.zeros((4, P.pulse_block_bytes(st.sh)), dtype=torch.uint8, device=DEV),
             stats=torch.zeros(2, dtype=torch.int64, device=DEV), out=torch.zeros((1, hq, D), device=DEV),
             dev_status=st.status)
    nb = P.pulse_workspace_bytes(st.sh, 1, 4, 4)
    ws = torch.zeros(nb, dtype=torch.uint8, device=DEV)
    a = P.pulse_layer_args()
    a.shape, a.B, a.total_blocks, a.k_max, a.max_blocks, a.n_free, a.n_slots, a.sm_scale = st.sh, 1, 4, 4, 4, 4, 4, SCALE
    a.host_kv, a.ws, a.ws_bytes = store.ptr, ws.data_ptr(), nb
    for f, t in o.items():
        setattr(a, f, t.data_ptr())
    sched = P.IrqScheduler(torch.cuda.Stream(), torch.cuda.Stream())
    torch.cuda.synchronize()
    stats, _ = sched.step([a], [n], mode="blocking")
    torch.cuda.synchronize()
    assert st.status.item() == 0 and stats["normal_layers"] == 1
    assert torch.equal(out, want) and torch.equal(lse, want_lse)
    assert torch.equal(xb.view(B, hq, D), want.bfloat16())
    xd, g64 = xb.view(B, -1).double().cpu(), wgu.double().cpu()
    # one rounding to bf16 and fp32 sums of products
    for got, ref, mass in ((bufs["gu"], xd @ g64.T, xd.abs() @ g64.abs().T),
                           (bufs["y"], bufs["h"].double().cpu() @ wd.double().cpu().T,
                            bufs["h"].double().cpu().abs() @ wd.double().cpu().abs().T)):
        assert ((got.double().cpu() - ref).abs() <= 2.0**-8 * ref.abs() + 2.0**-20 * mass).all()
    sched.destroy()
    store.free()
    n.slot_pool += 8
    s2 = P.IrqScheduler(torch.cuda.Stream(), torch.cuda.Stream())
    with pytest.raises(P.PulseError) as e:
        s2.step([a], [n], mode="blocking")
    assert e.value.status == P.PULSE_ERR_INVALID_ARG
    s2.destroy()
