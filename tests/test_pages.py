"""Forks, frees and compaction of the pool's blocks against loops over requests and blocks."""
import copy
import math

import numpy as np
import pytest
import torch

import plain8
import plain64
from paper_2609_34555_amd import pulse as P
from parity import say
from test_kv4 import check_attention
from test_kv4_step import Run
from test_kv8 import same_bytes

DEV = "cuda"
D = 128
FAKE = 0x1000
KEEP_ALL = 2**31 - 1


def dev(x, dtype=torch.int32):
    return torch.tensor(np.asarray(x), dtype=dtype, device=DEV)


class Wrong(Exception):
    pass


class Exhausted(Exception):
    pass


class Pages:
    """The state as numpy arrays; calls by their definitions, all or nothing."""

    def __init__(self, B, mb, n_slots, bs, seed):
        self.rng = np.random.default_rng(seed)
        self.B, self.mb, self.n_slots, self.bs = B, mb, n_slots, bs
        self.table = np.full((B, mb), -1, np.int32)
        self.shared = np.zeros(n_slots, np.int32)
        self.free = self.rng.permutation(n_slots).astype(np.int32)
        self.head = 0
        self.what = np.arange(n_slots)  # which block's contents lie in a slot
        self.ctx = np.zeros(B, np.int64)

    def take(self, r, n):
        """What the maps do for n more tokens."""
        for j in range(-(-self.ctx[r] // self.bs), -(-(self.ctx[r] + n) // self.bs)):
            self.table[r, j] = self.free[self.head]
            self.head += 1
        self.ctx[r] += n

    def do_free(self, keep, with_shared=True):
        freed, kept = [], set()
        for r in range(self.B):
            if keep[r] < 0:
                raise Wrong
            for j in range(self.mb):
                s = int(self.table[r, j])
                if j * self.bs < keep[r]:
                    if (j + 1) * self.bs > keep[r] and with_shared and s >= 0 and self.shared[s] > 0:
                        raise Wrong
                elif s != -1:
                    if not 0 <= s < self.n_slots:
                        raise Wrong
                    freed.append((r, j, s))
        held = {s: (int(self.shared[s]) if with_shared else 0) + 1 for _, _, s in freed}
        back = []
        for _, _, s in freed:
            held[s] -= 1
            if held[s] < 0:
                raise Wrong
            if held[s] == 0:
                back.append(s)
        if not 0 <= self.head <= len(self.free) or len(back) > self.head:
            raise Wrong
        for r, j, _ in freed:
            self.table[r, j] = -1
        if with_shared:
            for s, h in held.items():
                self.shared[s] = max(h - 1, 0)
        self.head -= len(back)
        self.free[self.head:self.head + len(back)] = back

    def do_fork(self, src, dst, ln):
        if len(set(dst)) != len(dst) or set(src) & set(dst):
            raise Wrong
        need = sum(x % self.bs != 0 for x in ln)
        for a, b, x in zip(src, dst, ln):
            if not (0 <= a < self.B and 0 <= b < self.B and x >= 0 and -(-x // self.bs) <= self.mb):
                raise Wrong
            w = x // self.bs
            if (self.table[b] != -1).any() or (self.table[a, :w] < -1).any() or (self.table[a, :w] >= self.n_slots).any():
                raise Wrong
            if x % self.bs and not 0 <= self.table[a, w] < self.n_slots:
                raise Wrong
        if not 0 <= self.head <= len(self.free):
            raise Wrong
        if need > len(self.free) - self.head:
            raise Exhausted
        new = self.free[self.head:self.head + need]
        if ((new < 0) | (new >= self.n_slots)).any():
            raise Wrong
        for a, b, x in zip(src, dst, ln):
            w = x // self.bs
            self.table[b, :w] = self.table[a, :w]
            for s in self.table[b, :w]:
                self.shared[s] += s >= 0
            if x % self.bs:
                s = self.free[self.head]
                self.head += 1
                self.table[b, w] = s
                self.what[s] = self.what[self.table[a, w]]

    def do_compact(self, n_keep, with_shared=True):
        t, rest = self.table, self.free[self.head:] if 0 <= self.head <= len(self.free) else None
        if rest is None or ((t < -1) | (t >= self.n_slots)).any() or ((rest < 0) | (rest >= self.n_slots)).any():
            raise Wrong
        live = set(t[t >= 0].tolist())
        if len(set(rest.tolist())) != len(rest) or live & set(rest.tolist()):
            raise Wrong
        high, low = sorted(s for s in live if s >= n_keep), [s for s in rest.tolist() if s < n_keep]
        if len(high) > len(low):
            raise Exhausted
        to = dict(zip(high, low))
        self.table = np.array([[to.get(int(s), int(s)) for s in row] for row in t], np.int32).reshape(t.shape)
        for a, b in to.items():
            self.what[b] = self.what[a]
            if with_shared:
                self.shared[b], self.shared[a] = self.shared[a], 0
        left = low[len(high):]
        self.head = len(self.free) - len(left)
        self.free[self.head:] = left


class Both:
    """The state on the device beside Pages; a call is made on both and everything compared."""

    def __init__(self, p, code=P.PULSE_BF16, hkv=1):
        self.p, self.sh = p, P.make_shape(hkv, hkv, D, p.bs, code)
        U = P.pulse_block_bytes(self.sh)
        self.start = torch.randint(0, 255, (p.n_slots, U), dtype=torch.uint8, device=DEV)
        self.pool = self.start[torch.from_numpy(p.what).to(DEV)].clone()
        self.status = dev([0])
        self.nb = P.pulse_pages_workspace_bytes(self.sh, p.B, p.mb, p.n_slots)
        self.push()

    def push(self):
        p = self.p
        self.table, self.shared, self.free, self.head = dev(p.table), dev(p.shared), dev(p.free), dev([p.head])

    def same(self, with_shared=True):
        p = self.p
        assert (self.table.cpu().numpy() == p.table).all()
        assert (self.free.cpu().numpy() == p.free).all() and self.head.item() == p.head
        assert (self.shared.cpu().numpy() == p.shared).all()
        assert torch.equal(self.pool, self.start[torch.from_numpy(p.what).to(DEV)])

    def call(self, what, *args, shared=True):
        p, want = self.p, 0
        before = copy.deepcopy(p)
        try:
            getattr(p, "do_" + what)(*args, **({} if what == "fork" else dict(with_shared=shared)))
        except Wrong:
            want, self.p = P.PULSE_ERR_BAD_INDEX, before
        except Exhausted:
            want, self.p = P.PULSE_ERR_POOL_EXHAUSTED, before
        ws = torch.randint(0, 255, (self.nb,), dtype=torch.uint8, device=DEV)
        sh = self.shared if shared else None
        tail = (self.status, ws, self.nb)
        if what == "free":
            P.pulse_free_blocks(self.sh, dev(args[0]), p.B, self.table, p.mb, sh, self.free, self.head, len(p.free),
                                p.n_slots, *tail)
        elif what == "fork":
            P.pulse_fork_blocks(self.sh, *(dev(x) for x in args), len(args[0]), self.table, p.B, p.mb, self.shared, self.free,
                                self.head, len(p.free), self.pool, p.n_slots, *tail)
        else:
            P.pulse_compact_blocks(self.sh, self.table, p.B, p.mb, args[0], sh, self.free, self.head, len(p.free), self.pool,
                                   p.n_slots, *tail)
        assert self.status.item() == want, (what, want)
        self.status.zero_()
        self.same()
        return want


def life(both, steps, rng):
    """Requests come, grow, fork, fall back and go; now and then the pool is compacted."""
    for _ in range(steps):
        p = both.p
        live, idle = [r for r in range(p.B) if p.ctx[r]], [r for r in range(p.B) if not p.ctx[r]]
        for r in idle[:2]:
            n = int(rng.integers(1, p.mb * p.bs // 2))
            if p.n_slots - p.head > 2 * -(-n // p.bs) + p.B:
                p.take(r, n)
        for r in live[::2]:
            if p.n_slots - p.head > p.B:
                p.take(r, int(min(rng.integers(0, 4), p.mb * p.bs - p.ctx[r])))
        both.push()
        live, idle = [r for r in range(p.B) if p.ctx[r]], [r for r in range(p.B) if not p.ctx[r]]
        k = min(len(idle), int(rng.integers(0, 6)))
        if live and k:
            src, dst = rng.choice(live, k).tolist(), rng.permutation(idle)[:k].tolist()
            ln = [int(p.ctx[a]) if rng.random() < 0.5 else int(rng.integers(0, p.ctx[a] + 1)) for a in src]
            if not both.call("fork", src, dst, ln):
                both.p.ctx[dst] = ln
        p = both.p
        keep = np.full(p.B, KEEP_ALL, np.int64)
        for r in range(p.B):
            u = rng.random()
            if u < 0.15:
                keep[r] = 0
            elif u < 0.35:
                keep[r] = max(0, p.ctx[r] - int(rng.integers(0, 3 * p.bs)))
        if not both.call("free", keep):
            both.p.ctx = np.minimum(both.p.ctx, keep)
        if rng.random() < 0.4:
            p = both.p
            used = len(set(p.table[p.table >= 0].tolist()))
            n_keep = int(rng.integers(used, p.n_slots + 1))
            if not both.call("compact", n_keep):  # the other slots leave the pool: put them behind the list again
                p = both.p
                rest = p.free[p.head:].tolist()
                out = sorted(set(range(n_keep, p.n_slots)))
                p.head = p.n_slots - len(rest) - len(out)
                p.free[p.head:] = rest + out
                both.push()


@pytest.mark.gpu
@pytest.mark.parametrize("B,mb,n_slots,bs,code,hkv", [
    (1, 1, 3, 16, P.PULSE_BF16, 1), (5, 7, 40, 16, P.PULSE_BF16_KV8, 3), (12, 33, 300, 32, P.PULSE_F16_KV4, 2),
    (40, 20, 700, 16, P.PULSE_F16, 1), (70, 1000, 9000, 16, P.PULSE_BF16_KV4, 1), (9, 64, 450, 64, P.PULSE_BF16, 5)])
def test_lives_of_requests(B, mb, n_slots, bs, code, hkv):
    """Up to 70 x 1000 entries, beyond what one workgroup takes."""
    say(f"\n[gpu] pages B={B} mb={mb} slots={n_slots} bs={bs}")
    both = Both(Pages(B, mb, n_slots, bs, B), code, hkv)
    life(both, 12, np.random.default_rng(B + mb))


def small(seed=1, B=6, mb=12, n_slots=60, bs=16):
    p = Pages(B, mb, n_slots, bs, seed)
    for r, n in enumerate((100, 64, 17, 0, 0, 0)):
        if n:
            p.take(r, n)
    return p


@pytest.mark.gpu
@pytest.mark.parametrize("wide", [False, True])
def test_refused_frees(wide):
    """Each leaves everything as it was; `wide`: the form of many workgroups."""
    def state(seed=1):
        p = small(seed, mb=20000 if wide else 12)
        return Both(p)

    b = state()
    every = [KEEP_ALL] * 6
    assert b.call("free", [-1] + every[1:]) == P.PULSE_ERR_BAD_INDEX
    b.call("fork", [0], [3], [100])
    for keep in (90, 33):  # inside a shared block
        assert b.call("free", [keep] + every[1:]) == P.PULSE_ERR_BAD_INDEX
    assert b.call("free", [96] + every[1:]) == 0 and b.call("free", [32] + every[1:]) == 0
    assert b.call("free", [0] * 6) == 0 and b.p.head == 0
    for bad in (60, -2, 2**31 - 1):
        b = state()
        b.p.table[1, 2] = bad
        b.push()
        assert b.call("free", [0] * 6) == P.PULSE_ERR_BAD_INDEX
        assert b.call("free", every) == 0  # what is kept is not looked at
    b = state()
    b.p.table[4, 5] = b.p.table[0, 1]  # named twice, counted once
    b.push()
    assert b.call("free", [0] * 6) == P.PULSE_ERR_BAD_INDEX
    assert b.call("free", [0] * 6, shared=False) == P.PULSE_ERR_BAD_INDEX
    for head in (-1, 61, 3):  # out of range; fewer slots out than come back
        b = state()
        b.p.head = head
        b.push()
        assert b.call("free", [0] * 6) == P.PULSE_ERR_BAD_INDEX
    b = state()
    b.p.shared[b.p.table[0, 0]] = -1
    b.push()
    assert b.call("free", [0] * 6) == P.PULSE_ERR_BAD_INDEX
    b = state()
    assert b.call("free", [17, 0, KEEP_ALL, 0, 0, 0], shared=False) == 0


@pytest.mark.gpu
def test_refused_forks():
    ok = ([0, 1, 0], [3, 4, 5], [100, 64, 7])
    assert Both(small()).call("fork", *ok) == 0
    for src, dst, ln in (([0, 0], [3, 3], [16, 16]), ([0, 3], [3, 4], [16, 16]), ([0], [0], [0]), ([-1], [3], [5]),
                         ([6], [3], [5]), ([0], [6], [5]), ([0], [-1], [5]), ([0], [3], [-1]), ([0], [3], [193]),
                         ([0], [1], [5]), ([0], [3], [113]), ([4], [3], [1]), ([0], [3], [2**31 - 1])):
        assert Both(small()).call("fork", src, dst, ln) == P.PULSE_ERR_BAD_INDEX, (src, dst, ln)
    b = Both(small())  # blocks that are not resident stay so; the one that is copied has to be
    b.p.table[0, 2] = -1
    b.push()
    assert b.call("fork", [0], [3], [100]) == 0 and b.p.table[3, 2] == -1
    assert b.call("fork", [0], [4], [40]) == P.PULSE_ERR_BAD_INDEX
    for bad in (60, -2):
        b = Both(small())
        b.p.table[0, 1] = bad
        b.push()
        assert b.call("fork", [0], [3], [100]) == P.PULSE_ERR_BAD_INDEX
        b = Both(small())
        b.p.free[b.p.head] = bad
        b.push()
        assert b.call("fork", [0], [3], [100]) == P.PULSE_ERR_BAD_INDEX
    b = Both(small())
    b.p.head = 59
    b.push()
    assert b.call("fork", *ok) == P.PULSE_ERR_POOL_EXHAUSTED
    for head in (-1, 61):
        b.p.head = head
        b.push()
        assert b.call("fork", *ok) == P.PULSE_ERR_BAD_INDEX


@pytest.mark.gpu
@pytest.mark.parametrize("wide", [False, True])
def test_refused_compactions(wide):
    def state():
        return Both(small(mb=20000 if wide else 12))

    used = 13
    assert state().call("compact", used) == 0
    assert state().call("compact", 60) == 0 and state().call("compact", used, shared=False) == 0
    assert state().call("compact", used - 1) == P.PULSE_ERR_POOL_EXHAUSTED
    assert state().call("compact", 0) == P.PULSE_ERR_POOL_EXHAUSTED
    for bad in (60, -2):
        b = state()
        b.p.table[1, 2] = bad
        b.push()
        assert b.call("compact", 30) == P.PULSE_ERR_BAD_INDEX
        b = state()
        b.p.free[-1] = bad
        b.push()
        assert b.call("compact", 30) == P.PULSE_ERR_BAD_INDEX
    b = state()
    b.p.free[-1] = b.p.free[-2]  # twice in the list
    b.push()
    assert b.call("compact", 30) == P.PULSE_ERR_BAD_INDEX
    b = state()
    b.p.free[-1] = b.p.table[0, 0]  # in the list and the table
    b.push()
    assert b.call("compact", 30) == P.PULSE_ERR_BAD_INDEX
    for head in (-1, 61):
        b = state()
        b.p.head = head
        b.push()
        assert b.call("compact", 30) == P.PULSE_ERR_BAD_INDEX
    b = state()
    b.p.head = 60  # no slot is free
    b.push()
    assert b.call("compact", 60) == 0


@pytest.mark.gpu
def test_blocks_past_32_bit_offsets():
    p = Pages(2, 4, 9500, 64, 3)
    p.free = np.concatenate([[9498, 9499], np.arange(9498)]).astype(np.int32)
    p.take(0, 100)
    b = Both(p, P.PULSE_BF16, 16)
    assert b.pool.numel() > 4 << 30
    assert b.call("fork", [0], [1], [100]) == 0
    assert b.call("compact", 100) == 0 and (b.p.table[:, :2] < 100).all()


# ------------------------------------------------------------------------------------------------ a run of them


@pytest.mark.gpu
@pytest.mark.parametrize("code,dtype", [(P.PULSE_BF16_KV8, torch.bfloat16), (P.PULSE_F16_KV8, torch.float16)])
def test_a_batch_from_prompts_to_the_end(code, dtype):
    """Prompts into the 8-bit cache and attended to, forks of them, decode steps, tokens taken back, drafted tokens
    verified, requests that end, a compacted pool, more steps: every result against 64 bits over what the cache holds."""
    prompt, hq, hkv, bs = [100, 37, 64, 1], 8, 2, 16
    B = len(prompt) + 3
    st = Run(prompt + [0] * 3, 60, hq, hkv, bs, code, dtype, 5)
    cache = plain8.Cache(st.n_slots, hkv, bs, dtype)
    shared, scale = torch.zeros(st.n_slots, dtype=torch.int32, device=DEV), 1 / math.sqrt(D)
    nb = P.pulse_pages_workspace_bytes(st.sh, B, st.mb, st.n_slots)
    ws = torch.zeros(nb, dtype=torch.uint8, device=DEV)
    ctx = prompt + [0] * 3

    def attend(new):
        pb = P.pulse_prompt_workspace_bytes(st.sh, B, st.T, st.mb)
        pws = torch.full((pb,), 255, dtype=torch.uint8, device=DEV)
        out = torch.full((st.T, hq * D), 3.0, device=DEV, dtype=dtype)
        lse = torch.zeros((st.T, hq), device=DEV)
        P.pulse_prompt_attn(st.sh, st.q, hq * D, st.tok, st.T, st.ctx, B, st.pool, st.n_slots, st.table, st.mb, scale, out,
                            hq * D, lse, st.status, pws, pb)
        assert st.status.item() == 0
        kv, row, u = cache.values(), 0, torch.finfo(dtype).eps / 2
        for r in range(B):
            b = st.table[r, : -(-ctx[r] // bs)].long().cpu()
            k, v = (x[b].transpose(0, 1).reshape(hkv, -1, D) for x in kv)
            for i in range(new[r]):
                p = ctx[r] - new[r] + i + 1
                want, want_lse, mass, reach = plain64.attention(st.q[row].cpu(), k[:, :p], v[:, :p], scale)
                logit = reach * 134 * 2.0**-24 + 2.0**-23
                rel = (2 * logit + u + (p + 16) * 2.0**-23)[:, None]
                low = 2.0**-25 * v[:, :p].abs().sum(1).repeat_interleave(hq // hkv, 0) if u < 2.0**-10 else 0
                got = out[row].view(hq, D).double().cpu()
                assert ((got - want).abs() <= (mass * rel + low) * (1 + u) + want.abs() * u + 2.0**-24).all()
                row += 1
        assert (out[row:] == 3).all()

    def step(new, decode):
        for r in range(B):
            ctx[r] += new[r] if decode else 0
        st.ctx.copy_(dev(ctx))
        st.new.copy_(dev(new))
        T = sum(new) + 2
        x = st.rows(T)
        st.buffers(T)
        st.write(x)
        assert st.status.item() == 0
        cache.append(st.k, x[:, (hq + hkv) * D:].unflatten(1, (hkv, D)), st.slot_map.tolist())
        same_bytes(st.pool, cache)
        attend(new)

    def free(keep):
        P.pulse_free_blocks(st.sh, dev(keep), B, st.table, st.mb, shared, st.free, st.head, st.n_slots, st.n_slots, st.status,
                            ws, nb)
        assert st.status.item() == 0
        for r in range(B):
            ctx[r] = min(ctx[r], keep[r])

    step(ctx, False)
    P.pulse_fork_blocks(st.sh, dev([0, 0, 2]), dev([4, 5, 6]), dev([100, 50, 64]), 3, st.table, B, st.mb, shared, st.free,
                        st.head, st.n_slots, st.pool, st.n_slots, st.status, ws, nb)
    assert st.status.item() == 0 and shared.sum().item() == 6 + 3 + 4
    for a, b, n in ((0, 4, 100), (0, 5, 50)):
        i, j = (int(st.table[r, n // bs]) for r in (a, b))
        cache.code[j], cache.exp[j], cache.known[j] = cache.code[i], cache.exp[i], cache.known[i]
    ctx[4:] = [100, 50, 64]
    for _ in range(3):
        step([1] * B, True)
    # decode attention sees the same
    full = [x for x in ctx]
    st.q = st.q[:B].contiguous()
    st.ctx.copy_(dev(full))
    P.pulse_build_tables(st.sh, st.ctx, dev([0] * B), B, st.table, st.mb, st.free, st.head, st.n_slots, st.n_slots, st.blk,
                         st.tok, st.slot_map, st.pos, st.T, st.status, st.tws, st.tws.numel())
    st.attend()
    kv = cache.values()
    for r in range(B):
        b = st.table[r, : -(-ctx[r] // bs)].long().cpu()
        k, v = (x[b].transpose(0, 1).reshape(hkv, -1, D)[:, : ctx[r]] for x in kv)
        check_attention(st.out[r], st.lse[r], *plain64.attention(st.q[r].cpu(), k, v, scale), ctx[r])
    step([4, 5, 1, 0, 3, 2, 5], True)                 # drafted tokens, of which some are refused
    free([ctx[0] - 2, ctx[1] - 5, KEEP_ALL, 0, ctx[4], ctx[5] - 1, ctx[6] - 1])
    step([1, 1, 1, 0, 1, 1, 1], True)
    free([0, KEEP_ALL, KEEP_ALL, 0, KEEP_ALL, KEEP_ALL, 0])  # a source ends before its forks
    used = int(torch.unique(st.table[st.table >= 0]).numel())
    n_keep = used + 3
    old = st.table.cpu().clone()
    P.pulse_compact_blocks(st.sh, st.table, B, st.mb, n_keep, shared, st.free, st.head, st.n_slots, st.pool, st.n_slots,
                           st.status, ws, nb)
    assert st.status.item() == 0 and st.table.max().item() < n_keep and st.n_slots - st.head.item() == 3
    now = st.table.cpu()
    for i, j in {(int(a), int(b)) for a, b in zip(old.reshape(-1), now.reshape(-1)) if a != b}:
        cache.code[j], cache.exp[j], cache.known[j] = cache.code[i], cache.exp[i], cache.known[i]
    for _ in range(2):
        step([0, 1, 1, 0, 1, 1, 0], True)


@pytest.mark.gpu
def test_captured_calls_replay_as_eager():
    """Free, fork and compaction in a graph, replayed on states that change between, beside an eager twin."""
    def state():
        p = Pages(8, 30, 200, 16, 4)
        for r, n in enumerate((200, 130, 77, 16)):
            p.take(r, n)
        return Both(p)

    keep, src, dst, ln = dev([KEEP_ALL] * 8), dev([0, 2]), dev([5, 6]), dev([100, 77])
    eager, rec = state(), state()
    rec.pool.copy_(eager.pool)

    def calls(b, ws):
        p, tail = b.p, (b.status, ws, b.nb)
        P.pulse_free_blocks(b.sh, keep, p.B, b.table, p.mb, b.shared, b.free, b.head, 200, 200, *tail)
        P.pulse_fork_blocks(b.sh, src, dst, ln, 2, b.table, p.B, p.mb, b.shared, b.free, b.head, 200, b.pool, 200, *tail)
        P.pulse_compact_blocks(b.sh, b.table, p.B, p.mb, 100, b.shared, b.free, b.head, 200, b.pool, 200, *tail)

    wse, wsr = (torch.zeros(eager.nb, dtype=torch.uint8, device=DEV) for _ in range(2))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        calls(rec, wsr)
    torch.cuda.current_stream().wait_stream(side)
    calls(eager, wse)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        calls(rec, wsr)
    for i in range(5):
        keep.copy_(dev([KEEP_ALL] * 5 + [0, 0, 0]))
        src.copy_(dev([i % 3, 1]))
        ln.copy_(dev([16 * i + 3, 129 - i]))
        g.replay()
        calls(eager, wse)
        torch.cuda.synchronize()
        for f in ("table", "shared", "free", "head", "pool", "status"):
            assert torch.equal(getattr(eager, f), getattr(rec, f)), (i, f)
        assert eager.status.item() == 0


# ------------------------------------------------------------------------------------------------ host entry


def test_pages_refusals():
    sh = P.make_shape(32, 8, D, 16, P.PULSE_BF16_KV8)
    assert P.pulse_pages_workspace_bytes(sh, 4, 100, 500) > 0
    assert P.pulse_pages_workspace_bytes(sh, 4097, 100, 500) == 0 and P.pulse_pages_workspace_bytes(sh, 4, 0, 500) == 0
    common = dict(block_table=FAKE, B=4, max_blocks=100, shared=FAKE, free_slots=FAKE, free_head=FAKE, n_free=10, n_slots=500,
                  dev_status=FAKE, ws=FAKE, ws_bytes=1, stream=0, check=False)
    calls = [(P.pulse_fork_blocks, dict(common, src=FAKE, dst=FAKE, fork_len=FAKE, n=2, slot_pool=FAKE),
              ("src", "dst", "fork_len", "shared", "slot_pool")),
             (P.pulse_free_blocks, dict(common, keep_len=FAKE), ("keep_len",)),
             (P.pulse_compact_blocks, dict(common, n_keep=7, slot_pool=FAKE), ("slot_pool",))]
    for fn, args, needs in calls:
        call = lambda s=sh, **kw: fn(s, **{**args, **kw})  # noqa: E731
        assert call() == P.PULSE_ERR_WORKSPACE
        for name in needs + ("block_table", "free_slots", "free_head", "dev_status"):
            assert call(**{name: None}) == P.PULSE_ERR_INVALID_ARG, name
        for kw in (dict(B=-1), dict(max_blocks=0), dict(n_free=-1), dict(n_slots=0)):
            assert call(**kw) == P.PULSE_ERR_INVALID_ARG, kw
        for kw in (dict(B=4097), dict(max_blocks=2**31 - 1), dict(n_slots=2**31 - 1)):
            assert call(**kw) == P.PULSE_ERR_UNSUPPORTED, kw
        assert call(P.make_shape(32, 8, 64, 16, P.PULSE_BF16)) == P.PULSE_ERR_UNSUPPORTED
        if "slot_pool" in args:
            assert call(slot_pool=FAKE + 8) == P.PULSE_ERR_INVALID_ARG
    fork = lambda **kw: calls[0][0](sh, **{**calls[0][1], **kw})  # noqa: E731
    assert fork(n=-1) == P.PULSE_ERR_INVALID_ARG and fork(n=5) == P.PULSE_ERR_INVALID_ARG
    assert fork(n=0, src=None) == P.PULSE_OK and calls[1][0](sh, **{**calls[1][1], "B": 0}) == P.PULSE_OK
    for n_keep in (-1, 501):
        assert calls[2][0](sh, **{**calls[2][1], "n_keep": n_keep}) == P.PULSE_ERR_INVALID_ARG
