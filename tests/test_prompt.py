"""Attention of new tokens over each form of the cache, against plain forms in 64 bits."""
import math

import numpy as np
import pytest
import torch

import plain8
import plain64
from paper_2609_34555_amd import pulse as P
from parity import say

DEV = "cuda"
D = 128
FAKE = 0x1000
SCALE = 1 / math.sqrt(D)
CODES = {("bf16", 16): P.PULSE_BF16, ("f16", 16): P.PULSE_F16, ("bf16", 8): P.PULSE_BF16_KV8, ("f16", 8): P.PULSE_F16_KV8,
         ("bf16", 4): P.PULSE_BF16_KV4, ("f16", 4): P.PULSE_F16_KV4}
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


def dev(x, dtype=torch.int32):
    return torch.tensor(np.asarray(x), dtype=dtype, device=DEV)


def pack(kv, bits, bs):
    """Keys and values [2][n][hkv][bs][128] -> (blocks as bytes, keys, values in 64 bits)."""
    n, hkv = kv.shape[1:3]
    if bits == 4:
        b = plain64.pack(kv[0], kv[1], bs)
        return (b, *plain64.unpack(b, hkv, bs))
    if bits == 8:
        b, cache = plain8.pack(kv[0], kv[1], bs)
        return (b, *cache.values())
    b = torch.cat([kv[0].reshape(n, -1), kv[1].transpose(2, 3).reshape(n, -1)], 1).contiguous().view(torch.uint8)
    return b, kv[0].double(), kv[1].double()


def spoil(pool, bits, hkv, bs, block, t):
    """What lies from token t of a block on becomes NaN."""
    b = pool[block]
    if bits == 16:
        k, v = b.view(torch.int16).view(2, -1)
        k.view(hkv, bs, D)[:, t:] = -1
        v.view(hkv, D, bs)[:, :, t:] = -1
    elif bits == 8:
        for h in range(hkv):
            r = b[h * 256 * bs:(h + 1) * 256 * bs]
            r[t * D:bs * D] = 0xFF
            tok, c = torch.meshgrid(torch.arange(t, bs), torch.arange(D), indexing="ij")
            r[128 * bs + ((tok // 8 * 16 + c % 16) * 8 + c // 16) * 8 + tok % 8] = 0x7F
    else:
        r = b.view(hkv, 136 * bs)
        r[:, 128 * bs + 4 * t:132 * bs] = 255
        r[:, 132 * bs:].view(hkv, 4, bs)[:, :, t:] = 255


class Case:
    def __init__(self, ctx, new, hq, hkv, bs, dt, bits, seed, pad=0, stride=0, mb=0, garbage=True):
        self.ctx, self.new, self.hq, self.hkv, self.bs, self.bits = ctx, new, hq, hkv, bs, bits
        self.dtype, self.B = TYPES[dt], len(ctx)
        gen = torch.Generator().manual_seed(seed)
        n = [-(-x // bs) for x in ctx]
        total = sum(n) + 2
        slots = np.random.default_rng(seed).permutation(total)
        kv = torch.randn((2, total, hkv, bs, D), generator=gen)
        kv = (kv * torch.exp2(torch.randint(-2, 3, kv.shape[:-2] + (1, 1), generator=gen).float())).to(self.dtype)
        self.pool, self.k, self.v = pack(kv, bits, bs)
        self.mb = max(max(n), 1) + mb
        self.table, g = torch.full((self.B, self.mb), -1, dtype=torch.int32), 0
        for r, m in enumerate(n):
            self.table[r, :m] = torch.from_numpy(slots[g:g + m].astype(np.int32))
            g += m
            if garbage and ctx[r] % bs:
                spoil(self.pool, bits, hkv, bs, int(self.table[r, m - 1]), ctx[r] % bs)
        self.off = np.concatenate([[0], np.cumsum(new)])
        self.T = int(self.off[-1]) + pad
        self.stride = hq * D + stride
        self.q = torch.randn((self.T, self.stride), generator=gen).mul_(1.5).to(self.dtype)
        self.sh = P.make_shape(hq, hkv, D, bs, CODES[dt, bits])
        self.d = dict(q=self.q.to(DEV), pool=self.pool.to(DEV), table=self.table.to(DEV), off=dev(self.off), ctx=dev(ctx))

    def run(self, scale=SCALE, lse=True, fill=255, status_want=0, T=None, **kw):
        d = dict(self.d, **kw)
        T = T or self.T
        nb = P.pulse_prompt_workspace_bytes(self.sh, self.B, T, self.mb)
        ws = torch.full((nb,), fill, dtype=torch.uint8, device=DEV)
        out = torch.full((T, self.stride), 3.0, device=DEV, dtype=self.dtype)
        ls = torch.full((T, self.hq), 3.0, device=DEV) if lse else None
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        P.pulse_prompt_attn(self.sh, d["q"], self.stride, d["off"], T, d["ctx"], self.B, d["pool"], self.pool.shape[0],
                            d["table"], self.mb, scale, out, self.stride, ls, status, ws, nb)
        assert status.item() == status_want
        return out, ls

    def keys(self, r, upto=None):
        b = self.table[r, : -(-self.ctx[r] // self.bs)].long()
        return (x[b].transpose(0, 1).reshape(self.hkv, -1, D)[:, : self.ctx[r]] for x in (self.k, self.v))

    def check(self, out, lse, scale=SCALE, requests=None, skip=None, parts=1):
        """`skip`: (request, mask of its tokens that count nothing).  `parts`: of the 16-bit type that hold a probability."""
        u = torch.finfo(self.dtype).eps / 2
        out, lse = out.double().cpu(), lse.double().cpu()
        worst = [0.0, 0.0]
        for r in requests if requests is not None else range(self.B):
            k, v = self.keys(r)
            for i in sample(self.new[r]):
                p = self.ctx[r] - self.new[r] + i
                row = int(self.off[r]) + i
                m = torch.arange(p + 1)
                if skip and skip[0] == r:
                    m = m[~skip[1][: p + 1]]
                q = self.q[row, : self.hq * D].view(self.hq, D) * (-1 if scale < 0 else 1)
                want, want_lse, mass, reach = plain64.attention(q, k[:, m], v[:, m], abs(scale))
                got = out[row, : self.hq * D].view(self.hq, D)
                if not len(m):
                    assert (got == 0).all() and (lse[row] == -math.inf).all()
                    continue
                # a logit is a sum of 128 fp32 products of exact factors, scaled (134 * 2^-24 of the sum of their sizes);
                # the exponential adds 2^-23 of its value and 2^-24 of an argument of up to twice `reach`; a probability is
                # rounded once to the 16-bit type (u; in fp16 2^-25 of 2^7 at least), summed over the tokens in fp32, and so is
                # the denominator; the result is rounded once more
                n = len(m)
                logit = reach * 134 * 2.0**-24 + 2.0**-23
                rel = (2 * logit + u**parts + (n + 16) * 2.0**-23)[:, None]  # (each part rounds what the last left)
                low = 2.0**-32 * v[:, m].abs().sum(1).repeat_interleave(self.hq // self.hkv, 0) if u < 2.0**-10 else 0
                bound = (mass * rel + low) * (1 + u) + want.abs() * u + 2.0**-24
                worst[0] = max(worst[0], ((got - want).abs() / bound).max().item())
                worst[1] = max(worst[1], ((lse[row] - want_lse).abs()
                                          / (logit + (n + 16) * 2.0**-23 + want_lse.abs() * 2.0**-22)).max().item())
        say(f"  {worst[0]:.4f} / {worst[1]:.4f} of the bound")
        assert worst[0] <= 1 and worst[1] <= 1, worst


def sample(n):
    """Rows of a request that are looked at: all of a few, else the ends, those around tiles' ends, and some between."""
    if n <= 40:
        return range(n)
    at = {0, 1, 7, 8, 15, 16, 31, 32, 63, 64, 127, 128, n // 3, n // 2, n - 65, n - 33, n - 2, n - 1}
    return sorted(i for i in at if 0 <= i < n)


# contexts, new tokens (None: all), hq, hkv, bs, dtype
CASES = [
    ([1], None, 1, 1, 16, "bf16"),
    ([1, 2, 3], None, 4, 2, 16, "f16"),
    ([15, 16, 17, 64, 65], None, 8, 2, 16, "bf16"),
    ([200, 0, 129, 1], None, 6, 3, 32, "f16"),                  # a request without a token
    ([77, 300], None, 16, 2, 64, "bf16"),                        # eight heads of a group
    ([300], None, 3, 1, 32, "bf16"),
    ([190, 33], None, 7, 1, 16, "f16"),
    ([150, 90], None, 12, 1, 64, "f16"),
    ([100, 260], None, 16, 1, 16, "bf16"),
    ([500, 31, 640], None, 32, 8, 16, "bf16"),
    ([1000, 900], None, 10, 2, 32, "bf16"),
    ([513, 700, 65, 64], [1, 5, 64, 3], 8, 2, 16, "bf16"),       # the last tokens of longer contexts
    ([4000, 100, 2500, 17], [1, 1, 1, 1], 32, 8, 16, "f16"),      # a decode step
    ([5000, 3000], [7, 0], 16, 4, 64, "bf16"),                    # split over the context
    ([9000], [3], 8, 8, 16, "f16"),
    ([2100, 1900, 64, 3], [5, 4, 6, 2], 28, 4, 32, "bf16"),
    ([1800, 2048], [600, 500], 4, 1, 16, "bf16"),                # a part of a prompt
    ([60] * 70, None, 2, 2, 16, "bf16"),                          # many short ones
    ([40 + 3 * i for i in range(100)], [1 + i % 9 for i in range(100)], 5, 1, 32, "f16"),
    # 32 rows a workgroup by the number of workgroups, a request of many rows among requests of few; more than that
    ([700], None, 8, 2, 32, "f16"),
    ([900, 30, 2000, 1], [200, 2, 3, 1], 8, 1, 16, "bf16"),
    ([260, 300, 280], None, 32, 8, 16, "bf16"),
    ([2000, 40, 1999], [64, 64 - 24, 64], 24, 8, 64, "f16"),
    # 128 rows a workgroup, split over the context
    ([6001], [300], 32, 8, 16, "bf16"),
    ([6001], [300], 32, 8, 32, "f16"),
    ([6001, 5300], [170, 150], 16, 4, 64, "bf16"),
]


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_new_tokens(case, bits):
    ctx, new, hq, hkv, bs, dt = CASES[case]
    say(f"\n[gpu] prompt {bits} bits ctx={ctx[:4]} new={(new or ctx)[:4]} hq={hq} hkv={hkv} bs={bs} {dt}")
    c = Case(ctx, new or ctx, hq, hkv, bs, dt, bits, case, pad=case % 4, stride=8 * (case % 3), mb=case % 2)
    out, lse = c.run()
    n = int(c.off[-1])
    c.check(out, lse)
    assert (out[n:] == 3).all() and (lse[n:] == 3).all() and (out[:, hq * D:] == 3).all()
    again = c.run(fill=0)
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])
    assert torch.equal(c.run(lse=False)[0], out)


@pytest.mark.gpu
@pytest.mark.parametrize("ctx,new,hq,hkv,bs,dt,bits", [
    ([4200], None, 32, 8, 16, "bf16", 16), ([2300, 2100], None, 64, 16, 32, "f16", 8), ([2900], [2700], 48, 8, 64, "bf16", 4),
    ([4111], None, 32, 2, 16, "f16", 4), ([2500, 1900], None, 32, 8, 64, "bf16", 16), ([2431, 1900], None, 36, 12, 32, "bf16", 8)])
def test_long_prompts(ctx, new, hq, hkv, bs, dt, bits):
    """Prompts long and wide enough for the workgroups of 256 rows."""
    say(f"\n[gpu] prompt {bits} bits ctx={ctx} hq={hq} hkv={hkv} bs={bs} {dt}")
    c = Case(ctx, new or ctx, hq, hkv, bs, dt, bits, sum(ctx))
    out, lse = c.run()
    c.check(out, lse)
    again = c.run(fill=0)
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])


@pytest.mark.gpu
@pytest.mark.parametrize("bits,scale", [(16, 0.0), (8, -0.1), (16, -0.2), (4, 1.0)])
def test_any_scale(bits, scale):
    c = Case([100, 300], [100, 40], 8, 2, 16, "bf16", bits, 5)
    c.check(*c.run(scale=scale), scale=scale)


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("new", [260, 3])
def test_blocks_without_a_slot_count_nothing(bits, new):
    c = Case([260, 90], [new, 9], 8, 2, 16, "bf16", bits, 6)
    for j, bad in ((3, -1), (5, c.pool.shape[0]), (16, -9), (0, 2**31 - 1)):
        t = c.table.clone()
        t[0, j] = bad
        out, lse = c.run(table=t.to(DEV), status_want=P.PULSE_ERR_BAD_INDEX)
        mask = torch.zeros(260, dtype=torch.bool)
        mask[j * 16:j * 16 + 16] = True
        c.check(out, lse, skip=(0, mask))


@pytest.mark.gpu
def test_lengths_out_of_range():
    c = Case([50, 60, 70], [50, 10, 70], 4, 2, 16, "bf16", 16, 7)
    want, want_lse = c.run()
    for ctx, r in (([50, 9, 70], 1), ([50, 81, 70], 1), ([-1, 60, 70], 0), ([50, 60, 2**31 - 1], 2)):
        out, lse = c.run(ctx=dev(ctx), status_want=P.PULSE_ERR_BAD_INDEX)
        for i in range(3):
            s = slice(int(c.off[i]), int(c.off[i + 1]))
            if i == r:
                assert (out[s] == 0).all() and (lse[s] == -math.inf).all()
            else:
                assert torch.equal(out[s], want[s]) and torch.equal(lse[s], want_lse[s])
    for off in ([0, 50, 60, 131], [0, 50, 40, 130], [-1, 50, 60, 130], [0, 50, 2**31 - 1, 130], [0, 0, 0, -5]):
        c.run(off=dev(off), status_want=P.PULSE_ERR_BAD_INDEX)
    # offsets as the maps leave them after an error: nothing to do
    out, lse = c.run(off=dev([0, 0, 0, 0]))
    assert (out == 3).all() and (lse == 3).all()


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [16, 8, 4])
def test_nan_stays_in_its_head_and_after_its_token(bits):
    """A key or value that is NaN reaches the rows that attend to it, of its head alone."""
    c = Case([200], [200], 8, 2, 16, "bf16", bits, 8, garbage=False)
    b = c.pool[c.table[0, 4]]  # tokens 64 .. 79, head 1, token 69
    if bits == 16:
        b.view(torch.int16)[(1 * 16 + 5) * D + 3] = 0x7FC0
    elif bits == 8:
        b[256 * 16 + 5 * D + 3] = 0x7F
    else:
        b[136 * 16 + 128 * 16 + 5 * 4] = 255
    out, lse = c.run(pool=c.pool.to(DEV))
    nan = out.isnan().view(200, 2, -1)
    assert not nan[:, 0].any() and not nan[:69, 1].any() and nan[69:, 1].all()
    assert lse.isnan().view(200, 2, 4)[69:, 1].all() and not lse.isnan()[:69].any()


@pytest.mark.gpu
def test_pools_past_32_bit_offsets():
    bs, hkv = 64, 8
    sh = P.make_shape(8, hkv, D, bs, P.PULSE_BF16)
    U = P.pulse_block_bytes(sh)
    n_slots = (9 << 29) // U + 1
    c = Case([128], [30], 8, hkv, bs, "bf16", 16, 9)
    pool = torch.zeros((n_slots, U), dtype=torch.uint8, device=DEV)
    pool[-2:] = c.pool[c.table[0].long()].to(DEV)
    c.d["table"] = dev([[n_slots - 2, n_slots - 1]])
    nb = P.pulse_prompt_workspace_bytes(sh, 1, c.T, 2)
    ws = torch.zeros(nb, dtype=torch.uint8, device=DEV)
    out, lse = torch.zeros((c.T, c.stride), device=DEV, dtype=c.dtype), torch.zeros((c.T, 8), device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    P.pulse_prompt_attn(sh, c.d["q"], c.stride, c.d["off"], c.T, c.d["ctx"], 1, pool, n_slots, c.d["table"], 2, SCALE, out,
                        c.stride, lse, status, ws, nb)
    assert status.item() == 0
    c.check(out, lse)


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [16, 8])
def test_large_logits_and_constant_rows(bits):
    """Logits that grow along the context by more than the exponential's range, and rows whose logits are all equal."""
    c = Case([700], [700], 4, 1, 16, "bf16", bits, 10, garbage=False)
    c.q[:350] = 0
    ramp = torch.linspace(-40, 40, 700)
    kv = torch.zeros((2, c.pool.shape[0], 1, 16, D))
    for t in range(700):
        kv[0, c.table[0, t // 16], 0, t % 16, 0] = ramp[t]
    kv[1] = torch.randn(kv[1].shape)
    c.pool, c.k, c.v = pack(kv.bfloat16(), bits, 16)
    c.q[350:, 0::D] = 50.0
    out, lse = c.run(q=c.q.to(DEV), pool=c.pool.to(DEV))
    c.check(out, lse)


@pytest.mark.gpu
@pytest.mark.parametrize("new", [3, 700])
def test_many_small_probabilities(new):
    """fp16: one token's probability is near 1 and its value 0; the result is the sum of the others', 2^-19.6 each."""
    c = Case([3000], [new], 16, 1 if new == 3 else 4, 16, "f16", 16, 21, garbage=False)
    k0 = torch.zeros((c.hkv, 1, D), dtype=torch.float64)
    k0[..., 0] = 16
    first = int(c.table[0, 0])
    c.k[:], c.v[:] = 0, c.v.abs() + 0.5
    c.k[first, :, 0], c.v[first, :, 0] = k0[:, 0], 0
    c.pool, c.k, c.v = pack(torch.stack([c.k, c.v]).to(c.dtype), 16, c.bs)
    c.q.zero_()
    c.q.view(c.T, c.hq, D)[..., 0] = 19.6424 / (16 * SCALE * 1.4426950408889634)
    c.d.update(q=c.q.to(DEV), pool=c.pool.to(DEV))
    c.check(*c.run())


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("bits", [16, 8])
def test_few_rows_keep_probabilities_in_two_parts(bits, dt):
    c = Case([3000, 900, 6], [5, 3, 6], 16, 4, 16, dt, bits, 24)
    # values of one sign, so that the bound is little more than the result's own rounding
    c.v.abs_()
    c.pool, c.k, c.v = pack(torch.stack([c.k, c.v]).to(c.dtype), bits, c.bs)
    c.d.update(pool=c.pool.to(DEV))
    c.check(*c.run(), parts=2)


@pytest.mark.gpu
@pytest.mark.parametrize("T,bits", [(5, 16), (5, 8), (70, 4), (300, 16)])
def test_rows_before_the_first_request_stay(T, bits):
    """The first request's rows need not begin at 0: what is before them is left as it was, whatever the splits."""
    c = Case([2000, 900], [T, T // 2], 8, 2, 16, "bf16", bits, 22)
    want, want_lse = c.run()
    lead = 3
    q = torch.cat([torch.zeros((lead, c.stride), device=DEV, dtype=c.dtype), c.d["q"]])
    for fill in (0, 255):
        out, lse = c.run(q=q, off=c.d["off"] + lead, T=c.T + lead, fill=fill)
        assert (out[:lead] == 3).all() and (lse[:lead] == 3).all()
        u = torch.finfo(c.dtype).eps / 2  # (the plan may be another: each form rounds as in `check`)
        assert ((out[lead:] - want).double().abs() <= 8 * u * want.double().abs() + 8 * u).all()


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("T", [96, 5])
def test_captured_calls_replay_as_eager(T, bits):
    """A padded step in a graph, replayed on other lengths, contexts and queries, with eager work between; few rows and a
    split over the context (T = 5) and more."""
    c = Case([1500, 700, 900], [T // 3, T // 3, T - 2 * (T // 3)], 8, 2, 16, "bf16", bits, 12, pad=4)
    d, st = c.d, dev([0])
    nb = P.pulse_prompt_workspace_bytes(c.sh, 3, c.T, c.mb)
    bufs = [dict(out=torch.zeros((c.T, c.stride), device=DEV, dtype=c.dtype), lse=torch.zeros((c.T, c.hq), device=DEV),
                 ws=torch.full((nb,), 255, dtype=torch.uint8, device=DEV)) for _ in range(2)]

    def call(b):
        P.pulse_prompt_attn(c.sh, d["q"], c.stride, d["off"], c.T, d["ctx"], 3, d["pool"], c.pool.shape[0], d["table"], c.mb,
                            SCALE, b["out"], c.stride, b["lse"], st, b["ws"], nb)

    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        call(bufs[0])
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        call(bufs[0])
    for i, new in enumerate(([T, 0, 0], [1, 1, 1], [0, 2, T - 2], [T // 3] * 3)):
        d["off"].copy_(dev(np.concatenate([[0], np.cumsum(new)])))
        d["ctx"].copy_(dev([1500 - i, 700 - 7 * i, 900]))
        d["q"].mul_(-1)
        for b in bufs:
            b["out"].fill_(3)
            b["lse"].fill_(3)
        g.replay()
        call(bufs[1])
        torch.cuda.synchronize()
        assert torch.equal(bufs[0]["out"], bufs[1]["out"]) and torch.equal(bufs[0]["lse"], bufs[1]["lse"]), i
        n = sum(new)
        assert (bufs[0]["out"][n:] == 3).all() and (bufs[0]["out"][:n, : c.hq * D] != 3).any() and st.item() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("new", [[7, 1, 5, 2], [400, 90, 300, 1]])
def test_contexts_of_all_lengths_in_a_wide_table(new, bits):
    """Rows that are split over their context beside rows that are not, and whatever was in the workspace before."""
    c = Case([new[0] + 7000, new[1], new[2] + 1500, new[3] + 20], new, 16, 2, 16, "bf16", bits, 23, pad=2, mb=2000)
    out, lse = c.run()
    c.check(out, lse)
    again, again_lse = c.run(fill=0)
    n = sum(new)
    assert torch.equal(out, again) and torch.equal(lse, again_lse) and (out[n:] == 3).all() and (lse[n:] == 3).all()


@pytest.mark.gpu
def test_two_calls_at_once():
    """Calls on two streams with workspaces of their own give what they give alone."""
    cases = [Case([5000, 3000], [7, 2], 16, 4, 64, "bf16", 8, 13), Case([300, 900], [300, 900], 8, 2, 16, "f16", 16, 14)]
    alone = [c.run() for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    sizes = [P.pulse_prompt_workspace_bytes(c.sh, c.B, c.T, c.mb) for c in cases]
    got = [dict(ws=torch.full((sizes[i % 2],), 255, dtype=torch.uint8, device=DEV), st=dev([0]),
                out=torch.full_like(alone[i % 2][0], 3), lse=torch.full_like(alone[i % 2][1], 3)) for i in range(6)]
    torch.cuda.synchronize()
    for i, b in enumerate(got):
        c = cases[i % 2]
        P.pulse_prompt_attn(c.sh, c.d["q"], c.stride, c.d["off"], c.T, c.d["ctx"], c.B, c.d["pool"], c.pool.shape[0],
                            c.d["table"], c.mb, SCALE, b["out"], c.stride, b["lse"], b["st"], b["ws"], sizes[i % 2],
                            stream=streams[i % 2])
    torch.cuda.synchronize()
    for i, b in enumerate(got):
        out, lse = alone[i % 2]
        assert b["st"].item() == 0 and torch.equal(b["out"], out) and torch.equal(b["lse"], lse)


def test_prompt_refusals():
    sh = P.make_shape(32, 8, D, 16, P.PULSE_BF16)
    a = dict(q=FAKE, q_stride=4096, tok_off=FAKE, max_tokens=100, ctx_len=FAKE, B=2, slot_pool=FAKE, n_slots=50,
             block_table=FAKE, max_blocks=100, sm_scale=0.1, out=FAKE, out_stride=4096, lse=None, dev_status=FAKE, ws=FAKE,
             ws_bytes=1, stream=0, check=False)
    call = lambda s=sh, **kw: P.pulse_prompt_attn(s, **{**a, **kw})  # noqa: E731
    assert call() == P.PULSE_ERR_WORKSPACE
    assert call(ws=None, ws_bytes=1 << 40) == P.PULSE_ERR_WORKSPACE
    for name in ("q", "tok_off", "ctx_len", "slot_pool", "block_table", "out", "dev_status"):
        assert call(**{name: None}) == P.PULSE_ERR_INVALID_ARG, name
    for name in ("q", "slot_pool", "out"):
        assert call(**{name: FAKE + 8}) == P.PULSE_ERR_INVALID_ARG, name
    for kw in (dict(q_stride=4088), dict(q_stride=4100), dict(out_stride=0), dict(B=-1), dict(max_tokens=-1),
               dict(n_slots=0), dict(max_blocks=0)):
        assert call(**kw) == P.PULSE_ERR_INVALID_ARG, kw
    for kw in (dict(B=4097), dict(max_tokens=1 << 26), dict(max_tokens=1 << 31)):
        assert call(**kw) == P.PULSE_ERR_UNSUPPORTED, kw
    assert call(P.make_shape(32, 8, 64, 16, P.PULSE_BF16)) == P.PULSE_ERR_UNSUPPORTED
    assert call(P.make_shape(32, 8, D, 16, 7)) == P.PULSE_ERR_UNSUPPORTED
    assert call(P.make_shape(64, 64, D, 16, P.PULSE_BF16), q_stride=8192, out_stride=8192,
                max_tokens=1 << 24) == P.PULSE_ERR_UNSUPPORTED
    assert call(P.make_shape(2048, 2048, D, 16, P.PULSE_BF16), q_stride=1 << 18,
                out_stride=1 << 18) == P.PULSE_ERR_UNSUPPORTED
    assert call(B=0, q=None) == P.PULSE_OK and call(max_tokens=0, q=None) == P.PULSE_OK
    assert P.pulse_prompt_workspace_bytes(sh, 2, 1 << 26, 8) == 0 and P.pulse_prompt_workspace_bytes(sh, -1, 5, 8) == 0
    assert P.pulse_prompt_workspace_bytes(sh, 2, 100, 8) > 0


def test_a_workspace_serves_smaller_calls():
    for hq, hkv, bs in ((32, 8, 16), (16, 1, 64), (28, 4, 32), (2, 2, 16), (48, 4, 64)):
        for code in (P.PULSE_BF16, P.PULSE_F16_KV8, P.PULSE_BF16_KV4):
            sh = P.make_shape(hq, hkv, D, bs, code)
            sizes = {}
            for B in (1, 2, 5, 16, 31, 64, 200):
                for T in (1, 3, 8, 31, 64, 200, 900, 5000, 40000):
                    for mb in (1, 7, 64, 500, 3000, 8192):
                        sizes[B, T, mb] = P.pulse_prompt_workspace_bytes(sh, B, T, mb)
            for (B, T, mb), n in sizes.items():
                assert n > 0
                for other in ((2, T, mb), (B, 200, mb), (B, T, 64), (1, 1, 8192), (5, 31, 3000)):
                    if all(x <= y for x, y in zip(other, (B, T, mb))):
                        assert sizes[other] <= n, (other, (B, T, mb))
