"""The 8-bit cache: rows written and read, scales that grow, attention over it, against plain forms in 64 bits."""
import math

import numpy as np
import pytest
import torch

import plain8
import plain64
from paper_2609_34555_amd import pulse as P
from parity import say
from test_kv4 import attend, check_attention

DEV = "cuda"
D = 128
FAKE = 0x1000
TYPES = {"bf16": (torch.bfloat16, P.PULSE_BF16_KV8), "f16": (torch.float16, P.PULSE_F16_KV8)}
SCALE = 1 / math.sqrt(D)


def dev(x, dtype=torch.int32):
    return torch.tensor(np.asarray(x), dtype=dtype, device=DEV)


def equal(a, b):
    a, b = a.double().cpu(), b.double().cpu()
    return bool(((a == b) | (a.isnan() & b.isnan())).all())


def same_bytes(pool, cache):
    """The pool's bytes where they are known (a zero has either sign, a NaN any of its two codes)."""
    got, (want, sure) = pool.cpu().numpy(), cache.bytes()
    assert got.shape == want.shape
    bad = sure & (got != want) & ~((got & 127 == 127) & (want & 127 == 127))
    assert not bad.any(), (np.argwhere(bad)[:5], got[bad][:5], want[bad][:5])


# ------------------------------------------------------------------------------------------------ rows

# calls one after another, of each the places of its rows (None: nowhere); bs
ROWS = [
    ([[0]], 16),
    ([[0], [1], [2], [3, 4, 5], [6]], 16),                    # token after token
    ([list(range(16)), list(range(16, 19)), [19], [20, 21]], 16),
    ([list(range(40))], 16),                                   # whole blocks and a part
    ([list(range(45)), list(range(45, 64)), [64]], 64),        # a block filled by two calls
    ([[7, 6, 5, 4, 3, 2, 1, 0]], 16),                          # tokens in any order
    ([[0, 2, 4, 6, 1, 3, 5, 7, 31], [30, 8]], 32),
    ([[0, 1, 2, 3, None, 16, 17, None, None, 32], [4, None, 18]], 16),
    ([[None] * 3], 16),
    ([list(range(32, 64)) + [0, 1, 2], [64, 65, 66, 96], [3, 67]], 32),
    ([list(range(64, 128)) + list(range(0, 64)) + list(range(192, 211)), list(range(211, 256)) + [128]], 64),
    ([[0, 1, 2, 3, 4], [0], [1, 2], list(range(3, 16))], 16),  # a block begun anew
    ([[48, 32, 16, 0], [49, 33, 17, 1], [50, 34, 18, 2]], 16),  # requests of a token each
]


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("hkv", [1, 3, 8])
@pytest.mark.parametrize("case", range(len(ROWS)))
def test_append_and_load(case, hkv, dt):
    calls, bs = ROWS[case]
    dtype, code = TYPES[dt]
    gen = torch.Generator(device=DEV)
    gen.manual_seed(case)
    n_slots = max([p or 0 for c in calls for p in c]) // bs + 3
    sh = P.make_shape(2 * hkv, hkv, D, bs, code)
    U = P.pulse_block_bytes(sh)
    assert U == hkv * 256 * bs + 128
    before = torch.randint(0, 255, (n_slots, U), generator=gen, device=DEV, dtype=torch.uint8)
    pool, status = before.clone(), torch.zeros(1, dtype=torch.int32, device=DEV)
    cache = plain8.Cache(n_slots, hkv, bs, dtype)
    for places in calls:
        T = len(places)
        # rows of different sizes inside wider ones
        wide = torch.randn((T, 2, hkv * D + 24), generator=gen, device=DEV)
        wide = (wide * torch.exp2(torch.randint(-6, 6, (T, 1, 1), generator=gen, device=DEV).float())).to(dtype)
        k, v = wide[:, 0, 8:8 + hkv * D], wide[:, 1, 16:16 + hkv * D]
        stride = wide.stride(0)
        P.pulse_append_kv(sh, k, stride, v, stride, dev([-1 if p is None else p for p in places], torch.int64), T, pool,
                          n_slots, status)
        assert status.item() == 0
        cache.append(*(x.unflatten(1, (hkv, D)) for x in (k, v)), places)
        same_bytes(pool, cache)
    untouched = ~cache.known.any(1)
    assert torch.equal(pool[untouched], before[untouched])
    assert torch.equal(pool[:, hkv * 256 * bs + 2 * hkv:], before[:, hkv * 256 * bs + 2 * hkv:])
    # and back, every token that is known, in an order of its own, into wider rows
    places = np.flatnonzero(cache.known.reshape(-1))
    places = places[np.random.default_rng(case).permutation(len(places))]
    places = np.concatenate([places, [-1, -1], np.sort(places)])
    T = len(places)
    out = torch.full((T, 2, hkv * D + 24), 5.0, device=DEV, dtype=dtype)
    P.pulse_load_kv(sh, pool, n_slots, dev(places, torch.int64), T, out[:, 0, 16:], out.stride(0), out[:, 1, 8:],
                    out.stride(0), status)
    assert status.item() == 0
    live = torch.from_numpy(places >= 0)
    for side, at in ((0, 16), (1, 8)):
        want = cache.values()[side].transpose(1, 2).reshape(-1, hkv, D)[places]
        got = out[:, side, at:at + hkv * D].unflatten(1, (hkv, D)).cpu()
        assert equal(got[live], want[live]) and (got[~live] == 5).all()
    assert (out[:, 0, :16] == 5).all() and (out[:, 0, 16 + hkv * D:] == 5).all() and (out[:, 1, :8] == 5).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f16"])
def test_rounding_of_every_value(dt):
    """Every 16-bit value as a block's largest and as a member below a larger one; ties, signs, subnormal codes, the
    ends of the exponents' range, infinities and NaN."""
    dtype, code = TYPES[dt]
    every = torch.arange(65536, dtype=torch.int32).to(torch.uint16).view(dtype)
    lead = torch.exp2(torch.floor(torch.log2(every.float().abs().nan_to_num(1).clamp(min=1e-30, max=1e38))) +
                      torch.arange(65536) % 19).clamp(max=torch.finfo(dtype).max)
    x = torch.zeros((2, 65536, 1, D), dtype=dtype)
    x[0, :, 0, 7] = every
    x[1, :, 0, 100], x[1, :, 0, 3] = every, lead.to(dtype)
    sh = P.make_shape(1, 1, D, 16, code)
    pool = torch.zeros((65536, P.pulse_block_bytes(sh)), dtype=torch.uint8, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    m = torch.arange(65536, device=DEV) * 16
    back = torch.empty(x.shape, dtype=dtype, device=DEV)
    xd = x.to(DEV)
    P.pulse_append_kv(sh, xd[0], D, xd[1], D, m, 65536, pool, 65536, status)
    P.pulse_load_kv(sh, pool, 65536, m, 65536, back[0], D, back[1], D, status)
    assert status.item() == 0
    for side in (0, 1):
        r = x[side, :, 0].double().numpy()
        e = plain8.exponent(np.where(np.isfinite(r), np.abs(r), 0).max(1), dtype)[:, None]
        want = torch.from_numpy(plain8.decode(plain8.encode(r, e), e))
        got = back[side, :, 0].double().cpu()
        bad = ~((got == want) | (got.isnan() & want.isnan()))
        assert not bad.any(), (r[bad][:4], got[bad][:4], want[bad][:4])
        assert torch.equal(want.isnan(), ~x[side, :, 0].isfinite())


@pytest.mark.gpu
@pytest.mark.parametrize("bs,hkv", [(16, 8), (32, 3), (64, 8), (64, 1)])
def test_many_rows(bs, hkv):
    """More rows and heads than the rule for one row per workgroup: runs that begin anywhere in a group and go on into
    the next, requests of one token among them, earlier tokens in the first blocks."""
    say(f"\n[gpu] kv8 rows bs={bs} hkv={hkv}")
    rng = np.random.default_rng(bs + hkv)
    sh = P.make_shape(hkv, hkv, D, bs, P.PULSE_BF16_KV8)
    lengths = [1, 1, 300, 7, 1, 64, 900, 33, 1, 1, 1500] + [1] * 40 + [1, 2, 3] * 20 + [6000 // hkv]
    start = [int(rng.integers(0, bs)) for _ in lengths]
    need = [-(-(s + n) // bs) for s, n in zip(start, lengths)]
    slots = rng.permutation(sum(need) + 3)
    cache = plain8.Cache(len(slots), hkv, bs, torch.bfloat16)
    pool = torch.zeros((len(slots), P.pulse_block_bytes(sh)), dtype=torch.uint8, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    first, then, g = [], [], 0
    for s, n, m in zip(start, lengths, need):
        t = np.arange(s + n)
        at = slots[g + t // bs] * bs + t % bs
        first += list(at[:s])
        then += list(at[s:])
        g += m
    for places in (first, then):
        T = len(places)
        x = (torch.randn((2, T, hkv, D)) * torch.exp2(torch.randn((2, T, 1, 1)))).bfloat16()
        xd = x.to(DEV)
        P.pulse_append_kv(sh, xd[0], hkv * D, xd[1], hkv * D, dev(places, torch.int64), T, pool, len(slots), status)
        assert status.item() == 0
        cache.append(x[0], x[1], [int(p) for p in places])
        same_bytes(pool, cache)
    assert len(then) * hkv > 8192


@pytest.mark.gpu
def test_codes_that_were_there_follow_the_scale():
    """A block whose tokens grow by a factor of two a token: codes are rounded again and again, down to nothing; then
    infinities and NaN, which set no scale."""
    for dt, bs in (("bf16", 64), ("f16", 16)):
        dtype, code = TYPES[dt]
        sh = P.make_shape(2, 2, D, bs, code)
        pool = torch.zeros((1, P.pulse_block_bytes(sh)), dtype=torch.uint8, device=DEV)
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        cache = plain8.Cache(1, 2, bs, dtype)
        for t in range(bs):
            x = (torch.randn((2, 1, 2, D)) * 2.0 ** (t * (1 if bs == 16 else 0.5) - 4)).to(dtype)
            x[0, 0, 1] = x[0, 0, 1] * 0  # the second head's keys stay nothing
            if t == 9:
                x[0, 0, 0, 5], x[1, 0, 1, 6], x[1, 0, 0, 7] = math.inf, -math.inf, math.nan
            xd = x.to(DEV)
            P.pulse_append_kv(sh, xd[0], 2 * D, xd[1], 2 * D, dev([t], torch.int64), 1, pool, 1, status)
            cache.append(x[0], x[1], [t])
            same_bytes(pool, cache)
        assert status.item() == 0


@pytest.mark.gpu
def test_places_out_of_range_are_reported_and_skipped():
    sh = P.make_shape(4, 2, D, 16, P.PULSE_BF16_KV8)
    for bad in (32, -2, 2**40, -2**62):
        k = torch.randn((3, 2, D), device=DEV).bfloat16()
        pool = torch.full((2, P.pulse_block_bytes(sh)), 9, dtype=torch.uint8, device=DEV)
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        m = dev([0, bad, 16], torch.int64)
        P.pulse_append_kv(sh, k, 2 * D, k, 2 * D, m, 3, pool, 2, status)
        assert status.item() == P.PULSE_ERR_BAD_INDEX
        cache = plain8.Cache(2, 2, 16, torch.bfloat16)
        cache.append(k, k, [0, None, 16])
        same_bytes(pool, cache)
        out = torch.full((2, 3, 2, D), 5.0, device=DEV).bfloat16()
        status.zero_()
        P.pulse_load_kv(sh, pool, 2, m, 3, out[0], 2 * D, out[1], 2 * D, status)
        assert status.item() == P.PULSE_ERR_BAD_INDEX
        for side, o in enumerate(out):
            want = cache.values()[side]
            assert equal(o[0], want[0, :, 0]) and equal(o[2], want[1, :, 0]) and (o[1] == 5).all()


@pytest.mark.gpu
def test_rows_past_32_bit_offsets():
    """A pool of more than 4 GiB: rows at its end are written there, and nothing else changes."""
    sh = P.make_shape(8, 8, D, 64, P.PULSE_BF16_KV8)
    U = P.pulse_block_bytes(sh)
    n_slots = (9 << 29) // U + 1
    pool = torch.zeros((n_slots, U), dtype=torch.uint8, device=DEV)
    T = 128
    k = torch.randn((2, T, 8, D)).bfloat16()
    kd = k.to(DEV)
    m = torch.arange(T, device=DEV) + (n_slots * 64 - T)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    out = torch.zeros_like(kd)
    P.pulse_append_kv(sh, kd[0], 8 * D, kd[1], 8 * D, m, T, pool, n_slots, status)
    P.pulse_load_kv(sh, pool, n_slots, m, T, out[0], 8 * D, out[1], 8 * D, status)
    assert status.item() == 0
    cache = plain8.Cache(2, 8, 64, torch.bfloat16)
    cache.append(k[0], k[1], list(range(128)))
    vals = cache.values()
    for side in (0, 1):
        assert equal(out[side], vals[side].transpose(1, 2).reshape(T, 8, D))
    assert not pool[:-2].any()
    q = torch.randn((1, 8, D)).bfloat16()
    got = attend(sh, q.to(DEV), pool, dev([[n_slots - 2, n_slots - 1]]), dev([[0, 1]]), dev([2]), dev([128]))
    ref = plain64.attention(q[0], *(x.transpose(0, 1).reshape(8, -1, D) for x in vals), SCALE)
    check_attention(got[0][0], got[1][0], *ref, 128)


# ------------------------------------------------------------------------------------------------ attention


def case_state(ctx, cnt, hq, hkv, bs, dt, gen, garbage=True):
    """A pool of drawn rows, packed by the plain form, whose blocks lie in slots of no order; behind a context's last
    token lie NaN codes."""
    dtype, code = TYPES[dt]
    B = len(ctx)
    n = [-(-x // bs) for x in ctx]
    total = max(1, sum(cnt))
    slots = np.random.default_rng(sum(ctx) + bs).permutation(total + 2)
    kv = torch.randn((2, total + 2, hkv, bs, D), generator=gen)
    kv = (kv * torch.exp2(torch.randint(-3, 3, kv.shape[:-2] + (1, 1), generator=gen).float())).to(dtype)
    pool, cache = plain8.pack(kv[0], kv[1], bs)
    vals = cache.values()
    table = np.full((B, max(1, max(n))), -1, np.int32)
    k_max = max(1, max(cnt))
    sel = np.full((B, k_max), -1, np.int32)
    g, rng = 0, np.random.default_rng(1)
    for r in range(B):
        j = np.sort(rng.choice(n[r], size=cnt[r], replace=False)) if cnt[r] else np.zeros(0, int)
        if cnt[r]:
            j[-1] = n[r] - 1  # the last block, partly filled
        sel[r, : cnt[r]], table[r, j] = j, slots[g:g + cnt[r]]
        g += cnt[r]
        left = n[r] * bs - ctx[r]
        if garbage and cnt[r] and left:
            cache.code[table[r, n[r] - 1], :, :, bs - left:] = 0xFF
    if garbage:  # the slots of no request: scales of no meaning
        pool = torch.from_numpy(cache.bytes()[0])
        pool[slots[total:]] = 255
    q = torch.randn((B, hq, D), generator=gen).mul_(1.5).to(dtype)
    sh = P.make_shape(hq, hkv, D, bs, code)
    return sh, q, pool, torch.from_numpy(table), torch.from_numpy(sel), vals


ATTEND = [
    ([1], [1], 1, 1, 16, "bf16"),
    ([1, 16, 17, 33], [1, 1, 2, 3], 4, 2, 16, "f16"),
    ([5, 0, 40], [1, 0, 2], 8, 2, 16, "bf16"),                      # a request without a block
    ([100, 90, 80], [0, 0, 0], 4, 1, 32, "bf16"),                   # no selection at all
    ([31, 32, 33, 64, 65], [1, 1, 2, 2, 3], 6, 3, 32, "f16"),
    ([63, 64, 65, 500], [1, 1, 2, 8], 16, 2, 64, "bf16"),           # eight query heads per head
    ([700, 333], [40, 21], 12, 1, 16, "f16"),                        # twelve
    ([700, 333], [40, 21], 16, 1, 16, "bf16"),
    ([300], [17], 5, 1, 16, "bf16"),
    ([300], [17], 7, 1, 32, "f16"),
    ([1999], [125], 32, 8, 16, "bf16"),                              # several workgroups per head
    ([4000, 100, 2500], [250, 7, 100], 3, 3, 16, "f16"),              # counts that differ
    ([3000, 2999, 17, 1], [40, 94, 1, 1], 28, 4, 32, "bf16"),
    ([1000] * 70, [5] * 70, 2, 2, 64, "bf16"),
    ([9000], [563], 8, 8, 16, "bf16"),
    ([1050] * 24, [66] * 24, 8, 8, 16, "bf16"),
    ([2100] + [1900] * 11, [132] + [119] * 11, 8, 8, 16, "bf16"),
    ([1300] * 130, [41] * 130, 2, 1, 32, "f16"),
    ([3200] + [16 * (7 * i % 60) for i in range(69)], [200] + [7 * i % 60 for i in range(69)], 2, 2, 16, "bf16"),
    ([16 * (5 * i % 77) for i in range(256)], [5 * i % 77 for i in range(256)], 1, 1, 16, "bf16"),
    ([16 * (5 * i % 77) for i in range(257)], [5 * i % 77 for i in range(257)], 16, 1, 16, "f16"),
]


@pytest.mark.gpu
@pytest.mark.parametrize("case", range(len(ATTEND)))
def test_attention_over_the_8_bit_cache(case):
    ctx, cnt, hq, hkv, bs, dt = ATTEND[case]
    cnt = [min(c, -(-x // bs)) for c, x in zip(cnt, ctx)]
    say(f"\n[gpu] kv8 attention ctx={ctx[:4]} cnt={cnt[:4]} hq={hq} hkv={hkv} bs={bs} {dt}")
    gen = torch.Generator().manual_seed(case)
    sh, q, pool, table, sel, vals = case_state(ctx, cnt, hq, hkv, bs, dt, gen)
    args = (sh, *(x.to(DEV) for x in (q, pool, table, sel)), dev(cnt), dev(ctx))
    out, lse = attend(*args)
    for r in range(len(ctx)):
        if not cnt[r]:
            assert (out[r] == 0).all() and (lse[r] == -math.inf).all()
            continue
        j = sel[r, : cnt[r]].long()
        k, v = (x[table[r, j].long()].transpose(0, 1).reshape(hkv, -1, D) for x in vals)
        n = (j[:, None] * bs + torch.arange(bs)).view(-1) < ctx[r]
        check_attention(out[r], lse[r], *plain64.attention(q[r], k[:, n], v[:, n], SCALE), int(n.sum()))
    again = attend(*args, ws_fill=0)
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])
    assert torch.equal(attend(*args, lse=False)[0], out)


@pytest.mark.gpu
def test_probabilities_keep_all_their_bits():
    """Values of one size and alternating signs: the sums cancel down to what the probabilities' last bits leave."""
    ctx, cnt, hq, hkv, bs = [2000], [125], 4, 1, 16
    gen = torch.Generator().manual_seed(5)
    sh, q, pool, table, sel, vals = case_state(ctx, cnt, hq, hkv, bs, "bf16", gen)
    out, _ = attend(sh, *(x.to(DEV) for x in (q, pool, table, sel)), dev(cnt), dev(ctx))
    j = sel[0, :125].long()
    k, v = (x[table[0, j].long()].transpose(0, 1).reshape(1, -1, D) for x in vals)
    want, _, mass, _ = plain64.attention(q[0], k, v, SCALE)
    # logits of up to 134 products, 2^-24 of their sizes each, move a probability by that much; the typical error is
    # the square root of such counts: 2^-20 of the mass leaves room, a probability of 16 bits would not
    err = ((out[0].double().cpu() - want).abs() / mass).mean().item()
    assert err < 2.0**-20, err


@pytest.mark.gpu
@pytest.mark.parametrize("which", ["key", "value"])
def test_a_nan_code_stays_in_its_head(which):
    ctx, cnt, bs, hq = [200, 200], [13, 13], 16, 8
    gen = torch.Generator().manual_seed(3)
    sh, q, pool, table, sel, _ = case_state(ctx, cnt, hq, 2, bs, "bf16", gen, garbage=False)
    head = pool[table[1, 4], 256 * bs:512 * bs]
    head[5 * D + 77 if which == "key" else 128 * bs + (77 % 16 * 8 + 77 // 16) * 8 + 5] = 0x7F
    out, _ = attend(sh, *(x.to(DEV) for x in (q, pool, table, sel)), dev(cnt), dev(ctx))
    nan = out.isnan().cpu().view(2, 2, hq // 2, D)
    assert not nan[0].any() and not nan[1, 0].any()
    if which == "key":
        assert nan[1, 1].all()
        for b in table[1]:  # every key of the request: nothing is left that is not NaN
            pool[b, 256 * bs:256 * bs + 128 * bs] = 0xFF
        nan = attend(sh, *(x.to(DEV) for x in (q, pool, table, sel)), dev(cnt), dev(ctx))[0].isnan().cpu().view(2, 2, -1)
        assert nan[1, 1].all() and not nan[0].any() and not nan[1, 0].any()
    else:
        assert nan[1, 1, :, 77].all() and nan[1, 1].sum() == hq // 2


@pytest.mark.gpu
def test_missing_blocks_are_reported():
    ctx, cnt = [200], [13]
    gen = torch.Generator().manual_seed(3)
    sh, q, pool, table, sel, _ = case_state(ctx, cnt, 4, 2, 16, "bf16", gen)
    for j, bad in ((3, -1), (5, pool.shape[0]), (12, -9)):
        t = table.clone()
        t[0, j] = bad
        attend(sh, *(x.to(DEV) for x in (q, pool, t, sel)), dev(cnt), dev(ctx), status_want=P.PULSE_ERR_BAD_INDEX)
    attend(sh, *(x.to(DEV) for x in (q, pool, table, sel)), dev([14]), dev(ctx), status_want=P.PULSE_ERR_BAD_INDEX)


# ------------------------------------------------------------------------------------------------ host entry


def test_kv8_sizes_and_refusals():
    sh = P.make_shape(32, 8, D, 16, P.PULSE_BF16_KV8)
    assert P.pulse_block_bytes(sh) == 32 * 1024 + 128
    assert P.pulse_block_bytes(P.make_shape(6, 3, D, 64, P.PULSE_F16_KV8)) == 3 * 256 * 64 + 128
    assert P.pulse_block_bytes(P.make_shape(65, 65, D, 16, P.PULSE_F16_KV8)) == 65 * 256 * 16 + 256
    assert P.pulse_block_bytes(P.make_shape(32, 8, 64, 16, P.PULSE_BF16_KV8)) == 0
    assert P.pulse_workspace_bytes(sh, 4, 64, 100) > 0 and P.pulse_attention_workgroups(sh, 4, 64) > 0
    assert P.pulse_mam_workspace_bytes(sh, 2, 8) == 0
    assert P.pulse_mam(sh, FAKE, FAKE, 10, FAKE, 4, FAKE, 2, 1, 8, 0.1, FAKE, FAKE, FAKE, 1 << 30, stream=0,
                       check=False) == P.PULSE_ERR_UNSUPPORTED
    with pytest.raises(P.PulseError) as e:
        P.GatherScatterEngine(sh, 1, 8, 8)
    assert e.value.status == P.PULSE_ERR_UNSUPPORTED
    r = dict(host_kv=FAKE, blk_off=FAKE, B=2, sel_idx=FAKE, sel_cnt=FAKE, k_max=16, block_table=FAKE, max_blocks=100,
             free_slots=FAKE, free_head=FAKE, n_free=10, slot_pool=FAKE, n_slots=50, stats=FAKE, dev_status=FAKE, ws=FAKE,
             ws_bytes=1, stream=0, check=False)
    t = dict(q=FAKE, slot_pool=FAKE, n_slots=50, block_table=FAKE, max_blocks=100, sel_idx=FAKE, sel_cnt=FAKE, k_max=16,
             ctx_len=FAKE, B=2, sm_scale=0.1, out=FAKE, lse=None, dev_status=FAKE, ws=FAKE, ws_bytes=1, stream=0,
             check=False)
    assert P.pulse_recall_gather(sh, **r) == P.PULSE_ERR_WORKSPACE
    assert P.pulse_recall_gather(sh, **{**r, "host_kv": FAKE + 8}) == P.PULSE_ERR_INVALID_ARG
    assert P.pulse_recall_gather(sh, **{**r, "slot_pool": FAKE + 8}) == P.PULSE_ERR_INVALID_ARG
    assert P.pulse_sparse_decode_attn(sh, **t) == P.PULSE_ERR_WORKSPACE
    assert P.pulse_sparse_decode_attn(sh, **{**t, "slot_pool": FAKE + 8}) == P.PULSE_ERR_INVALID_ARG
    a = dict(k=FAKE, k_stride=1024, v=FAKE, v_stride=1024, slot_map=FAKE, n_rows=3, slot_pool=FAKE, n_slots=9,
             dev_status=FAKE, stream=0, check=False)
    for fn in (P.pulse_append_kv, P.pulse_load_kv):
        call = lambda s=sh, **kw: fn(s, **{**a, **kw})  # noqa: E731
        for name in ("k", "v", "slot_pool"):
            assert call(**{name: FAKE + 8}) == P.PULSE_ERR_INVALID_ARG, name
        for kw in (dict(k_stride=1016), dict(v_stride=1028), dict(n_rows=-1), dict(n_slots=0), dict(slot_map=None)):
            assert call(**kw) == P.PULSE_ERR_INVALID_ARG, kw
        assert call(n_rows=0, k=None) == P.PULSE_OK


def test_plain_form():
    """The levels are e4m3's; codes are the nearest, as torch's cast has them; an append token by token ends within half
    a step of every rounding."""
    every = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert (every == plain8.LEVELS).all()
    x = np.concatenate([np.linspace(-448, 448, 9001), plain8.MIDS, -plain8.MIDS])
    cast = torch.from_numpy(x).float().to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    ok = torch.from_numpy(x).float().double().numpy() == x
    assert (plain8.decode(plain8.encode(x, 0), 0) == plain8.decode(cast, 0))[ok].all()
    gen = torch.Generator().manual_seed(1)
    kv = torch.randn((2, 16, 2, D), generator=gen).bfloat16()
    one, whole = (plain8.Cache(1, 2, 16, torch.bfloat16) for _ in range(2))
    whole.append(kv[0], kv[1], range(16))
    for t in range(16):
        one.append(kv[0, t:t + 1], kv[1, t:t + 1], [t])
    assert (one.exp == whole.exp).all()
    for a, b in zip(one.values(), whole.values()):
        assert ((a - b).abs() <= 2.0**-9 * 2.0 ** torch.from_numpy(one.exp).max()).all()


@pytest.mark.parametrize("dt", ["bf16", "f16"])
def test_a_workspace_serves_smaller_calls(dt):
    for hq, hkv, bs in ((32, 8, 16), (16, 1, 64), (28, 4, 32), (2, 2, 16), (48, 4, 64), (3, 3, 32)):
        sh = P.make_shape(hq, hkv, D, bs, TYPES[dt][1])
        before = None
        for B in [1, 2, 3, 7, 16, 17, 31, 33, 64, 65, 86, 128, 129, 256, 257, 512, 1000]:
            row, most = [], 0
            for k in [1, 2, 3, 8, 9, 17, 63, 64, 65, 127, 130, 256, 257, 500, 513, 1000, 4100]:
                n = P.pulse_workspace_bytes(sh, B, k, 0)
                assert n >= 4 * (B * k + 3 * B) + P.pulse_attention_workgroups(sh, B, k) * B * hq * (4 * D + 8)
                most = max(most, n)
                assert n == most
                row.append(n)
            assert before is None or all(a <= b for a, b in zip(before, row))
            before = row
