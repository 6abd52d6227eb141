"""The 4-bit cache: rows written and read, attention over it, recall of its blocks and the layer-step, against plain
forms in 64 bits."""
import math

import numpy as np
import pytest
import torch

import plain64
from paper_2609_34555_amd import pulse as P
from parity import say

DEV = "cuda"
D = 128
FAKE = 0x1000
TYPES = {"bf16": (torch.bfloat16, P.PULSE_BF16, P.PULSE_BF16_KV4), "f16": (torch.float16, P.PULSE_F16, P.PULSE_F16_KV4)}
SCALE = 1 / math.sqrt(D)


def dev(x, dtype=torch.int32):
    return torch.tensor(np.asarray(x), dtype=dtype, device=DEV)


def equal(a, b):
    """Equal values, NaN where the other is NaN (a zero has no sign)."""
    a, b = a.double().cpu(), b.double().cpu()
    return bool(((a == b) | (a.isnan() & b.isnan())).all())


# ------------------------------------------------------------------------------------------------ rows

ROWS = [  # places of the rows (None: nowhere), bs
    ([0], 16),
    ([15, 16, 31, 32], 16),                                 # octets' and blocks' ends
    (list(range(40)), 16),                                   # whole octets and blocks
    (list(range(5, 61)), 64),                                # a run that begins and ends inside an octet
    ([7, 6, 5, 4, 3, 2, 1, 0], 16),                          # every row its own run, all in one octet
    ([0, 2, 4, 6, 1, 3, 5, 7], 32),
    ([3, 4, 5, None, 6, 7, None, None, 8], 16),
    ([None] * 3, 16),
    ([60, 61, 62, 63, 100, 101, 8, 9, 10, 11, 12, 13, 14, 15, 16, 17], 32),
    (list(range(64, 128)) + list(range(0, 64)) + list(range(200, 219)), 64),
]


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("four", [True, False])
@pytest.mark.parametrize("hkv", [1, 3, 8])
@pytest.mark.parametrize("case", range(len(ROWS)))
def test_append_and_load(case, hkv, four, dt):
    places, bs = ROWS[case]
    dtype, code16, code4 = TYPES[dt]
    gen = torch.Generator(device=DEV)
    gen.manual_seed(case)
    T, n_slots = len(places), max([p or 0 for p in places]) // bs + 3
    sh = P.make_shape(2 * hkv, hkv, D, bs, code4 if four else code16)
    U = P.pulse_block_bytes(sh)
    assert U == (hkv * 136 * bs if four else hkv * bs * 512)
    # rows of different sizes inside wider ones
    wide = torch.randn((T, 2, hkv * D + 24), generator=gen, device=DEV)
    wide = (wide * torch.exp2(torch.randint(-6, 6, (T, 1, 1), generator=gen, device=DEV).float())).to(dtype)
    k, v = wide[:, 0, 8:8 + hkv * D], wide[:, 1, 16:16 + hkv * D]
    before = torch.randint(0, 255, (n_slots, U), generator=gen, device=DEV, dtype=torch.uint8)
    pool, status = before.clone(), torch.zeros(1, dtype=torch.int32, device=DEV)
    m = dev([-1 if p is None else p for p in places], torch.int64)
    stride = wide.stride(0)
    P.pulse_append_kv(sh, k, stride, v, stride, m, T, pool, n_slots, status)
    assert status.item() == 0
    # the blocks: what was there, with the rows' tokens in their places
    live = [(i, p) for i, p in enumerate(places) if p is not None]
    kr, vr = (x.unflatten(1, (hkv, D)).cpu() for x in (k, v))
    if four:
        kd, vd = torch.zeros((2, n_slots, hkv, bs, D), dtype=dtype)
        for i, p in live:
            kd[p // bs, :, p % bs], vd[p // bs, :, p % bs] = kr[i], vr[i]
        want = plain64.pack(kd, vd, bs).numpy().reshape(n_slots, hkv, -1)
        old = before.cpu().numpy().reshape(n_slots, hkv, -1)
        mask = np.zeros((n_slots, 136 * bs), np.uint8)  # the bits that the rows own
        for _, p in live:
            b, t = p // bs, p % bs
            mask[b, t * 64:(t + 1) * 64] = 255
            for w in range(D):
                mask[b, 64 * bs + 4 * (t // 8 * 128 + w) + t % 8 // 2] |= 15 << (4 * (t % 2))
            mask[b, 128 * bs + 4 * t:128 * bs + 4 * t + 4] = 255
            mask[b, 132 * bs + t::bs] = 255
        mask = mask[:, None]
        want = (want & mask) | (old & ~mask)
        got = pool.cpu().numpy().reshape(want.shape)
        assert (got == want).all(), np.argwhere(got != want)[:5]
    else:
        want = before.cpu().view(torch.int16).clone().view(n_slots, 2, hkv, -1)
        for i, p in live:
            want[p // bs, 0].view(hkv, bs, D)[:, p % bs] = kr[i].contiguous().view(torch.int16)
            want[p // bs, 1].view(hkv, D, bs)[:, :, p % bs] = vr[i].contiguous().view(torch.int16)
        assert torch.equal(pool.cpu().view(torch.int16).view_as(want), want)
    # and back, into wider rows
    out = torch.full_like(wide, 5.0)
    P.pulse_load_kv(sh, pool, n_slots, m, T, out[:, 0, 16:], stride, out[:, 1, 8:], stride, status)
    assert status.item() == 0
    ko, vo = out[:, 0, 16:16 + hkv * D].unflatten(1, (hkv, D)), out[:, 1, 8:8 + hkv * D].unflatten(1, (hkv, D))
    for x, y in ((kr, ko), (vr, vo)):
        x = plain64.quantise(x)[2] if four else x
        for i, p in enumerate(places):
            assert equal(y[i], x[i]) if p is not None else (y[i] == 5).all()
    assert (out[:, 0, :16] == 5).all() and (out[:, 0, 16 + hkv * D:] == 5).all() and (out[:, 1, :8] == 5).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f16"])
def test_rounding_of_every_value(dt):
    """Every finite 16-bit value as a group's largest and as a member below a larger one; ties, signs, the ends of the
    exponents' range; groups with an infinity or a NaN."""
    dtype, _, code = TYPES[dt]
    every = torch.arange(65536, dtype=torch.int32).to(torch.uint16).view(dtype)
    every = every.view(-1, 1)
    alone = torch.zeros((65536, 32), dtype=dtype)
    alone[:, 7:8] = every
    # beside a power of two up to 2^4 above: all members from nothing to all 7 codes
    lead = torch.exp2(torch.floor(torch.log2(every.float().abs().clamp(min=1e-30, max=1e38))) +
                      torch.arange(65536).view(-1, 1) % 5).clamp(max=torch.finfo(dtype).max)
    pair = torch.zeros((65536, 32), dtype=dtype)
    pair[:, 31:32], pair[:, 0:1] = every, lead.to(dtype)
    x = torch.cat([alone.view(-1, 4, 32), pair.view(-1, 4, 32)]).view(-1, 1, D).to(DEV)  # 4 groups a row
    T, bs = x.shape[0], 64
    n_slots = T // bs
    sh = P.make_shape(1, 1, D, bs, code)
    pool = torch.zeros((n_slots, P.pulse_block_bytes(sh)), dtype=torch.uint8, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    m = torch.arange(T, device=DEV)
    back = torch.empty((2,) + x.shape, dtype=dtype, device=DEV)
    P.pulse_append_kv(sh, x, D, x, D, m, T, pool, n_slots, status)
    P.pulse_load_kv(sh, pool, n_slots, m, T, back[0], D, back[1], D, status)
    assert status.item() == 0
    codes, scales, want = plain64.quantise(x)
    assert want.isnan().any() and want[~want.isnan()].isfinite().all()
    for got in back:
        bad = ~((got.double().cpu() == want) | (got.cpu().isnan() & want.isnan()))
        assert not bad.any(), (x.cpu()[bad][:4], got.cpu()[bad][:4], want[bad][:4])


@pytest.mark.gpu
def test_places_out_of_range_are_reported_and_skipped():
    sh = P.make_shape(4, 2, D, 16, P.PULSE_BF16_KV4)
    for bad in (32, -2, 2**40, -2**62):
        k = torch.randn((3, 2, D), device=DEV).bfloat16()
        pool = torch.full((2, P.pulse_block_bytes(sh)), 9, dtype=torch.uint8, device=DEV)
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        m = dev([3, bad, 31], torch.int64)
        P.pulse_append_kv(sh, k, 2 * D, k, 2 * D, m, 3, pool, 2, status)
        assert status.item() == P.PULSE_ERR_BAD_INDEX
        out = torch.full((2, 3, 2, D), 5.0, device=DEV).bfloat16()
        status.zero_()
        P.pulse_load_kv(sh, pool, 2, m, 3, out[0], 2 * D, out[1], 2 * D, status)
        assert status.item() == P.PULSE_ERR_BAD_INDEX
        want = plain64.quantise(k)[2]
        for o in out:
            assert equal(o[0], want[0]) and equal(o[2], want[2]) and (o[1] == 5).all()


@pytest.mark.gpu
def test_rows_past_32_bit_offsets():
    """A pool of more than 4 GiB: rows at its end are written there, and nothing else changes."""
    sh = P.make_shape(8, 8, D, 64, P.PULSE_BF16_KV4)
    U = P.pulse_block_bytes(sh)
    n_slots = (9 << 29) // U + 1
    pool = torch.zeros((n_slots, U), dtype=torch.uint8, device=DEV)
    T = 70
    k = torch.randn((2, T, 8, D), device=DEV).bfloat16()
    m = torch.arange(T, device=DEV) + (n_slots * 64 - T)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    out = torch.zeros_like(k)
    P.pulse_append_kv(sh, k[0], 8 * D, k[1], 8 * D, m, T, pool, n_slots, status)
    P.pulse_load_kv(sh, pool, n_slots, m, T, out[0], 8 * D, out[1], 8 * D, status)
    assert status.item() == 0
    assert equal(out, plain64.quantise(k)[2])
    assert not pool[:-2].any()
    # attention over the last blocks
    q = torch.randn((1, 8, D), device=DEV).bfloat16()
    table = torch.full((1, 2), 0, dtype=torch.int32, device=DEV)
    table[0] = dev([n_slots - 2, n_slots - 1])
    ctx = dev([128])
    got = attend(sh, q, pool, table, dev([[0, 1]]), dev([2]), ctx)
    kd, vd = plain64.unpack(pool[-2:], 8, 64)
    out, lse, mass, reach = plain64.attention(q[0].cpu(), *(x.transpose(0, 1).reshape(8, -1, D) for x in (kd, vd)), SCALE)
    check_attention(got[0][0], got[1][0], out, lse, mass, reach, 128)


# ------------------------------------------------------------------------------------------------ attention


def attend(sh, q, pool, table, sel, cnt, ctx, lse=True, ws_fill=255, status_want=0):
    B, k_max = sel.shape
    nb = P.pulse_workspace_bytes(sh, B, k_max, 0)
    ws = torch.full((max(nb, 1),), ws_fill, dtype=torch.uint8, device=DEV)
    out = torch.full((B, sh.num_q_heads, D), 3.0, device=DEV)
    ls = torch.full((B, sh.num_q_heads), 3.0, device=DEV) if lse else None
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    P.pulse_sparse_decode_attn(sh, q, pool, pool.shape[0], table, table.shape[1], sel, cnt, k_max, ctx, B, SCALE, out,
                               ls, status, ws, nb)
    assert status.item() == status_want
    return out, ls


def check_attention(out, lse, want, want_lse, mass, reach, n):
    """A logit is a sum of 128 fp32 products of exact factors (132 * 2^-24 of the sum of their sizes covers it and the
    scaling), the exponential adds 2^-23 of its value and 2^-24 of its argument, which no larger than twice `reach` is;
    the probability is a sum of bf16 parts (2^-16 at most), summed over n tokens in fp32 (as is the denominator)."""
    logit = reach * 134 * 2.0**-24 + 2.0**-23
    rel = (2 * logit + 2.0**-16 + (n + 16) * 2.0**-23)[:, None]
    over = ((out.double().cpu() - want).abs() / (mass * rel + 1e-30)).max().item()
    over_lse = ((lse.double().cpu() - want_lse).abs() / (logit + (n + 16) * 2.0**-23 + want_lse.abs() * 2.0**-22)).max().item()
    say(f"  {over:.4f} / {over_lse:.4f} of the bound")
    assert over <= 1 and over_lse <= 1


def case_state(ctx, cnt, hq, hkv, bs, dt, gen, garbage=True):
    """A pool of drawn rows, quantised by the plain form, whose blocks lie in slots of no order; the bytes behind the
    last token of a context are garbage (every scale byte 255 among them)."""
    dtype, _, code = TYPES[dt]
    B = len(ctx)
    n = [-(-x // bs) for x in ctx]
    total = max(1, sum(cnt))
    slots = np.random.default_rng(sum(ctx) + bs).permutation(total + 2)
    kv = torch.randn((2, total + 2, hkv, bs, D), generator=gen)
    kv = (kv * torch.exp2(torch.randint(-4, 4, kv.shape[:-1] + (1,), generator=gen).float())).to(dtype)
    pool = plain64.pack(kv[0], kv[1], bs)
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
            b = pool.view(total + 2, hkv, 136 * bs)[table[r, n[r] - 1]]
            t = bs - left
            b[:, t * 64:bs * 64] = 0x77
            b[:, 128 * bs + 4 * t:132 * bs] = 255
            b[:, 132 * bs:].view(hkv, 4, bs)[:, :, t:] = 255
    q = torch.randn((B, hq, D), generator=gen).mul_(1.5).to(dtype)
    sh = P.make_shape(hq, hkv, D, bs, code)
    return sh, q, pool, torch.from_numpy(table), torch.from_numpy(sel)


# contexts, selected blocks, hq, hkv, bs, dtype
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
    # more than a round of workgroups: equal counts in one and in two workgroups each, counts that fit a round with
    # more entries per wave, more requests than lanes, as many as a plan takes, one more
    ([1050] * 24, [66] * 24, 8, 8, 16, "bf16"),
    ([2100] * 12, [132] * 12, 16, 8, 16, "f16"),
    ([2100] + [1900] * 11, [132] + [119] * 11, 8, 8, 16, "bf16"),
    ([1300] * 130, [41] * 130, 2, 1, 32, "f16"),
    ([3200] + [16 * (7 * i % 60) for i in range(69)], [200] + [7 * i % 60 for i in range(69)], 2, 2, 16, "bf16"),
    ([32 * (11 * i % 50) + 32 for i in range(199)] + [4000], [11 * i % 50 + 1 for i in range(199)] + [125], 16, 1, 32, "f16"),
    ([16 * (5 * i % 77) for i in range(256)], [5 * i % 77 for i in range(256)], 1, 1, 16, "bf16"),
    ([16 * (5 * i % 77) for i in range(257)], [5 * i % 77 for i in range(257)], 1, 1, 16, "f16"),
]


@pytest.mark.gpu
@pytest.mark.parametrize("case", range(len(ATTEND)))
def test_attention_over_the_4_bit_cache(case):
    ctx, cnt, hq, hkv, bs, dt = ATTEND[case]
    cnt = [min(c, -(-x // bs)) for c, x in zip(cnt, ctx)]
    say(f"\n[gpu] kv4 attention ctx={ctx[:4]} cnt={cnt[:4]} hq={hq} hkv={hkv} bs={bs} {dt}")
    gen = torch.Generator().manual_seed(case)
    sh, q, pool, table, sel = case_state(ctx, cnt, hq, hkv, bs, dt, gen)
    d = [x.to(DEV) for x in (q, pool, table, sel)]
    args = (sh, d[0], d[1], d[2], d[3], dev(cnt), dev(ctx))
    out, lse = attend(*args)
    for r in range(len(ctx)):
        if not cnt[r]:
            assert (out[r] == 0).all() and (lse[r] == -math.inf).all()
            continue
        j = sel[r, : cnt[r]].long()
        k, v = (x.transpose(0, 1).reshape(hkv, -1, D) for x in plain64.unpack(pool[table[r, j].long()], hkv, bs))
        n = (j[:, None] * bs + torch.arange(bs)).view(-1) < ctx[r]
        ref = plain64.attention(q[r], k[:, n], v[:, n], SCALE)
        check_attention(out[r], lse[r], *ref, int(n.sum()))
    again = attend(*args, ws_fill=0)
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])
    assert torch.equal(attend(*args, lse=False)[0], out)


@pytest.mark.gpu
@pytest.mark.parametrize("hq", [4, 8, 16])
@pytest.mark.parametrize("which", ["key", "value"])
def test_a_nan_group_stays_in_its_head(hq, which):
    """A group that holds NaN makes its head's (keys) or its channels' (values) results NaN, in no other head."""
    ctx, cnt, bs = [200, 200], [13, 13], 16
    gen = torch.Generator().manual_seed(3)
    sh, q, pool, table, sel = case_state(ctx, cnt, hq, 2, bs, "bf16", gen, garbage=False)
    head = pool.view(-1, 2, 136 * bs)[table[1, 4], 1]
    head[(128 if which == "key" else 132) * bs + (5 * 4 + 2 if which == "key" else 2 * bs + 5)] = 255
    out, _ = attend(sh, *(x.to(DEV) for x in (q, pool, table, sel)), dev(cnt), dev(ctx))
    nan = out.isnan().cpu().view(2, 2, hq // 2, 4, 32)
    assert not nan[0].any() and not nan[1, 0].any()
    assert nan[1, 1].all() if which == "key" else nan[1, 1, :, 2].all() and not nan[1, 1, :, [0, 1, 3]].any()
    if which == "key":  # every key of the request: nothing is left that is not NaN
        for b in table[1]:
            pool.view(-1, 2, 136 * bs)[b, 1, 128 * bs:132 * bs] = 255
        out, _ = attend(sh, *(x.to(DEV) for x in (q, pool, table, sel)), dev(cnt), dev(ctx))
        nan = out.isnan().cpu().view(2, 2, -1)
        assert nan[1, 1].all() and not nan[0].any() and not nan[1, 0].any()


@pytest.mark.gpu
def test_missing_blocks_are_reported():
    ctx, cnt = [200], [13]
    gen = torch.Generator().manual_seed(3)
    sh, q, pool, table, sel = case_state(ctx, cnt, 4, 2, 16, "bf16", gen)
    for j, bad in ((3, -1), (5, pool.shape[0]), (12, -9)):
        t = table.clone()
        t[0, j] = bad
        attend(sh, *(x.to(DEV) for x in (q, pool, t, sel)), dev(cnt), dev(ctx), status_want=P.PULSE_ERR_BAD_INDEX)
    attend(sh, *(x.to(DEV) for x in (q, pool, table, sel)), dev([14]), dev(ctx), status_want=P.PULSE_ERR_BAD_INDEX)


# ------------------------------------------------------------------------------------------------ host entry


def test_kv4_sizes_and_refusals():
    sh = P.make_shape(32, 8, D, 16, P.PULSE_BF16_KV4)
    assert P.pulse_block_bytes(sh) == 17 * 1024
    assert P.pulse_block_bytes(P.make_shape(6, 3, D, 64, P.PULSE_F16_KV4)) == 3 * 136 * 64
    assert P.pulse_block_bytes(P.make_shape(32, 8, 64, 16, P.PULSE_BF16_KV4)) == 0
    assert P.pulse_block_bytes(P.make_shape(32, 8, D, 16, 4)) == 0
    assert P.pulse_workspace_bytes(sh, 4, 64, 100) > 0 and P.pulse_attention_workgroups(sh, 4, 64) > 0
    # what has no 4-bit form refuses the type
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
        for name in ("k", "v", "slot_map", "slot_pool", "dev_status"):
            assert call(**{name: None}) == P.PULSE_ERR_INVALID_ARG, name
        for name in ("k", "v", "slot_pool"):
            assert call(**{name: FAKE + 8}) == P.PULSE_ERR_INVALID_ARG, name
        for kw in (dict(k_stride=1016), dict(v_stride=1028), dict(v_stride=0), dict(n_rows=-1), dict(n_slots=0)):
            assert call(**kw) == P.PULSE_ERR_INVALID_ARG, kw
        assert call(P.make_shape(32, 8, D, 8, P.PULSE_BF16_KV4)) == P.PULSE_ERR_UNSUPPORTED
        assert call(n_rows=0, k=None) == P.PULSE_OK


def test_plain_form_packs_what_it_unpacks():
    gen = torch.Generator().manual_seed(1)
    for dt, bs in ((torch.bfloat16, 16), (torch.float16, 32)):
        kv = torch.randn((2, 2, 3, bs, D), generator=gen).to(dt)
        k, v = plain64.unpack(plain64.pack(kv[0], kv[1], bs), 3, bs)
        assert torch.equal(k, plain64.quantise(kv[0])[2]) and torch.equal(v, plain64.quantise(kv[1])[2])
        # a code is never further than half a step of its group's largest step, or what 6 stands for up to 7
        top = kv.double().unflatten(-1, (4, 32)).abs().amax(-1, keepdim=True)
        err = (torch.stack([k, v]) - kv.double()).unflatten(-1, (4, 32)).abs()
        assert (err <= top / 3.5).all()


@pytest.mark.gpu
@pytest.mark.parametrize("scale", [0.0, -0.1, 3.0])
def test_any_scale(scale):
    ctx, cnt = [200, 77], [13, 5]
    gen = torch.Generator().manual_seed(8)
    sh, q, pool, table, sel = case_state(ctx, cnt, 4, 2, 16, "bf16", gen)
    d = [x.to(DEV) for x in (q, pool, table, sel)]
    out, lse = torch.zeros((2, 4, D), device=DEV), torch.zeros((2, 4), device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    nb = P.pulse_workspace_bytes(sh, 2, 13, 0)
    ws = torch.zeros(nb, dtype=torch.uint8, device=DEV)
    P.pulse_sparse_decode_attn(sh, d[0], d[1], pool.shape[0], d[2], table.shape[1], d[3], dev(cnt), 13, dev(ctx), 2, scale,
                               out, lse, status, ws, nb)
    assert status.item() == 0
    for r in range(2):
        j = sel[r, : cnt[r]].long()
        k, v = (x.transpose(0, 1).reshape(2, -1, D) for x in plain64.unpack(pool[table[r, j].long()], 2, 16))
        n = (j[:, None] * 16 + torch.arange(16)).view(-1) < ctx[r]
        check_attention(out[r], lse[r], *plain64.attention(q[r] * (-1 if scale < 0 else 1), k[:, n], v[:, n], abs(scale)),
                        int(n.sum()))


@pytest.mark.gpu
@pytest.mark.parametrize("B,hq,bs,least", [(132, 4, 32, 130), (132, 2, 32, 3), (256, 2, 32, 130), (256, 2, 32, 100),
                                           (256, 2, 64, 1), (256, 32, 64, 50), (257, 2, 32, 100)])
def test_requests_and_heads_beyond_a_round(B, hq, bs, least):
    """Counts of `least` to 4160 tokens (all that, three quarters and less on average) over blocks that requests share."""
    say(f"\n[gpu] kv4 attention B={B} hq={hq} bs={bs} least={least}")
    hkv, most, n_slots = 2, 4160 // bs, 140
    gen = torch.Generator().manual_seed(B + bs)
    rng = np.random.default_rng(B + bs + least)
    kv = torch.randn((2, n_slots, hkv, bs, D), generator=gen).bfloat16()
    pool = plain64.pack(kv[0], kv[1], bs)
    cnt = rng.integers(min(least, most), most + 1, size=B)
    cnt[rng.integers(B)] = most
    ctx = most * bs - rng.integers(0, bs, size=B)
    table = rng.permuted(np.tile(np.arange(n_slots, dtype=np.int32), (B, 1)), axis=1)[:, :most].copy()
    sel = np.full((B, most), -1, np.int32)
    for r in range(B):
        sel[r, :cnt[r]] = np.sort(rng.choice(most, size=cnt[r], replace=False))
    q = torch.randn((B, hq, D), generator=gen).bfloat16()
    sh = P.make_shape(hq, hkv, D, bs, P.PULSE_BF16_KV4)
    out, lse = attend(sh, q.to(DEV), pool.to(DEV), dev(table), dev(sel), dev(cnt), dev(ctx))
    k, v = (x.transpose(0, 1).reshape(hkv, n_slots, bs, D) for x in plain64.unpack(pool, hkv, bs))
    for r in range(0, B, 3):
        j = sel[r, :cnt[r]]
        n = torch.from_numpy(((j[:, None] * bs + np.arange(bs)) < ctx[r]).reshape(-1))
        rows = [x[:, table[r, j].astype(np.int64)].reshape(hkv, -1, D)[:, n] for x in (k, v)]
        check_attention(out[r], lse[r], *plain64.attention(q[r], *rows, SCALE), int(n.sum()))


@pytest.mark.gpu
@pytest.mark.parametrize("B", [3, 64, 100])
def test_counts_out_of_range_among_others(B):
    """Such a request has no output, whichever lane holds its count, and takes nothing from the others."""
    ctx, cnt = [1600 + 16 * (r % 9) for r in range(B)], [60 + r % 41 for r in range(B)]
    gen = torch.Generator().manual_seed(B)
    sh, q, pool, table, sel = case_state(ctx, cnt, 2, 1, 16, "bf16", gen)
    d = [x.to(DEV) for x in (q, pool, table, sel)]
    bad = cnt[:]
    bad[1], bad[B - 1] = -1, sel.shape[1] + 1
    out, lse = attend(sh, *d, dev(bad), dev(ctx), status_want=P.PULSE_ERR_BAD_INDEX)
    for r in range(B):
        if r in (1, B - 1):
            assert (out[r] == 0).all() and (lse[r] == -math.inf).all()
            continue
        j = sel[r, : cnt[r]].long()
        k, v = (x.transpose(0, 1).reshape(1, -1, D) for x in plain64.unpack(pool[table[r, j].long()], 1, 16))
        n = (j[:, None] * 16 + torch.arange(16)).view(-1) < ctx[r]
        check_attention(out[r], lse[r], *plain64.attention(q[r], k[:, n], v[:, n], SCALE), int(n.sum()))


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("kv4", [False, True])
def test_a_workspace_serves_smaller_calls(dt, kv4):
    """Batches around a round of workgroups and a plan's limits, selections around whole splits; the partials of every
    call fit beside the lists."""
    for hq, hkv, bs in ((32, 8, 16), (16, 1, 64), (28, 4, 32), (2, 2, 16), (48, 4, 64), (3, 3, 32)):
        sh = P.make_shape(hq, hkv, D, bs, TYPES[dt][2 if kv4 else 1])
        ks = [1, 2, 3, 8, 9, 17, 63, 64, 65, 127, 128, 130, 255, 256, 257, 500, 512, 513, 1000, 4100]
        before = None
        for B in [1, 2, 3, 7, 16, 17, 31, 32, 33, 43, 64, 65, 85, 86, 128, 129, 256, 257, 300, 512, 1000]:
            row, most = [], 0
            for k in ks:
                n = P.pulse_workspace_bytes(sh, B, k, 0)
                lists = 4 * (B * k + 3 * B)
                assert n >= lists + P.pulse_attention_workgroups(sh, B, k) * B * hq * (4 * D + 8)
                most = max(most, n)
                assert n == most
                row.append(n)
            assert before is None or all(a <= b for a, b in zip(before, row))
            before = row


def test_kv4_attention_workgroups():
    """One workgroup of eight waves, hence no merge launch, up to two 32-token steps of each wave (more than eight query
    heads per KV head), three, or four (more than 64 requests and heads); splits over several beyond."""
    def groups(hq, hkv, bs, B, k):
        return P.pulse_attention_workgroups(P.make_shape(hq, hkv, D, bs, P.PULSE_BF16_KV4), B, k)

    for hq, hkv, bs, B, k in ((32, 8, 16, 2, 48), (64, 8, 32, 8, 24), (64, 4, 64, 2, 8), (8, 8, 64, 2, 12),
                              (32, 8, 16, 9, 64), (64, 4, 64, 17, 16)):
        assert groups(hq, hkv, bs, B, k) == 1
        assert groups(hq, hkv, bs, B, k + 1) > 1
    assert groups(32, 8, 16, 32, 256) == 1  # 256 requests and heads take a round of workgroups between them
