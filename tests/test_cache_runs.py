"""Rows into the cache and back on either side of the rule that gives a wave eight rows instead of one (more than 8192
rows times heads): runs that begin and end anywhere, go over from one wave's rows to the next's, or are cut by rows
without a place; the whole pool is compared."""
import numpy as np
import pytest
import torch

import plain64
from paper_2609_34555_amd import pulse as P
from parity import say
from test_kv4 import DEV, TYPES, D, dev, equal

pytestmark = pytest.mark.gpu


def places(kind, T, bs, rng):
    """Places of T rows (-1: none) and the slots of the pool."""
    n_slots = -(-(T + 600) // bs) + 3
    if kind == "shifted":  # one run from the middle of an octet on: every wave's rows lie in two octets
        m = 3 + np.arange(T)
    elif kind == "unordered":
        m = rng.permutation(n_slots * bs)[:T]
    elif kind == "backwards":
        m = 3 + np.arange(T)[::-1]
    else:  # runs of 1 to 29 rows in no order, ends of the pool among them
        m, at = [], 0
        while at < n_slots * bs:
            n = min(int(rng.integers(1, 30)), n_slots * bs - at)
            m.append(np.arange(at, at + n))
            at += n
        rng.shuffle(m)
        m = np.concatenate(m)[:T]
    m = m.astype(np.int64)
    if kind != "backwards":
        for i in (1, 12, 13, 23, 24, 40, T // 2, T - 2):  # inside a wave's rows, its first and its last
            m[i] = -1
    return m, n_slots


SIZES = [(1024, 8), (1025, 8), (1031, 8), (8192, 1), (8193, 1), (2733, 3)]  # rows, heads


@pytest.mark.parametrize("dt,four", [("bf16", True), ("f16", True), ("bf16", False)])
@pytest.mark.parametrize("kind", ["shifted", "runs", "unordered", "backwards"])
@pytest.mark.parametrize("T,hkv", SIZES)
def test_rows_and_whole_pool(T, hkv, kind, dt, four):
    bs = {8: 16, 1: 64, 3: 32}[hkv]
    say(f"\n[gpu] cache runs rows={T} hkv={hkv} bs={bs} {kind} {dt} four={four}")
    dtype, code16, code4 = TYPES[dt]
    gen = torch.Generator(device=DEV).manual_seed(T + hkv)
    m, n_slots = places(kind, T, bs, np.random.default_rng(T))
    bad = kind == "runs"
    if bad:  # reported, skipped, and its neighbours are runs of their own
        m[100], m[777], m[T - 1] = n_slots * bs, -2, 2**40
    on = np.flatnonzero((m >= 0) & (m < n_slots * bs))
    assert len(np.unique(m[on])) == len(on)
    slot, tok = m[on] // bs, m[on] % bs
    sh = P.make_shape(2 * hkv, hkv, D, bs, code4 if four else code16)
    U = P.pulse_block_bytes(sh)
    wide = torch.randn((T, 2, hkv * D + 24), generator=gen, device=DEV)  # rows inside wider ones
    wide = (wide * torch.exp2(torch.randint(-6, 6, (T, 1, 1), generator=gen, device=DEV).float())).to(dtype)
    k, v = wide[:, 0, 8:8 + hkv * D], wide[:, 1, 16:16 + hkv * D]
    before = torch.randint(0, 255, (n_slots, U), generator=gen, device=DEV, dtype=torch.uint8)
    pool, status = before.clone(), torch.zeros(1, dtype=torch.int32, device=DEV)
    P.pulse_append_kv(sh, k, wide.stride(0), v, wide.stride(0), dev(m, torch.int64), T, pool, n_slots, status)
    assert status.item() == (P.PULSE_ERR_BAD_INDEX if bad else 0)
    kr, vr = (x.unflatten(1, (hkv, D)).cpu()[torch.from_numpy(on)] for x in (k, v))
    if four:
        kd, vd = torch.zeros((2, n_slots, hkv, bs, D), dtype=dtype)
        kd[slot, :, tok], vd[slot, :, tok] = kr, vr
        want = plain64.pack(kd, vd, bs).numpy().reshape(n_slots, hkv, -1)
        mask = np.zeros((n_slots, 136 * bs), np.uint8)  # the bits that the rows own
        mask[:, : 64 * bs].reshape(n_slots, bs, 64)[slot, tok] = 255
        words = mask[:, 64 * bs:128 * bs].reshape(n_slots, bs // 8, D, 4)
        for b, t in zip(slot, tok):
            words[b, t // 8, :, t % 8 // 2] |= np.uint8(240 if t % 2 else 15)
        mask[:, 128 * bs:132 * bs].reshape(n_slots, bs, 4)[slot, tok] = 255
        mask[:, 132 * bs:].reshape(n_slots, 4, bs)[slot, :, tok] = 255
        mask = mask[:, None]
        want = (want & mask) | (before.cpu().numpy().reshape(want.shape) & ~mask)
        got = pool.cpu().numpy().reshape(want.shape)
        assert (got == want).all(), np.argwhere(got != want)[:5]
    else:
        want = before.cpu().view(torch.int16).clone().view(n_slots, 2, hkv, bs * D)
        want[:, 0].view(n_slots, hkv, bs, D)[slot, :, tok] = kr.contiguous().view(torch.int16)
        want[:, 1].view(n_slots, hkv, D, bs)[slot, :, :, tok] = vr.contiguous().view(torch.int16)
        assert torch.equal(pool.cpu().view(torch.int16).view_as(want), want)
    # and back, into wider rows; rows without a place stay as they were
    out = torch.full_like(wide, 5.0)
    status.zero_()
    P.pulse_load_kv(sh, pool, n_slots, dev(m, torch.int64), T, out[:, 0, 16:], wide.stride(0), out[:, 1, 8:],
                    wide.stride(0), status)
    assert status.item() == (P.PULSE_ERR_BAD_INDEX if bad else 0)
    want = torch.full((T, 2, hkv * D + 24), 5.0, dtype=torch.float64)
    for i, (x, at) in enumerate(((kr, 16), (vr, 8))):
        x = plain64.quantise(x)[2] if four else x.double()
        want[torch.from_numpy(on), i, at:at + hkv * D] = x.flatten(1)
    assert equal(out, want)


@pytest.mark.parametrize("four", [True, False])
def test_more_rows_than_one_pass_of_the_grid(four):
    """65535 workgroups of 32 rows each, and 1000 rows more, from the middle of an octet on."""
    say(f"\n[gpu] cache, more rows than the grid four={four}")
    T, bs = 65535 * 32 + 1000, 64
    sh = P.make_shape(1, 1, D, bs, P.PULSE_BF16_KV4 if four else P.PULSE_BF16)
    n_slots = (T + 5) // bs + 2
    k, v = torch.randn((2, T, D), device=DEV, dtype=torch.bfloat16)
    pool = torch.zeros((n_slots, P.pulse_block_bytes(sh)), dtype=torch.uint8, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    m = torch.arange(T, device=DEV) + 5
    P.pulse_append_kv(sh, k, D, v, D, m, T, pool, n_slots, status)
    out = torch.zeros((2, T, D), dtype=torch.bfloat16, device=DEV)
    P.pulse_load_kv(sh, pool, n_slots, m, T, out[0], D, out[1], D, status)
    assert status.item() == 0
    if not four:
        assert torch.equal(out[0], k) and torch.equal(out[1], v)
        return
    for x, y in ((k, out[0]), (v, out[1])):
        for at in (0, 65535 * 32 - 500, T - 1000):
            assert equal(y[at:at + 1000], plain64.quantise(x[at:at + 1000])[2])
        assert ((x.float() - y.float()).view(T, 4, 32).abs().amax(-1) <= x.float().view(T, 4, 32).abs().amax(-1) / 3.5).all()
