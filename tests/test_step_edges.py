"""The step around the attention where no other test goes: more rows than one pass of the rotation's grid, selections of
every kind for a 4-bit cache, and steps of two batches on two streams at once."""
import numpy as np
import pytest
import torch

import plain64
from paper_2609_34555_amd import pulse as P
from parity import say
from test_kv4_step import Run
from test_norm_rope import bound, inv_freq

pytestmark = pytest.mark.gpu
DEV, D = "cuda", 128


@pytest.mark.parametrize("inter,rot", [(0, 128), (1, 48)])
def test_more_rows_than_one_pass_of_the_rotation(inter, rot):
    """2^20 workgroups of a row each and 777 rows more, every seventh row without a position."""
    T = (1 << 20) + 777
    say(f"\n[gpu] norm_rope rows={T} inter={inter} rot={rot}")
    sh = P.make_shape(1, 1, D, 16, P.PULSE_BF16)
    gen = torch.Generator(device=DEV).manual_seed(rot)
    x = torch.randn((T, 2 * D), generator=gen, device=DEV).bfloat16()
    qw, kw = torch.randn((2, D), generator=gen, device=DEV).add_(1).bfloat16()
    pos = torch.randint(0, 1 << 20, (T,), generator=gen, device=DEV).int()
    skip = torch.arange(T, device=DEV) % 7 == 4
    pos[skip] = -1
    out = torch.full((2, T, 2 * D), 7.0, dtype=torch.bfloat16, device=DEV)
    f = inv_freq(rot)

    def call(o, a, b):
        P.pulse_qk_norm_rope(sh, x[a:], 2 * D, x[a:, D:], 2 * D, b - a, pos[a:], qw, kw, 1e-6, f, rot, inter, o[a:], 2 * D,
                             o[a:, D:], 2 * D)

    call(out[0], 0, T)
    half = 600_000  # the same in calls that one pass holds
    call(out[1], 0, half)
    call(out[1], half, T)
    assert torch.equal(out[0], out[1])
    assert (out[0][skip] == 7).all()
    for a in (0, (1 << 20) - 100, T - 200):
        rows = slice(a, a + 200)
        live = (~skip[rows]).cpu()
        for c, w in ((0, qw), (D, kw)):
            part = x[rows, c:c + D].unflatten(1, (1, D))
            want, size = plain64.norm_rope(part, w, 1e-6, pos[rows], f, rot, inter)
            err = (out[0][rows, c:c + D].double().cpu().unflatten(1, (1, D)) - want).abs()
            assert (err <= bound(want, size, torch.bfloat16))[live].all()


@pytest.mark.parametrize("n16,n4", [(P.PULSE_F16, P.PULSE_F16_KV4), (P.PULSE_BF16, P.PULSE_BF16_KV4)])
@pytest.mark.parametrize("lens", [[20, 1, 33], [700, 650, 3]])
def test_selections_read_queries_and_digests_alone(lens, n16, n4):
    dtype = torch.float16 if n16 == P.PULSE_F16 else torch.bfloat16
    B, total, hq, hkv, k_max = len(lens), sum(lens), 12, 3, 40
    gen = torch.Generator(device=DEV).manual_seed(total)
    off = torch.tensor(np.concatenate([[0], np.cumsum(lens)]), device=DEV)
    q = torch.randn((B, hq, D), generator=gen, device=DEV).to(dtype)
    dig = torch.randn((hkv, total, 2, D), generator=gen, device=DEV).sort(2).values.to(dtype)
    k_mid = torch.tensor([30, 2, 25], dtype=torch.int32, device=DEV)
    got = []
    for code in (n16, n4):
        sh = P.make_shape(hq, hkv, D, 16, code)
        nb = max(P.pulse_workspace_bytes(sh, B, k_max, total), P.pulse_average_workspace_bytes(sh, B, k_max, total),
                 P.pulse_headwise_workspace_bytes(sh, B, k_max, total))
        ws = torch.full((nb,), 255, dtype=torch.uint8, device=DEV)
        i32 = lambda *s: torch.full(s, -1, dtype=torch.int32, device=DEV)  # noqa: E731
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        one, avg = [(i32(B, k_max), i32(B), torch.zeros(total, device=DEV)) for _ in range(2)]
        head = (i32(hkv, B, k_max), i32(hkv, B), i32(hkv, B), i32(hkv, B))
        P.pulse_select_solohead(sh, q, dig[1], off, B, total, 1, k_mid, 1, 2, k_max, *one, status, ws, nb)
        P.pulse_select_average(sh, q, dig, off, B, total, k_mid, 1, 2, k_max, *avg, status, ws, nb)
        P.pulse_select_headwise(sh, q, dig, off, B, total, k_mid, 1, 2, k_max, i32(B, max(lens)), max(lens), 5, *head,
                                status, ws, nb)
        assert status.item() == 0
        got.append([*one, *avg, *head])
    assert all(torch.equal(a, b) for a, b in zip(*got))
    assert (got[0][1] > 0).all() and (got[0][7] > 0).all()


def test_two_batches_on_two_streams():
    """A step of two batches each with buffers of its own, enqueued side by side; the results are those of one after the
    other."""
    say("\n[gpu] two batches on two streams")

    def make():
        return [Run([900, 3000, 17], 40, 8, 2, 16, P.PULSE_BF16_KV4, torch.bfloat16, 1),
                Run([2100] * 9, 40, 16, 1, 32, P.PULSE_F16_KV4, torch.float16, 2)]

    def prompt(st):
        x = st.rows(int(st.new.sum().item()) + 1)
        st.buffers(x.shape[0])
        st.write(x)
        st.new.fill_(1)
        st.x = [st.rows(st.B + 2) for _ in range(12)]
        st.buffers(st.B + 2)

    def step(st, i):
        st.ctx.add_(1)
        st.write(st.x[i])
        st.attend()

    want, got = make(), make()
    for st in want + got:
        prompt(st)
    torch.cuda.synchronize()
    for st in want:
        for i in range(12):
            step(st, i)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for i in range(12):
        for st, s in zip(got, streams):
            with torch.cuda.stream(s):
                step(st, i)
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert a.status.item() == 0 == b.status.item()
        for x, y in zip(a.snapshot(), b.snapshot()):
            assert torch.equal(x, y)
