"""Head norms with the position rotation, against the formulas in 64 bits."""
import pytest
import torch

import plain64
from paper_2609_34555_amd import pulse as P
from parity import say

DEV = "cuda"
D = 128
FAKE = 0x1000
DT = {"bf16": (torch.bfloat16, P.PULSE_BF16), "f16": (torch.float16, P.PULSE_F16)}


def inv_freq(rot, base=10000.0):
    return base ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=DEV) / max(rot, 1))


def bound(want, size, dt):
    """Half a step of the rounding, and before it, in units of 2^-24 of what an element is a sum of: 12 for the sum of
    128 squares (8 in a lane, 4 exchanges), halved by the root, 4 for root, division and two products, 8 for an angle
    that is a float fraction of a turn (2^-26 turns, times 2 pi) and its sine and cosine, 3 for the rotation."""
    before = size * 24 * 2.0**-24
    return (want.abs() + before) * torch.finfo(dt).eps / 2 + before + torch.finfo(dt).tiny * torch.finfo(dt).eps


# rows, hq, hkv, rot, interleaved, weights, largest position, gaps between the rows, dtype
CASES = [
    (1, 8, 2, 128, 0, True, 1, 0, "bf16"),
    (1, 32, 8, 128, 0, True, 131072, 0, "f16"),
    (3, 6, 3, 64, 1, True, 5000, 8, "bf16"),
    (5, 16, 1, 16, 0, True, 2**31 - 1, 24, "f16"),
    (7, 1, 1, 112, 0, True, 2**20, 0, "bf16"),
    (4, 40, 8, 96, 1, True, 2**20, 128, "f16"),
    (33, 64, 8, 128, 1, False, 10**6, 0, "bf16"),
    (2, 12, 1, 0, 0, True, 100, 0, "bf16"),
    (3, 4, 4, 32, 0, False, 100, 0, "f16"),
    (1000, 28, 4, 128, 0, True, 262144, 16, "bf16"),
    (2, 256, 16, 128, 0, True, 4096, 0, "f16"),
]


@pytest.mark.gpu
@pytest.mark.parametrize("T,hq,hkv,rot,inter,weights,far,gap,dt", CASES)
def test_norm_rope(T, hq, hkv, rot, inter, weights, far, gap, dt):
    say(f"\n[gpu] norm_rope T={T} hq={hq} hkv={hkv} rot={rot} inter={inter} {dt}")
    dtype, code = DT[dt]
    gen = torch.Generator(device=DEV)
    gen.manual_seed(T + rot)
    width = (hq + 2 * hkv) * D + gap
    qkv = torch.randn((T, width), generator=gen, device=DEV).mul_(3).to(dtype)
    qkv[0, :D] = 0  # a head of zeros
    pos = torch.randint(0, far, (T,), generator=gen, device=DEV, dtype=torch.int64).int()
    pos[-1] = far - 1
    skip = torch.arange(T, device=DEV) % 5 == 3
    pos[skip] = -1
    qw, kw = (torch.randn((2, D), generator=gen, device=DEV).add_(1).to(dtype) if weights else (None, None))
    f = inv_freq(rot)
    qo = torch.full((T, hq * D + gap), 7.0, dtype=dtype, device=DEV)
    ko = torch.full((T, hkv * D + 2 * gap), 7.0, dtype=dtype, device=DEV)
    keep = qkv.clone()
    P.pulse_qk_norm_rope(P.make_shape(hq, hkv, D, 16, code), qkv, width, qkv[:, hq * D:], width, T, pos, qw, kw, 1e-6,
                         f, rot, inter, qo, qo.shape[1], ko, ko.shape[1])
    assert torch.equal(qkv, keep)
    for name, x, w, out in (("q", qkv[:, : hq * D], qw, qo), ("k", qkv[:, hq * D:(hq + hkv) * D], kw, ko)):
        heads = x.shape[1] // D
        want, size = plain64.norm_rope(x.unflatten(1, (heads, D)), w, 1e-6, pos, f, rot, inter)
        got = out[:, : heads * D].unflatten(1, (heads, D)).double().cpu()
        live = (~skip).cpu()
        over = ((got - want).abs() / bound(want, size, dtype))[live].max().item()
        say(f"  {name}: {over:.3f} of the bound")
        assert over <= 1
        assert (got[~live] == 7).all() and (out[:, heads * D:] == 7).all()
    # in place
    P.pulse_qk_norm_rope(P.make_shape(hq, hkv, D, 16, code), qkv, width, qkv[:, hq * D:], width, T, pos, qw, kw, 1e-6,
                         f, rot, inter, qkv, width, qkv[:, hq * D:], width)
    live = ~skip
    assert torch.equal(qkv[live][:, : hq * D], qo[live][:, : hq * D])
    assert torch.equal(qkv[live][:, hq * D:(hq + hkv) * D], ko[live][:, : hkv * D])
    assert torch.equal(qkv[skip], keep[skip]) and torch.equal(qkv[:, (hq + hkv) * D:], keep[:, (hq + hkv) * D:])


@pytest.mark.gpu
@pytest.mark.parametrize("which", ["q", "k"])
def test_one_weight_alone(which):
    """Only the side that has a weight is normed."""
    gen = torch.Generator(device=DEV).manual_seed(2)
    q, k = (torch.randn((3, h, D), generator=gen, device=DEV).mul_(3).bfloat16() for h in (4, 2))
    w = torch.randn(D, generator=gen, device=DEV).bfloat16()
    pos = torch.tensor([0, 17, 4000], dtype=torch.int32, device=DEV)
    qo, ko = torch.zeros_like(q), torch.zeros_like(k)
    qw, kw = (w, None) if which == "q" else (None, w)
    P.pulse_qk_norm_rope(P.make_shape(4, 2, D, 16, P.PULSE_BF16), q, 4 * D, k, 2 * D, 3, pos, qw, kw, 1e-6, inv_freq(D),
                         D, 0, qo, 4 * D, ko, 2 * D)
    for x, y, wt in ((q, qo, qw), (k, ko, kw)):
        want, size = plain64.norm_rope(x, wt, 1e-6, pos, inv_freq(D), D, 0)
        assert ((y.double().cpu() - want).abs() <= bound(want, size, torch.bfloat16)).all()


@pytest.mark.gpu
def test_norm_rope_non_finite_stays_in_its_head():
    q = torch.randn((2, 4, D), device=DEV).bfloat16()
    k = torch.randn((2, 2, D), device=DEV).bfloat16()
    q[0, 1, 5], k[1, 0, 9] = float("nan"), float("inf")
    w = torch.ones(D, device=DEV).bfloat16()
    qo, ko = torch.zeros_like(q), torch.zeros_like(k)
    P.pulse_qk_norm_rope(P.make_shape(4, 2, D, 16, P.PULSE_BF16), q, 4 * D, k, 2 * D, 2,
                         torch.tensor([3, 4], dtype=torch.int32, device=DEV), w, w, 1e-6, inv_freq(128), 128, 0, qo,
                         4 * D, ko, 2 * D)
    bad_q, bad_k = qo.isnan().any(-1).cpu(), ko.isnan().any(-1).cpu()
    assert bad_q.tolist() == [[False, True, False, False], [False] * 4]
    assert bad_k.tolist() == [[False, False], [True, False]]


def test_norm_rope_refusals():
    sh = P.make_shape(8, 2, D, 16, P.PULSE_BF16)
    a = dict(q=FAKE, q_stride=1024, k=FAKE, k_stride=256, n_rows=3, positions=FAKE, q_weight=FAKE, k_weight=FAKE,
             eps=1e-6, inv_freq=FAKE, rot_dim=128, interleaved=0, q_out=FAKE, q_out_stride=1024, k_out=FAKE,
             k_out_stride=256, stream=0, check=False)
    call = lambda s=sh, **kw: P.pulse_qk_norm_rope(s, **{**a, **kw})  # noqa: E731
    for name in ("q", "k", "positions", "inv_freq", "q_out", "k_out"):
        assert call(**{name: None}) == P.PULSE_ERR_INVALID_ARG, name
    for name in ("q", "k", "q_out", "k_out", "q_weight", "k_weight"):
        assert call(**{name: FAKE + 8}) == P.PULSE_ERR_INVALID_ARG, name
    for kw in (dict(q_stride=1016), dict(k_stride=248), dict(q_stride=1028), dict(q_out_stride=0),
               dict(k_out_stride=-256), dict(n_rows=-1), dict(rot_dim=-16), dict(rot_dim=144), dict(interleaved=2),
               dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf"))):
        assert call(**kw) == P.PULSE_ERR_INVALID_ARG, kw
    for rot in (8, 24, 100, 127):
        assert call(rot_dim=rot) == P.PULSE_ERR_UNSUPPORTED
    assert call(P.make_shape(8, 2, 64, 16, P.PULSE_BF16)) == P.PULSE_ERR_UNSUPPORTED
    assert call(P.make_shape(8, 2, D, 16, 9)) == P.PULSE_ERR_UNSUPPORTED
    assert call(n_rows=0, q=None, positions=None) == P.PULSE_OK
