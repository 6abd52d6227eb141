"""pulse_decode_layer_noalloc at sizes where a workspace that also serves smaller calls would not fit the library's
array: the call needs room for its own partials alone."""
import numpy as np
import pytest
import torch

from paper_2609_34555_amd import pulse as P
from parity import say

D = 128
FAKE = 0x1000
POINTERS = ("ctx_len", "blk_off", "q", "digests", "k_mid", "sel_idx", "sel_cnt", "host_kv", "block_table", "free_slots",
            "free_head", "slot_pool", "stats", "out", "dev_status")


def align(x):
    return (x + 255) & ~255


def own_bytes(sh, B, k_max, total_blocks):
    """The lists of a call and one partial per workgroup of its attention."""
    G = sh.num_q_heads // sh.num_kv_heads
    units = B * sh.num_kv_heads * P.pulse_attention_workgroups(sh, B, k_max)
    return (align(4 * total_blocks) + align(4 * B * k_max) + 3 * align(4 * B) + align(64) + align(4 * units * G * D)
            + align(8 * units * G))


# query heads, KV heads, bs, requests, k_max
SIZES = [(64, 8, 64, 429, 591), (128, 16, 32, 92, 2016), (256, 16, 32, 149, 204), (32, 8, 16, 1900, 64),
         (128, 8, 16, 400, 64), (64, 4, 16, 900, 128)]


@pytest.mark.parametrize("dtype", [P.PULSE_F16, P.PULSE_BF16, P.PULSE_F16_KV4, P.PULSE_BF16_KV4])
@pytest.mark.parametrize("hq,hkv,bs,B,k_max", SIZES)
def test_a_call_that_fits_the_array_is_taken(hq, hkv, bs, B, k_max, dtype):
    """Both sides of the limit, by the number of blocks. (Without `out` a call that fits ends at the check of its
    arguments, before any device work.)"""
    la = P.pulse_layer_args()
    la.shape = P.make_shape(hq, hkv, D, bs, dtype)
    for f in POINTERS:
        setattr(la, f, FAKE)
    la.B, la.k_max, la.max_blocks, la.n_free, la.n_slots, la.n_sink_blocks, la.n_local_blocks = B, k_max, k_max, 10, 50, 1, 8
    la.out = None
    base = own_bytes(la.shape, B, k_max, 0)
    assert base <= P.pulse_workspace_bytes(la.shape, B, k_max, 0)
    most = (P.NOALLOC_SCRATCH_BYTES - base) // 256 * 64  # blocks, a score of 4 bytes each
    if dtype in (P.PULSE_F16, P.PULSE_BF16):
        assert base < P.NOALLOC_SCRATCH_BYTES < P.pulse_workspace_bytes(la.shape, B, k_max, most)
    for total, want in ((B, P.PULSE_ERR_INVALID_ARG), (most, P.PULSE_ERR_INVALID_ARG), (most + 1, P.PULSE_ERR_WORKSPACE)):
        if total < 0 or (total == B and B > most):
            continue
        la.total_blocks = total
        assert P.pulse_decode_layer_noalloc(la, stream=0, check=False) == want, total


@pytest.mark.gpu
@pytest.mark.parametrize("hq,hkv,bs,B,k_max", [(128, 8, 16, 400, 64), (32, 8, 16, 1900, 64)])
def test_a_large_batch_equals_the_call_with_a_workspace(hq, hkv, bs, B, k_max):
    """1 to 12 blocks a request, far fewer than k_max; resident, so that nothing is recalled."""
    say(f"\n[gpu] noalloc batch B={B} hq={hq} hkv={hkv} bs={bs} k_max={k_max}")
    dev = "cuda"
    rng = np.random.default_rng(B)
    ctx = rng.integers(1, 12 * bs, size=B)
    n = -(-ctx // bs)
    total, mb = int(n.sum()), int(n.max())
    sh = P.make_shape(hq, hkv, D, bs, P.PULSE_BF16)
    gen = torch.Generator(device=dev).manual_seed(B)
    n_slots = 200  # requests share slots
    pool = torch.randn((n_slots, P.pulse_block_bytes(sh) // 2), generator=gen, device=dev).bfloat16()
    table = torch.randint(0, n_slots, (B, mb), generator=gen, device=dev, dtype=torch.int32)
    t = lambda x, d=torch.int32: torch.tensor(np.asarray(x), dtype=d, device=dev)  # noqa: E731
    in_ = dict(ctx_len=t(ctx), blk_off=t(np.concatenate([[0], np.cumsum(n)]), torch.int64),
               q=torch.randn((B, hq, D), generator=gen, device=dev).bfloat16(), digests=torch.zeros(
                   (total, 2, D), dtype=torch.bfloat16, device=dev), k_mid=t(rng.integers(0, 5, size=B)),
               free_slots=t([0]))
    got = []
    for own in (True, False):
        out = dict(sel_idx=torch.full((B, k_max), -1, dtype=torch.int32, device=dev), sel_cnt=t([0] * B),
                   block_table=table.clone(), free_head=t([0]), slot_pool=pool,
                   stats=torch.zeros(2, dtype=torch.int64, device=dev), out=torch.full((B, hq, D), np.nan, device=dev),
                   lse=torch.full((B, hq), np.nan, device=dev), dev_status=t([0]))
        a = P.pulse_layer_args()
        a.shape, a.B, a.total_blocks, a.n_sink_blocks, a.n_local_blocks, a.k_max, a.max_blocks = sh, B, total, 1, 2, k_max, mb
        a.n_free, a.n_slots, a.sm_scale, a.host_kv = 1, n_slots, 0.1, pool.data_ptr()  # (nothing is missing)
        for f, x in {**in_, **out}.items():
            setattr(a, f, x.data_ptr())
        if own:
            nb = P.pulse_workspace_bytes(sh, B, k_max, total)
            assert nb > P.NOALLOC_SCRATCH_BYTES
            ws = torch.full((nb,), 255, dtype=torch.uint8, device=dev)
            a.ws, a.ws_bytes = ws.data_ptr(), nb
            P.pulse_decode_layer(a)
        else:
            P.pulse_decode_layer_noalloc(a)
        torch.cuda.synchronize()
        assert out["dev_status"].item() == 0 and out["stats"].sum().item() == 0
        got.append(out)
    for f in ("sel_idx", "sel_cnt", "out", "lse", "block_table", "free_head"):
        assert torch.equal(got[0][f], got[1][f]), f
    assert got[0]["out"].isfinite().all().item() and got[0]["lse"].isfinite().all().item()
