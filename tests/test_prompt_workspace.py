"""Attention of new tokens writes within the workspace that its size function gives, and no further."""
import numpy as np
import pytest
import torch

from paper_2609_34555_amd import pulse as P
from test_prompt import CODES, DEV, SCALE, D, dev

# query heads, KV heads, bs
SIZES = [(32, 8, 16), (16, 1, 64), (28, 4, 32), (2, 2, 16), (48, 4, 64)]


@pytest.mark.gpu
@pytest.mark.parametrize("hq,hkv,bs", SIZES)
@pytest.mark.parametrize("bits", [16, 8, 4])
def test_what_lies_behind_the_workspace_stays(hq, hkv, bs, bits):
    """Every call writes within the size that pulse_prompt_workspace_bytes gives for it, whatever its splits."""
    sh = P.make_shape(hq, hkv, D, bs, CODES["bf16", bits])
    pool = torch.zeros((4, P.pulse_block_bytes(sh)), dtype=torch.uint8, device=DEV)
    guard = torch.arange(1 << 20, device=DEV).to(torch.uint8)
    status = dev([0])
    for mb in (1, 17, 300, 4096):
        table = torch.randint(0, 4, (64, mb), dtype=torch.int32, device=DEV)
        for B in (1, 2, 7, 64):
            for T in (1, 3, 17, 64, 200, 300, 1000, 1500):
                if mb * bs * max(T, 64) * hq > 1 << 32 or T < B or T // B > mb * bs:
                    continue
                nb = P.pulse_prompt_workspace_bytes(sh, B, T, mb)
                buf = torch.full((nb + guard.numel(),), 255, dtype=torch.uint8, device=DEV)
                buf[nb:] = guard
                q = torch.zeros((T, hq * D), dtype=torch.bfloat16, device=DEV)
                out, lse = torch.empty_like(q), torch.zeros((T, hq), device=DEV)
                off = np.arange(B + 1) * (T // B)
                P.pulse_prompt_attn(sh, q, hq * D, dev(off), T, dev([mb * bs] * B), B, pool, 4, table, mb, SCALE, out, hq * D,
                                    lse, status, buf, nb)
                assert torch.equal(buf[nb:], guard), (mb, B, T)
    assert status.item() == 0
