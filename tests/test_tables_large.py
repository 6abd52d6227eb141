"""Maps of steps with room for more tokens than the tiles have at their smallest: one workspace for every smaller step,
and tiles that a workgroup takes in several parts."""
import random

import pytest
import torch

import plain64
from paper_2609_34555_amd import pulse as P
from parity import say
from test_tables import Step, shape, start


@pytest.mark.parametrize("bs", [16, 32, 64])
def test_a_workspace_serves_smaller_steps(bs):
    """Around the rooms at which a tile grows (1024 tiles of 8192 tokens each, twice that, ..) and the rules' limits."""
    rooms = sorted({0, 1, 4096, 4097, 16384, 16385, 100_000, 1 << 30, 2**31 - 1}
                   | {m * (1 << 23) + d for m in (1, 2, 3, 5) for d in (-200_000, -20_000, -129, -1, 0, 1, 11_392, 150_000)})
    before = None
    for B in (0, 1, 2, 32, 33, 256, 257, 1000, 4096):
        row = [P.pulse_tables_workspace_bytes(shape(bs), B, n) for n in rooms]
        assert row == sorted(row), (B, row)
        assert before is None or all(a <= b for a, b in zip(before, row)), B
        before = row


@pytest.mark.gpu
@pytest.mark.parametrize("what", ["", "exhausted", "slot", "entry"])
def test_tiles_taken_in_parts(what):
    """Room for 8.5M tokens makes tiles of 1024 blocks, which a workgroup's 512 threads take in two parts; the step has
    2065 blocks (the last tile's second part is empty). A fault lies in a second part, or shows only behind it."""
    say(f"\n[gpu] tables, tiles of two parts {what}")
    rng = random.Random(2)
    bs, room = 16, 8_500_000
    ctx, new = [20000, 7, 0, 12345, 800], [20000, 3, 0, 12300, 700]
    table, free, n_slots = start(ctx, new, bs, rng, later=0.2)
    want = plain64.tables(ctx, new, bs, table, free, 0, sum(new))
    need = want[5]
    assert 1024 < need < 2048
    code = 0
    if what == "exhausted":
        free, code = free[: need - 1], P.PULSE_ERR_POOL_EXHAUSTED
    elif what == "slot":
        free[need - 1], code = n_slots, P.PULSE_ERR_BAD_INDEX
    elif what == "entry":
        table[0][700], code = n_slots, P.PULSE_ERR_BAD_INDEX
    s = Step(ctx, new, bs, table, free, n_slots, room).run()
    assert s.status.item() == code
    assert (s.pos[room:] == 77).all() and (s.place[room:] == 77).all()
    T = 0 if code else sum(new)
    assert (s.pos[T:room] == -1).all() and (s.place[T:room] == -1).all()
    if code:
        assert not s.blk.any() and not s.tok.any() and s.table.tolist() == table and s.head.item() == 0
        return
    got = (s.blk.tolist(), s.tok.tolist(), s.place[:T].tolist(), s.pos[:T].tolist(), s.table.tolist(), s.head.item())
    assert got == tuple(want)
    s.run()  # once more on its own result: every block has its slot
    again = (s.blk.tolist(), s.tok.tolist(), s.place[:T].tolist(), s.pos[:T].tolist(), s.table.tolist(), s.head.item())
    assert s.status.item() == 0 and again == got
