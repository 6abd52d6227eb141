"""Holder counts and free lists that do not agree with the table: frees and forks refuse them before they write."""
import copy

import numpy as np
import pytest

from paper_2609_34555_amd import pulse as P
from parity import say
from test_pages import KEEP_ALL, Both, Pages, Wrong, life, small


class Strict(Pages):
    """Pages whose frees look at the entries that stay too."""

    def do_free(self, keep, with_shared=True):
        inside = (self.table >= 0) & (self.table < self.n_slots)
        gone = (np.arange(self.mb) * self.bs)[None] >= np.asarray(keep, np.int64)[:, None]
        freed, kept = (np.bincount(self.table[inside & m], minlength=self.n_slots) for m in (gone, ~gone))
        if ((freed > (self.shared if with_shared else 0)) & (kept > 0)).any():
            raise Wrong
        super().do_free(keep, with_shared)

    def do_fork(self, src, dst, ln):
        """The slots that are taken: none twice, none that an entry names, none with a count."""
        need = sum(x % self.bs != 0 for x in ln)
        if 0 <= self.head <= len(self.free) - need:
            new = self.free[self.head:self.head + need]
            inside = new[(new >= 0) & (new < self.n_slots)]
            if len(set(new.tolist())) < need or np.isin(inside, self.table).any() or self.shared[inside].any():
                raise Wrong
        super().do_fork(src, dst, ln)


def state(mb, **kw):
    p = small(mb=mb, **kw)
    p.__class__ = Strict
    return Both(p)


WIDTHS = [12, 600, 20000]  # one workgroup, with two and four entries a lane; a launch a pass


@pytest.mark.gpu
@pytest.mark.parametrize("mb", WIDTHS)
def test_a_slot_that_a_kept_entry_names_is_not_given_back(mb):
    """Named twice and counted once, one of the two kept: the slot would be in the list and in the table."""
    say(f"\n[gpu] frees with kept holders, {mb} blocks a request")
    every = [KEEP_ALL] * 6
    for shared in (True, False):
        b = state(mb)
        b.p.table[4, 5] = b.p.table[0, 1]
        b.push()
        assert b.call("free", [0] + every[1:], shared=shared) == P.PULSE_ERR_BAD_INDEX
        assert b.call("free", every[:4] + [0, KEEP_ALL], shared=shared) == P.PULSE_ERR_BAD_INDEX
        assert b.call("free", [32] + every[1:], shared=shared) == 0  # (neither of the two is freed)
    b = state(mb)  # twice in one row
    b.p.table[0, 6] = b.p.table[0, 1]
    b.push()
    assert b.call("free", [96] + every[1:]) == P.PULSE_ERR_BAD_INDEX
    for rows, ok in (([0], True), ([4], True), ([0, 4], False), ([4, 5], False), ([0, 4, 5], False)):
        b = state(mb)  # three names, two of them counted
        b.p.table[4, 5] = b.p.table[5, 7] = b.p.table[0, 1]
        b.p.shared[b.p.table[0, 1]] = 1
        b.push()
        assert (b.call("free", [0 if r in rows else KEEP_ALL for r in range(6)]) == 0) == ok
        if ok:  # (nothing went back; it would with the next)
            assert b.call("free", every[:5] + [0]) == P.PULSE_ERR_BAD_INDEX
    b = state(mb)  # counted as they are: the last holder gives the slot back
    b.p.table[4, 5] = b.p.table[5, 7] = b.p.table[0, 1]
    b.p.shared[b.p.table[0, 1]] = 2
    b.push()
    for r, back in ((4, 0), (0, 6), (5, 1)):  # (request 0 has six more blocks, which nobody shares)
        head = b.p.head
        assert b.call("free", [0 if x == r else KEEP_ALL for x in range(6)]) == 0
        assert head - b.p.head == back


@pytest.mark.gpu
@pytest.mark.parametrize("mb", WIDTHS)
def test_counts_may_hold_entries_of_other_tables(mb):
    """A count above what the table shows (a call on the first requests of a larger table) keeps the slot."""
    b = state(mb)
    b.p.shared[b.p.table[0, :7]] = 1
    b.push()
    head = b.p.head
    assert b.call("free", [0] + [KEEP_ALL] * 5) == 0 and b.p.head == head


@pytest.mark.gpu
@pytest.mark.parametrize("B,mb,n_slots", [(6, 20, 150), (30, 100, 900), (60, 500, 4000)])
def test_lives_with_a_wrong_entry_now_and_then(B, mb, n_slots):
    """Requests that come, fork and go; between, an entry is written over a free place of the table, and a free of its
    slot is refused, with or without the others that hold it."""
    say(f"\n[gpu] pages with wrong entries B={B} mb={mb}")
    rng = np.random.default_rng(B)
    both = Both(Strict(B, mb, n_slots, 16, B))
    refused = 0
    for _ in range(10):
        life(both, 2, rng)
        p, start = both.p, copy.deepcopy(both.p)
        named, r = p.table[p.table >= 0], int(rng.integers(0, B))
        for part in (0.1, 0.9):
            if not len(named) or p.table[r, mb - 1] != -1:
                continue
            both.p.table[r, mb - 1] = rng.choice(named)
            both.push()
            keep = np.where(rng.random(B) < part, 0, KEEP_ALL)
            if part < 0.5:
                keep[r] = (mb - 1) * 16  # the wrong entry goes, the slot's others may stay
            refused += both.call("free", keep) != 0
            both.p = p = copy.deepcopy(start)
            both.push()
    assert refused > 0


@pytest.mark.gpu
@pytest.mark.parametrize("mb", WIDTHS)
def test_slots_that_a_fork_takes(mb):
    """A slot twice in the list would be two forks' block; one that an entry names would be written over."""
    say(f"\n[gpu] forks over wrong lists, {mb} blocks a request")
    ok = ([0, 1, 0], [3, 4, 5], [100, 63, 7])
    assert state(mb).call("fork", *ok) == 0
    for i, j in ((0, 1), (0, 2), (1, 2)):
        b = state(mb)
        b.p.free[b.p.head + i] = b.p.free[b.p.head + j]
        b.push()
        assert b.call("fork", *ok) == P.PULSE_ERR_BAD_INDEX
        assert b.call("fork", [0, 1, 0], [3, 4, 5], [96, 64, 16]) == 0  # whole blocks alone: no slot is taken
    for i in range(3):
        for r, j in ((0, 0), (0, 6), (2, 1)):
            b = state(mb)
            b.p.free[b.p.head + i] = b.p.table[r, j]
            b.push()
            assert b.call("fork", *ok) == P.PULSE_ERR_BAD_INDEX
        for count in (1, -1):
            b = state(mb)
            b.p.shared[b.p.free[b.p.head + i]] = count
            b.push()
            assert b.call("fork", *ok) == P.PULSE_ERR_BAD_INDEX
    b = state(mb)  # a request that is no part of the call, at the end of its row
    b.p.table[2, mb - 1] = b.p.free[b.p.head + 2]
    b.push()
    assert b.call("fork", *ok) == P.PULSE_ERR_BAD_INDEX
    b = state(mb)  # what lies behind the taken slots is not looked at
    b.p.free[b.p.head + 3:b.p.head + 6] = [b.p.free[b.p.head], b.p.table[0, 0], -7]
    b.push()
    assert b.call("fork", *ok) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("n", [255, 256, 257, 2048, 4095])
def test_many_forks_over_wrong_lists(n):
    """As many forks as a table has rows, of one request, each with a slot of its own; one of them wrong, anywhere."""
    say(f"\n[gpu] {n} forks")

    def fresh():
        p = Strict(n + 1, 2, n + 40, 16, n)
        p.take(0, 20)
        return Both(p)

    call = ([0] * n, list(range(1, n + 1)), [5 + i % 11 + 16 * (i % 5 == 0) for i in range(n)])
    b = fresh()
    assert b.call("fork", *call) == 0
    need = b.p.head - 2
    assert need > n - 100
    assert b.call("free", [KEEP_ALL] + [0] * n) == 0 and b.p.head == 2
    rng = np.random.default_rng(n)
    for _ in range(4):
        i, j = rng.choice(need, 2, replace=False) + 2
        b = fresh()
        b.p.free[i] = b.p.free[j]
        b.push()
        assert b.call("fork", *call) == P.PULSE_ERR_BAD_INDEX
        b = fresh()
        b.p.free[i] = b.p.table[0, 1]
        b.push()
        assert b.call("fork", *call) == P.PULSE_ERR_BAD_INDEX
