"""nat_kv_reserve around the sizes at which its launches change: lengths and counts in place of the inputs or not, up to and above 1024 sequences and 4096 rows; arrays of
millions of rows."""
import numpy as np
import pytest
import torch

from nat_testlib import DEV
from oracle import pages as opage

pytestmark = pytest.mark.gpu


def dev(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def state(seed, lens, page, width, spare):
    rng = np.random.default_rng(seed)
    need = [opage.pages_of(n, page) for n in lens]
    order = [int(p) for p in rng.permutation(sum(need) + spare)]
    table, at = [[-1] * width for _ in lens], 0
    for i, c in enumerate(need):
        table[i][:c] = order[at:at + c]
        at += c
    return table, order[at:] + [-9] * at, [spare, 0]


def reserve(table, lens, new, free, counts, page, cap, counts_in_place, lens_in_place):
    """nat_kv_reserve and the oracle on copies of the same state; everything that the call may write is compared."""
    import paper_2603_06619_amd as nat
    n = len(lens)
    t, f, c, l = dev(table), dev(free), dev(counts), dev(lens)
    c_out, l_out = c if counts_in_place else dev([77, 77]), l if lens_in_place else dev([77] * n)
    start, cu = dev([77] * n), dev([77] * (n + 1))
    slots, pos = torch.full((cap + 3,), 77, dtype=torch.int64, device=DEV), torch.full((cap + 3,), 77, dtype=torch.int32, device=DEV)
    ws = torch.empty(nat.kv_reserve_workspace_bytes(n), dtype=torch.uint8, device=DEV)
    nat.nat_kv_reserve(t, l, dev(new), f, c, page, cap, c_out, l_out, start, cu, slots[:cap], pos[:cap], ws)
    mine = [list(row) for row in table]
    want = opage.reserve(mine, lens, new, list(free), counts, page, cap)
    same = lambda got, ref: np.array_equal(got.cpu().numpy(), np.asarray(ref))
    assert same(c_out, want["counts"]) and same(l_out, want["seq_lens"]) and same(start, want["start"]) and same(cu, want["cu_new"])
    assert same(t, mine) and same(f, free)
    assert same(slots, want["slots"] + [77] * 3) and same(pos, want["position_ids"] + [77] * 3)
    if not counts_in_place:
        assert same(c, counts)
    if not lens_in_place:
        assert same(l, lens)
    return want


IN_PLACE = [(True, True), (True, False), (False, True), (False, False)]


@pytest.mark.parametrize("in_place", IN_PLACE)
@pytest.mark.parametrize("cap", [1023, 1024, 1025, 4095, 4096, 4097, 9000])
def test_rows_of_some_hundred_sequences(cap, in_place):
    rng = np.random.default_rng(cap)
    n, page = 300, 16
    lens = [int(x) for x in rng.integers(0, 200, n)]
    new = [int(x) for x in rng.multinomial(cap, np.ones(n) / n)]                  # as many rows as there is room for
    table, free, counts = state(1, lens, page, 20, 10 + cap // 20)                # not enough pages for the last ones
    want = reserve(table, lens, new, free, counts, page, cap, *in_place)
    assert want["counts"][1] > 0 and max(want["slots"][:cap]) > 0
    table, free, counts = state(2, lens, page, 20, 3000)
    reserve(table, lens, [2 * x for x in new], free, counts, page, cap, *in_place)               # more rows than fit


@pytest.mark.parametrize("in_place", IN_PLACE)
@pytest.mark.parametrize("n", [1023, 1024, 1025, 2500])
@pytest.mark.parametrize("most", [1, 9])
def test_many_sequences(n, most, in_place):
    rng = np.random.default_rng(n)
    page = 32
    lens = [int(x) for x in rng.integers(0, 300, n)]
    new = [int(x) for x in rng.integers(0, most + 1, n)]
    table, free, counts = state(3, lens, page, 10, max(1, n // 40))
    reserve(table, lens, new, free, counts, page, sum(new), *in_place)


@pytest.mark.parametrize("in_place", [(True, True), (False, False)])
@pytest.mark.parametrize("n", [5, 700])
def test_millions_of_rows(n, in_place):
    rng = np.random.default_rng(n)
    page, rows = 256, 1_500_000
    lens = [int(x) for x in rng.integers(0, 3000, n)]
    new = [int(x) for x in rng.multinomial(rows - 1000, np.ones(n) / n)]
    width = max(opage.pages_of(a + b, page) for a, b in zip(lens, new))
    table, free, counts = state(4, lens, page, width, sum(new) // page + 2 * n)
    reserve(table, lens, new, free, counts, page, rows, *in_place)


def test_a_step_among_rows_for_many():
    """Room for two million rows, of which three are used."""
    table, free, counts = state(5, [31, 32, 5], 16, 4, 2)
    for in_place in IN_PLACE:
        reserve(table, [31, 32, 5], [1, 1, 1], free, counts, 16, 2_000_000, *in_place)
