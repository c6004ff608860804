"""Block tables whose entries and counts do not agree: flagged where a call meets them, and no two rows end up on one block because of
it."""
import pytest
import torch

import paper_2601_03700_gb300 as adept

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    adept.load_library()


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def pages(n_blocks, table, ref):
    p = adept.KVPages(n_blocks, len(table), len(table[0]))
    p.block_table.copy_(i32(table))
    p.ref.copy_(i32(ref))
    return p


def flagged(p):
    with pytest.raises(adept.AdeptError) as ei:
        p.check()
    assert ei.value.status == 6
    p.check()


def compact(p):
    n = p.ref.numel() // 2
    used, src, dst = i32([-9]), *(torch.full((n,), -9, dtype=torch.int32, device="cuda") for _ in range(2))
    adept.adept_kv_compact(p, used, src, dst)
    return used.tolist()[0], src.tolist(), dst.tolist()


def test_compaction_onto_a_block_that_a_row_holds():
    """Row 0 holds block 0, which is counted as free: row 1's block moves there, and row 0 holds it no more."""
    p = pages(2, [[0], [1]], [0, 1])
    assert compact(p) == (1, [1], [0])
    assert p.block_table.tolist() == [[-1], [0]] and p.ref.tolist() == [1, 0]
    flagged(p)


def test_compaction_of_a_large_table():
    """Counted as free below the border, at it and past it, among 40000 entries that are sound."""
    n = 50000
    table, ref = torch.full((40, 1000), -1, dtype=torch.int32), torch.zeros(n, dtype=torch.int32)
    order = torch.randperm(n, generator=torch.Generator().manual_seed(3))[:40000].int()
    table.view(-1)[:] = order
    ref[order.long()] = 1
    bad = [int((table.view(-1) == b).nonzero()[0, 0]) for b in sorted(order.tolist())[5:39000:3000]]   # entries
    ids = table.view(-1)[bad].tolist()
    ref[ids] = 0
    p = pages(n, table.tolist(), ref.tolist())
    used, src, dst = compact(p)
    flagged(p)
    assert used == 40000 - len(bad)
    held = [i for i in order.tolist() if i not in ids]
    move = {s: d for s, d in zip(src, dst) if s >= 0}
    assert sorted(move) == sorted(i for i in held if i >= used)
    want = [[move.get(e, e) for e in row] for row in table.tolist()]
    for at, e in zip(bad, ids):   # below the border a block may have come there
        want[at // 1000][at % 1000] = -1 if e < used else e
    assert p.block_table.tolist() == want
    assert p.ref.tolist() == [1] * used + [0] * (n - used)


def reserve(p, length, want):
    out = [torch.full((len(length),), -9, dtype=torch.int32, device="cuda") for _ in range(3)]
    adept.adept_kv_reserve(p, i32(length), i32(want), *out)
    return [o.tolist() for o in out]


@pytest.mark.parametrize("blocks", [3, 9])   # of a row: few, many
def test_growth_into_an_entry_that_is_counted_as_free(blocks):
    """Row 0 holds block 0 behind its length, counted as free: the entry counts as -1 and gets a block like the others; block 0 is
    given once."""
    n = 4 * blocks
    p = pages(n, [[blocks, 0] + [-1] * blocks, [-1] * (blocks + 2)], [0] * blocks + [1] + [0] * (n - blocks - 1))
    got, src, dst = reserve(p, [16, 0], [16 + 16 * blocks, 20])
    assert (got, src, dst) == ([16 + 16 * blocks, 20], [-1, -1], [-1, -1])
    free = [i for i in range(n) if i != blocks]
    assert p.block_table.tolist() == [[blocks] + free[:blocks] + [-1], free[blocks:blocks + 2] + [-1] * blocks]
    assert p.ref.tolist() == [int(i in [blocks] + free[:blocks + 2]) for i in range(n)]
    flagged(p)


def test_growth_into_a_first_block_that_is_counted_as_free():
    """The block of positions that stay: its row gets another, without a copy, and nobody's count falls below 0."""
    p = pages(6, [[2, -1], [4, -1]], [1, 1, 0, 1, 1, 0])
    assert reserve(p, [5, 5], [9, 9]) == [[9, 9], [-1, -1], [-1, -1]]
    assert p.block_table.tolist() == [[2, -1], [4, -1]] and p.ref.tolist() == [1, 1, 1, 1, 1, 0]
    flagged(p)


def test_growth_that_is_not_served():
    """Nothing else of the row changes."""
    p = pages(4, [[0, 3, -1], [1, 2, -1]], [1, 1, 1, 0])
    assert reserve(p, [16, 20], [48, 30]) == [[16, 30], [-1, -1], [-1, -1]]   # two blocks asked for, one free
    assert p.block_table.tolist() == [[0, -1, -1], [1, 2, -1]] and p.ref.tolist() == [1, 1, 1, 0]
    flagged(p)


def fork(p, source, length):
    adept.adept_kv_fork(p, i32(source), i32(length))


@pytest.mark.parametrize("cols", [4, 30000])   # in one launch, in two
@pytest.mark.parametrize("entry", [1, 9, -3])
def test_fork_of_an_entry_that_is_no_block(cols, entry):
    """Row 0's second entry is counted as free (1), or no block (9, -3).  Rows that take it get -1 there, a row that has the same number there
    already too; no count changes for it."""
    rest = [-1] * (cols - 2)
    p = pages(8, [[0, entry] + rest, [2, entry] + rest, [3, -1] + rest], [1, 0, 1, 1, 0, 0, 0, 0])
    fork(p, [0, 0, 0], [32, 32, 32])
    assert p.block_table[:, :3].tolist() == [[0, entry, -1], [0, -1, -1], [0, -1, -1]]
    assert p.ref.tolist() == [3, 0, 0, 0, 0, 0, 0, 0]
    flagged(p)


@pytest.mark.parametrize("cols", [4, 30000])
def test_fork_that_drops_an_entry_counted_as_free(cols):
    rest = [-1] * (cols - 2)
    p = pages(8, [[0, 1] + rest, [2, 1] + rest, [3, -1] + rest], [1, 0, 1, 1, 0, 0, 0, 0])
    fork(p, [0, 1, 2], [16, 16, 16])
    assert p.block_table[:, :2].tolist() == [[0, -1], [2, -1], [3, -1]]
    assert p.ref.tolist() == [1, 0, 1, 1, 0, 0, 0, 0]
    flagged(p)


@pytest.mark.parametrize("cols", [4, 30000])
def test_fork_takes_what_another_row_drops(cols):
    """Not a fault: row 0 drops the block that row 1 takes from it, whichever comes first."""
    rest = [-1] * (cols - 1)
    for _ in range(20):
        p = pages(8, [[5] + rest, [6] + rest], [0, 0, 0, 0, 0, 1, 1, 0])
        fork(p, [1, 0], [16, 16])
        assert p.block_table[:, 0].tolist() == [6, 5] and p.ref.tolist() == [0, 0, 0, 0, 0, 1, 1, 0]
        fork(p, [-1, 0], [16, 16])
        assert p.block_table[:, 0].tolist() == [-1, 6] and p.ref.tolist() == [0, 0, 0, 0, 0, 0, 1, 0]
        p.check()
