"""The pages behind a paged cache against their block-by-block statement: rows grown, forked, cut back and dropped in long random
sequences, pools that run out, blocks that rows share, compaction, blocks copied in every layer, inputs out of range, graphs."""
import random

import pytest
import torch

from serve_reference import Pool, up

import paper_2601_03700_gb300 as adept

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    adept.load_library()


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Both:
    """The same calls on the GPU's pages and on the plain ones."""

    def __init__(self, n_blocks, n_seq, cols, bt=16):
        self.gpu, self.plain = adept.KVPages(n_blocks, n_seq, cols, block_tokens=bt), Pool(n_blocks, n_seq, cols, bt)
        self.n = n_seq

    def same(self):
        assert self.gpu.block_table.tolist() == self.plain.table
        assert self.gpu.ref.tolist() == self.plain.ref
        self.gpu.check()

    def fork(self, source, length):
        adept.adept_kv_fork(self.gpu, i32(source), i32(length))
        self.plain.fork(source, length)
        self.same()

    def reserve(self, length, want):
        out = [torch.full((self.n,), -9, dtype=torch.int32, device="cuda") for _ in range(3)]
        adept.adept_kv_reserve(self.gpu, i32(length), i32(want), *out)
        exp = self.plain.reserve(length, want)
        assert [o.tolist() for o in out] == [list(e) for e in exp]
        self.same()
        return exp

    def compact(self):
        n = len(self.plain.ref) // 2
        used, src, dst = i32([-9]), *(torch.full((n,), -9, dtype=torch.int32, device="cuda") for _ in range(2))
        adept.adept_kv_compact(self.gpu, used, src, dst)
        u, s, d = self.plain.compact()
        assert (used.tolist(), src.tolist(), dst.tolist()) == ([u], s, d)
        self.same()


@pytest.mark.parametrize("n_blocks,n_seq,cols,bt", [(1, 1, 1, 16), (7, 1, 20, 1), (40, 5, 9, 16), (64, 33, 40, 5), (300, 8, 70, 16), (1000, 100, 40, 3),
                                                    (9001, 257, 130, 16), (40000, 40, 1500, 16)])
def test_random_calls(n_blocks, n_seq, cols, bt):
    rng = random.Random(n_blocks)
    p = Both(n_blocks, n_seq, cols, bt)
    lens = [0] * n_seq
    most = max(1, min(cols * bt, n_blocks * bt * 2 // n_seq))
    for step in range(24):
        kind = rng.choice(["grow", "grow", "fork", "cut", "compact"])
        if kind == "grow":
            want = [min(cols * bt, n + rng.choice([0, 0, 1, bt, rng.randint(0, most)])) for n in lens]
            want = [w if rng.random() < 0.9 else n - 1 for n, w in zip(lens, want)]   # (fewer than there are: nothing is asked for)
            got = p.reserve(lens, want)[0]
            lens = [max(n, w) if g == w else n for n, w, g in zip(lens, want, got)]
        elif kind == "fork":
            source = [b if rng.random() < 0.5 else rng.choice([-1, rng.randrange(n_seq)]) for b in range(n_seq)]
            lens = [0 if s < 0 else lens[s] if rng.random() < 0.6 else rng.randint(0, lens[s]) for s in source]
            p.fork(source, lens)
        elif kind == "cut":
            lens = [rng.randint(n // 2, n) for n in lens]
            p.fork(list(range(n_seq)), lens)
        else:
            p.compact()
        p.plain.check()


def test_a_prompt_that_branches():
    """Three branches of a prompt of 20 positions that grow at once: two get a copy of the block they write, the last keeps it; with the
    prompt itself kept by its row, all three get one."""
    p = Both(20, 4, 5)
    p.reserve([0] * 4, [20, 0, 0, 0])
    p.fork([0, 0, 0, -1], [20, 20, 20, 0])
    got, src, dst = p.reserve([20, 20, 20, 0], [21, 25, 40, 0])
    assert got == [21, 25, 40, 0] and src == [1, 1, -1, -1] and dst == [2, 3, -1, -1]
    p = Both(20, 4, 5)
    p.reserve([0] * 4, [20, 0, 0, 0])
    p.fork([0, 0, 0, 0], [20] * 4)
    got, src, dst = p.reserve([20] * 4, [20, 25, 25, 25])
    assert src == [-1, 1, 1, 1] and dst == [-1, 2, 3, 4]


def test_rows_of_different_lengths_share_the_block():
    """Cut back to different places of one block: each that grows gets a copy but the last; one that is not served keeps sharing, and then
    nobody behind it may keep the block."""
    p = Both(4, 3, 4)
    p.reserve([0, 0, 0], [30, 0, 0])
    p.fork([0, 0, 0], [30, 18, 25])
    assert p.reserve([30, 18, 25], [31, 19, 26])[0] == [31, 19, 26]   # two copies, two free blocks
    p = Both(3, 3, 4)
    p.reserve([0, 0, 0], [30, 0, 0])
    p.fork([0, 0, 0], [30, 18, 25])
    got, src, dst = p.reserve([30, 18, 25], [31, 19, 26])
    assert got == [31, 18, 25] and src == [1, -1, -1]   # the third may not write where the second still reads


def test_a_pool_that_runs_out():
    p = Both(10, 5, 8)
    got = p.reserve([0] * 5, [50, 64, 1, 100, 0])[0]   # 4, 4 and 1 of ten blocks, 7 are not there
    assert got == [50, 64, 1, 0, 0]
    got = p.reserve([50, 64, 1, 0, 0], [64, 70, 16, 1, 0])[0]   # the first and the third have what they need, the second takes the last
    assert got == [64, 70, 16, 0, 0]
    got = p.reserve([64, 70, 16, 0, 0], [65, 71, 17, 0, 0])[0]   # nothing is left, but the second has room
    assert got == [64, 71, 16, 0, 0]


def test_entries_behind_the_length_are_the_rows():
    """Blocks that a row holds behind its length are used; those of them that others hold too are replaced, without a copy."""
    p = Both(30, 2, 8)
    p.reserve([0, 0], [100, 0])
    got, src, dst = p.reserve([20, 0], [90, 0])
    assert got == [90, 0]
    p.fork([0, 0], [100, 100])
    got, src, dst = p.reserve([32, 100], [90, 101])
    assert src == [-1, 6]


def test_blocks_that_the_program_holds():
    p = Both(12, 2, 4)
    p.reserve([0, 0], [40, 10])
    p.gpu.ref[0] += 1
    p.plain.ref[0] += 1
    p.fork([-1, 1], [0, 10])
    assert p.plain.ref[0] == 1
    p.compact()
    got, src, _ = p.reserve([0, 10], [64, 64])
    assert got == [64, 64]


def test_simultaneous_rows():
    """Rows that swap, chains of rows, a row that drops what others take from it."""
    p = Both(40, 5, 6)
    p.reserve([0] * 5, [90, 17, 33, 1, 16])
    p.fork([1, 0, 2, 3, 4], [17, 90, 33, 1, 16])
    p.fork([1, 2, 3, 4, 0], [90, 33, 1, 16, 17])
    p.fork([-1, 0, 0, 0, 0], [0, 90, 70, 16, 1])
    p.fork([4, 4, 4, 4, -1], [1, 1, 1, 1, 99])
    p.fork([-5, -1, 0, 1, 2], [3, 0, -4, 1, 1])


@pytest.mark.parametrize("case", ["source", "length", "entry", "entry_negative", "free_but_held"])
def test_fork_out_of_range(case):
    p = Both(10, 3, 4)
    p.reserve([0] * 3, [40, 20, 10])
    source, length = [0, 1, 2], [40, 20, 10]
    want = [list(r) for r in p.plain.table]
    if case == "source":
        source[1] = 3
    elif case == "length":
        length[1] = 65
    elif case == "entry":
        p.gpu.block_table[1, 1] = 10
        source[2], length[2] = 1, 20
        want[2] = [want[1][0], -1, -1, -1]
        want[1][1] = 10
    elif case == "entry_negative":
        p.gpu.block_table[1, 1] = -2
        length[1] = 3
        want[1] = [want[1][0], -1, -1, -1]
    else:
        p.gpu.ref[want[1][1]] = 0
        length[1] = 3
        want[1] = [want[1][0], -1, -1, -1]
    adept.adept_kv_fork(p.gpu, i32(source), i32(length))
    assert p.gpu.block_table.tolist() == want
    with pytest.raises(adept.AdeptError) as ei:
        p.gpu.check()
    assert ei.value.status == 6
    p.gpu.check()


@pytest.mark.parametrize("length,want,ok", [([-1, 0], [5, 5], False), ([0, 0], [65, 5], False), ([-3, 0], [-4, 5], True), ([70, 0], [70, 5], True)])
def test_reserve_out_of_range(length, want, ok):
    p = adept.KVPages(10, 2, 4)
    out = [torch.full((2,), -9, dtype=torch.int32, device="cuda") for _ in range(3)]
    adept.adept_kv_reserve(p, i32(length), i32(want), *out)
    assert out[0].tolist() == [length[0], 5] and p.block_table.tolist() == [[-1] * 4, [0, -1, -1, -1]]
    if not ok:
        with pytest.raises(adept.AdeptError):
            p.check()
    p.check()


def test_entries_out_of_range_are_replaced_or_left():
    p = adept.KVPages(10, 2, 4)
    p.block_table[0, 1] = 99
    out = [torch.full((2,), -9, dtype=torch.int32, device="cuda") for _ in range(3)]
    adept.adept_kv_reserve(p, i32([16, 0]), i32([20, 0]), *out)
    assert p.block_table[0].tolist() == [-1, 0, -1, -1] and out[0].tolist() == [20, 0]
    with pytest.raises(adept.AdeptError):
        p.check()
    p.block_table[1, 0], p.block_table[1, 1], p.block_table[1, 2] = 99, -3, 7   # (7: counted as free)
    used, s, d = i32([0]), i32([0] * 5), i32([0] * 5)
    adept.adept_kv_compact(p, used, s, d)
    assert used.tolist() == [1] and p.block_table[1].tolist() == [99, -3, 7, -1]
    with pytest.raises(adept.AdeptError):
        p.check()


def test_the_most_rows():
    n = 4096
    p = Both(9000, n, 3, 4)
    lens = [b % 9 for b in range(n)]
    p.reserve([0] * n, lens)
    source = [b // 2 for b in range(n)]
    lens = [lens[s] for s in source]
    p.fork(source, lens)
    p.reserve(lens, [n + 1 for n in lens])
    p.compact()
    big = adept.KVPages(5, n + 1, 1)
    z = torch.zeros(n + 1, dtype=torch.int32, device="cuda")
    with pytest.raises(adept.AdeptError) as ei:
        adept.adept_kv_reserve(big, z, z, z.clone(), z.clone(), z.clone())
    assert ei.value.status == 3
    adept.adept_kv_fork(big, z, z)


@pytest.mark.parametrize("n_blocks", [16000, 200000])
def test_blocks_that_become_free_are_not_given(n_blocks):
    """Two rows get away from 400 blocks that only they hold; the third row's come from those that were free before.  In the larger pool counts are
    read after the first blocks have been given."""
    p = Both(n_blocks, 4, 1000)
    low, shared = n_blocks // 200, n_blocks // 10
    ref = [0] * low + [1] * (shared - low) + [2] * 400 + [0] * (n_blocks - shared - 400)
    row = list(range(shared, shared + 400)) + [-1] * 600
    p.plain.ref, p.plain.table = list(ref), [list(row), list(row), [-1] * 1000, [-1] * 1000]
    p.gpu.ref.copy_(i32(ref))
    p.gpu.block_table[:2] = i32(row)
    got = p.reserve([0, 0, 0, 0], [6400, 6400, 9600, 300])[0]
    assert got == [6400, 6400, 9600, 300] and p.plain.ref[shared:shared + 400] == [0] * 400


def test_results_over_the_lengths():
    p, q = (adept.KVPages(9000, 300, 40) for _ in range(2))
    want = i32([(b * 7) % 400 for b in range(300)])
    for step in (0, 1, 150, 40):
        length = want.clone() if step else torch.zeros_like(want)
        more = want + step
        out = [[torch.empty_like(want) for _ in range(3)] for _ in range(2)]
        adept.adept_kv_reserve(p, length, more, *out[0])
        for place in ((length, 0), (more, 1)):
            if place[1] == 0:
                save = q.block_table.clone(), q.ref.clone()
            else:
                q.block_table.copy_(save[0])
                q.ref.copy_(save[1])
            args = [length.clone(), more.clone()]
            adept.adept_kv_reserve(q, *args, args[place[1]], *out[1][1:])
            assert torch.equal(args[place[1]], out[0][0])
            assert torch.equal(out[0][1], out[1][1]) and torch.equal(out[0][2], out[1][2])
            assert torch.equal(p.block_table, q.block_table) and torch.equal(p.ref, q.ref)
        want = out[0][0]


def test_a_long_row():
    """A row of 2^30 positions in blocks of one, of which the last are reserved."""
    p = adept.KVPages(300, 1, 1 << 26, block_tokens=16)
    out = [i32([0]) for _ in range(3)]
    adept.adept_kv_reserve(p, i32([(1 << 30) - 1000]), i32([1 << 30]), *out)
    n = 1000 // 16 + 1
    assert out[0].tolist() == [1 << 30] and p.block_table[0, -n:].tolist() == list(range(n)) and int((p.block_table >= 0).sum()) == n
    adept.adept_kv_fork(p, i32([0]), i32([(1 << 30) - 16]))
    assert int((p.block_table >= 0).sum()) == n - 1 and int(p.ref.sum()) == n - 1
    p.check()


def test_another_stream_and_graphs():
    """A round of fork, reserve, copy as one captured graph, replayed on other lengths; two graphs with workspaces of their own."""
    p, plain = adept.KVPages(60, 4, 10), Pool(60, 4, 10)
    c = adept.KVCache(60, 2, 64, 4, 10, pages=p)
    source, length, want = i32([0, 1, 2, 3]), i32([0] * 4), i32([0] * 4)
    out, ws = [i32([0] * 4) for _ in range(3)], p.workspace()

    def run():
        adept.adept_kv_fork(p, source, length, workspace=ws)
        adept.adept_kv_reserve(p, length, want, *out, workspace=ws)
        adept.adept_kv_copy_blocks(c, out[1], out[2])

    torch.cuda.synchronize()   # (what the side stream reads is made on this one)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        run()
    s.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run()
    for src, ln, wt in (([0, 1, 2, 3], [0] * 4, [40, 3, 0, 100]), ([0, 0, 1, 3], [35, 40, 3, 90], [50, 41, 20, 95]), ([3, 3, 3, 3], [70] * 4, [71] * 4)):
        for t, v in ((source, src), (length, ln), (want, wt)):
            t.copy_(i32(v))
        before = c.k.normal_().clone()
        g.replay()
        plain.fork(src, ln)
        exp = plain.reserve(ln, wt)
        assert [o.tolist() for o in out] == [list(e) for e in exp]
        assert p.block_table.tolist() == plain.table and p.ref.tolist() == plain.ref
        for a, b in zip(exp[1], exp[2]):
            if a >= 0:
                before[b] = before[a]
        assert torch.equal(c.k, before)
    p.check()


# ---- blocks copied

def caches(n, n_blocks, hk, dh, bt, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    out = []
    for _ in range(n):
        c = adept.KVCache(n_blocks, hk, dh, 1, 1, dtype=dtype, block_tokens=bt)
        for x in (c.k, c.v, c.k_exp, c.v_exp):
            if x is not None:
                x.copy_(torch.randint(0, 256, x.shape, generator=g, device="cuda").to(x.dtype) if x.dtype is torch.uint8 else
                        torch.randn(x.shape, generator=g, device="cuda").to(x.dtype))
        out.append(c)
    return out


@pytest.mark.parametrize("dtype", ["f32", "bf16", "e4m3"])
@pytest.mark.parametrize("layers,hk,dh,bt", [(1, 1, 32, 1), (2, 3, 32, 5), (3, 12, 64, 16), (33, 1, 32, 3), (70, 2, 64, 16), (2, 32, 128, 16), (1, 5, 128, 33),
                                             (1, 64, 128, 64)])
def test_copied_blocks(dtype, layers, hk, dh, bt):
    n = 41
    cs = caches(layers, n, hk, dh, bt, dtype, layers * hk)
    order = torch.randperm(n, generator=torch.Generator().manual_seed(bt)).tolist()
    src, dst = order[:20], order[20:40]
    src[3:6] = [src[2]] * 3   # one block to several
    src[7], dst[9] = -1, -1
    dst[11] = src[11]         # onto itself
    exp = []
    for c in cs:
        exp.append([None if x is None else x.clone() for x in (c.k, c.v, c.k_exp, c.v_exp)])
        for s, d in zip(src, dst):
            if s >= 0 and d >= 0:
                for x in exp[-1]:
                    if x is not None:
                        x[d] = x[s]
    adept.adept_kv_copy_blocks(adept.KVLayers(cs), i32(src), i32(dst))
    for c, e in zip(cs, exp):
        for x, y in zip((c.k, c.v, c.k_exp, c.v_exp), e):
            assert y is None or torch.equal(x.view(torch.uint8), y.view(torch.uint8))
        c.check()


@pytest.mark.parametrize("pairs", [0, 1, 700, 5000])
def test_many_pairs(pairs):
    """More pairs than there are blocks: most of them empty."""
    c = caches(1, 3000, 1, 32, 16, "bf16", 5)[0]
    g = torch.Generator().manual_seed(pairs)
    src, dst = torch.full((2, pairs), -1, dtype=torch.int32)
    live = torch.randperm(max(pairs, 1), generator=g)[:min(pairs, 1400)] if pairs else torch.zeros(0, dtype=torch.int64)
    order = torch.randperm(3000, generator=g).int()
    src[live], dst[live] = order[:len(live)], order[1500:1500 + len(live)]
    exp = c.k.clone(), c.v.clone()
    for x in exp:
        x[order[1500:1500 + len(live)].long().cuda()] = x[order[:len(live)].long().cuda()]
    adept.adept_kv_copy_blocks(c, src.cuda(), dst.cuda())
    assert torch.equal(c.k, exp[0]) and torch.equal(c.v, exp[1])


def test_pairs_out_of_range():
    c = caches(1, 6, 2, 64, 16, "e4m3", 6)[0]
    exp = c.k.clone()
    exp[1] = exp[0]
    adept.adept_kv_copy_blocks(c, i32([0, 6, 2]), i32([1, 2, 6]))
    assert torch.equal(c.k, exp)
    with pytest.raises(adept.AdeptError):
        c.check()


def test_a_pool_past_2_31_bytes():
    """Blocks of 1 MB at offsets that 32 bits do not hold."""
    c = adept.KVCache(2300, 128, 128, 1, 1, dtype="bf16", block_tokens=32)
    c.k[2299].normal_()
    c.v[0].normal_()
    adept.adept_kv_copy_blocks(c, i32([2299, 0]), i32([1, 2298]))
    assert torch.equal(c.k[1], c.k[2299]) and torch.equal(c.v[2298], c.v[0]) and not bool(c.k[2:2299].any())


def test_up():
    assert [up(n, 16) for n in (0, 1, 16, 17)] == [0, 1, 1, 2]
