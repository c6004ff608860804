"""The operators on a caller-owned paged K/V cache (adept_kv_append, adept_kv_gather, adept_chunk_attention) against their
64-bit statements: types, head layouts, ragged and empty chunks, block ends, strides, hidden NaN, streams and graphs."""
import math

import pytest
import torch

import kv_reference as R
import paper_2601_03700_gb300 as adept

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    adept.load_library()


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def make_cache(dtype, hk, dh, lens, seed, bt=16, spare=2):
    """A cache with random entries at positions below lens[b] in shuffled blocks; everything else holds NaN."""
    g = _gen(seed)
    need = [(n + bt - 1) // bt for n in lens]
    width, total = max(max(need), 1), sum(need) + spare
    c = adept.KVCache(total, hk, dh, len(lens), width, dtype=dtype, block_tokens=bt)
    if dtype == "e4m3":
        c.k.fill_(0x7f)
        c.v.fill_(0x7f)
    else:
        c.k.fill_(math.nan)
        c.v.fill_(math.nan)
    order = torch.randperm(total, generator=g, device="cuda").to(torch.int32)
    at = 0
    for b, n in enumerate(need):
        c.block_table[b, :n] = order[at:at + n]
        at += n
    for b, n in enumerate(lens):
        if n:
            kv = 1.5 * torch.randn(2, n, hk, dh, generator=g, device="cuda")
            kv[1] *= torch.exp2(torch.randn(dh, generator=g, device="cuda"))
            adept.adept_kv_append(c, kv[0], kv[1], _i32([b] * n), _i32(list(range(n))))
    c.check()
    return c


def make_q(dtype, new, heads, dh, seed, extra=0, pad=0):
    """Queries as a view into wider rows, and the rows' starts."""
    g = _gen(seed)
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    rows = sum(new) + extra
    q = torch.randn(rows, heads * dh + pad, generator=g, device="cuda").to(dt)[:, :heads * dh]
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    return q.unflatten(1, (heads, dh)), starts


def attend(c, q, starts, lens, **kw):
    out = torch.full(q.shape, -7.0, dtype=q.dtype, device="cuda")
    max_q = max(b - a for a, b in zip(starts, starts[1:]))
    adept.adept_chunk_attention(c, q, _i32(starts), _i32(lens), max_q, max(lens), out, **kw)
    return out


def assert_attention(c, q, starts, lens, out):
    want, tol = R.attention(c, q, starts, lens)
    n = starts[-1]
    err = (out[:n].double() - want[:n]).abs()
    worst = (err / (tol[:n] + 1e-30)).max().item() if n else 0.0
    assert torch.isfinite(out).all() and (err <= tol[:n] + 1e-30).all(), f"error {worst:.3f} of its bound"
    assert (out[n:] == -7).all()


# (new tokens, cached positions before them) per sequence
CHUNKS = [
    ([1], [0]),
    ([1], [15]),
    ([1], [16]),
    ([2, 1, 1], [0, 130, 62]),
    ([0, 3, 0], [5, 0, 0]),
    ([17, 5], [64, 97]),
    ([16, 1, 33, 0, 8], [16, 300, 1, 40, 127]),
    ([130], [45]),
    ([1] * 37, [7 * i % 90 for i in range(37)]),
]


@pytest.mark.parametrize("new,past", CHUNKS)
@pytest.mark.parametrize("heads,hk,dh", [(3, 3, 64), (8, 2, 128), (4, 4, 32), (5, 1, 64)])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "e4m3"])
def test_attention_of_ragged_chunks(dtype, heads, hk, dh, new, past):
    lens = [a + b for a, b in zip(new, past)]
    c = make_cache(dtype, hk, dh, lens, 3)
    q, starts = make_q(dtype, new, heads, dh, 4, extra=3, pad=24)
    out = attend(c, q, starts, lens)
    c.check()
    assert_attention(c, q, starts, lens, out)


@pytest.mark.parametrize("dtype,heads,hk,dh,new,past", [
    ("bf16", 32, 32, 128, [1], [2500]),
    ("e4m3", 32, 8, 128, [1, 1, 1], [1999, 3, 700]),
    ("bf16", 12, 12, 64, [300], [1000]),
    ("e4m3", 16, 2, 64, [70, 257], [900, 0]),
    ("bf16", 8, 2, 128, [513], [129]),
    ("e4m3", 8, 8, 128, [129, 64, 40], [0, 640, 1111]),
    ("bf16", 40, 2, 64, [1, 3, 90], [100, 2, 30]),     # 20 query heads on a K/V head
    ("e4m3", 33, 1, 128, [2, 50], [1030, 17]),
    ("f32", 6, 3, 64, [40, 1], [700, 1500]),
])
def test_attention_of_longer_chunks(dtype, heads, hk, dh, new, past):
    lens = [a + b for a, b in zip(new, past)]
    c = make_cache(dtype, hk, dh, lens, 5)
    q, starts = make_q(dtype, new, heads, dh, 6)
    out = attend(c, q, starts, lens)
    c.check()
    assert_attention(c, q, starts, lens, out)
    assert torch.equal(out, attend(c, q, starts, lens)), "the same call gave other bits"


@pytest.mark.parametrize("new,past", [
    ([16, 1, 33, 0, 8, 400], [16, 300, 1, 40, 127, 5]),
    ([300, 257, 17, 5], [64, 0, 0, 97]),
    ([600], [45]),
    ([9, 400, 2, 1, 270], [-3, -250, -1, 128, -15]),   # chunks longer than what is held: their first rows attend nothing
])
@pytest.mark.parametrize("heads,hk,dh", [(3, 3, 64), (8, 2, 128), (5, 1, 64), (24, 2, 128)])
@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_attention_of_chunks_beside_a_long_one(dtype, heads, hk, dh, new, past):
    lens = [a + b for a, b in zip(new, past)]
    c = make_cache(dtype, hk, dh, lens, 9)
    q, starts = make_q(dtype, new, heads, dh, 10, extra=3)
    out = attend(c, q, starts, lens)
    c.check()
    assert_attention(c, q, starts, lens, out)
    for b, (n, p) in enumerate(zip(new, past)):
        assert (out[starts[b]:starts[b] + max(0, -p)] == 0).all()


@pytest.mark.parametrize("heads,hk,dh,new,past", [
    (16, 4, 128, [1, 200, 3, 0, 17], [4600, 300, 90, 8, 0]),   # the few rows' keys split over the GPU, joined beside the longer chunks'
    (4, 4, 64, [40, 1, 1], [60, 2300, 0]),
    (16, 4, 128, [1, 200, 3], [700, 300, 90]),                 # over clusters
    (16, 4, 128, [1, 2, 30], [3, 90, 50]),                     # not split
    (16, 4, 128, [200, 300], [4600, 10]),                      # no sequence of few
])
def test_few_and_many_tokens_over_8_bit_entries(heads, hk, dh, new, past):
    lens = [a + b for a, b in zip(new, past)]
    c = make_cache("e4m3", hk, dh, lens, 7)
    q, starts = make_q("bf16", new, heads, dh, 8, extra=2)
    ws = c.attention_workspace(heads, q.shape[0], max(new), max(lens))
    outs = [attend(c, q, starts, lens, workspace=ws) for _ in range(6)]
    c.check()
    assert_attention(c, q, starts, lens, outs[0])
    assert all(torch.equal(outs[0], o) for o in outs)


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("bt", [1, 8, 48])
def test_attention_over_other_block_sizes(dtype, bt):
    new, past = [9, 1], [50, 200]
    lens = [a + b for a, b in zip(new, past)]
    c = make_cache(dtype, 2, 64, lens, 7, bt=bt)
    q, starts = make_q(dtype, new, 4, 64, 8)
    assert_attention(c, q, starts, lens, attend(c, q, starts, lens))


@pytest.mark.parametrize("shift,pad", [(1, 0), (0, 1), (4, 3)])
def test_attention_of_rows_off_16_bytes(shift, pad):
    new, lens = [20, 1], [100, 50]
    c = make_cache("bf16", 2, 64, lens, 9)
    buf = torch.randn(21 * (256 + pad) + shift, generator=_gen(10), device="cuda").to(torch.bfloat16)
    q = buf[shift:].view(21, 256 + pad)[:, :256].unflatten(1, (4, 64))
    room = torch.full((21 * (256 + pad) + shift,), -7.0, dtype=torch.bfloat16, device="cuda")
    out = room[shift:].view(21, 256 + pad)[:, :256].unflatten(1, (4, 64))
    adept.adept_chunk_attention(c, q, _i32([0, 20, 21]), _i32(lens), 20, 100, out)
    assert_attention(c, q, [0, 20, 21], lens, out)
    assert (room[:shift] == -7).all() and (room[shift:].view(21, 256 + pad)[:, 256:] == -7).all()


@pytest.mark.parametrize("dtype,heads,hk,dh,new,past", [
    ("f32", 2, 2, 64, 20, 3), ("bf16", 8, 2, 128, 4, 30), ("bf16", 4, 4, 64, 200, 10), ("e4m3", 8, 2, 128, 4, 30),
    ("e4m3", 4, 2, 128, 150, 100), ("e4m3", 2, 2, 64, 40, 0),
])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_later_positions_may_hold_anything(dtype, heads, hk, dh, new, past, bad):
    """A NaN or infinite entry at position p: rows before p are what they were, rows from p on show it in its column."""
    if dtype == "e4m3" and not math.isnan(bad):
        pytest.skip("stored as NaN")
    n = new + past
    c = make_cache(dtype, hk, dh, [n], 11)
    q, starts = make_q(dtype, [new], heads, dh, 12)
    clean = attend(c, q, starts, [n])
    p, col = past + new // 2, 5
    k = R.positions(c, "k", 0, n).float()[p:p + 1].clone()
    v = R.positions(c, "v", 0, n).float()[p:p + 1].clone()
    v[0, hk - 1, col] = bad
    adept.adept_kv_append(c, k, v, _i32([0]), _i32([p]))
    out = attend(c, q, starts, [n])
    hit = torch.zeros_like(out, dtype=torch.bool)
    hit[new // 2:, heads - heads // hk:, col] = True
    assert not torch.isfinite(out[hit]).any()
    if dtype != "e4m3":
        assert torch.equal(out[~hit], clean[~hit])
    else:   # (without that element the head's exponent may be another)
        assert torch.isfinite(out[~hit]).all() and torch.equal(out[:new // 2], clean[:new // 2])
    k[0, hk - 1, col] = bad   # and in K: the rows from p on, the heads of that K/V head, whole
    adept.adept_kv_append(c, k, v, _i32([0]), _i32([p]))
    out = attend(c, q, starts, [n])
    assert torch.equal(out[:new // 2], clean[:new // 2])
    assert torch.equal(out[:, :heads - heads // hk], clean[:, :heads - heads // hk])


@pytest.mark.parametrize("dtype,heads,hk,dh", [("f32", 4, 2, 64), ("bf16", 8, 2, 128), ("bf16", 6, 6, 64), ("e4m3", 8, 2, 128),
                                               ("bf16", 4, 4, 32)])
@pytest.mark.parametrize("new,keep", [([6, 1, 0, 9], 0.6), ([700, 40, 1, 3], 0.5), ([300, 2, 260, 0], 0.95)])
def test_rows_at_given_positions(dtype, heads, hk, dh, new, keep):
    """Rows of some of a chunk's tokens only, at their own positions: the same rows of the whole chunk's reference."""
    past = [130, 0, 77, 500]
    lens = [a + b for a, b in zip(new, past)]
    c = make_cache(dtype, hk, dh, lens, 50)
    q, starts = make_q(dtype, new, heads, dh, 51)
    want, tol = R.attention(c, q, starts, lens)
    g = torch.Generator().manual_seed(52)
    pick = torch.rand(sum(new), generator=g) < keep
    pos = torch.cat([torch.arange(p, p + n) for n, p in zip(new, past)])
    rows = pick.nonzero().flatten()
    st = [int((rows < s).sum()) for s in starts]
    sub = torch.cat([q[rows.cuda()], q[:2]])                 # two rows behind the last sequence's
    out = torch.full_like(sub, -7.0)
    row_pos = _i32(pos[rows].tolist() + [0, 0])
    adept.adept_chunk_attention(c, sub, _i32(st), _i32(lens), max(new), max(lens), out, row_pos=row_pos)
    c.check()
    assert (out[len(rows):] == -7).all()
    err = (out[:len(rows)].double() - want[rows.cuda()]).abs()
    assert (err <= tol[rows.cuda()] + 1e-30).all()
    again = torch.full_like(sub, -7.0)
    adept.adept_chunk_attention(c, sub, _i32(st), _i32(lens), max(new), max(lens), again, row_pos=row_pos)
    assert torch.equal(out, again)


@pytest.mark.parametrize("heads,hk,dh,new,past", [(8, 2, 128, 2, 30), (3, 3, 64, 8, 700), (4, 4, 32, 5, 20), (2, 1, 128, 4, 5000)])
def test_eight_rows_over_8_bit_entries(heads, hk, dh, new, past):
    """At most 8 rows a K/V head: NaN at later positions; rows at given positions."""
    test_later_positions_may_hold_anything("e4m3", heads, hk, dh, new, past, math.nan)
    test_rows_at_given_positions("e4m3", heads, hk, dh, [new, 1, 0, 2], 0.7)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "e4m3"])
@pytest.mark.parametrize("n", [6, 700])
def test_positions_that_do_not_ascend_touch_no_other_sequence(dtype, n):
    """A sequence's rows in descending, then in shuffled order of position: its own rows may hold anything."""
    new, lens = [n, 20, n], [3000, 90, 3000]
    c = make_cache(dtype, 2, 128, lens, 53)
    q, starts = make_q(dtype, new, 8, 128, 54, extra=2)
    want, tol = R.attention(c, q, starts, lens)
    down = torch.arange(2999, 2999 - n, -1)
    mixed = torch.randint(-5, 4000, (n,), generator=torch.Generator().manual_seed(55))
    row_pos = _i32(torch.cat([down, torch.arange(70, 90), mixed, torch.zeros(2)]).long().tolist())
    out = torch.full_like(q, -7.0)
    adept.adept_chunk_attention(c, q, _i32(starts), _i32(lens), max(new), 3000, out, row_pos=row_pos)
    torch.cuda.synchronize()
    mid = slice(n, n + 20)
    assert ((out[mid].double() - want[mid]).abs() <= tol[mid] + 1e-30).all()
    assert (out[-2:] == -7).all()


@pytest.mark.parametrize("dtype,heads,hk,dh", [("f32", 2, 1, 64), ("bf16", 8, 2, 128), ("e4m3", 4, 4, 64)])
def test_rows_without_keys_are_zero(dtype, heads, hk, dh):
    c = make_cache(dtype, hk, dh, [4, 0, 20], 13)
    q, starts = make_q(dtype, [9, 6, 33], heads, dh, 14)
    out = attend(c, q, starts, [4, 0, 20])
    assert (out[:5] == 0).all() and (out[9:15] == 0).all() and (out[15:28] == 0).all()
    assert_attention(c, q, starts, [4, 0, 20], out)
    c.check()


@pytest.mark.parametrize("dtype,dh", [("f32", 64), ("bf16", 128), ("e4m3", 128), ("bf16", 32)])
def test_large_and_small_scores(dtype, dh):
    """Scores in the thousands (one key takes all the weight) and all alike."""
    c = make_cache(dtype, 1, dh, [300], 15)
    q, starts = make_q(dtype, [5], 2, dh, 16)
    for f in (0.0, 300.0):
        qq = (q.float() * f).to(q.dtype)
        assert_attention(c, qq, starts, [300], attend(c, qq, starts, [300]))


def test_inputs_out_of_range_are_flagged_and_left_out():
    new, lens = [3, 2, 4], [40, 30, 50]
    for dtype, heads, hk, dh in (("bf16", 4, 2, 64), ("f32", 2, 2, 32), ("e4m3", 8, 8, 128)):
        c = make_cache(dtype, hk, dh, lens, 17)
        q, starts = make_q(dtype, new, heads, dh, 18)
        good = attend(c, q, starts, lens)

        def call(starts=starts, lens=lens, max_q=4, max_kv=50):
            out = torch.full(q.shape, -7.0, dtype=q.dtype, device="cuda")
            adept.adept_chunk_attention(c, q, _i32(starts), _i32(lens), max_q, max_kv, out)
            with pytest.raises(adept.AdeptError) as ei:
                c.check()
            assert ei.value.status == 6
            c.check()   # cleared
            return out

        out = call(max_q=3)                      # sequence 2 brings 4 rows
        assert torch.equal(out[:5], good[:5]) and (out[5:] == -7).all()
        out = call(max_kv=45)                    # and its 50 positions
        assert torch.equal(out[:5], good[:5]) and (out[5:] == -7).all()
        out = call(lens=[40, -1, 50])
        assert torch.equal(out[:3], good[:3]) and (out[3:5] == -7).all() and torch.equal(out[5:], good[5:])
        # sequence 1 would have -1 rows (the bound of 9 rows may pick another kernel: held against the reference)
        out = call(starts=[0, 3, 2, 9], max_q=9)
        assert_attention(c, q[:2], [0, 2, 2, 2], [39, 0, 0], out[:2])
        call(starts=[0, 3, 5, 10], max_q=9)      # a row behind the last
        call(starts=[-1, 3, 5, 9], max_q=9)
        for blk in (-1, 10 ** 6):
            held = c.block_table[0, 1].item()
            c.block_table[0, 1] = blk
            out = call()
            c.block_table[0, 1] = held
            assert torch.equal(out[3:], good[3:]) and torch.isfinite(out).all()


# ---- writing and reading back ---------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["f32", "bf16", "e4m3"])
@pytest.mark.parametrize("bt", [8, 16])
def test_keys_of_a_missing_block_are_left_out(dtype, bt):
    """The last block of positions is in no table: its rows attend what is before it, and the call says so."""
    lens = [3 * bt, 10]
    c = make_cache(dtype, 2, 64, lens, 19, bt=bt)
    q, starts = make_q(dtype, [1, 2], 4, 64, 20)
    c.block_table[0, 2] = -1
    out = attend(c, q, starts, lens)
    with pytest.raises(adept.AdeptError):
        c.check()
    assert_attention(c, q, starts, [2 * bt, 10], out)


def test_sequences_that_share_rows_beyond_any_count():
    """Row ranges that go up and down (flagged) over and over: 4000 times 8192 rows at 8192 positions of 512 heads are 2^32 pairs of
    tiles, though the call's 8192 rows are not; nothing is done."""
    n, c = 8000, 8192
    cache = adept.KVCache(1, 512, 64, n, c // 16)
    cache.block_table.zero_()
    start = torch.zeros(n + 1, dtype=torch.int32, device="cuda")
    start[1::2] = c
    q = torch.ones(c, 512, 64, dtype=torch.bfloat16, device="cuda")
    out = torch.full_like(q, 7)
    adept.adept_chunk_attention(cache, q, start, torch.full((n,), c, dtype=torch.int32, device="cuda"), c, c, out)
    with pytest.raises(adept.AdeptError):
        cache.check()
    assert (out == 7).all()


@pytest.mark.parametrize("src", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "e4m3"])
@pytest.mark.parametrize("hk,dh", [(3, 32), (5, 64), (1, 128), (2, 128)])
def test_write_and_read_back(src, dtype, hk, dh):
    g = _gen(20)
    rows, bt = 83, 16
    c = adept.KVCache(12, hk, dh, 3, 4, dtype=dtype, block_tokens=bt)
    c.block_table.copy_(torch.randperm(12, generator=g, device="cuda").view(3, 4).to(torch.int32))
    slots = torch.randperm(3 * 4 * bt, generator=g, device="cuda")[:rows]
    seq, pos = (slots // (4 * bt)).to(torch.int32), (slots % (4 * bt)).to(torch.int32)
    seq[5] = seq[-1] = -1   # left out
    kv = (torch.randn(2, rows, hk, dh, generator=g, device="cuda") * torch.exp2(6 * torch.randn(2, rows, hk, 1, generator=g, device="cuda"))).to(src)
    before = [R.entries(c, w) for w in ("k", "v")]
    adept.adept_kv_append(c, kv[0], kv[1], seq, pos)
    c.check()
    keep = seq >= 0
    blk = c.block_table[seq[keep].long(), pos[keep].long() // bt].long()
    for w, x, old in zip(("k", "v"), kv, before):
        want = old.clone()
        x = x[keep].double()
        want[blk, :, pos[keep].long() % bt] = R.quantise(x)[0] if dtype == "e4m3" else \
            (x if dtype == "f32" else x.to(torch.bfloat16).double())
        assert torch.equal(R.entries(c, w), want)
    for dst in (torch.float32, torch.bfloat16):
        out = torch.full((2, rows, hk, dh), -7.0, dtype=dst, device="cuda")
        adept.adept_kv_gather(c, seq, pos, out[0], out[1])
        for w, o in zip(("k", "v"), out):
            got = R.entries(c, w)[blk, :, pos[keep].long() % bt]
            assert torch.equal(o[keep], got.to(dst)) and (o[~keep] == -7).all()
    c.check()


def test_every_code_ties_and_exponents():
    """All 254 finite codes at several exponents come back as themselves, halfway points go to the even code, and the
    largest element decides the exponent on both sides of 448."""
    codes = torch.arange(256, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn).float()
    vals = codes[torch.isfinite(codes)]
    mid = (vals.sort().values[1:] + vals.sort().values[:-1]) / 2
    c = adept.KVCache(64, 1, 128, 1, 64, dtype="e4m3")
    c.block_table.copy_(torch.arange(64, device="cuda").view(1, 64))
    x = torch.cat([vals, vals[:2], mid, mid[:3]])
    x = x[:x.numel() // 127 * 127].view(-1, 127)
    x = torch.cat([x, torch.full((x.shape[0], 1), 448.0, device="cuda")], 1)   # pins the exponent at 0
    rows = torch.cat([x * 2.0 ** e for e in (-100, -3, 0, 11, 100)])
    tops = [448.0, 448.0000305, 447.9, 449.0, 1.0, 0.875, 0.8750001, 1e-38, 1.2e-41, 3.4e38, 3e-45, 0.0]
    more = torch.randn(len(tops), 128, generator=_gen(21), device="cuda").clamp(-1, 1) * torch.tensor(tops, device="cuda")[:, None]
    more[:, 7] = -torch.tensor(tops, device="cuda")
    rows = torch.cat([rows, more]).view(-1, 1, 128)
    n = rows.shape[0]
    seq, pos = _i32([0] * n), _i32(list(range(n)))
    adept.adept_kv_append(c, rows, -rows, seq, pos)
    c.check()
    want, ex = R.quantise(rows)
    p = torch.arange(n, device="cuda")
    assert torch.equal(c.k_exp.view(-1)[:n].int(), ex.view(-1) + 127)
    assert torch.equal(R.entries(c, "k")[p // 16, :, p % 16], want)
    assert torch.equal(R.entries(c, "v")[p // 16, :, p % 16], -want)
    out = torch.empty(2, n, 1, 128, device="cuda")
    adept.adept_kv_gather(c, seq, pos, out[0], out[1])
    # 3.4e38 rounds to 2^128, which fp32 does not hold: it reads back as infinity; everything else as it is (4 bits)
    assert torch.equal(out[0], want.float()) and torch.equal(out[1], -want.float())
    assert (want.float().double() != want).sum() == (want.abs() == 2.0 ** 128).sum() > 0


def test_nan_and_infinity_are_stored_as_nan():
    c = adept.KVCache(1, 2, 64, 1, 1, dtype="e4m3")
    c.block_table.zero_()
    x = torch.randn(3, 2, 64, generator=_gen(22), device="cuda")
    clean = R.quantise(x)[0]
    bad = x.clone()
    bad[0, 0, 3], bad[1, 1, 9], bad[2, 0, 60] = math.nan, math.inf, -math.inf
    for dt in (torch.float32, torch.bfloat16):
        adept.adept_kv_append(c, bad.to(dt), x.to(dt), _i32([0, 0, 0]), _i32([0, 1, 2]))
        out = torch.empty(2, 3, 2, 64, device="cuda")
        adept.adept_kv_gather(c, _i32([0, 0, 0]), _i32([0, 1, 2]), out[0], out[1])
        fin = torch.isfinite(bad)
        assert torch.isnan(out[0][~fin]).all() and torch.isfinite(out[0][fin]).all()
        assert torch.equal(out[1].double(), R.quantise(x.to(dt))[0])
    all_bad = torch.full((1, 2, 64), math.inf, device="cuda")
    adept.adept_kv_append(c, all_bad, x[:1], _i32([0]), _i32([0]))
    assert (c.k_exp[0, :, 0] == 127).all() and clean is not None


@pytest.mark.parametrize("src", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shift,pad", [(0, 0), (1, 0), (0, 1), (8, 16)])
def test_strided_and_misaligned_rows(src, shift, pad):
    g = _gen(23)
    rows, w = 19, 3 * 64
    buf = torch.randn(2, rows * (w + pad) + shift, generator=g, device="cuda").to(src)
    kv = [b[shift:].view(rows, w + pad)[:, :w] for b in buf]
    c = adept.KVCache(2, 3, 64, 1, 2, dtype="e4m3")
    c.block_table.copy_(torch.tensor([[1, 0]]))
    seq, pos = _i32([0] * rows), _i32(list(range(rows)))
    adept.adept_kv_append(c, kv[0], kv[1], seq, pos)
    room = torch.full_like(buf, -7.0)
    out = [b[shift:].view(rows, w + pad)[:, :w] for b in room]
    adept.adept_kv_gather(c, seq, pos, out[0], out[1])
    for x, o, b in zip(kv, out, room):
        assert torch.equal(o.unflatten(1, (3, 64)).double(), R.quantise(x.unflatten(1, (3, 64)))[0])
        assert (b[:shift] == -7).all() and (b[shift:].view(rows, w + pad)[:, w:] == -7).all()


def test_rows_out_of_range_are_flagged_and_left_out():
    c = adept.KVCache(3, 1, 64, 2, 2, dtype="bf16")
    c.block_table.copy_(torch.tensor([[0, -1], [2, 99]]))
    x = torch.ones(6, 1, 64, device="cuda")
    for seq, pos in ((2, 0), (0, -1), (0, 32), (0, 17), (1, 16)):
        adept.adept_kv_append(c, x[:1], x[:1], _i32([seq]), _i32([pos]))
        with pytest.raises(adept.AdeptError) as ei:
            c.check()
        assert ei.value.status == 6
        out = torch.full((2, 1, 1, 64), -7.0, device="cuda")
        adept.adept_kv_gather(c, _i32([seq]), _i32([pos]), out[0], out[1])
        with pytest.raises(adept.AdeptError):
            c.check()
        assert (out == -7).all()
    assert (c.k == 0).all() and (c.v == 0).all()
    adept.adept_kv_append(c, x[:0], x[:0], _i32([]), _i32([]))
    c.check()


# ---- as they are used together --------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_a_conversation_grows(dtype):
    """Turns of several users: their new K/V are written, their new tokens attend; prompts, checks and steps mixed."""
    g = _gen(30)
    heads, hk, dh, users = 8, 2, 128, 3
    c = adept.KVCache(users * 40, hk, dh, users, 40, dtype=dtype)
    c.block_table.copy_(torch.randperm(users * 40, generator=g, device="cuda").view(users, 40).to(torch.int32))
    lens = [0] * users
    for new in ([150, 1, 33], [1, 5, 0], [1, 1, 1], [17, 290, 2]):
        rows = sum(new)
        qkv = torch.randn(rows, heads + 2 * hk, dh, generator=g, device="cuda").to(torch.bfloat16)
        lens = [a + b for a, b in zip(lens, new)]
        seq = [b for b, n in enumerate(new) for _ in range(n)]
        pos = [p for b, n in enumerate(new) for p in range(lens[b] - n, lens[b])]
        adept.adept_kv_append(c, qkv[:, heads:heads + hk], qkv[:, heads + hk:], _i32(seq), _i32(pos))
        starts = [sum(new[:b]) for b in range(users + 1)]
        q = qkv[:, :heads]
        out = attend(c, q, starts, lens)
        c.check()
        assert_attention(c, q, starts, lens, out)


def test_a_captured_step_follows_its_lengths():
    """A generation step's two calls captured once and replayed as the contexts grow, beside a second captured step with a
    workspace of its own; each equal to the direct calls."""
    g = _gen(31)
    heads, hk, dh, users = 16, 4, 128, 2
    caches = [make_cache("e4m3", hk, dh, [600, 2000], 32 + i) for i in range(2)]
    steps = []
    for c in caches:
        s = dict(c=c, kv=torch.randn(2, users, hk, dh, generator=g, device="cuda").to(torch.bfloat16),
                 q=torch.randn(users, heads, dh, generator=g, device="cuda").to(torch.bfloat16),
                 seq=_i32([0, 1]), pos=_i32([40, 900]), lens=_i32([41, 901]), starts=_i32([0, 1, 2]))
        s["out"] = torch.zeros_like(s["q"])
        s["ws"] = c.attention_workspace(heads, users, 1, 2000)
        steps.append(s)

    def step(s, out, ws):
        adept.adept_kv_append(s["c"], s["kv"][0], s["kv"][1], s["seq"], s["pos"])
        adept.adept_chunk_attention(s["c"], s["q"], s["starts"], s["lens"], 1, 2000, out, ws)

    side = torch.cuda.Stream()
    graphs = []
    for s in steps:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step(s, s["out"], s["ws"])
        graphs.append(graph)
    for turn in range(4):
        for s in steps:
            s["q"].copy_(torch.randn(s["q"].shape, generator=g, device="cuda"))
            s["kv"].copy_(torch.randn(s["kv"].shape, generator=g, device="cuda"))
            s["pos"].copy_(_i32([40 + 130 * turn, 900 + turn]))
            s["lens"].copy_(s["pos"] + 1)
        for graph in graphs:
            graph.replay()
        for s in steps:
            got = s["out"].clone()
            direct = torch.zeros_like(got)
            step(s, direct, None)
            assert torch.equal(got, direct)
            assert_attention(s["c"], s["q"], [0, 1, 2], s["lens"].tolist(), got)


def test_other_streams():
    """Calls on streams of their own, side by side, each with its workspace."""
    lens, new = [3000, 40], [2, 40]
    c = make_cache("bf16", 4, 64, lens, 33)
    q, starts = make_q("bf16", new, 8, 64, 34)
    want = attend(c, q, starts, lens)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    outs = []
    for _ in range(4):
        for s in streams:
            with torch.cuda.stream(s):
                outs.append(attend(c, q, starts, lens))
        s = streams[0]
        s.wait_stream(torch.cuda.current_stream())
        out = torch.empty_like(want)
        s.wait_stream(torch.cuda.current_stream())
        adept.adept_chunk_attention(c, q, _i32(starts), _i32(lens), 40, 3000, out, stream=s)
        torch.cuda.synchronize()
        outs.append(out)
    assert all(torch.equal(o, want) for o in outs)


@pytest.mark.parametrize("dtype", ["e4m3", "bf16"])
def test_offsets_past_32_bits(dtype):
    """Blocks whose elements lie past 2^32 of the pool."""
    hk, dh, bt = 8, 128, 16
    n_blocks = (2 ** 32 // (hk * dh * bt)) + 64
    c = adept.KVCache(n_blocks, hk, dh, 1, 8, dtype=dtype)
    c.block_table.copy_(torch.arange(n_blocks - 8, n_blocks, device="cuda").view(1, 8))
    g = _gen(35)
    kv = torch.randn(2, 128, hk, dh, generator=g, device="cuda").to(torch.bfloat16)
    seq, pos = _i32([0] * 128), _i32(list(range(128)))
    adept.adept_kv_append(c, kv[0], kv[1], seq, pos)
    back = torch.empty_like(kv)
    adept.adept_kv_gather(c, seq, pos, back[0], back[1])
    small = adept.KVCache(8, hk, dh, 1, 8, dtype=dtype)
    small.block_table.copy_(torch.arange(8, device="cuda").view(1, 8))
    adept.adept_kv_append(small, back[0], back[1], seq, pos)
    assert torch.equal(back.double(), R.quantise(kv)[0] if dtype == "e4m3" else kv.double())
    for new in (1, 5, 100):
        q, starts = make_q(dtype, [new], 16, dh, 36)
        out = attend(c, q, starts, [128])
        assert_attention(small, q, starts, [128], out)


@pytest.mark.parametrize("dtype,new", [("bf16", [1]), ("e4m3", [2]), ("bf16", [200]), ("e4m3", [150])])
def test_waits_of_one_cycle(dtype, new):
    """A wait that has to be taken up again gives up at once: the call either comes through (the hardware's own wait was long
    enough) or reports the time-out, its copies landed; the next call is whole again."""
    lens = [n + 700 for n in new]
    c = make_cache(dtype, 4, 128, lens, 60)
    q, starts = make_q(dtype, new, 8, 128, 61)
    want = attend(c, q, starts, lens)
    try:
        adept.adept_set_wait_limit(1)
        out = attend(c, q, starts, lens)
        try:
            c.check()
            assert torch.equal(out, want)
        except adept.AdeptError as e:
            assert e.status == 5
    finally:
        adept.adept_set_wait_limit(0)
    assert torch.equal(attend(c, q, starts, lens), want)
    c.check()
