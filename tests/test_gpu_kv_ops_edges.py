"""Calls at the edges of what the operators on a paged K/V cache take: sequences that hold nothing, or nothing that is there."""
import math

import pytest
import torch

import kv_reference as R
import paper_2601_03700_gb300 as adept
from test_gpu_kv_ops import _i32, _lib, assert_attention, attend, make_cache, make_q  # noqa: F401  (_lib: the module's fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16", "e4m3"])
@pytest.mark.parametrize("new", [[1], [300], [3, 0, 200], [1, 1]])
@pytest.mark.parametrize("heads,hk,dh", [(4, 2, 64), (8, 2, 128), (4, 4, 32)])
def test_no_positions_at_all(dtype, new, heads, hk, dh):
    """max_kv_len = 0: every row is zero, rows of no sequence stay."""
    c = adept.KVCache(4, hk, dh, len(new), 4, dtype=dtype)
    q, starts = make_q(dtype, new, heads, dh, 90, extra=2)
    out = torch.full(q.shape, -7.0, dtype=q.dtype, device="cuda")
    adept.adept_chunk_attention(c, q, _i32(starts), _i32([0] * len(new)), max(new), 0, out)
    c.check()
    assert (out[:-2] == 0).all() and (out[-2:] == -7).all()


# the CUDA-core kernel whole and split, the few-row kernel whole, over a cluster and split, the tcgen05 kernel whole and in parts
MISSING = [
    ("f32", 4, 2, 64, [3, 20, 5], [50, 30, 9]),
    ("f32", 4, 2, 64, [1, 2, 1], [1500, 700, 90]),
    ("bf16", 4, 4, 32, [2, 3, 1], [900, 40, 3]),
    ("bf16", 8, 2, 128, [4, 2, 1], [20, 30, 9]),
    ("bf16", 8, 2, 128, [1, 2, 1], [700, 500, 60]),
    ("e4m3", 8, 2, 128, [1, 2, 3], [700, 500, 60]),
    ("bf16", 32, 32, 128, [1, 1, 1], [4000, 3000, 60]),
    ("e4m3", 32, 32, 128, [5, 1, 2], [4000, 3000, 60]),
    ("bf16", 32, 2, 64, [300, 290, 280], [0, 0, 20]),
    ("bf16", 8, 2, 128, [200, 1, 40], [3000, 900, 10]),
    ("e4m3", 8, 2, 128, [200, 1, 40], [3000, 900, 10]),
    ("e4m3", 4, 4, 64, [300, 2, 1], [1000, 2000, 10]),
]


@pytest.mark.parametrize("dtype,heads,hk,dh,new,past", MISSING, ids=str)
@pytest.mark.parametrize("gone", [0, 1])
def test_rows_of_missing_blocks_alone_are_zero(dtype, heads, hk, dh, new, past, gone):
    """A sequence none of whose blocks is there: flagged, its rows zero, the others' what they are."""
    lens = [a + b for a, b in zip(new, past)]
    c = make_cache(dtype, hk, dh, lens, 91)
    q, starts = make_q(dtype, new, heads, dh, 92)
    c.block_table[gone] = -1
    out = attend(c, q, starts, lens)
    with pytest.raises(adept.AdeptError) as ei:
        c.check()
    assert ei.value.status == 6
    assert (out[starts[gone]:starts[gone + 1]] == 0).all()
    held = [0 if b == gone else n for b, n in enumerate(lens)]   # (without keys the reference's rows are zero too)
    assert_attention(c, q, starts, held, out)


@pytest.mark.parametrize("dtype,heads,hk,dh,new,past", [m for m in MISSING if m[0] != "e4m3"], ids=str)
def test_scores_of_minus_infinity_alone_give_zeros(dtype, heads, hk, dh, new, past):
    """K of one head at -infinity in a column where Q is positive: that head's rows are zero, the others' what they are."""
    lens = [a + b for a, b in zip(new, past)]
    c = make_cache(dtype, hk, dh, lens, 93)
    q, starts = make_q(dtype, new, heads, dh, 94)
    q = q.clone()
    q[..., 7] = q[..., 7].abs() + 1
    clean = attend(c, q, starts, lens)
    c.k[:, 0, :, 7] = -math.inf
    out = attend(c, q, starts, lens)
    c.check()
    g = heads // hk
    assert (out[:, :g] == 0).all() and torch.equal(out[:, g:], clean[:, g:])


def test_a_flag_set_right_behind_a_check_is_reported():
    """Flags on a side stream, each right behind the check of the one before: every check reports its own."""
    c = adept.KVCache(2, 1, 64, 1, 2)
    c.block_table.zero_()
    x = torch.ones(1, 1, 64, device="cuda")
    seq, pos = _i32([0]), _i32([99])
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(2000):
        adept.adept_kv_append(c, x, x, seq, pos, stream=side)
        with pytest.raises(adept.AdeptError):
            c.check(side)
    c.check(side)
    assert c.err.item() == 0


def test_a_check_takes_what_it_reports_only():
    """Bits that other streams set are reported by this check or the next, and cleared by that."""
    c = adept.KVCache(2, 1, 64, 1, 2)
    c.err.fill_(1 << 30)   # (a bit no kernel sets)
    with pytest.raises(adept.AdeptError, match="0x40000000"):
        c.check()
    c.check()
    c.check(torch.cuda.Stream())


def test_a_check_in_capture_is_refused():
    c = adept.KVCache(2, 1, 64, 1, 2)
    x = torch.zeros(1, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        x += 1
        with pytest.raises(adept.AdeptError, match="captured") as ei:
            c.check()
    assert ei.value.status == 1
    graph.replay()
    assert x.item() == 1   # the capture is whole
    c.check()


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("heads,hk", [(128, 1), (160, 1), (258, 2), (21, 7)])
@pytest.mark.parametrize("new,past", [([1], [300]), ([40, 3], [100, 20])])
def test_many_query_heads_on_a_head(dtype, heads, hk, new, past):
    lens = [a + b for a, b in zip(new, past)]
    c = make_cache(dtype, hk, 64, lens, 97)
    q, starts = make_q(dtype, new, heads, 64, 98)
    out = attend(c, q, starts, lens)
    c.check()
    assert_attention(c, q, starts, lens, out)


@pytest.mark.parametrize("dtype,heads,hk,dh,new,past", MISSING, ids=str)
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_a_query_that_is_not_finite_reaches_no_other_row(dtype, heads, hk, dh, new, past, bad):
    lens = [a + b for a, b in zip(new, past)]
    c = make_cache(dtype, hk, dh, lens, 99)
    q, starts = make_q(dtype, new, heads, dh, 100)
    q = q.clone()
    clean = attend(c, q, starts, lens)
    row, head = starts[-1] // 2, heads - 1
    q[row, head, 3] = bad
    out = attend(c, q, starts, lens)
    c.check()
    assert not torch.isfinite(out[row, head]).any()
    out[row, head] = clean[row, head]
    assert torch.equal(out, clean)


def test_few_and_many_tokens_over_8_bit_entries_on_several_streams():
    """The form whose launches run side by side (widening, few rows, longer chunks), itself on three streams at once, with a
    workspace each, and replayed from two graphs."""
    new, past = [1, 200, 3, 0, 17], [4600, 300, 90, 8, 0]
    lens = [a + b for a, b in zip(new, past)]
    c = make_cache("e4m3", 4, 128, lens, 101)
    q, starts = make_q("bf16", new, 16, 128, 102)
    want = attend(c, q, starts, lens)
    assert_attention(c, q, starts, lens, want)
    at, n = _i32(starts), _i32(lens)
    streams = [torch.cuda.Stream() for _ in range(3)]
    sets = [(torch.empty_like(want), c.attention_workspace(16, q.shape[0], max(new), max(lens))) for _ in streams]
    torch.cuda.synchronize()
    for _ in range(20):
        for s, (out, ws) in zip(streams, sets):
            with torch.cuda.stream(s):
                out.fill_(-7)
                adept.adept_chunk_attention(c, q, at, n, max(new), max(lens), out, ws)
    torch.cuda.synchronize()
    assert all(torch.equal(out, want) for out, _ in sets)
    graphs = []
    for out, ws in sets[:2]:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            adept.adept_chunk_attention(c, q, at, n, max(new), max(lens), out, ws)
    for _ in range(10):
        for g, s, (out, _) in zip(graphs, streams, sets):
            with torch.cuda.stream(s):
                out.fill_(-7)
                g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(out, want) for out, _ in sets)
    c.check()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "e4m3"])
@pytest.mark.parametrize("heads,hk,dh,new,past", [(8, 2, 128, [3, 1], [700, 60]), (8, 2, 128, [200, 40], [700, 60]),
                                                  (4, 4, 64, [150, 2], [90, 600])])
@pytest.mark.parametrize("e", [100, -100])
def test_values_far_from_one(dtype, heads, hk, dh, new, past, e):
    """V around 2^100 and 2^-100, the bounds within which nothing overflows or loses bits."""
    lens = [a + b for a, b in zip(new, past)]
    c = make_cache(dtype, hk, dh, lens, 103)
    if dtype == "e4m3":
        c.v_exp.copy_((c.v_exp.int() + e).clamp(1, 254).to(torch.uint8))
    else:
        c.v.mul_(2.0 ** e)
    q, starts = make_q(dtype, new, heads, dh, 104)
    out = attend(c, q, starts, lens)
    c.check()
    want, tol = R.attention(c, q, starts, lens)
    assert torch.isfinite(out).all() and ((out.double() - want).abs() <= tol).all()


@pytest.mark.parametrize("dtype,heads,hk,dh,new,past", MISSING, ids=str)
def test_bounds_far_above_the_lengths(dtype, heads, hk, dh, new, past):
    """max_q_len up to the largest int: the same rows (another kernel may take them)."""
    lens = [a + b for a, b in zip(new, past)]
    c = make_cache(dtype, hk, dh, lens, 105)
    q, starts = make_q(dtype, new, heads, dh, 106)
    for max_q in (2 ** 31 - 1, 2 ** 31 - 3, 2 ** 20):
        out = torch.full_like(q, -7.0)
        adept.adept_chunk_attention(c, q, _i32(starts), _i32(lens), max_q, 16 * c.block_table.shape[1], out)
        c.check()
        assert_attention(c, q, starts, lens, out)
