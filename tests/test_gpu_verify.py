"""adept_verify_drafts against its 64-bit statement: vocabularies of one to 2^20 tokens, ragged chunks, strided and unaligned rows, masks,
temperatures, drafts without probabilities, tests next to their border, drawn tokens' distribution, inputs out of range, streams and
graphs.  Whole numbers are equal; a log probability is off by at most LP."""
import math

import pytest
import torch

from serve_reference import verify

import paper_2601_03700_gb300 as adept

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    adept.load_library()


def lp_tol(vocab, value):
    """Half a step of the fp32 result, and the 32-bit sum of exponentials: a chain of at most vocab / 1024 + 1 additions and
    rescalings a thread of 2^-22 each and 13 joins of 2^-21, exponents rounded thrice by 2^-24 of up to log2(vocab) + 2 units on average."""
    return 2.0 ** -24 * abs(value) + 2.0 ** -22 * (vocab / 1024 + 1) + 13 * 2.0 ** -21 + 3 * 2.0 ** -24 * (math.log2(vocab) + 2)


def make(drafts, vocab, seed, spread=2.0, td=F32, dd=F32, near=0.5, pad=0, off=0):
    """Chunks of drafts[b] + 1 rows (None: no row), drafted from the draft's own distribution."""
    g = torch.Generator().manual_seed(seed)
    n = [0 if d is None else d + 1 for d in drafts]
    rows, start = sum(n), [0]
    for k in n:
        start.append(start[-1] + k)
    wide = lambda: torch.randn(rows, vocab + pad + off, generator=g)  # noqa: E731
    t = spread * wide()
    q = t + near * wide()
    t, q = t.to(td), q.to(dd)
    x = (q[:, off:off + vocab].float() - torch.empty(rows, vocab).exponential_(generator=g).log()).argmax(1)
    tokens = torch.cat([torch.zeros(1, dtype=torch.int64), x])[:rows].int() if rows else torch.zeros(0, dtype=torch.int32)
    return dict(target=t.cuda()[:, off:off + vocab], draft=q.cuda()[:, off:off + vocab], tokens=tokens, start=start, u=torch.rand(rows, generator=g))


def call(c, temp=None, stream=None, ws=None, err=None, draft=True):
    n_seq = len(c["start"]) - 1
    acc, nxt = (torch.full((n_seq,), -7, dtype=torch.int32, device="cuda") for _ in range(2))
    lp = torch.full((len(c["tokens"]),), 77.0, device="cuda")
    adept.adept_verify_drafts(c["target"], c["draft"] if draft else None, c["tokens"].int().cuda(), torch.tensor(c["start"], dtype=torch.int32).cuda(),
                              c["u"].float().cuda(), acc, nxt, logprob=lp, temperature=None if temp is None else torch.tensor(temp).float().cuda(),
                              workspace=ws, err=err, stream=stream)
    return acc, nxt, lp


def check(c, temp=None, draft=True):
    got = call(c, temp, draft=draft)
    acc, nxt, lp = verify(c["target"].cpu(), c["draft"].cpu() if draft else None, c["tokens"].tolist(), c["start"], c["u"], temp)
    assert got[0].tolist() == acc
    assert got[1].tolist() == nxt
    for r, v in enumerate(got[2].tolist()):
        if r not in lp:
            assert v == 77.0   # not written
        else:
            assert abs(v - lp[r]) <= lp_tol(c["target"].shape[1], lp[r]), (r, v, lp[r])
    for a, b in zip(got, call(c, temp, draft=draft)):
        assert torch.equal(a, b)
    return acc, nxt


@pytest.mark.parametrize("vocab", [1, 2, 3, 7, 31, 33, 255, 1000, 4097, 32000, 50257, 131073])
@pytest.mark.parametrize("td,dd", [(F32, F32), (F32, BF16), (BF16, F32), (BF16, BF16)])
def test_vocabularies_and_types(vocab, td, dd):
    c = make([4, 0, None, 1, 7, 2], vocab, vocab, td=td, dd=dd)
    check(c)
    check(c, draft=False)
    check(c, [0.0, 0.7, 1.0, 2.0, 0.0, 0.3])


@pytest.mark.parametrize("drafts", [[0], [12], [None, None, 3], [None], [700, 0, 3], [1] * 300])
def test_chunks(drafts):
    c = make(drafts, 50, 3, near=0.05)
    acc, _ = check(c)
    if drafts == [700, 0, 3]:   # (a chunk of more rows than a CTA has threads, all of it accepted)
        c["draft"] = c["target"]
        assert check(c)[0][0] == 700
        check(c, [0.0] * 3)
    check(c, draft=False)


@pytest.mark.parametrize("td", [F32, BF16])
@pytest.mark.parametrize("pad,off", [(1, 0), (3, 1), (5, 2), (8, 3), (0, 5), (16, 8)])
def test_strides_and_alignments(td, pad, off):
    check(make([3, 5, 0], 1237, pad * 16 + off, td=td, dd=td, pad=pad, off=off))


@pytest.mark.parametrize("low", [-math.inf, torch.finfo(F32).min, torch.finfo(BF16).min])
@pytest.mark.parametrize("td", [F32, BF16])
def test_masked_tokens(low, td):
    """Most of a row masked, its beginning and its end too; a draft that the target has masked does not hold."""
    if td is BF16 and low == torch.finfo(F32).min:
        low = -math.inf   # (fp32's lowest rounds to it)
    c = make([4, 4, 4, 4], 3001, 5, td=td, dd=td)
    keep = torch.rand(3001, generator=torch.Generator().manual_seed(6)) < 0.02
    keep[:700] = keep[2500:] = False
    for x in (c["target"], c["draft"]):
        x.masked_fill_(~keep.cuda(), low)
    ids = keep.nonzero()[:, 0]
    c["tokens"] = ids[torch.randint(len(ids), (len(c["tokens"]),), generator=torch.Generator().manual_seed(7))].int()
    acc, nxt = check(c)
    assert all(bool(keep[i]) for i in nxt)
    check(c, draft=False)
    check(c, [0.0, 0.5, 1.5, 1024.0])
    c["tokens"][1] = 0   # masked for the target: nothing makes it hold
    assert check(c, draft=False)[0][0] == 0


def test_a_row_of_the_lowest_value_alone_is_even():
    c = make([0, 0, 0, 0], 8, 8)
    c["target"].fill_(torch.finfo(F32).min)
    c["u"] = torch.tensor([0.0, 0.3, 0.6, 1 - 2.0 ** -24])
    assert check(c)[1] == [0, 2, 4, 7]


def test_numbers_at_their_ends():
    """u = 0 draws the first token that has a share of 2^-25, u next to 1 the last."""
    c = make([0, 0, 2, 2], 1000, 9, spread=8.0)
    c["u"] = torch.tensor([0.0, 1 - 2.0 ** -24, 0.0, 0.0, 0.0, 1 - 2.0 ** -24, 1 - 2.0 ** -24, 1 - 2.0 ** -24])
    acc, _ = check(c)
    assert acc[2] == 2   # u = 0 accepts what the target has any share of
    check(c, draft=False)


@pytest.mark.parametrize("seed", range(4))
def test_next_to_the_border(seed):
    """Numbers u within a few steps of p / q: 32-bit sums do not tell the sides apart."""
    B, V = 96, 5003
    c = make([3] * B, V, seed + 20, near=0.3)
    lt, ld = torch.log_softmax(c["target"].double(), 1).cpu(), torch.log_softmax(c["draft"].double(), 1).cpu()
    r = torch.arange(4 * B - 1)
    ratio = (lt[r, c["tokens"][1:].long()] - ld[r, c["tokens"][1:].long()]).exp()
    near = ratio.float() * (1 + torch.randint(-3, 4, ratio.shape, generator=torch.Generator().manual_seed(seed)) * 2.0 ** -23)
    use = ratio < 0.999
    c["u"][:-1][use] = near[use]
    acc, _ = check(c)
    assert 0 < sum(acc) < 3 * B
    # the same without probabilities of the drafts: u next to p itself
    ok = lt[r, c["tokens"][1:].long()].exp().float()
    c["u"][:-1] = torch.where(ok > 0, ok * (1 + torch.randint(-3, 4, ok.shape, generator=torch.Generator().manual_seed(seed)) * 2.0 ** -23), c["u"][:-1]).clamp(max=1 - 2.0 ** -24)
    check(c, draft=False)


def test_the_draft_is_the_target():
    """Every draft holds, however near u is to 1."""
    c = make([5] * 40, 2000, 30, near=0.0)
    c["u"][:120] = 1 - 2.0 ** -24
    assert check(c)[0] == [5] * 40


def test_nothing_left_to_draw_from():
    """p = q, and a draft that neither has: it does not hold, and max(p - q, 0) is empty: drawn from p."""
    c = make([1] * 8, 300, 31, near=0.0)
    for x in (c["target"], c["draft"]):
        x[:, 17] = -math.inf
    c["draft"] = c["target"].clone()
    c["tokens"][1::2] = 17
    acc, nxt = check(c)
    assert acc == [0] * 8 and 17 not in nxt
    # all but 2^-22 of p and q alike: below what is drawn from
    c["draft"][:, 0] += 2.0 ** -12 * (torch.rand(16, generator=torch.Generator().manual_seed(1)).cuda() - 0.5)
    check(c)


def test_equal_logits_greedy():
    c = make([2, 2], 4000, 32, td=BF16)
    c["target"].fill_(1.0)
    c["target"][:, 777] = c["target"][:, 778] = c["target"][:, 3999] = 2.0
    c["tokens"] = torch.tensor([0, 777, 777, 0, 778, 777], dtype=torch.int32)
    assert check(c, [0.0, 0.0])[0] == [2, 0]


def test_the_distribution_is_the_targets():
    """The first token that a chunk yields, over 40000 chunks of one draft: within 5 standard deviations of the target's share."""
    n, V = 40000, 6
    p, q = torch.tensor([0.4, 0.05, 0.25, 0.1, 0.15, 0.05]), torch.tensor([0.1, 0.3, 0.2, 0.1, 0.2, 0.1])
    g = torch.Generator().manual_seed(33)
    x = torch.multinomial(q, n, True, generator=g).int()
    tokens = torch.stack([torch.zeros(n, dtype=torch.int32), x], 1).reshape(-1)
    c = dict(target=p.log().cuda().expand(2 * n, V).contiguous(), draft=q.log().cuda().expand(2 * n, V).contiguous(), tokens=tokens,
             start=list(range(0, 2 * n + 1, 2)), u=torch.rand(2 * n, generator=g))
    for draft in (True, False):
        acc, nxt, _ = (t.cpu() for t in call(c, draft=draft))
        first = torch.where(acc > 0, x, nxt)
        share = torch.bincount(first.long(), minlength=V) / n
        assert ((share - p).abs() <= 5 * (p * (1 - p) / n).sqrt()).all(), share
        second = torch.bincount(nxt[acc > 0].long(), minlength=V)
        k = int((acc > 0).sum())
        assert ((second / k - p).abs() <= 5 * (p * (1 - p) / k).sqrt()).all()
    # at temperature 1/2 the target's shares are p^2
    acc, nxt, _ = (t.cpu() for t in call(c, [0.5] * n, draft=False))
    p2 = p * p / (p * p).sum()
    share = torch.bincount(torch.where(acc > 0, x, nxt).long(), minlength=V) / n
    assert ((share - p2).abs() <= 5 * (p2 * (1 - p2) / n).sqrt()).all()


BAD = {
    "nan": lambda c: c["target"][8].index_fill_(0, torch.tensor([99]).cuda(), math.nan),
    "inf": lambda c: c["target"][8].index_fill_(0, torch.tensor([98]).cuda(), math.inf),
    "nothing": lambda c: c["target"][8].fill_(-math.inf),
    "draft_nan": lambda c: c["draft"][8].index_fill_(0, torch.tensor([3]).cuda(), math.nan),
    "draft_nothing": lambda c: c["draft"][8].fill_(-math.inf),
    "token": lambda c: c["tokens"].index_fill_(0, torch.tensor([9]), 100),
    "token_negative": lambda c: c["tokens"].index_fill_(0, torch.tensor([9]), -1),
    "u_one": lambda c: c["u"].index_fill_(0, torch.tensor([8]), 1.0),
    "u_negative": lambda c: c["u"].index_fill_(0, torch.tensor([8]), -1e-9),
    "u_nan": lambda c: c["u"].index_fill_(0, torch.tensor([8]), math.nan),
    "rows": lambda c: c["start"].__setitem__(3, 21),
    "rows_negative": lambda c: c["start"].__setitem__(0, -1),
    "temp_negative": lambda c: c.__setitem__("temp", [1.0, -1.0, 1.0]),
    "temp_nan": lambda c: c.__setitem__("temp", [1.0, math.nan, 1.0]),
    "temp_small": lambda c: c.__setitem__("temp", [1.0, 2.0 ** -11, 1.0]),
    "temp_inf": lambda c: c.__setitem__("temp", [1.0, math.inf, 1.0]),
}


@pytest.mark.parametrize("bad", BAD)
def test_inputs_out_of_range(bad):
    """Sequence 1 (2 and 0 for the rows) is left out and flagged, the others are as without it; where it is decided before it meets the
    input, that has no part in it."""
    def fresh():
        c = make([6, 6, 5], 100, 40)
        c["draft"] = c["target"].clone()   # every draft holds
        return c
    good = [t.tolist() for t in call(fresh())]
    c = fresh()
    BAD[bad](c)
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    which = {"rows": 2, "rows_negative": 0}.get(bad, 1)
    got = [t.tolist() for t in call(c, c.get("temp"), err=err)]
    for b in range(3):
        assert (got[0][b], got[1][b]) == ((-1, -1) if b == which else (good[0][b], good[1][b]))
    with pytest.raises(adept.AdeptError) as ei:
        adept.adept_error_check(err)
    assert ei.value.status == 6
    adept.adept_error_check(err)
    if "temp" in bad or "rows" in bad:
        return
    # the draft before is refused: row 8 and what follows do not enter
    c = fresh()
    c["draft"][7, c["tokens"][8].long()] += 30.0
    c["u"][7] = 1 - 2.0 ** -24
    want = [t.tolist() for t in call(c)][:2]
    assert want[0][1] == 0
    BAD[bad](c)
    assert [t.tolist() for t in call(c, err=err)][:2] == want
    adept.adept_error_check(err)


def test_u_of_the_last_row_is_what_draws():
    c = make([2], 64, 41, near=0.0)
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    c["u"][2] = 1.5
    assert [t.tolist() for t in call(c, err=err)][:2] == [[-1], [-1]]
    assert [t.tolist()[0] for t in call(c, [0.0], err=err)][1] >= 0   # greedy: not looked at


def test_no_rows_and_no_sequences():
    c = make([None, None], 10, 42)
    assert [t.tolist() for t in call(c)][:2] == [[0, 0], [-1, -1]]
    c["start"] = [0]
    assert call(c)[0].numel() == 0


def test_the_most_sequences():
    n, g = 1 << 16, torch.Generator().manual_seed(44)
    c = dict(target=torch.randn(n, 4, generator=g).cuda(), draft=torch.zeros(n, 4).cuda(), tokens=torch.zeros(n, dtype=torch.int32),
             start=list(range(n + 1)), u=torch.rand(n, generator=g))
    w = c["target"].cpu().double().softmax(1)
    want = (w.cumsum(1) <= (c["u"].double() + 2.0 ** -25).unsqueeze(1) * w.sum(1, keepdim=True)).sum(1)
    acc, nxt, lp = (t.cpu() for t in call(c))
    assert not acc.any() and torch.equal(nxt.long(), want)
    assert (lp - w.gather(1, want.unsqueeze(1))[:, 0].log()).abs().max() <= lp_tol(4, 16)
    acc, nxt, _ = (t.cpu() for t in call(c, [0.0] * n))
    assert not acc.any() and torch.equal(nxt.long(), w.argmax(1))


def test_the_largest_vocabulary():
    c = make([2, 1], 1 << 20, 43)
    check(c)
    check(c, draft=False)
    check(c, [0.0, 0.9])


def test_rows_of_other_sequences_and_a_wider_product():
    """Chunks in a buffer that holds more: rows in front of the first and behind the last belong to nobody."""
    c = make([2, 3], 500, 44)
    want = [t.tolist() for t in call(c)]
    pad = lambda x, v: torch.cat([torch.full_like(x[:2], v), x, torch.full_like(x[:2], v)])  # noqa: E731
    d = dict(target=pad(c["target"], math.nan), draft=pad(c["draft"], math.nan), tokens=pad(c["tokens"], -5), start=[s + 2 for s in c["start"]],
             u=pad(c["u"], math.nan))
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = [t.tolist() for t in call(d, err=err)]
    adept.adept_error_check(err)
    assert got[:2] == want[:2] and got[2] == [77.0, 77.0] + want[2] + [77.0, 77.0]


def test_another_stream_and_two_at_once():
    cs = [make([4] * 20, 8000, 45 + i) for i in range(2)]
    want = [[t.clone() for t in call(c)] for c in cs]
    streams = [torch.cuda.Stream() for _ in cs]
    torch.cuda.synchronize()
    got = []
    for _ in range(3):
        for c, s in zip(cs, streams):
            with torch.cuda.stream(s):
                got.append(call(c))
    torch.cuda.synchronize()
    for k, g in enumerate(got):
        assert all(torch.equal(a, b) for a, b in zip(g, want[k % 2]))


def test_captured_and_replayed():
    c, d = make([4, 0, 3], 3000, 47), make([4, 0, 3], 3000, 48)
    dev = lambda c: [c["target"].clone(), c["draft"].clone(), c["tokens"].cuda(), torch.tensor(c["start"], dtype=torch.int32).cuda(), c["u"].cuda()]  # noqa: E731
    x, y = dev(c), dev(d)
    out = [torch.zeros(3, dtype=torch.int32, device="cuda") for _ in range(2)]
    ws = adept.verify_workspace(10)
    run = lambda: adept.adept_verify_drafts(*x, *out, workspace=ws)  # noqa: E731
    torch.cuda.synchronize()   # (what the side stream reads is made on this one)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        run()
    s.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run()
    for src, k in ((y, d), (dev(c), c)):
        for a, b in zip(x, src):
            a.copy_(b)
        g.replay()
        acc, nxt, _ = verify(k["target"].cpu(), k["draft"].cpu(), k["tokens"].tolist(), k["start"], k["u"])
        assert [o.tolist() for o in out] == [acc, nxt]


def test_a_larger_calls_workspace_serves_a_smaller_call():
    ws = adept.verify_workspace(700)
    for drafts, vocab in (([8] * 70, 200), ([3], 131072), ([0], 1)):
        c = make(drafts, vocab, 49)
        want = call(c)
        assert all(torch.equal(a, b) for a, b in zip(call(c, ws=ws), want))


@pytest.mark.parametrize("noise", [0.0, 1e-7, 1e-6, 1e-5])
@pytest.mark.parametrize("share", [0.5, 0.98])
def test_tokens_that_both_give_nearly_the_same(noise, share):
    """Most tokens with the same probability in target and draft, but for noise of the order of fp32's steps, the others exchanged in
    pairs (so that both sums are the same): which side a token is on hangs on the sums' last bits."""
    B, V = 48, 20002
    g = torch.Generator().manual_seed(60)
    t = (2.0 * torch.randn(B * 2, V, generator=g)).double()
    d = t.clone()
    n = int(V * (1 - share)) // 2 * 2
    d[:, 0:n:2], d[:, 1:n:2] = t[:, 1:n:2], t[:, 0:n:2]
    d[:, n:] += noise * torch.randn(B * 2, V - n, generator=g)
    t, d = t.float(), d.float()
    # drafts that the draft gives much more than the target
    x = (torch.log_softmax(d[0::2], 1) - torch.log_softmax(t[0::2], 1)).argmax(1)
    tokens = torch.stack([torch.zeros(B, dtype=torch.int64), x], 1).reshape(-1).int()
    c = dict(target=t.cuda(), draft=d.cuda(), tokens=tokens, start=list(range(0, 2 * B + 1, 2)), u=torch.rand(2 * B, generator=g))
    acc, _ = check(c)
    assert acc.count(0) > B // 2
    check(c, [0.6] * B)


@pytest.mark.parametrize("noise", [1e-7, 3e-7, 1e-6])
def test_few_tokens_that_both_give_nearly_the_same(noise):
    """Twelve tokens that hold half of both distributions, in the same ratio to each other but for that noise, before 400000 small ones
    whose borders lie 10^-6 apart: the twelve move the drawn token where they are counted on the wrong side."""
    B, V = 16, 400000
    g = torch.Generator().manual_seed(61)
    t = torch.randn(B * 2, V, generator=g).double()
    d = t.clone()
    d[:, 0::2], d[:, 1::2] = t[:, 1::2], t[:, 0::2]
    big = torch.logsumexp(t, 1, keepdim=True) - math.log(12) + 0.1 * torch.randn(B * 2, 12, generator=g).double()
    t[:, :12], d[:, :12] = big, big + noise * torch.randn(B * 2, 12, generator=g)
    t, d = t.float(), d.float()
    x = (torch.log_softmax(d[0::2], 1) - torch.log_softmax(t[0::2], 1)).argmax(1)
    tokens = torch.stack([torch.zeros(B, dtype=torch.int64), x], 1).reshape(-1).int()
    c = dict(target=t.cuda(), draft=d.cuda(), tokens=tokens, start=list(range(0, 2 * B + 1, 2)), u=torch.rand(2 * B, generator=g))
    acc, _ = check(c)
    assert acc.count(0) > B // 2


def test_masked_tokens_where_both_sums_are_the_same():
    """Target and draft with the same sum of weights, and thousands of tokens masked in both: those are next to each other in p and q, but
    nothing of either; vocabularies that end within a warp's tokens."""
    for V in (4099, 20011):
        g = torch.Generator().manual_seed(V)
        B = 24
        t = 2.0 * torch.randn(2 * B, V, generator=g)
        t[:, torch.rand(V, generator=g) < 0.6] = -math.inf
        keep = (t[0] > -math.inf).nonzero()[:, 0]
        keep = keep[:len(keep) // 2 * 2]
        d = t.clone()
        d[:, keep[0::2]], d[:, keep[1::2]] = t[:, keep[1::2]], t[:, keep[0::2]]
        x = (torch.log_softmax(d[0::2][:, keep], 1) - torch.log_softmax(t[0::2][:, keep], 1)).argmax(1)
        tokens = torch.stack([torch.zeros(B, dtype=torch.int64), keep[x]], 1).reshape(-1).int()
        c = dict(target=t.cuda(), draft=d.cuda(), tokens=tokens, start=list(range(0, 2 * B + 1, 2)), u=torch.rand(2 * B, generator=g))
        acc, nxt = check(c)
        assert acc.count(0) > B // 2 and all(i in keep for i in nxt)


@pytest.mark.parametrize("scale,offset", [(1.0, 1e4), (1.0, -1e4), (1.0, 3e6), (1e3, 0.0), (1e6, -1e7), (1e30, 0.0), (1e37, 0.0), (1e-4, 0.0), (1e-30, 0.0), (0.0, 7.0)])
def test_logits_of_any_size(scale, offset):
    """Far from zero, far apart, next to each other, all the same."""
    c = make([3, 2, 0, 4], 2003, 70)
    for k in ("target", "draft"):
        c[k] = (c[k] * scale + offset).contiguous()
    check(c)
    check(c, draft=False)
    check(c, [0.0, 2.0 ** -10, 1024.0, 0.5])
    check({**c, "target": c["target"].bfloat16(), "draft": c["draft"].bfloat16()})


@pytest.mark.parametrize("t", [2.0 ** -10, 0.01, 0.3, 3.0, 100.0, 1024.0])
def test_temperatures(t):
    c = make([4] * 12, 5000, 71)
    check(c, [t] * 12)
    check(c, [t] * 12, draft=False)


def test_drafts_that_were_never_likely():
    """Tokens with shares down to 2^-100 and below as drafts: tested by their logarithms."""
    c = make([3] * 16, 700, 72, spread=40.0, near=20.0)
    g = torch.Generator().manual_seed(73)
    c["tokens"] = torch.randint(700, c["tokens"].shape, generator=g).int()
    c["u"][::2] = 1e-30
    check(c)
    check(c, draft=False)


@pytest.mark.parametrize("t", [0.3, 0.7, 2.0])
def test_next_to_the_border_at_a_temperature(t):
    B, V = 64, 3001
    c = make([3] * B, V, 80, near=0.3, td=F32, dd=BF16)
    lt, ld = (torch.log_softmax(c[k].double() / torch.tensor(t).float().double().item(), 1).cpu() for k in ("target", "draft"))
    r = torch.arange(4 * B - 1)
    x = c["tokens"][1:].long()
    ratio = (lt[r, x] - ld[r, x]).exp()
    near = ratio.float() * (1 + torch.randint(-3, 4, ratio.shape, generator=torch.Generator().manual_seed(81)) * 2.0 ** -23)
    use = ratio < 0.999
    c["u"][:-1][use] = near[use]
    acc, _ = check(c, [float(torch.tensor(t).float())] * B)
    assert 0 < sum(acc) < 3 * B
