"""The operators on a paged cache together, as a server uses them: rounds in which rows grow, a chunk of drafts is written and attended, its
drafts are verified, rows are cut back to what was accepted, branch, drop and take others' places, and the pool is compacted.  What the
cache holds of every row is compared with the row's own history, the attention and the verification with their 64-bit statements."""
import random

import pytest
import torch

from kv_reference import attention
from serve_reference import Pool, verify

import paper_2601_03700_gb300 as adept

pytestmark = pytest.mark.gpu

HK, H, DH, V, LAYERS, BT = 2, 4, 64, 61, 2, 16


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    adept.load_library()


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rounds_of_drafts(dtype):
    rng, B, cols, blocks = random.Random(3), 6, 12, 60
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    g = torch.Generator(device="cuda").manual_seed(4)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    ek, ev, eq = rnd(LAYERS, V, HK, DH), rnd(LAYERS, V, HK, DH), rnd(V, H, DH)
    place, w_out = rnd(cols * BT, HK, DH), rnd(H * DH, V) / 16   # (logits of the order of 1)
    key = lambda l, tok, pos: ((ek[l][tok] + place[pos]).to(dt), (ev[l][tok] - place[pos]).to(dt))  # noqa: E731

    pages, plain = adept.KVPages(blocks, B, cols, block_tokens=BT), Pool(blocks, B, cols, BT)
    layers = adept.KVLayers([adept.KVCache(blocks, HK, DH, B, cols, dtype=dtype, pages=pages) for _ in range(LAYERS)])
    out3 = [i32([0] * B) for _ in range(3)]

    def reserve(lens, want):
        adept.adept_kv_reserve(pages, i32(lens), i32(want), *out3)
        exp = plain.reserve(lens, want)
        assert [o.tolist() for o in out3] == [list(e) for e in exp]
        adept.adept_kv_copy_blocks(layers, out3[1], out3[2])
        return exp[0]

    def write(chunks, lens):
        seq = [b for b, c in enumerate(chunks) for _ in c]
        pos = [lens[b] + j for b, c in enumerate(chunks) for j in range(len(c))]
        tok = torch.tensor([t for c in chunks for t in c], device="cuda")
        for l, cache in enumerate(layers.caches):
            k, v = key(l, tok, torch.tensor(pos, device="cuda"))
            adept.adept_kv_append(cache, k.contiguous(), v.contiguous(), i32(seq), i32(pos))

    def held(history):
        """Every row's entries are those of its history."""
        for b, h in enumerate(history):
            if not h:
                continue
            n, tok = len(h), torch.tensor(h, device="cuda")
            for l, cache in enumerate(layers.caches):
                k, v = (torch.empty(n, HK, DH, dtype=dt, device="cuda") for _ in range(2))
                adept.adept_kv_gather(cache, i32([b] * n), i32(list(range(n))), k, v)
                ek_, ev_ = key(l, tok, torch.arange(n, device="cuda"))
                assert torch.equal(k, ek_) and torch.equal(v, ev_), (b, l)

    # rows 0 and 1 start with a prompt; a row's last token is not in the cache yet
    history = [[rng.randrange(V) for _ in range(37)], [rng.randrange(V) for _ in range(5)]] + [[] for _ in range(B - 2)]
    last = [rng.randrange(V) for _ in range(B)]
    got = reserve([0] * B, [len(h) for h in history])
    assert got == [len(h) for h in history]
    write(history, [0] * B)
    temp = [1.0, 0.0, 0.7, 1.0, 2.0, 1.0]
    total = 0
    for step in range(14):
        if step % 3 == 0:   # branches, dropped rows, places changed
            source = [0, 1, 0, 1, 0, -1] if step == 0 else [rng.choice([b, b, rng.randrange(B), -1]) if b > 1 else b for b in range(B)]
            history = [list(history[s]) if s >= 0 else [] for s in source]
            last = [last[s] if s >= 0 else last[b] for b, s in enumerate(source)]
            adept.adept_kv_fork(pages, i32(source), i32([len(h) for h in history]))
            plain.fork(source, [len(h) for h in history])
        lens = [len(h) for h in history]
        drafts = [[rng.randrange(V) for _ in range(rng.randint(0, 4))] if n and n + 5 < cols * BT else None for n in lens]
        want = [n if d is None else n + 1 + len(d) for n, d in zip(lens, drafts)]
        got = reserve(lens, want)
        chunks = [[] if d is None or g_ < w else [t] + d for d, t, g_, w in zip(drafts, last, got, want)]
        write(chunks, lens)
        now = [n + len(c) for n, c in zip(lens, chunks)]
        held([h + c for h, c in zip(history, chunks)])
        start = [0]
        for c in chunks:
            start.append(start[-1] + len(c))
        toks = [t for c in chunks for t in c]
        q = eq[torch.tensor(toks, device="cuda")].to(dt).contiguous()
        att = torch.empty_like(q)
        adept.adept_chunk_attention(layers.caches[-1], q, i32(start), i32(now), max(map(len, chunks)), max(now), att)
        exp, tol = attention(layers.caches[-1], q, start, now)
        assert ((att.double() - exp).abs() <= tol).all()
        logits = (att.float().reshape(len(toks), H * DH) @ w_out).contiguous()
        # the drafts' own distribution: even
        u = torch.rand(len(toks), generator=g, device="cuda")
        acc, nxt = i32([0] * B), i32([0] * B)
        adept.adept_verify_drafts(logits, torch.zeros_like(logits), i32(toks), i32(start), u, acc, nxt, temperature=torch.tensor(temp, device="cuda"),
                                  err=pages.err)
        acc, nxt = acc.tolist(), nxt.tolist()
        assert (acc, nxt) == verify(logits.cpu(), torch.zeros(logits.shape), toks, start, u.cpu(), temp)[:2]
        total += sum(acc)
        history = [h + c[:1 + a] for h, c, a in zip(history, chunks, acc)]
        last = [n if c else t for n, c, t in zip(nxt, chunks, last)]
        adept.adept_kv_fork(pages, i32(list(range(B))), i32([len(h) for h in history]))   # what was not accepted goes
        plain.fork(list(range(B)), [len(h) for h in history])
        if step % 4 == 3:
            used, s, d = i32([0]), i32([0] * (blocks // 2)), i32([0] * (blocks // 2))
            adept.adept_kv_compact(pages, used, s, d)
            u_, s_, d_ = plain.compact()
            assert (used.tolist(), s.tolist(), d.tolist()) == ([u_], s_, d_)
            adept.adept_kv_copy_blocks(layers, s, d)
        assert pages.block_table.tolist() == plain.table and pages.ref.tolist() == plain.ref
        held(history)
        pages.check()
    assert total > 0


def test_a_round_captured_and_replayed():
    """A whole round whose lengths never leave the device (rows grown, chunk written and attended, verified, cut back), captured once and
    replayed: the same bits as calls one by one."""
    B, D, cols, blocks = 4, 3, 10, 48
    n = B * (D + 1)
    g = torch.Generator(device="cuda").manual_seed(9)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    emb, w_out = rnd(V, (H + 2 * HK), DH).bfloat16(), rnd(H * DH, V) / 16
    drafts = [torch.randint(V, (B, D), generator=g, device="cuda", dtype=torch.int32) for _ in range(8)]
    us = [torch.rand(n, generator=g, device="cuda") for _ in range(8)]

    class State:
        def __init__(self):
            self.pages = adept.KVPages(blocks, B, cols, block_tokens=BT)
            self.cache = adept.KVCache(blocks, HK, DH, B, cols, pages=self.pages)
            self.layers = adept.KVLayers([self.cache])
            self.len, self.tok = i32([0] * B), i32([[7, 0, 0, 0]] * B)
            self.own, self.start = i32(list(range(B))), i32([b * (D + 1) for b in range(B + 1)])
            self.seq = self.own.repeat_interleave(D + 1).contiguous()
            self.got, self.src, self.dst, self.acc, self.nxt = (i32([0] * B) for _ in range(5))
            self.draft, self.u = torch.zeros_like(drafts[0]), torch.zeros_like(us[0])
            self.q, self.att = (torch.zeros(n, H, DH, dtype=torch.bfloat16, device="cuda") for _ in range(2))
            self.ws = [self.pages.workspace(), self.cache.attention_workspace(H, n, D + 1, cols * BT), adept.verify_workspace(n)]
            self.logits = torch.zeros(n, V, device="cuda")

        def round(self):
            want = self.len + (D + 1)
            adept.adept_kv_reserve(self.pages, self.len, want, self.got, self.src, self.dst, workspace=self.ws[0])
            adept.adept_kv_copy_blocks(self.layers, self.src, self.dst)
            self.tok[:, 1:] = self.draft
            x = emb[self.tok.view(-1).long()]
            pos = (self.len[:, None] + torch.arange(D + 1, device="cuda", dtype=torch.int32)).view(-1).contiguous()
            adept.adept_kv_append(self.cache, x[:, H:H + HK], x[:, H + HK:], self.seq, pos)
            self.q.copy_(x[:, :H])
            adept.adept_chunk_attention(self.cache, self.q, self.start, want, D + 1, cols * BT, self.att, self.ws[1])
            torch.matmul(self.att.float().view(n, -1), w_out, out=self.logits)
            adept.adept_verify_drafts(self.logits, None, self.tok.view(-1), self.start, self.u, self.acc, self.nxt, workspace=self.ws[2],
                                      err=self.pages.err)
            self.len += 1 + self.acc
            self.tok[:, 0] = self.nxt
            adept.adept_kv_fork(self.pages, self.own, self.len, workspace=self.ws[0])

        def all(self):
            return [self.pages.state, self.cache.k, self.cache.v, self.len, self.tok, self.acc, self.nxt, self.logits]

    one, two = State(), State()
    torch.cuda.synchronize()   # (what the side stream reads is made on this one)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        State().round()
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        two.round()
    for d, u in zip(drafts, us):
        for st in (one, two):
            st.draft.copy_(d)
            st.u.copy_(u)
        one.round()
        graph.replay()
        assert all(torch.equal(x, y) for x, y in zip(one.all(), two.all()))
    one.pages.check()
    two.pages.check()
    assert int(one.len.max()) > 8 and int((one.pages.block_table >= 0).sum()) == sum(-(-int(x) // BT) for x in one.len)
