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
