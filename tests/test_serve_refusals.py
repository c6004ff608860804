"""Refusals of the pages' calls and of the verification that need no GPU: checked before anything is enqueued."""
import ctypes

import pytest
import torch


@pytest.fixture(scope="module")
def lib():
    from paper_2601_03700_gb300 import build
    build.build()
    import paper_2601_03700_gb300 as adept
    return adept.load_library()


def pages(**kw):
    import paper_2601_03700_gb300 as adept
    c = dict(n_blocks=8, block_tokens=16, n_seq=3, max_blocks_per_seq=4, d_block_table=512, d_ref=1024, d_err=None)
    c.update(kw)
    return adept.AdeptKVPages(**c)


@pytest.mark.parametrize("bad", [dict(n_blocks=0), dict(block_tokens=0), dict(n_seq=0), dict(max_blocks_per_seq=0), dict(d_block_table=None),
                                 dict(d_ref=None), dict(d_block_table=514), dict(d_ref=1028), dict(d_err=2),
                                 dict(max_blocks_per_seq=2 ** 27, block_tokens=16)], ids=str)
def test_bad_pages(lib, bad):
    p = ctypes.byref(pages(**bad))
    assert lib.adept_kv_pages_workspace(p) == -1
    assert lib.adept_kv_fork(p, 64, 64, 64, 2 ** 40, None) == 1
    assert lib.adept_kv_reserve(p, 64, 64, 64, 64, 64, 64, 2 ** 40, None) == 1
    assert lib.adept_kv_compact(p, 64, 64, 64, 64, 2 ** 40, None) == 1
    assert lib.adept_last_error(None)
    assert lib.adept_kv_fork(None, 64, 64, 64, 2 ** 40, None) == 1
    assert lib.adept_kv_pages_workspace(None) == -1


def test_bad_calls_on_pages(lib):
    p = ctypes.byref(pages())
    n = lib.adept_kv_pages_workspace(p)
    assert n >= 4 * (8 + 3)
    for args in ((None, 64, 64, n), (64, None, 64, n), (64, 64, None, n), (64, 64, 72, n), (64, 64, 64, n - 1), (66, 64, 64, n), (64, 65, 64, n)):
        assert lib.adept_kv_fork(p, *args, None) == 1
    for at in range(5):
        for bad in (None, 66):
            args = [64] * 5
            args[at] = bad
            assert lib.adept_kv_reserve(p, *args, 64, n, None) == 1
    assert lib.adept_kv_reserve(p, *[64] * 5, 64, n - 1, None) == 1
    for args in ((None, 64, 64), (64, None, 64), (64, 64, None), (65, 64, 64), (64, 66, 64), (64, 64, 67)):
        assert lib.adept_kv_compact(p, *args, 64, n, None) == 1
    assert lib.adept_kv_compact(p, 64, 64, 64, None, n, None) == 1
    big = ctypes.byref(pages(n_seq=4097))
    assert lib.adept_kv_reserve(big, *[64] * 5, 64, 2 ** 40, None) == 3


def cache(**kw):
    import paper_2601_03700_gb300 as adept
    c = dict(kv_type=2, n_blocks=8, n_kv_heads=2, head_dim=64, block_tokens=16, n_seq=3, max_blocks_per_seq=4, d_k=4096,
             d_v=8192, d_k_exp=1024, d_v_exp=2048, d_block_table=512, d_err=None)
    c.update(kw)
    return adept.AdeptKVCache(**c)


def test_bad_copies(lib):
    import paper_2601_03700_gb300 as adept
    two = lambda **kw: (adept.AdeptKVCache * 2)(cache(), cache(**kw))  # noqa: E731
    assert lib.adept_kv_copy_blocks(None, 1, 1, 64, 64, None) == 1
    assert lib.adept_kv_copy_blocks(two(), 0, 1, 64, 64, None) == 1
    assert lib.adept_kv_copy_blocks(two(), 2, -1, 64, 64, None) == 1
    for args in ((None, 64), (64, None), (66, 64), (64, 65)):
        assert lib.adept_kv_copy_blocks(two(), 2, 1, *args, None) == 1
    for kw in (dict(kv_type=1), dict(n_blocks=9), dict(n_kv_heads=1), dict(head_dim=32), dict(block_tokens=8), dict(d_k=None), dict(d_v=8200)):
        assert lib.adept_kv_copy_blocks(two(**kw), 2, 1, 64, 64, None) == 1, kw
    assert lib.adept_kv_copy_blocks(two(n_seq=9, max_blocks_per_seq=1), 2, 0, None, None, None) == 0


GOOD = dict(n_seq=2, n_rows=5, vocab=100, td=0, target=64, ld_t=100, dd=1, draft=64, ld_d=100, tokens=64, start=64, temp=None, u=64, acc=64, nxt=64,
            lp=None, err=None, ws=64, nb=2 ** 40)


@pytest.mark.parametrize("bad", [dict(n_seq=-1), dict(n_rows=-1), dict(vocab=0), dict(vocab=2 ** 20 + 1), dict(td=2), dict(dd=-1), dict(target=None),
                                 dict(ld_t=99), dict(ld_d=99), dict(tokens=None), dict(start=None), dict(u=None), dict(acc=None), dict(nxt=None),
                                 dict(target=66), dict(draft=65), dict(tokens=66), dict(start=66), dict(temp=66), dict(u=66), dict(acc=66),
                                 dict(nxt=66), dict(lp=66), dict(err=66), dict(ws=None), dict(ws=72), dict(nb=0), dict(n_seq=2 ** 24 + 1),
                                 dict(n_rows=2 ** 24 + 1)], ids=str)
def test_bad_verifications(lib, bad):
    a = {**GOOD, **bad}
    assert lib.adept_verify_drafts(*a.values(), None) == (3 if max(a["n_seq"], a["n_rows"]) > 2 ** 24 else 1)


def test_as_many_sequences_as_a_verification_takes(lib):
    assert lib.adept_verify_drafts(*{**GOOD, "n_seq": 2 ** 16 + 1}.values(), None) == 3
    assert lib.adept_verify_drafts(*{**GOOD, "n_seq": 2 ** 16, "vocab": 0}.values(), None) == 1


def test_verification_workspaces(lib):
    assert lib.adept_verify_workspace(-1) == -1 and lib.adept_verify_workspace(2 ** 24 + 1) == -1
    sizes = [lib.adept_verify_workspace(n) for n in (0, 1, 2, 100, 5000, 2 ** 24)]
    assert sizes == sorted(sizes) and sizes[0] >= 0
    assert lib.adept_verify_drafts(*{**GOOD, "n_seq": 0}.values(), None) == 0   # nothing to do
    assert lib.adept_error_check(None, None) == 1 and lib.adept_error_check(66, None) == 1


def test_binding_checks_pages(lib):
    import paper_2601_03700_gb300 as adept
    p = adept.KVPages(8, 3, 4, device="cpu")
    assert p.block_table.shape == (3, 4) and p.ref.tolist() == [0] * 8 and p.ref.data_ptr() % 16 == p.state.data_ptr() % 16
    c = adept.KVCache(8, 2, 64, 3, 4, pages=p)
    assert c.block_table is p.block_table and c.err is p.err
    for args in ((9, 2, 64, 3, 4), (8, 2, 64, 2, 4), (8, 2, 64, 3, 5)):
        with pytest.raises(ValueError, match="pages"):
            adept.KVCache(*args, pages=p)
    with pytest.raises(ValueError, match="pages"):
        adept.KVCache(8, 2, 64, 3, 4, block_tokens=8, pages=p)
    n = torch.zeros(3, dtype=torch.int32)
    for bad in (n.long(), n[:2], torch.zeros(6, dtype=torch.int32)[::2]):
        with pytest.raises(ValueError):
            adept.adept_kv_fork(p, bad, n)
        with pytest.raises(ValueError):
            adept.adept_kv_fork(p, n, bad)
        for at in range(5):
            args = [n] * 5
            args[at] = bad
            with pytest.raises(ValueError):
                adept.adept_kv_reserve(p, *args)
    with pytest.raises(ValueError):
        adept.adept_kv_compact(p, n, n, n)
    with pytest.raises(ValueError, match="GPU"):
        adept.adept_kv_fork(p, n, n)
    with pytest.raises(ValueError, match="GPU"):
        adept.adept_kv_copy_blocks(c, n, n)
    with pytest.raises(ValueError):
        adept.adept_kv_copy_blocks(c, n, n[:2])
    with pytest.raises(ValueError):
        adept.KVLayers([])
    with pytest.raises(ValueError, match="GPU"):
        p.check()


def test_binding_checks_verifications(lib):
    import paper_2601_03700_gb300 as adept
    t, i, f = torch.zeros(5, 10), torch.zeros(5, dtype=torch.int32), torch.zeros(5)
    s, r = torch.tensor([0, 2, 5], dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    good = dict(target=t, draft=t, tokens=i, start=s, u=f, accepted=r, next_token=r, logprob=f, temperature=torch.ones(2), err=torch.zeros(1, dtype=torch.int32))
    for key, bad in (("target", t.half()), ("target", t[0]), ("draft", t[:, :9]), ("draft", t[:4]), ("draft", t.half()), ("target", torch.zeros(10, 5).T),
                     ("target", torch.zeros(1, 10).expand(5, 10)), ("tokens", i.long()), ("tokens", i[:4]), ("start", s.long()), ("start", s[None]),
                     ("u", f.double()), ("u", f[:4]), ("accepted", i), ("next_token", r.long()), ("logprob", f[:2]), ("temperature", torch.ones(3)),
                     ("err", r)):
        with pytest.raises(ValueError):
            adept.adept_verify_drafts(**{**good, key: bad})
    with pytest.raises(ValueError, match="GPU"):
        adept.adept_verify_drafts(**good)


def test_the_check_takes_the_word_on_its_stream():
    """As the other checks: cudaMemset works on the legacy stream, for which others do not wait."""
    import re
    from test_error_words import body
    calls = body("serve_ops.cu", "adept_error_check")
    assert "take_error_word(" in calls and not re.search(r"\bcudaMem(set|cpy)\s*\(", calls)
