"""Refusals of the operators on a caller-owned paged K/V cache that need no GPU: checked before anything is enqueued."""
import ctypes

import pytest
import torch


@pytest.fixture(scope="module")
def lib():
    from paper_2601_03700_gb300 import build
    build.build()
    import paper_2601_03700_gb300 as adept
    return adept.load_library()


def cache(**kw):
    import paper_2601_03700_gb300 as adept
    c = dict(kv_type=2, n_blocks=8, n_kv_heads=2, head_dim=64, block_tokens=16, n_seq=3, max_blocks_per_seq=4, d_k=4096,
             d_v=8192, d_k_exp=1024, d_v_exp=2048, d_block_table=512, d_err=None)
    c.update(kw)
    return adept.AdeptKVCache(**c)


BAD_CACHES = [dict(kv_type=3), dict(kv_type=-1), dict(head_dim=48), dict(head_dim=0), dict(n_blocks=0), dict(n_kv_heads=0),
              dict(block_tokens=0), dict(n_seq=0), dict(max_blocks_per_seq=0), dict(d_k=None), dict(d_v=None),
              dict(d_block_table=None), dict(d_k_exp=None), dict(d_v_exp=None), dict(d_k=4104), dict(d_v=8200),
              dict(d_k_exp=1032), dict(max_blocks_per_seq=2 ** 30, block_tokens=16), dict(n_kv_heads=2 ** 20)]


@pytest.mark.parametrize("bad", BAD_CACHES, ids=str)
def test_bad_caches(lib, bad):
    c = ctypes.byref(cache(**bad))
    assert lib.adept_kv_append(c, 1, 1, 64, 128, 64, 128, 64, 64, None) == 1
    assert lib.adept_kv_gather(c, 1, 1, 64, 128, 64, 128, 64, 64, None) == 1
    assert lib.adept_chunk_attention(c, 4, 1, 64, 256, 64, 64, None, 1, 16, 64, 256, None, 0, None) == 1
    assert lib.adept_chunk_attention_workspace(c, 4, 1, 1, 16) == -1
    assert lib.adept_last_error(None)
    assert lib.adept_kv_append(None, 1, 1, 64, 128, 64, 128, 64, 64, None) == 1
    assert lib.adept_kv_check(None, None) == 1


@pytest.mark.parametrize("args", [(-1, 1, 64, 128, 64, 128, 64, 64), (1, 2, 64, 128, 64, 128, 64, 64),
                                  (1, 1, None, 128, 64, 128, 64, 64), (1, 1, 64, 128, None, 128, 64, 64),
                                  (1, 1, 64, 128, 64, 128, None, 64), (1, 1, 64, 128, 64, 128, 64, None),
                                  (1, 1, 64, 127, 64, 128, 64, 64), (1, 1, 64, 128, 64, 0, 64, 64),
                                  (1, 1, 65, 128, 64, 128, 64, 64), (1, 0, 66, 128, 64, 128, 64, 64)])
def test_bad_rows(lib, args):
    c = ctypes.byref(cache())
    assert lib.adept_kv_append(c, *args, None) == 1
    assert lib.adept_kv_gather(c, *args, None) == 1


def test_no_rows_are_no_work(lib):
    c = ctypes.byref(cache())
    assert lib.adept_kv_append(c, 0, 1, None, 0, None, 0, None, None, None) == 0
    assert lib.adept_kv_gather(c, 0, 1, None, 0, None, 0, None, None, None) == 0
    assert lib.adept_chunk_attention(c, 4, 0, None, 0, None, None, None, 5, 16, None, 0, None, 0, None) == 0
    assert lib.adept_chunk_attention(c, 4, 3, None, 0, None, None, None, 0, 16, None, 0, None, 0, None) == 0
    assert lib.adept_kv_check(c, None) == 1   # no error word


@pytest.mark.parametrize("kw", [dict(n_heads=3), dict(n_heads=0), dict(n_heads=-2), dict(n_rows=-1), dict(max_q=-1),
                                dict(max_kv=-1), dict(max_kv=65), dict(q=None), dict(start=None), dict(kv_len=None),
                                dict(ld_q=255), dict(out=None), dict(ld_out=8), dict(q=65), dict(out=63), dict(ws=None),
                                dict(ws=72), dict(nb=-1)], ids=str)
def test_bad_attention_calls(lib, kw):
    a = dict(n_heads=4, n_rows=40, q=64, ld_q=256, start=64, kv_len=64, row_pos=None, max_q=40, max_kv=64, out=64, ld_out=256,
             ws=128, nb=None)
    a.update(kw)
    c = ctypes.byref(cache(kv_type=0, n_seq=1))
    need = lib.adept_chunk_attention_workspace(c, 4, 40, 40, 64)
    assert need == 0   # (one unit of keys: not split)
    c = ctypes.byref(cache(kv_type=0, n_seq=1, max_blocks_per_seq=4, block_tokens=64))
    if "max_kv" not in kw:
        a["max_kv"] = 256
    elif kw["max_kv"] == 65:
        a["max_kv"] = 257
    need = lib.adept_chunk_attention_workspace(c, 4, 40, 40, 256)
    assert need > 0
    nb = need + kw["nb"] if "nb" in kw else need
    assert lib.adept_chunk_attention(c, a["n_heads"], a["n_rows"], a["q"], a["ld_q"], a["start"], a["kv_len"], a["row_pos"],
                                     a["max_q"], a["max_kv"], a["out"], a["ld_out"], a["ws"], nb, None) == 1


def test_capacity(lib):
    assert lib.adept_chunk_attention(ctypes.byref(cache()), 64, 2 ** 25, 64, 64 * 64, 64, 64, None, 5, 16, 64, 64 * 64, None, 0,
                                     None) == 3


def test_capacity_of_sequences(lib):
    """More tiles than a grid has CTAs."""
    for n_seq, heads in ((2 ** 25, 64), (2 ** 16, 2 ** 15)):
        c = ctypes.byref(cache(n_seq=n_seq))
        assert lib.adept_chunk_attention_workspace(c, heads, 40, 5, 16) == -1
        assert lib.adept_chunk_attention(c, heads, 40, 64, heads * 64, 64, 64, None, 5, 16, 64, heads * 64, 128, 2 ** 40, None) == 3


@pytest.mark.parametrize("at", [dict(start=66), dict(kv_len=65), dict(row_pos=67), dict(table=514), dict(err=2)], ids=str)
def test_misaligned_lengths_and_tables(lib, at):
    a = dict(start=64, kv_len=64, row_pos=None, table=512, err=None)
    a.update(at)
    c = ctypes.byref(cache(kv_type=0, d_block_table=a["table"], d_err=a["err"]))
    assert lib.adept_chunk_attention(c, 4, 40, 64, 256, a["start"], a["kv_len"], a["row_pos"], 40, 64, 64, 256, None, 0, None) == 1


@pytest.mark.parametrize("seq,pos", [(65, 64), (64, 66)])
def test_misaligned_places(lib, seq, pos):
    c = ctypes.byref(cache())
    assert lib.adept_kv_append(c, 1, 1, 64, 128, 64, 128, seq, pos, None) == 1
    assert lib.adept_kv_gather(c, 1, 1, 64, 128, 64, 128, seq, pos, None) == 1


def test_binding_checks_tensors(lib):
    import paper_2601_03700_gb300 as adept
    with pytest.raises(ValueError):
        adept.KVCache(1, 1, 64, 1, 1, dtype="fp4", device="cpu")
    c = adept.KVCache(2, 2, 64, 1, 2, dtype="e4m3", device="cpu")
    k = torch.zeros(3, 2, 64)
    i = torch.zeros(3, dtype=torch.int32)
    good = (k, k.clone(), i, i)
    for at, bad in ((0, k[:2]), (0, k.half()), (0, k[:, :1]), (0, torch.zeros(3, 64, 2).transpose(1, 2)), (1, k.bfloat16()),
                    (2, i.long()), (2, i[:2]), (3, torch.zeros(6, dtype=torch.int32)[::2]), (0, torch.zeros(1, 2, 64).expand(3, 2, 64))):
        args = list(good)
        args[at] = bad
        with pytest.raises(ValueError):
            adept.adept_kv_append(c, *args)
    with pytest.raises(ValueError, match="GPU"):
        adept.adept_kv_append(c, *good)
    q = torch.zeros(3, 4, 64, dtype=torch.bfloat16)
    s, n = torch.tensor([0, 3], dtype=torch.int32), torch.tensor([3], dtype=torch.int32)
    ws = torch.zeros(16, dtype=torch.uint8)
    for bad in (dict(q=q.float()), dict(out=q.float()), dict(out=q[:2]), dict(s=s[:1]), dict(n=s), dict(row_pos=n)):
        with pytest.raises(ValueError):
            adept.adept_chunk_attention(c, bad.get("q", q), bad.get("s", s), bad.get("n", n), 3, 3, bad.get("out", q.clone()), ws,
                                        row_pos=bad.get("row_pos"))
    with pytest.raises(ValueError, match="overlap"):
        adept.adept_chunk_attention(c, q, s, n, 3, 3, q, ws)


def test_models_that_an_8_bit_cache_does_not_fit(lib):
    import paper_2601_03700_gb300 as adept
    import synth
    for kw, word in ((dict(dtype="f32"), "8-bit"), (dict(dtype="bf16", kv_block_tokens=8), "8-bit"),
                     (dict(dtype="bf16", family=synth.BERT, max_pos=128, n_classes=2), "8-bit")):
        cfg = synth.tiny_config(**kw)
        cfg.kv_type = "e4m3"
        with pytest.raises(adept.AdeptError, match=word) as ei:
            adept.adept_model_load(cfg, {})
        assert ei.value.status == 1
    cfg = synth.tiny_config(dtype="bf16")
    cfg.kv_type = 1
    with pytest.raises(adept.AdeptError, match="kv_type"):
        adept.adept_model_load(cfg, {})
