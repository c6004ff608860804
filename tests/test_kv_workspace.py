"""The chunk attention's workspace: a model takes it once, for its largest batch, pass and context, so no smaller call may need
more; and what 8-bit entries are widened into is never more than the pool in bf16.  (The sizes are host arithmetic.)"""
import ctypes
import itertools

import pytest


@pytest.fixture(scope="module")
def lib():
    from paper_2601_03700_gb300 import build
    build.build()
    import paper_2601_03700_gb300 as adept
    return adept.load_library()


def size(lib, kv_type, n_blocks, hk, dh, heads, n_seq, width, max_q, max_kv):
    import paper_2601_03700_gb300 as adept
    c = adept.AdeptKVCache(kv_type=kv_type, n_blocks=n_blocks, n_kv_heads=hk, head_dim=dh, block_tokens=16, n_seq=n_seq,
                           max_blocks_per_seq=width, d_k=4096, d_v=8192, d_k_exp=1024, d_v_exp=2048, d_block_table=512)
    n = lib.adept_chunk_attention_workspace(ctypes.byref(c), heads, max_q, max_q, max_kv)
    assert n >= 0
    return n


POOLS = [  # pool blocks, K/V heads, head_dim, heads, table rows, table columns
    (8192, 32, 64, 32, 512, 8192),        # a small pool under many long rows: 2^26 positions in the table
    (16384, 32, 128, 32, 64, 2048),
    (3000, 8, 128, 32, 64, 2048),
    (40, 2, 128, 8, 3, 40),
    (40, 2, 128, 8, 1, 64),
    (8192, 4, 64, 4, 1, 512),             # a large pool under one short row
    (8192, 1, 64, 96, 16, 512),
]


@pytest.mark.parametrize("kv_type", [0, 1, 2])
@pytest.mark.parametrize("pool", POOLS, ids=str)
def test_no_smaller_call_needs_more(lib, kv_type, pool):
    n_blocks, hk, dh, heads, n_seq, width = pool
    cap, most_q = 16 * width, 4096
    most = size(lib, kv_type, n_blocks, hk, dh, heads, n_seq, width, most_q, cap)
    up_to = lambda n: sorted({1, 2, 3, 15, 16, 17, 63, 128, 200, 256, 257, 1000, 4096, n // 3, n // 2, n - 1, n} & set(range(1, n + 1)))  # noqa: E731
    for b, q, kv in itertools.product(up_to(n_seq), up_to(most_q), up_to(cap)):
        assert size(lib, kv_type, n_blocks, hk, dh, heads, b, width, q, kv) <= most, (b, q, kv)


@pytest.mark.parametrize("pool", POOLS, ids=str)
def test_widened_entries_are_at_most_the_pool(lib, pool):
    n_blocks, hk, dh, heads, n_seq, width = pool
    at = (hk, dh, heads, n_seq, width, 4096, 16 * width)
    plain, codes = size(lib, 1, n_blocks, *at), size(lib, 2, n_blocks, *at)
    # beside the partials of the longer chunks' kernel: K and V in bf16, and the few-row kernel's own partials
    assert codes <= 2 * plain + 256 + 2 * 2 * n_blocks * hk * 16 * dh
