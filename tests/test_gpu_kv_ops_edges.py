"""Calls at the edges of what the operators on a paged K/V cache take: sequences that hold nothing at all."""
import pytest
import torch

import paper_2601_03700_gb300 as adept
from test_gpu_kv_ops import _i32, _lib, make_q  # noqa: F401  (_lib: the module's fixture)

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
