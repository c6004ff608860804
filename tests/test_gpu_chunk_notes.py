"""Many segments a CTA on the tcgen05 chunk kernel, some with a NaN or infinite V entry in the middle of a long chunk, most of them
of one sub-tile only: each chunk shows its own entry, in its own rows and column, and nobody else's."""
import math

import pytest
import torch

from test_gpu_kv_ops import _lib, attend, make_cache, make_q  # noqa: F401  (_lib: the module's fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("heads,hk,dh", [(1, 1, 128), (2, 1, 64)])
def test_non_finite_entries_among_many_segments(dtype, heads, hk, dh):
    n = 1200
    new = [200 if b % 9 == 4 else 40 + b % 11 for b in range(n)]
    past = [7 * b % 90 for b in range(n)]
    lens = [a + b for a, b in zip(new, past)]
    c = make_cache(dtype, hk, dh, lens, 95)
    q, starts = make_q(dtype, new, heads, dh, 96)
    clean = attend(c, q, starts, lens)
    hit = torch.zeros_like(clean, dtype=torch.bool)
    for b in range(n):
        if b % 9 != 4 and b % 5:
            continue
        p, col = past[b] + new[b] // 2, 3 * b % dh
        blk = int(c.block_table[b, p // 16])
        c.v[blk, 0, p % 16, col] = 0x7f if dtype == "e4m3" else (math.nan if b % 2 else math.inf)
        hit[starts[b] + new[b] // 2:starts[b + 1], :, col] = True
    for _ in range(3):
        out = attend(c, q, starts, lens)
        assert not torch.isfinite(out[hit]).any()
        assert torch.equal(out[~hit], clean[~hit])
    c.check()
