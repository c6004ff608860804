"""Where 8-bit entries are widened to: calls whose workspace goes by the pool and by the table, blocks that sequences share, and a
model whose block table spans 2^31 rows of K (more than a tensor map takes) over a small pool."""
import pytest
import torch

import synth
from parity_utils import assert_rows_close
from test_gpu_kv_ops import _lib, assert_attention, attend, make_cache, make_q  # noqa: F401  (_lib: the module's fixture)

import paper_2601_03700_gb300 as adept

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("new,past,spare", [
    ([150, 130], [400, 400], 2),       # by the table: as many blocks as both rows take, two over in the pool
    ([150, 130], [900, 200], 0),       # by the pool: the second row is half empty
    ([150, 1, 3, 260], [900, 700, 0, 250], 40),
])
def test_shared_blocks(dtype, new, past, spare):
    """The first positions of all sequences in the same blocks (a prompt that users share)."""
    lens = [a + b for a, b in zip(new, past)]
    c = make_cache(dtype, 2, 128, lens, 80, spare=spare)
    n = min(b for b in lens if b >= 100) // 16 - 1
    for b in range(1, len(lens)):
        if lens[b] >= 100:
            c.block_table[b, :n] = c.block_table[0, :n]
    q, starts = make_q(dtype, new, 8, 128, 81)
    out = attend(c, q, starts, lens)
    c.check()
    assert_attention(c, q, starts, lens, out)
    assert torch.equal(out, attend(c, q, starts, lens))


def test_a_table_of_more_rows_than_a_tensor_map_takes():
    """512 sequences of 131072 positions of 32 heads in the table, one such sequence in the pool: a prompt and a chunk of one
    sequence as in a model made for it."""
    shape = dict(family=synth.LLAMA, n_layers=3, d_model=256, n_heads=32, head_dim=64, d_ffn=256, vocab=300, dtype="bf16",
                 max_pass_tokens=512)
    out = []
    for kw in (dict(max_batch=512, max_seq=131072, kv_pool_blocks=8192), dict(max_batch=1, max_seq=1024)):
        cfg = synth.ModelConfig(**shape, **kw)
        cfg.kv_type = "e4m3"
        m = adept.Model(cfg, synth.make_weights(cfg, seed=82))
        t = synth.make_tokens(83, 1, 500, cfg.vocab).cuda()
        f = synth.forced_exits_uniform(84, 500, 2, 3).cuda()
        run = []
        run += [m.prefill(t[:, :300], 0.9, f[:300])[1].cpu().numpy(), m.final_states(300).cpu().numpy()]
        run += [m.extend([200], t[0, 300:], 0.9, f[300:])[1].cpu().numpy(), m.final_states(200).cpu().numpy()]
        m.check()
        out.append(run)
        m.close()
    for a, b in zip(*out):
        assert_rows_close(a, b, 2e-2, "states and logits")
