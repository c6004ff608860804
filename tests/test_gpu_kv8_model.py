"""Models whose cache is held in 8 bits (kv_type e4m3): prompt passes, chunks, generation steps and fills.

The first layer's entries come from the same products as in a bf16 cache, so they are exactly its entries quantised.  Whole
passes are held against the oracle with a cache that quantises what it is given.  Bounds: an entry of either side is within
2^-4 of its value before rounding (half a step of a 4-bit significand), those are within the parity tolerance of each other
in a row's norm, so rows of the two caches differ by at most 2^-4 (1 + 1.02) + 2e-2 < 0.15 of the norm.  A code may round to the other
neighbour on the GPU, which moves an entry by at most a step, twice what quantising moved it: states and logits may be off by
the parity tolerance and twice the effect that quantising has on the oracle itself (taken from the oracle, without the GPU)."""
import numpy as np
import pytest
import torch

import kv_reference as R
import synth
from oracle import adept_oracle as O
from parity_utils import assert_rows_close, row_rel_err
from test_gpu_extend import CONFIGS, oracle_extend

import paper_2601_03700_gb300 as adept

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    adept.load_library()


class QuantisedCache(O.OracleCache):
    def write(self, i, seq, pos, k, v):
        super().write(i, seq, pos, *(R.quantise(torch.as_tensor(np.asarray(x)))[0].numpy() for x in (k, v)))


def models(name, n=3, seq=640, **kw):
    base = dict(max_batch=n, max_seq=seq, **CONFIGS[name])
    base.update(kw)
    cfg = synth.ModelConfig(**base)
    cfg8 = synth.ModelConfig(**base)
    cfg8.kv_type = "e4m3"
    W = synth.make_weights(cfg, seed=70)
    return cfg, W, adept.Model(cfg, W), adept.Model(cfg8, W)


def dev(x):
    return torch.as_tensor(np.asarray(x), dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("name", ["llama_gqa", "gpt2", "llama_32"])
def test_the_first_layers_entries_are_the_bf16_ones_quantised(name):
    cfg, W, m, m8 = models(name)
    t = synth.make_tokens(71, 3, 150, cfg.vocab).cuda()
    f = synth.forced_exits_uniform(72, 450, 2, cfg.n_layers).cuda()
    nx = dev([5, 6, 7])
    for x in (m, m8):
        x.prefill(t, 0.9, f)
        x.extend([0, 200, 3], t.reshape(-1)[:203], 0.9, f[:203])
        for _ in range(3):
            x.decode_step(nx, 0.9, dev([2, 3, 4]))
        x.check()
    for b, n in enumerate((153, 353, 156)):
        for want, got in zip(m.read_kv(1, b, 0, n), m8.read_kv(1, b, 0, n)):
            assert torch.equal(got.double(), R.quantise(want)[0])
    m.close()
    m8.close()


@pytest.mark.parametrize("name", ["llama_gqa", "gpt2", "llama_32"])
def test_against_the_oracle_with_a_quantised_cache(name):
    cfg, W, m, m8 = models(name)
    m.close()
    om = O.OracleModel(cfg, W)
    q, exact = QuantisedCache(cfg, 3, 640), O.OracleCache(cfg, 3, 640)
    tokens = synth.make_tokens(73, 3, 40, cfg.vocab).numpy()
    law = lambda s, n: synth.forced_exits_uniform(s, n, 2, cfg.n_layers).numpy()  # noqa: E731

    def compare(got, res, ref, rows):
        tol = [2e-2 + 2 * float(row_rel_err(a, b).max()) for a, b in ((res.final, ref.final), (res.logits, ref.logits))]
        assert max(tol) < 0.5   # (the bound still says something)
        assert_rows_close(m8.final_states(rows).cpu().numpy(), res.final, tol[0], "final states")
        assert_rows_close(got[1].cpu().numpy(), res.logits, tol[1], "logits")
        np.testing.assert_array_equal(got[0].cpu().numpy(), res.exit_layer)

    f = law(74, 120).reshape(3, 40)
    compare(m8.prefill(dev(tokens), 0.9, dev(f)), O.prefill(om, q, tokens, 0.9, f), O.prefill(om, exact, tokens, 0.9, f), 120)
    for seed, lens in ((75, [7, 300, 1]), (76, [1, 2, 20])):
        tk = synth.make_tokens(seed, 1, sum(lens), cfg.vocab).numpy()[0]
        f = law(seed + 10, sum(lens))
        compare(m8.extend(lens, dev(tk), 0.9, dev(f)), oracle_extend(om, q, lens, tk, 0.9, f)[0],
                oracle_extend(om, exact, lens, tk, 0.9, f)[0], sum(lens))
    for step in range(4):
        tk = synth.make_tokens(90 + step, 1, 3, cfg.vocab).numpy()[0]
        f = law(95 + step, 3)
        compare(m8.decode_step(dev(tk), 0.9, dev(f)), O.decode_step(om, q, tk, 0.9, f), O.decode_step(om, exact, tk, 0.9, f), 3)
    m8.check()
    for b in range(3):
        n = int(q.lens[b])
        for l in range(1, cfg.n_layers + 1):
            for got, want in zip(m8.read_kv(l, b, 0, n), (q.K[l - 1][b, :n], q.V[l - 1][b, :n])):
                assert_rows_close(got.float().cpu().numpy(), want, 0.15, f"cache of layer {l}")
    m8.close()


def test_steps_replayed_equal_direct_steps():
    _, _, m, m8 = models("llama_gqa")
    m.close()
    t = synth.make_tokens(77, 3, 60, 500).cuda()
    outs = []
    for graph in (0, 1):
        adept.adept_set_option(m8.h, adept.OPT_DECODE_GRAPH, graph)
        m8.prefill(t, 9.0)
        run = []
        for s in range(4):
            run += [x.clone() for x in m8.decode_step(dev([s, 2 * s, 9]), 9.0, dev([2 + s % 3, 0, 4]))]
        run += [x for layer in (1, 3, 5) for b in range(3) for x in m8.read_kv(layer, b, 0, 64)]
        outs.append(run)
    m8.check()
    assert all(torch.equal(torch.nan_to_num(a.float(), nan=-1), torch.nan_to_num(b.float(), nan=-1)) for a, b in zip(*outs))
    m8.close()


@pytest.mark.parametrize("n", [3, 40, 300])
def test_fills(n):
    cfg, W, m, m8 = models("llama_gqa")
    h = synth.make_mapped_states(78, n, cfg.d_model).cuda()
    el = synth.forced_exits_uniform(79, n, 1, cfg.n_layers, name="el").cuda().to(torch.int32)
    seq, pos = dev(np.arange(n) % 3), dev(np.arange(n) // 3)
    for x in (m, m8):
        adept.adept_seq_reserve(x.h, [640] * 3)
        adept.adept_skip_kv_fill(x.h, n, h, el, seq, pos)
        x.check()
    for r in range(2, cfg.n_layers + 1):
        sel = (el < r).nonzero().flatten()
        for b in range(3):
            rows = pos[sel[seq[sel] == b]].long()
            if rows.numel() == 0:
                continue
            for want, got in zip(m.read_kv(r, b, 0, 640), m8.read_kv(r, b, 0, 640)):
                assert_rows_close(got[rows].float().cpu().numpy(), want[rows].float().cpu().numpy(), 0.15, f"fill of layer {r}")
    with pytest.raises(adept.AdeptError) as ei:
        adept.adept_skip_kv_fill_noalloc(m8.h, n, h, el, seq, pos)
    assert ei.value.status == 1
    m.close()
    m8.close()
