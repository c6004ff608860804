"""Models with an 8-bit cache in the paths that the method's options take: exits all at once, threshold calibration, profiling, the
CUDA-core products, an encoder-decoder's turns, a model of two layers.

Each against the oracle with a cache that quantises, or against the same model by its ordinary path; bounds as in
test_gpu_kv8_model.py: the parity tolerance, and for a code that rounds to its other neighbour twice the effect that quantising
has on the oracle."""
import numpy as np
import pytest
import torch

import synth
from oracle import adept_oracle as O
from parity_utils import assert_rows_close, row_rel_err
from test_gpu_extend import CONFIGS, oracle_extend
from test_gpu_kv8_model import QuantisedCache, _lib, dev, models  # noqa: F401  (_lib: the module's fixture)

import paper_2601_03700_gb300 as adept

pytestmark = pytest.mark.gpu


def compare(m8, got, res, ref, rows):
    tol = [2e-2 + 2 * float(row_rel_err(a, b).max()) for a, b in ((res.final, ref.final), (res.logits, ref.logits))]
    assert max(tol) < 0.5
    np.testing.assert_array_equal(got[0].cpu().numpy(), res.exit_layer)
    assert_rows_close(m8.final_states(rows).cpu().numpy(), res.final, tol[0], "final states")
    assert_rows_close(got[1].cpu().numpy(), res.logits, tol[1], "logits")


def test_exits_all_at_once():
    cfg, W, m, m8 = models("llama_gqa")
    m.close()
    om = O.OracleModel(cfg, W)
    tokens = synth.make_tokens(100, 3, 90, cfg.vocab).numpy()
    # the sequences' exits, by their last prompt token
    f = np.full((3, 90), cfg.n_layers, dtype=np.int32)
    f[:, -1] = [2, 4, cfg.n_layers]
    adept.adept_set_option(m8.h, adept.OPT_ALL_AT_ONCE, 1)
    res, ref = (O.prefill(om, c(cfg, 3, 640), tokens, 0.9, f, all_at_once=True) for c in (QuantisedCache, O.OracleCache))
    compare(m8, m8.prefill(dev(tokens), 0.9, dev(f)), res, ref, 270)
    m8.check()
    m8.close()


def test_calibration():
    """The threshold that calibration gives cuts the batch's computation by what it says."""
    cfg, _, m, m8 = models("llama_gqa")
    m.close()
    t = synth.make_tokens(101, 3, 120, cfg.vocab).cuda()
    delta, rdc, _ = adept.adept_calibrate_threshold(m8.h, 3, 120, t.view(-1).contiguous(), 0.25, tol=0.05)
    ex = m8.prefill(t, delta)[0]
    m8.check()
    assert abs(1 - ex.float().sum().item() / (360 * cfg.n_layers) - rdc) < 1e-6 and 0 < rdc < 1
    m8.close()


@pytest.mark.parametrize("option", ["profile", "simt"])
def test_the_same_by_other_options(option):
    """Launches in line instead of side by side give the same bits; CUDA-core products the same up to rounding."""
    runs = []
    for on in (0, 1):
        cfg, _, m, m8 = models("llama_gqa")
        m.close()
        adept.adept_set_option(m8.h, adept.OPT_PROFILE if option == "profile" else adept.OPT_GEMM_SIMT, on)
        t = synth.make_tokens(102, 3, 100, cfg.vocab).cuda()
        f = synth.forced_exits_uniform(103, 300, 2, cfg.n_layers).cuda()
        run = [m8.prefill(t, 0.9, f)[1], m8.extend([1, 150, 20], t.view(-1)[:171], 0.9, f[:171])[1], m8.final_states(171)]
        run.append(m8.decode_step(dev([5, 6, 7]), 0.9, dev([2, 3, 5]))[1])
        m8.check()
        runs.append([x.cpu().numpy() for x in run])
        m8.close()
    for a, b in zip(*runs):
        if option == "profile":
            assert np.array_equal(a, b)
        else:   # (a code that rounds the other way moves an entry by up to 2^-3 of it, as the bf16 noise of either side may)
            assert_rows_close(a, b, 0.1, "the other products")


def test_an_encoder_decoders_turns():
    dec = dict(family=synth.GPT2, n_layers=4, d_model=256, n_heads=4, head_dim=64, d_ffn=512, vocab=500, max_pos=128, dtype="bf16",
               max_batch=2, max_seq=128, max_src=24)
    cfg = synth.ModelConfig(**dec)
    W = synth.make_weights(cfg, seed=105)
    om = O.OracleModel(cfg, W)
    cfg8 = synth.ModelConfig(**dec)
    cfg8.kv_type = "e4m3"
    m8 = adept.Model(cfg8, W)
    src = [24, 9]
    states = torch.randn(sum(src), 256, generator=torch.Generator().manual_seed(106))
    cross = O.CrossSource(om, [states[:24].numpy(), states[24:].numpy()])
    m8.set_cross_source(src, states.cuda())
    q, exact = QuantisedCache(cfg, 2, 128), O.OracleCache(cfg, 2, 128)
    law = lambda s, n: synth.forced_exits_uniform(s, n, 2, 4).numpy()  # noqa: E731
    tokens, f = synth.make_tokens(107, 2, 20, 500).numpy(), law(108, 40).reshape(2, 20)
    res, ref = (O.prefill(om, c, tokens, 0.9, f, cross=cross) for c in (q, exact))
    compare(m8, m8.prefill(dev(tokens), 0.9, dev(f)), res, ref, 40)
    tk, f = synth.make_tokens(109, 1, 35, 500).numpy()[0], law(110, 35)
    res, ref = (oracle_extend(om, c, [30, 5], tk, 0.9, f, cross)[0] for c in (q, exact))
    compare(m8, m8.extend([30, 5], dev(tk), 0.9, dev(f)), res, ref, 35)
    m8.check()
    m8.close()


def test_two_layers():
    shape = dict(CONFIGS["llama_gqa"], n_layers=2)
    cfg = synth.ModelConfig(max_batch=2, max_seq=96, **shape)
    W = synth.make_weights(cfg, seed=111)
    om = O.OracleModel(cfg, W)
    cfg8 = synth.ModelConfig(max_batch=2, max_seq=96, **shape)
    cfg8.kv_type = "e4m3"
    m8 = adept.Model(cfg8, W)
    q, exact = QuantisedCache(cfg, 2, 96), O.OracleCache(cfg, 2, 96)
    tokens = synth.make_tokens(112, 2, 40, cfg.vocab).numpy()
    res, ref = (O.prefill(om, c, tokens, 0.9) for c in (q, exact))
    compare(m8, m8.prefill(dev(tokens), 0.9), res, ref, 80)
    res, ref = (O.decode_step(om, c, np.array([3, 4]), 0.9) for c in (q, exact))
    compare(m8, m8.decode_step(dev([3, 4]), 0.9), res, ref, 2)
    m8.check()
    m8.close()
