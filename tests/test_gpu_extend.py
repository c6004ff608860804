"""adept_extend (chunks of new tokens behind what the sequences hold) against the oracle: turns of ragged and empty chunks after a
prompt, with forced exits and by threshold, generation steps in between; prompts of different lengths from nothing; a prompt
in pieces against the prompt in one pass; refusals."""
import numpy as np
import pytest
import torch

import synth
from oracle import adept_oracle as O
from parity_utils import Pair, assert_rows_close, band_tokens, compare_decode, compare_prefill, decisions_agree_outside_band

import paper_2601_03700_gb300 as adept

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    adept.load_library()


def oracle_extend(om, cache, lens, tokens, delta, forced=None, cross=None):
    """The oracle's pass over the chunks: its layer loop at the positions behind cache.lens."""
    seq = np.repeat(np.arange(len(lens)), lens)
    pos = np.concatenate([cache.lens[b] + np.arange(n) for b, n in enumerate(lens)]).astype(np.int64)
    cache.lens[:len(lens)] += np.asarray(lens)
    res = O.early_exit_pass(om, cache, om.embed(tokens, pos), seq, pos, delta, forced, True, cache.lens.copy(), cross=cross)
    last = np.cumsum(lens) - 1
    live = [b for b, n in enumerate(lens) if n]
    res.logits = np.zeros((len(lens), om.cfg.vocab))
    res.logits[live] = om.lm_logits(res.final[last[live]])
    return res, live


def compare_extend(pair, cache, lens, seed, delta, forced=None):
    tokens = synth.make_tokens(seed, 1, int(sum(lens)), pair.cfg.vocab).numpy()[0]
    lens0 = cache.lens.copy()
    kv0 = [(k.copy(), v.copy()) for k, v in zip(cache.K, cache.V)]
    res, live = oracle_extend(pair.om, cache, lens, tokens, delta, forced, pair.cross)
    if forced is None and band_tokens(res.sim, delta).any():
        # a similarity next to the threshold: the oracle's exits forced on both sides
        forced = res.exit_layer
        cache.lens[:] = lens0
        for l, (k, v) in enumerate(kv0):
            cache.K[l][:], cache.V[l][:] = k, v
        res, live = oracle_extend(pair.om, cache, lens, tokens, delta, forced, pair.cross)
    dev = lambda x: None if x is None else torch.as_tensor(np.asarray(x), dtype=torch.int32, device="cuda")  # noqa: E731
    ex, lg, nx, sim = pair.gm.extend(lens, dev(tokens), delta, dev(forced))
    pair.gm.check()
    np.testing.assert_array_equal(ex.cpu().numpy(), res.exit_layer)
    decisions_agree_outside_band(sim.cpu().numpy(), res.sim, delta, res.exit_layer)
    assert_rows_close(pair.gm.final_states(len(tokens)).cpu().numpy(), res.final, pair.tol, "final states")
    lg, nx = lg.cpu().numpy(), nx.cpu().numpy()
    assert_rows_close(lg[live], res.logits[live], pair.tol, "logits")
    np.testing.assert_array_equal(nx[live], lg[live].argmax(-1))
    idle = [b for b in range(len(lens)) if b not in live]
    assert (lg[idle] == 0).all() and (nx[idle] == 0).all()
    for b in range(len(lens)):
        n = int(cache.lens[b])
        for l in range(1, pair.cfg.n_layers + 1) if n else ():
            k, v = pair.gpu_kv(l, b, n)
            assert_rows_close(k, cache.K[l - 1][b, :n], pair.tol, f"K layer {l} seq {b}")
            assert_rows_close(v, cache.V[l - 1][b, :n], pair.tol, f"V layer {l} seq {b}")
    return res


CONFIGS = {
    "llama_f32": dict(family=synth.LLAMA, n_layers=4, d_model=256, n_heads=4, head_dim=64, d_ffn=512, vocab=500, dtype="f32"),
    "llama_gqa": dict(family=synth.LLAMA, n_layers=5, d_model=256, n_heads=4, n_kv_heads=2, head_dim=128, d_ffn=512, vocab=500,
                      dtype="bf16", hsm_m1=512, hsm_m2=1024, block_shuffle_seed=3),
    "gpt2": dict(family=synth.GPT2, n_layers=4, d_model=384, n_heads=6, head_dim=64, d_ffn=512, vocab=500, max_pos=640,
                 dtype="bf16", block_shuffle_seed=5),
    "llama_32": dict(family=synth.LLAMA, n_layers=4, d_model=256, n_heads=8, head_dim=32, d_ffn=512, vocab=500, dtype="bf16"),
    "llama_blocks_of_8": dict(family=synth.LLAMA, n_layers=4, d_model=256, n_heads=4, head_dim=64, d_ffn=512, vocab=500,
                              dtype="bf16", kv_block_tokens=8),
}


@pytest.mark.parametrize("name", CONFIGS)
@pytest.mark.parametrize("threshold", [False, True])
def test_turns_of_a_conversation(name, threshold):
    cfg = synth.ModelConfig(max_batch=3, max_seq=640, **CONFIGS[name])
    pair = Pair(cfg, seed=11)
    B, P = 3, 20
    law = lambda s, n: None if threshold else synth.forced_exits_uniform(s, n, 2, cfg.n_layers).numpy()  # noqa: E731
    tokens = synth.make_tokens(12, B, P, cfg.vocab).numpy()
    f = law(13, B * P)
    _, cache, _ = compare_prefill(pair, tokens, 0.9, None if f is None else f.reshape(B, P))
    delta = 0.9
    for turn, lens in enumerate(([5, 130, 1], [0, 1, 17], [301, 0, 2], [1, 1, 1])):
        res = compare_extend(pair, cache, lens, 20 + turn, delta, law(30 + turn, sum(lens)))
        if threshold and turn == 0:   # from here on about half of the tokens leave at layer 2
            delta = float(np.median(res.sim[:, 1][~np.isnan(res.sim[:, 1])]))
    nx = synth.make_tokens(40, 1, B, cfg.vocab).numpy()[0]
    steps = None if threshold else law(41, 3 * B).reshape(3, B)
    compare_decode(pair, cache, nx, 3, delta, steps)
    compare_extend(pair, cache, [3, 4, 40], 50, delta, law(51, 47))
    pair.close()


def test_prompts_of_different_lengths_from_nothing():
    cfg = synth.ModelConfig(max_batch=4, max_seq=320, **CONFIGS["llama_gqa"])
    pair = Pair(cfg, seed=14)
    cache = O.OracleCache(cfg, 4, 320)
    adept.adept_seq_reserve(pair.gm.h, [0] * 4)
    lens = [200, 1, 0, 33]
    compare_extend(pair, cache, lens, 15, 0.9, synth.forced_exits_uniform(16, sum(lens), 2, cfg.n_layers).numpy())
    compare_extend(pair, cache, [3, 1, 9, 0], 17, 0.9, None)
    pair.close()


def test_a_prompt_in_pieces_is_the_prompt():
    """Pieces of 1 to 200 tokens against one pass of the library itself, exits forced: states, cache and logits within the
    parity tolerance of each other (both are within it of the oracle, which computes the same in any pieces)."""
    cfg = synth.ModelConfig(max_batch=1, max_seq=512, **CONFIGS["gpt2"])
    W = synth.make_weights(cfg, seed=18)
    n = 420
    tokens = synth.make_tokens(19, 1, n, cfg.vocab).cuda()
    forced = synth.forced_exits_uniform(20, n, 2, cfg.n_layers).cuda()
    whole, parts = adept.Model(cfg, W), adept.Model(cfg, W)
    ex, lg, _, _ = whole.prefill(tokens, 0.9, forced.view(1, n))
    fin = whole.final_states(n)
    adept.adept_seq_reserve(parts.h, [0])
    at, got_ex, got_fin = 0, [], []
    for k in (1, 200, 16, 17, 128, 58):
        e, l, _, _ = parts.extend([k], tokens[0, at:at + k], 0.9, forced[at:at + k])
        got_ex.append(e)
        got_fin.append(parts.final_states(k))
        at += k
    assert at == n
    parts.check()
    assert torch.equal(torch.cat(got_ex), ex)
    assert_rows_close(torch.cat(got_fin).cpu().numpy(), fin.cpu().numpy(), 2e-2, "final states")
    assert_rows_close(l.cpu().numpy(), lg.cpu().numpy(), 2e-2, "logits")
    for layer in range(1, cfg.n_layers + 1):
        for a, b in zip(parts.read_kv(layer, 0, 0, n), whole.read_kv(layer, 0, 0, n)):
            assert_rows_close(a.float().cpu().numpy(), b.float().cpu().numpy(), 2e-2, f"cache of layer {layer}")
    whole.close()
    parts.close()


def test_encoder_decoder_turns():
    enc = synth.ModelConfig(family=synth.BERT, n_layers=3, d_model=256, n_heads=4, head_dim=64, d_ffn=512, vocab=500,
                            max_pos=64, n_classes=3, dtype="bf16", max_batch=2, max_seq=24)
    dec = synth.ModelConfig(family=synth.GPT2, n_layers=4, d_model=256, n_heads=4, head_dim=64, d_ffn=512, vocab=500,
                            max_pos=128, dtype="bf16", max_batch=2, max_seq=128, max_src=24)
    pe, pd = Pair(enc, seed=21), Pair(dec, seed=22)
    oe, _, _ = compare_prefill(pe, synth.make_tokens(23, 2, 24, 500).numpy(), 0.9,
                               synth.forced_exits_uniform(24, 48, 2, 3).view(2, 24).numpy())
    src = [24, 9]
    pd.cross = O.CrossSource(pd.om, [oe.final.reshape(2, 24, -1)[b, :src[b]] for b in range(2)])
    g = pe.gm.final_states(48).view(2, 24, -1)
    pd.gm.set_cross_source(src, torch.cat([g[b, :src[b]] for b in range(2)]).contiguous())
    _, cache, _ = compare_prefill(pd, synth.make_tokens(25, 2, 8, 500).numpy(), 0.9,
                                  synth.forced_exits_uniform(26, 16, 2, 4).view(2, 8).numpy())
    compare_extend(pd, cache, [30, 5], 27, 0.9, synth.forced_exits_uniform(28, 35, 2, 4).numpy())
    compare_extend(pd, cache, [0, 1], 29, 0.9, None)
    pe.close()
    pd.close()


def test_refusals_leave_the_model_as_it_was():
    cfg = synth.ModelConfig(max_batch=2, max_seq=64, max_pass_tokens=40, **CONFIGS["llama_gqa"])
    m = adept.Model(cfg, synth.make_weights(cfg, seed=30))
    t = torch.zeros(64, dtype=torch.int32, device="cuda")

    def refused(status, lens, tokens=t, delta=0.9):
        with pytest.raises(adept.AdeptError) as ei:
            adept.adept_extend(m.h, lens, tokens, delta)
        assert ei.value.status == status

    refused(1, [1, 0])              # nothing reserved
    m.prefill(t[:20].view(2, 10), 9.0)
    refused(1, [0, 0])
    refused(1, [-1, 3])
    refused(1, [3, 3], delta=float("nan"))
    refused(3, [1, 1, 1])           # batch
    refused(3, [55, 0])             # max_seq
    refused(3, [21, 20])            # the pass workspace
    adept.adept_set_option(m.h, adept.OPT_ALL_AT_ONCE, 1)
    refused(1, [1, 1])
    adept.adept_set_option(m.h, adept.OPT_ALL_AT_ONCE, 0)
    adept.adept_set_alloc_fail_after(0)
    refused(2, [1, 1])
    adept.adept_set_alloc_fail_after(-1)
    with pytest.raises(ValueError):
        m.extend([2, 1], t[:4], 0.9)
    m.extend([20, 20], t[:40], 9.0)
    m.check()
    with pytest.raises(adept.AdeptError):   # a token id out of range is flagged on the device
        m.extend([1, 1], torch.tensor([5, 10 ** 6], device="cuda"), 9.0)
        m.check()
    enc = synth.ModelConfig(family=synth.BERT, n_layers=2, d_model=64, n_heads=1, head_dim=64, d_ffn=64, vocab=64, max_pos=64,
                            n_classes=2, dtype="bf16", max_batch=1, max_seq=32)
    e = adept.Model(enc, synth.make_weights(enc, seed=31))
    with pytest.raises(adept.AdeptError):
        adept.adept_extend(e.h, [1], t, 0.9)
    e.close()
    m.close()


@pytest.mark.parametrize("kv", [None, "e4m3"])
def test_a_stream_in_capture_is_refused(kv):
    """The chunks' lengths come from the host: a replay would read them again."""
    cfg = synth.ModelConfig(max_batch=2, max_seq=64, **CONFIGS["llama_gqa"])
    if kv:
        cfg.kv_type = kv
    m = adept.Model(cfg, synth.make_weights(cfg, seed=32))
    t = synth.make_tokens(33, 2, 10, cfg.vocab).cuda()
    m.prefill(t, 9.0)
    before = m.extend([3, 1], t.view(-1)[:4], 9.0)[1].clone()
    m.prefill(t, 9.0)
    x = torch.zeros(1, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.graph(torch.cuda.CUDAGraph()):
        x += 1
        with pytest.raises(adept.AdeptError, match="captured"):
            adept.adept_extend(m.h, [3, 1], t.view(-1)[:4], 9.0)
        if kv:
            with pytest.raises(adept.AdeptError, match="captured"):
                adept.adept_prefill(m.h, 2, 10, t.view(-1), 9.0)
    assert torch.equal(m.extend([3, 1], t.view(-1)[:4], 9.0)[1], before)   # and nothing has moved
    m.check()
    m.close()
