"""adept_extend_verify and adept_seq_trim: the pass against adept_extend on a model of its own, its verification against the 64-bit
statement on its own logits; generation by a model's own early exits, checked at full depth, against full-depth generation; refusals."""
import numpy as np
import pytest
import torch

import synth
from parity_utils import assert_rows_close
from serve_reference import verify

import paper_2601_03700_gb300 as adept

pytestmark = pytest.mark.gpu

CONFIGS = {
    "llama_f32": dict(family=synth.LLAMA, n_layers=4, d_model=256, n_heads=4, head_dim=64, d_ffn=512, vocab=500, dtype="f32"),
    "llama_gqa": dict(family=synth.LLAMA, n_layers=5, d_model=256, n_heads=4, n_kv_heads=2, head_dim=128, d_ffn=512, vocab=501,
                      dtype="bf16", hsm_m1=512, hsm_m2=1024, block_shuffle_seed=3),
    "gpt2": dict(family=synth.GPT2, n_layers=4, d_model=384, n_heads=6, head_dim=64, d_ffn=512, vocab=500, max_pos=640, dtype="bf16"),
    "llama_e4m3": dict(family=synth.LLAMA, n_layers=4, d_model=256, n_heads=4, head_dim=64, d_ffn=512, vocab=500, dtype="bf16"),
}
TOL = {"f32": 1e-4, "bf16": 2e-2}   # of the parity tests


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    adept.load_library()


def make(name, batch=3, max_seq=320, seed=11):
    cfg = synth.ModelConfig(max_batch=batch, max_seq=max_seq, **CONFIGS[name])
    if name.endswith("e4m3"):
        cfg.kv_type = "e4m3"
    return cfg, adept.Model(cfg, synth.make_weights(cfg, seed=seed))


def i32(x):
    return torch.as_tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("name", CONFIGS)
def test_the_pass_and_its_verification(name):
    cfg, m = make(name)
    _, ref = make(name)
    B, P, V = 3, 20, cfg.vocab
    g = torch.Generator(device="cuda").manual_seed(1)
    prompt = synth.make_tokens(12, B, P, V).cuda()
    for x in (m, ref):
        x.prefill(prompt, 0.9)
    held, temp = [P] * B, [1.0, 0.0, 0.5]
    for turn, lens in enumerate(([5, 1, 3], [0, 4, 9], [1, 1, 1], [40, 2, 0])):
        n = sum(lens)
        tokens = synth.make_tokens(20 + turn, 1, n, V).cuda().view(-1).int()
        forced = synth.forced_exits_uniform(30 + turn, n, 2, cfg.n_layers).cuda().int()
        u = torch.rand(n, generator=g, device="cuda")
        draft = None if turn == 1 else torch.randn(n, V, generator=g, device="cuda").to(torch.bfloat16 if turn == 2 else torch.float32)
        t = torch.tensor(temp, device="cuda")
        acc, nx, lg, lp, ex, sim = m.verify(lens, tokens, 0.9, u, draft, t, forced)
        m.check()
        # the pass is adept_extend's
        ex2, lg2, nx2, _ = ref.extend(lens, tokens, 0.9, forced)
        assert torch.equal(ex, ex2)
        start = np.concatenate([[0], np.cumsum(lens)])
        live = [b for b in range(B) if lens[b]]
        assert_rows_close(lg[start[1:][live] - 1].cpu().numpy(), lg2[live].cpu().numpy(), TOL[cfg.dtype], "logits")
        assert_rows_close(m.final_states(n).cpu().numpy(), ref.final_states(n).cpu().numpy(), TOL[cfg.dtype], "final states")
        # every row's logits: the head of its state, as a pass that ends there gives it (prefill's last row, by pieces, in the next test)
        exp = verify(lg.cpu(), None if draft is None else draft.cpu(), tokens.tolist(), start.tolist(), u.cpu(), temp)
        assert (acc.tolist(), nx.tolist()) == exp[:2]
        for r, v in enumerate(lp.tolist()):
            assert np.isnan(v) if r not in exp[2] else abs(v - exp[2][r]) < 1e-4
        # both go on behind what was accepted
        held = [h + (1 + a if n_ else 0) for h, a, n_ in zip(held, acc.tolist(), lens)]
        for x in (m, ref):
            x.trim(held)
    for l in range(1, cfg.n_layers + 1):
        for b in range(B):
            k, v = m.read_kv(l, b, 0, held[b])
            k2, v2 = ref.read_kv(l, b, 0, held[b])
            assert_rows_close(k.float().reshape(held[b], -1).cpu().numpy(), k2.float().reshape(held[b], -1).cpu().numpy(), 2 * TOL[cfg.dtype], "K")
            assert_rows_close(v.float().reshape(held[b], -1).cpu().numpy(), v2.float().reshape(held[b], -1).cpu().numpy(), 2 * TOL[cfg.dtype], "V")
    m.close()
    ref.close()


@pytest.mark.parametrize("name", ["llama_f32", "gpt2"])
def test_logits_of_every_token(name):
    """Row j of a chunk has the logits that the chunk cut behind token j has as its last."""
    cfg, m = make(name, batch=1)
    prompt, chunk = synth.make_tokens(1, 1, 30, cfg.vocab).cuda(), synth.make_tokens(2, 1, 12, cfg.vocab).cuda().view(-1).int()
    m.prefill(prompt, float("inf"))
    lg = m.verify([12], chunk, float("inf"), torch.rand(12, device="cuda"))[2]
    for j in (0, 4, 11):
        m.trim([30])
        one = m.extend([j + 1], chunk[:j + 1], float("inf"))[1]
        assert_rows_close(lg[j:j + 1].cpu().numpy(), one.cpu().numpy(), TOL[cfg.dtype], "logits")
    m.close()


@pytest.mark.parametrize("name", ["llama_f32", "llama_e4m3"])
def test_generation_by_own_early_exits(name):
    """Drafts by generation steps that leave at layer 2, cut back, verified at full depth (greedy): the tokens of full-depth generation,
    as far as its best token stands out by more than the two ways' rounding."""
    cfg, m = make(name, batch=2)
    _, ref = make(name, batch=2)
    inf, B, P, D = float("inf"), 2, 16, 4
    prompt = synth.make_tokens(5, B, P, cfg.vocab).cuda()
    _, lg, nx, _ = ref.prefill(prompt, inf)
    want, margin = [[] for _ in range(B)], [[] for _ in range(B)]
    for _ in range(24):
        for b in range(B):
            top = lg[b].topk(2).values
            want[b].append(int(nx[b]))
            margin[b].append(float((top[0] - top[1]) / lg[b].norm()))
        _, lg, nx, _ = ref.decode_step(nx, inf)
    _, _, nx, _ = m.prefill(prompt, inf)
    got, held, zero = [[] for _ in range(B)], [P] * B, torch.zeros(B, device="cuda")
    accepted = 0
    while min(len(x) for x in got) < 20:
        drafts, t = [nx], nx
        for _ in range(D):   # (every draft token leaves at layer 2)
            _, _, t, _ = m.decode_step(t, 0.9, i32([2] * B))
            drafts.append(t)
        m.trim(held)
        chunk = torch.stack(drafts, 1).reshape(-1)
        acc, nx, *_ = m.verify([1 + D] * B, chunk, inf, torch.zeros(B * (1 + D), device="cuda"), temperature=zero)
        m.check()
        for b, a in enumerate(acc.tolist()):
            got[b] += chunk[b * (1 + D):b * (1 + D) + 1 + a].tolist()
            held[b] += 1 + a
            accepted += a
        m.trim(held)
    for b in range(B):
        for i, (x, y) in enumerate(zip(got[b], want[b])):
            if x != y:
                assert margin[b][i] < 2 * TOL[cfg.dtype], (b, i)
                break
    m.close()
    ref.close()


def test_refusals():
    cfg, m = make("llama_f32")
    n, V = 6, cfg.vocab
    tok, u, lg = i32([1] * n), torch.rand(n, device="cuda"), torch.zeros(n, V, device="cuda")
    acc, nx = i32([0] * 3), i32([0] * 3)

    def go(lens=(2, 3, 1), **kw):
        a = dict(u=u, logits_out=lg, accepted_out=acc, next_token_out=nx)
        a.update(kw)
        adept.adept_extend_verify(m.h, list(lens), tok, 0.9, **a)

    def refused(status, f):
        with pytest.raises(adept.AdeptError) as ei:
            f()
        assert ei.value.status == status

    refused(1, go)   # not reserved
    adept.adept_seq_reserve(m.h, [0, 0, 0])
    for k in ("u", "logits_out", "accepted_out", "next_token_out"):
        refused(1, lambda: go(**{k: None}))
    refused(1, lambda: go(lens=(0, 0, 0)))
    refused(1, lambda: go(lens=(-1, 3, 4)))
    refused(3, lambda: go(lens=(400, 0, 0)))
    refused(1, lambda: go(draft=torch.zeros(n, V - 1, device="cuda")))
    with pytest.raises(ValueError):
        go(draft=torch.zeros(n, V, device="cuda").half())
    with pytest.raises(ValueError):
        m.verify([2, 3], tok, 0.9, u)
    with pytest.raises(ValueError):
        m.verify([2, 3, 1], tok, 0.9, u, torch.zeros(n, V + 1, device="cuda"))
    go()
    m.check()
    for lens, status in (([3, 3, 1], 1), ([-1, 3, 1], 1), ([1, 1, 1, 1], 3), ([], 1)):
        refused(status, lambda: m.trim(lens))
    m.trim([2, 0])
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()   # (what the side stream reads is made on this one)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        g.capture_begin()
        try:
            refused(1, lambda: m.trim([1, 0]))
            refused(1, go)
        finally:
            g.capture_end()
    # a draft out of the vocabulary: the pass flags it, and so does the verification, which leaves the sequence out
    tok[1] = V
    go(lens=(2, 3, 1))
    assert acc.tolist()[0] == -1 and nx.tolist()[0] == -1 and acc.tolist()[1] >= 0
    refused(6, m.check)
    m.close()


def test_memory_that_is_not_there():
    """An allocation that fails leaves the sequences as they were; the call can be made again."""
    cfg, m = make("llama_f32")
    m.prefill(synth.make_tokens(1, 3, 10, cfg.vocab).cuda(), 0.9)
    tok, u = i32([1] * 3), torch.rand(3, device="cuda")
    for k in range(2):   # the first and the second of the call's own two, behind those of the extension
        m.extend([1, 1, 1], tok, 0.9)
        adept.adept_set_alloc_fail_after(k)
        try:
            with pytest.raises(adept.AdeptError) as ei:
                m.verify([1, 1, 1], tok, 0.9, u)
        finally:
            adept.adept_set_alloc_fail_after(-1)
        assert ei.value.status == 2
        m.trim([11 + k] * 3)   # (they hold that many: else refused, or more left)
        with pytest.raises(adept.AdeptError):
            m.trim([12 + k] * 3)
    m.verify([1, 1, 1], tok, 0.9, u)
    m.check()
    m.close()


def test_the_head_over_many_tokens():
    """Chunks of more tokens than the head's rows of any other call (a prompt verified as drafts)."""
    cfg, m = make("llama_gqa", batch=2)
    adept.adept_seq_reserve(m.h, [0, 0])
    n = 300
    tokens = synth.make_tokens(9, 1, n, cfg.vocab).cuda().view(-1).int()
    u = torch.rand(n, device="cuda")
    acc, nx, lg, lp, _, _ = m.verify([170, 130], tokens, float("inf"), u)
    m.check()
    exp = verify(lg.cpu(), None, tokens.tolist(), [0, 170, 300], u.cpu())
    assert (acc.tolist(), nx.tolist()) == exp[:2]
    m.trim([0, 0])
    last = m.extend([170, 130], tokens, float("inf"))[1]
    assert_rows_close(lg[[169, 299]].cpu().numpy(), last.cpu().numpy(), 2e-2, "logits")
    m.close()


def test_a_decoder_with_cross_attention():
    """An encoder-decoder's decoder: drafts verified behind its source, its logits as the chunk's without drafts."""
    cfg = synth.ModelConfig(family=synth.GPT2, n_layers=4, d_model=384, n_heads=6, head_dim=64, d_ffn=512, vocab=500, max_pos=256, dtype="bf16",
                            max_batch=2, max_seq=128, max_src=40)
    m = adept.Model(cfg, synth.make_weights(cfg, seed=7))
    prompt = synth.make_tokens(8, 2, 10, cfg.vocab).cuda()
    states = torch.randn(60, cfg.d_model, device="cuda")
    u = torch.rand(7, device="cuda")
    chunk = synth.make_tokens(9, 1, 7, cfg.vocab).cuda().view(-1).int()
    with pytest.raises(adept.AdeptError):
        m.verify([4, 3], chunk, 0.9, u)   # no source yet
    m.set_cross_source([40, 20], states)
    m.prefill(prompt, float("inf"))
    acc, nx, lg, *_ = m.verify([4, 3], chunk, float("inf"), u)
    m.check()
    exp = verify(lg.cpu(), None, chunk.tolist(), [0, 4, 7], u.cpu())
    assert (acc.tolist(), nx.tolist()) == exp[:2]
    m.trim([10, 10])
    last = m.extend([4, 3], chunk, float("inf"))[1]
    assert_rows_close(lg[[3, 6]].cpu().numpy(), last.cpu().numpy(), 2e-2, "logits")
    m.close()


def test_profiled_and_without_graphs():
    """The passes' other modes: events around launches, no captured steps, SIMT products."""
    cfg, m = make("llama_gqa")
    out = []
    for option in (None, adept.OPT_PROFILE, adept.OPT_DECODE_GRAPH, adept.OPT_GEMM_SIMT):
        if option is not None:
            adept.adept_set_option(m.h, option, 0 if option == adept.OPT_DECODE_GRAPH else 1)
        m.prefill(synth.make_tokens(1, 3, 12, cfg.vocab).cuda(), float("inf"))
        tok = synth.make_tokens(2, 1, 9, cfg.vocab).cuda().view(-1).int()
        acc, nx, lg, *_ = m.verify([2, 3, 4], tok, float("inf"), torch.full((9,), 0.5, device="cuda"))
        m.check()
        assert (acc.tolist(), nx.tolist()) == verify(lg.cpu(), None, tok.tolist(), [0, 2, 5, 9], torch.full((9,), 0.5))[:2]
        out.append(lg.cpu().numpy())
        if option is not None:
            adept.adept_set_option(m.h, option, 1 if option == adept.OPT_DECODE_GRAPH else 0)
    for x in out[1:]:
        assert_rows_close(x, out[0], 2e-2, "logits")
    m.close()
