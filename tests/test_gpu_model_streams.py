"""A model's calls on another stream than the current one, while that is still busy: what the wrapper makes and converts is ordered with the
call."""
import pytest
import torch

import synth

import paper_2601_03700_gb300 as adept

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def model():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    cfg = synth.ModelConfig(family=synth.LLAMA, n_layers=3, d_model=128, n_heads=2, head_dim=64, d_ffn=256, vocab=300, dtype="bf16", max_batch=2, max_seq=64)
    m = adept.Model(cfg, synth.make_weights(cfg, seed=2))
    yield cfg, m
    m.close()


def cases(cfg):
    """A call that leaves both sequences with their prompts and what it takes in, from inputs that need converting."""
    g = torch.Generator().manual_seed(3)
    prompt = synth.make_tokens(1, 2, 10, cfg.vocab).cuda().long()
    tok = torch.randint(cfg.vocab, (7,), generator=g).cuda()
    u, draft = torch.rand(7, generator=g, dtype=torch.float64).cuda(), torch.randn(7, cfg.vocab, generator=g).cuda()
    t = torch.tensor([1.0, 0.5], dtype=torch.float64).cuda()
    forced = torch.full((7,), 2).cuda()
    return {
        "prefill": lambda m, s: m.prefill(prompt, 0.9, stream=s),
        "extend": lambda m, s: m.extend([7, 0], tok, 0.9, forced, stream=s),
        "decode_step": lambda m, s: m.decode_step(tok[:2], 0.9, stream=s),
        "verify": lambda m, s: m.verify([4, 3], tok, 0.9, u, draft, t, forced, stream=s),
    }


@pytest.mark.parametrize("raw", [False, True])
@pytest.mark.parametrize("name", ["prefill", "extend", "decode_step", "verify"])
def test_a_busy_current_stream(model, name, raw):
    cfg, m = model
    run = cases(cfg)[name]
    start = lambda: (adept.adept_seq_reserve(m.h, [0, 0]), m.prefill(synth.make_tokens(1, 2, 10, cfg.vocab).cuda(), 0.9), torch.cuda.synchronize())  # noqa: E731
    start()
    want = [t.clone() for t in run(m, None)]
    start()
    s = torch.cuda.Stream()
    torch.cuda._sleep(200_000_000)   # about a tenth of a second
    busy = torch.cuda.Event()
    busy.record()
    got = run(m, s.cuda_stream if raw else s)
    s.synchronize()
    assert not busy.query()   # (the call did not wait for the current stream)
    with torch.cuda.stream(s):
        first = [t.cpu() for t in got]
    torch.cuda.synchronize()
    for a, b, c in zip(first, got, want):
        assert torch.equal(a.nan_to_num(7.0), c.cpu().nan_to_num(7.0))
        assert torch.equal(b.cpu().nan_to_num(7.0), c.cpu().nan_to_num(7.0))   # nothing came later
    m.check()


def test_trim_on_a_stream(model):
    cfg, m = model
    m.prefill(synth.make_tokens(1, 2, 10, cfg.vocab).cuda(), 0.9)
    torch.cuda.synchronize()
    tok = synth.make_tokens(5, 1, 4, cfg.vocab).cuda().view(-1)
    want = [t.clone() for t in m.extend([4, 0], tok, 0.9)]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    m.trim([10, 10], stream=s)
    got = m.extend([4, 0], tok, 0.9, stream=s)
    s.synchronize()
    assert all(torch.equal(a.nan_to_num(7.0), b.nan_to_num(7.0)) for a, b in zip(got, want))
