"""adept_extend_verify's buffers against the sizes of the model that the handle is of."""
import pytest
import torch

import synth

import paper_2601_03700_gb300 as adept

pytestmark = pytest.mark.gpu


def test_buffers_of_another_models_sizes():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    cfg = synth.ModelConfig(family=synth.LLAMA, n_layers=2, d_model=128, n_heads=2, head_dim=64, d_ffn=256, vocab=300, dtype="f32", max_batch=2, max_seq=32)
    m = adept.Model(cfg, synth.make_weights(cfg, seed=1))
    m.prefill(synth.make_tokens(1, 2, 8, cfg.vocab).cuda(), 0.9)
    tok = torch.ones(4, dtype=torch.int32, device="cuda")
    r = torch.full((2,), -7, dtype=torch.int32, device="cuda")
    good = dict(u=torch.rand(4, device="cuda"), logits_out=torch.zeros(4, 300, device="cuda"), accepted_out=r, next_token_out=r.clone(),
                draft=torch.zeros(4, 300, device="cuda"), sim_out=torch.zeros(4, 2, device="cuda"))
    for name, bad, status in (("logits_out", torch.zeros(4, 299, device="cuda"), 3), ("sim_out", torch.zeros(4, 1, device="cuda"), 3),
                              ("draft", torch.zeros(4, 310, device="cuda")[:, :299], 1), ("draft", torch.zeros(3, 300, device="cuda"), 3)):
        with pytest.raises(adept.AdeptError) as ei:
            adept.adept_extend_verify(m.h, [3, 1], tok, 0.9, **{**good, name: bad})
        assert ei.value.status == status, name
    for bad in (dict(u=torch.rand(4)), dict(draft=torch.zeros(4, 300)), dict(temperature=torch.ones(2))):   # on the host
        with pytest.raises(ValueError):
            adept.adept_extend_verify(m.h, [3, 1], tok, 0.9, **{**good, **bad})
        with pytest.raises(ValueError):
            m.verify([3, 1], tok, 0.9, **{"u": good["u"], **bad})
    m.trim([8, 8])   # nothing was taken in
    adept.adept_extend_verify(m.h, [3, 1], tok, 0.9, **good)
    m.check()
    assert r.min() >= 0
    m.close()
