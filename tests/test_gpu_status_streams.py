"""adept_check_device_status on a stream of its own: what a pass flagged right behind the check of the one before is reported."""
import pytest
import torch

import synth
from test_gpu_extend import CONFIGS

import paper_2601_03700_gb300 as adept

pytestmark = pytest.mark.gpu


def test_a_flag_set_right_behind_a_check_is_reported():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    cfg = synth.ModelConfig(max_batch=2, max_seq=64, **CONFIGS["llama_gqa"])
    m = adept.Model(cfg, synth.make_weights(cfg, seed=34))
    good = synth.make_tokens(35, 2, 4, cfg.vocab).cuda()
    bad = good.clone()
    bad[1, 2] = 10 ** 6
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(200):
            m.prefill(bad, 9.0)
            with pytest.raises(adept.AdeptError) as ei:
                m.check()
            assert ei.value.status == 6
        m.prefill(good, 9.0)
        m.check()
    m.close()
