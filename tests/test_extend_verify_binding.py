"""What the binding of adept_extend_verify refuses before the library sees a pointer."""
import pytest
import torch


@pytest.fixture(scope="module")
def adept():
    from paper_2601_03700_gb300 import build
    build.build()
    import paper_2601_03700_gb300 as adept
    return adept


N, V, B = 6, 50, 3


def arguments():
    i, f = torch.zeros(N, dtype=torch.int32), torch.zeros(N)
    r = torch.zeros(B, dtype=torch.int32)
    return dict(tokens=i, u=f, logits_out=torch.zeros(N, V), accepted_out=r, next_token_out=r.clone(), draft=torch.zeros(N, V), temperature=torch.ones(B),
                forced=i.clone(), exit_layer_out=i.clone(), logprob_out=f.clone(), sim_out=torch.zeros(N, 4))


class Handle:
    """Stands for a model's handle: no call reaches the library."""
    vocab, n_layers = V, 4


def call(adept, lens=(2, 3, 1), **kw):
    a = {**arguments(), **kw}
    adept.adept_extend_verify(Handle(), list(lens), a.pop("tokens"), 0.9, **a)


@pytest.mark.parametrize("name", [k for k in arguments()])
def test_types_and_strides(adept, name):
    t = arguments()[name]
    bad = [t.double(), t.new_zeros((2 * t.shape[0],) + t.shape[1:])[::2]]
    if name == "draft":   # (its rows may lie apart)
        bad = [t.double(), t.half(), t[None], t.new_zeros(V, N).T]
    for x in bad:
        with pytest.raises(ValueError):
            call(adept, **{name: x})


@pytest.mark.parametrize("name", [k for k in arguments()])
def test_too_few_rows(adept, name):
    with pytest.raises(adept.AdeptError) as ei:
        call(adept, **{name: arguments()[name][:-1]})
    assert ei.value.status == 3


def test_too_few_columns(adept):
    for name, bad in (("logits_out", torch.zeros(N, V - 1)), ("sim_out", torch.zeros(N, 3))):
        with pytest.raises(adept.AdeptError) as ei:
            call(adept, **{name: bad})
        assert ei.value.status == 3
    for bad in (torch.zeros(N, V - 1), torch.zeros(N, V + 8)[:, :V - 1]):   # (the second's rows as far apart as the vocabulary)
        with pytest.raises(adept.AdeptError) as ei:
            call(adept, draft=bad)
        assert ei.value.status == 1


def test_no_gpu(adept):
    for kw in ({}, dict(lens=(1, 1, 1)), dict(tokens=torch.zeros(2, 3, dtype=torch.int32))):   # (buffers for more; tokens in any shape)
        with pytest.raises(ValueError, match="GPU"):
            call(adept, **kw)


def test_another_device(adept):
    with pytest.raises(ValueError, match="on cpu"):
        call(adept, u=torch.zeros(N, device="meta"))
    with pytest.raises(ValueError, match="on cpu"):
        call(adept, draft=torch.zeros(N, V, device="meta"))

