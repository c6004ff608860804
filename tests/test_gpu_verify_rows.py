"""adept_verify_drafts where d_start does not ascend: rows that two sequences name belong to the first."""
import pytest
import torch

from serve_reference import verify

import paper_2601_03700_gb300 as adept

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    adept.load_library()


@pytest.mark.parametrize("temp", [[1.0, 1.0, 1.0], [0.0, 1.0, 1.0], [0.5, 1.0, 0.0], [-1.0, 1.0, 1.0]])
@pytest.mark.parametrize("start", [[0, 4, 2, 8], [0, 6, 3, 6], [4, 6, 0, 8], [2, 4, 4, 3], [0, 8, 8, 0]])
def test_rows_that_two_sequences_name(start, temp):
    """A sequence that meets a row of an earlier one, or whose rows end before they begin, is left out; the others are as they are alone."""
    V, n = 700, 8
    g = torch.Generator().manual_seed(start[1] * 8 + start[2])
    target = 2.0 * torch.randn(n, V, generator=g)
    draft = target + 0.3 * torch.randn(n, V, generator=g)
    tokens = torch.cat([torch.zeros(1, dtype=torch.int64), draft.argmax(1)])[:n].int()
    u = torch.rand(n, generator=g)
    ws = adept.verify_workspace(n)
    ws.fill_(0x3f)   # (any contents)
    acc, nxt = (torch.full((3,), -7, dtype=torch.int32, device="cuda") for _ in range(2))
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    adept.adept_verify_drafts(target.cuda(), draft.cuda(), tokens.cuda(), torch.tensor(start, dtype=torch.int32).cuda(), u.cuda(), acc, nxt,
                              temperature=torch.tensor(temp).cuda(), workspace=ws, err=err)
    taken = set()
    for b in range(3):
        s, e = start[b], start[b + 1]
        want = (-1, -1) if e < s else (0, -1)
        if e > s and temp[b] >= 0:
            k, x, _ = verify(target[s:e], draft[s:e], tokens[s:e].tolist(), [0, e - s], u[s:e], [temp[b]])
            want = (-1, -1) if taken & set(range(s, s + k[0] + 1)) else (k[0], x[0])
        elif e > s:
            want = (-1, -1)
        taken |= set(range(s, e))
        assert (acc[b].item(), nxt[b].item()) == want, b
    with pytest.raises(adept.AdeptError) as ei:
        adept.adept_error_check(err)
    assert ei.value.status == 6
