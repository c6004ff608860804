"""The token that adept_verify_drafts draws where little of p is left to draw from: numbers u next to the borders between two tokens,
against the 64-bit statement."""
import math

import pytest
import torch

from serve_reference import logs, verify

import paper_2601_03700_gb300 as adept

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    adept.load_library()


def pair(kind, t, seed=90):
    """Logits of a target and of a draft that is the target but for noise, fp32.  eight: eight tokens, the first, hold half of both."""
    V, noise = {"few": (1 << 17, 2e-3), "eight": (1 << 17, 2e-3), "many": (32000, 1e-3), "small": (32000, 1e-4)}[kind]
    g = torch.Generator().manual_seed(seed)
    x = (3.0 * t if kind in ("many", "small") else 1.0) * torch.randn(V, generator=g).double()
    if kind == "eight":
        x[:8] = t * (torch.logsumexp(x / t, 0) - math.log(8)) + 0.3 * torch.randn(8, generator=g).double()
    p = x.float()
    return p, (p.double() + noise * torch.randn(V, generator=g).double()).float()


def next_to_borders(w, least, n):
    """n numbers u with u + 2^-25 next to a border of w's cumulative shares, but no nearer than `least`."""
    c = w.cumsum(0) / w.sum()
    k = ((c - 2.0 ** -25) * 2.0 ** 24).round().clamp(0, 2 ** 24 - 1)
    off = (c - (k * 2.0 ** -24 + 2.0 ** -25)).abs()
    off[off < least] = 1.0
    return (k[off.argsort()[:n]] * 2.0 ** -24).float()


@pytest.mark.parametrize("t", [0.3, 0.7, 1.0])
@pytest.mark.parametrize("kind", ["few", "eight", "many", "small"])
def test_drawn_where_target_and_draft_are_close(kind, t):
    """max(p - q, 0) sums to s, 2^-8 to 2^-15; a weight is off by 2^-39 or so, every one by its own, so that those of a row's sums
    average to 2^-40 of p at most, 2^-40 / s of what is drawn from: borders are that far from u, or farther."""
    t = float(torch.tensor(t).float())
    p, q = pair(kind, t)
    w = (logs(p, t).exp() - logs(q, t).exp()).clamp(min=0)
    s = float(w.sum())
    assert 2.0 ** -15 < s < 2.0 ** -6
    n = 64
    x = int((logs(q, t) - logs(p, t)).argmax())   # the draft that q gives more than p: refused by a number next to 1
    u = torch.full((2 * n,), 1 - 2.0 ** -24)
    u[1::2] = next_to_borders(w, 2.0 ** -40 / s, n)
    start = list(range(0, 2 * n + 1, 2))
    tokens = torch.tensor([0, x] * n, dtype=torch.int32)
    target, draft = (v.expand(2 * n, -1).contiguous() for v in (p, q))
    acc, nxt = (torch.full((n,), -7, dtype=torch.int32, device="cuda") for _ in range(2))
    adept.adept_verify_drafts(target.cuda(), draft.cuda(), tokens.cuda(), torch.tensor(start, dtype=torch.int32).cuda(), u.cuda(), acc, nxt,
                              temperature=torch.full((n,), t).cuda())
    c = w.cumsum(0)
    want = [int((c <= (float(v) + 2.0 ** -25) * s).sum()) for v in u[1::2]]
    assert verify(target[:2], draft[:2], [0, x], [0, 2], u[:2], [t])[1] == want[:1]
    assert not acc.any()
    assert nxt.tolist() == want
