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


def drawn_without_probabilities(target, x, u):
    """The token behind a refused draft x of one row, for every number in u."""
    n = len(u)
    acc, nxt = (torch.full((n,), -7, dtype=torch.int32, device="cuda") for _ in range(2))
    both = torch.full((2 * n,), 1 - 2.0 ** -24)
    both[1::2] = torch.tensor(u)
    adept.adept_verify_drafts(target.expand(2 * n, -1).contiguous().cuda(), None, torch.tensor([0, x] * n, dtype=torch.int32).cuda(),
                              torch.arange(0, 2 * n + 1, 2, dtype=torch.int32).cuda(), both.cuda(), acc, nxt)
    assert not acc.any()
    return nxt.tolist()


@pytest.mark.parametrize("V", [32000, 50257])
@pytest.mark.parametrize("lg", [-19.9, -18.0, -14.0, -9.0])
def test_a_refused_draft_that_has_nearly_all_of_the_target(V, lg):
    """All but s = 2^lg of p is the draft's.  Token 10, a few places before it, has 2^-24.2 of the rest: u = 0, which stands for 2^-25, draws
    it, and no other u does."""
    x, s = 50, 2.0 ** lg
    g = torch.Generator().manual_seed(91)
    w = torch.rand(V, generator=g, dtype=torch.float64) * (torch.rand(V, generator=g) < 0.01)
    w[:4000] = 0.0
    w *= s / w.sum()
    w[10], w[x] = s * 2.0 ** -24.2, 1 - s
    target = w.log().float()
    assert float(logs(target, 1)[x]) < math.log(1 - 2.0 ** -24)   # refused
    u = [0.0, 2.0 ** -24, 0.25, 0.5, 0.75, 1 - 2.0 ** -24]
    want = [verify(target.expand(2, V), None, [0, x], [0, 2], torch.tensor([1 - 2.0 ** -24, v]))[1][0] for v in u]
    assert want[0] == 10 and 10 not in want[1:]
    assert drawn_without_probabilities(target, x, u) == want
