"""Pins of the 64-bit definitions of the operators on rows of logits: closed forms, library functions and
differences.  No GPU."""
import math

import pytest
import torch

from oracle import rows as R


def _case(n=5, V=11, seed=0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(n, V, generator=g, dtype=torch.float64) * 2
    tok = torch.randint(0, V, (n,), generator=g)
    return g, x, tok


def _differences(f, x, grad, places):
    for r, v in places:
        h = 1e-5
        hi, lo = x.clone(), x.clone()
        hi[r, v] += h
        lo[r, v] -= h
        assert abs((f(hi) - f(lo)) / (2 * h) - grad[r, v]) < 1e-7 * max(1.0, abs(float(grad[r, v])))


def test_top_logits_orders_ties_by_index_and_skips_masks():
    x = torch.tensor([[1.0, 3.0, 3.0, -math.inf, 2.0], [-0.0, 0.0, -math.inf, -1.0, 0.0]])
    v, i, lse = R.top_logits(x, 5, 1.0)
    assert i.tolist() == [[1, 2, 4, 0, -1], [0, 1, 4, 3, -1]]
    assert v[0].tolist() == [3.0, 3.0, 2.0, 1.0, -math.inf]
    assert torch.allclose(lse, torch.logsumexp(x.double(), 1))


def test_token_logprobs_match_cross_entropy_and_differences():
    g, x, tok = _case()
    T = 0.7
    o = R.token_logprobs(x, tok, T, torch.ones(5), torch.full((5,), 0.3))
    assert torch.allclose(o.logp, -torch.nn.functional.cross_entropy(x / T, tok, reduction="none"))
    assert torch.allclose(o.entropy, torch.distributions.Categorical(logits=x / T).entropy())
    f = lambda y: float((lambda q: (q.logp + 0.3 * q.entropy).sum())(R.token_logprobs(y, tok, T)))
    _differences(f, x, o.grad, [(0, 0), (1, int(tok[1])), (4, 10)])


def test_policy_gradient_stops_at_the_clip_and_matches_differences():
    g, x, tok = _case(n=6)
    logp = R.token_logprobs(x, tok, 1.0).logp
    ratio = torch.tensor([1.05, 0.9, 1.5, 1.5, 0.5, 0.5])
    adv = torch.tensor([1.0, -1.0, 1.0, -1.0, 1.0, -1.0])
    old = logp - ratio.log()
    o = R.policy(x, tok, 1.0, old, adv, clip_low=0.2, clip_high=0.28)
    zero = (o.grad.abs().sum(1) < 1e-12).tolist()
    assert zero == [False, False, True, False, False, True]
    want = -torch.minimum(ratio.double() * adv.double(), ratio.clamp(0.8, 1.28).double() * adv.double())
    assert torch.allclose(o.loss, want, atol=1e-6)
    ref = logp + 0.3
    kw = dict(ref=ref, kl_coef=0.1, entropy_coef=0.05)
    o = R.policy(x, tok, 1.0, old, adv, **kw)
    assert torch.allclose(o.kl, torch.full((6,), math.exp(0.3) - 0.3 - 1, dtype=torch.float64), atol=1e-6)
    f = lambda y: float(R.policy(y, tok, 1.0, old, adv, **kw).loss.sum())
    _differences(f, x, o.grad, [(0, 1), (1, int(tok[1])), (3, 2)])


@pytest.mark.parametrize("kind", ["forward_kl", "reverse_kl", "jsd"])
@pytest.mark.parametrize("tail", [True, False])
def test_distill_against_the_full_distribution_and_differences(kind, tail):
    if kind == "reverse_kl" and not tail:
        return
    g, t, _ = _case(n=4, V=9, seed=3)
    x = t + torch.randn(4, 9, generator=g, dtype=torch.float64)
    T, k = 1.3, 4
    vals, ids, lse = R.top_logits(t, k, T)
    kw = dict(lse=lse if tail else None, kind=kind, mix=0.3)
    o = R.distill(x, T, vals, ids, **kw)
    # the k + 1 outcomes written out
    p = torch.softmax(t / T, 1)
    q = torch.softmax(x / T, 1)
    pk, qk = p.gather(1, ids), q.gather(1, ids)
    if tail:
        pk = torch.cat([pk, 1 - pk.sum(1, keepdim=True)], 1)
    else:
        pk = torch.cat([pk / pk.sum(1, keepdim=True), torch.zeros(4, 1, dtype=torch.float64)], 1)
    qk = torch.cat([qk, 1 - qk.sum(1, keepdim=True)], 1)
    kl = lambda a, b: torch.where(a > 0, a * (a / b).log(), 0.0).sum(1)
    m = 0.3 * pk + 0.7 * qk
    want = {"forward_kl": lambda: kl(pk, qk), "reverse_kl": lambda: kl(qk, pk), "jsd": lambda: 0.3 * kl(pk, m) + 0.7 * kl(qk, m)}[kind]()
    assert torch.allclose(o.loss, want, atol=1e-9)
    f = lambda y: float(R.distill(y, T, vals, ids, **kw).loss.sum())
    _differences(f, x, o.grad, [(0, int(ids[0, 0])), (1, int(ids[1, -1])), (2, 0), (3, 5), (2, 8)])
    assert torch.allclose(o.grad.sum(1), torch.zeros(4, dtype=torch.float64), atol=1e-12)


def test_whole_vocabulary_listed_is_the_ordinary_divergence():
    g, t, _ = _case(n=3, V=6, seed=5)
    x = t + 0.5 * torch.randn(3, 6, generator=g, dtype=torch.float64)
    vals, ids, lse = R.top_logits(t, 6, 1.0)
    o = R.distill(x, 1.0, vals, ids, lse=lse.float())
    want = torch.nn.functional.kl_div(torch.log_softmax(x, 1), torch.softmax(t, 1), reduction="none").sum(1)
    assert torch.allclose(o.loss, want, atol=2e-6)
