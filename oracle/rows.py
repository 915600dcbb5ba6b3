"""64-bit definitions of the operators on rows of logits, with the gradients taken by differentiating
them (torch float64 on the CPU).  Test side only: shares nothing with the CUDA library.

Every function takes logits as [n, V] of any float type and returns float64 tensors.  Besides outputs and
gradients the results carry ``scale`` [n, V]: the size of the terms a gradient entry is made of, which is
what its rounding errors are proportional to.
"""
from __future__ import annotations

import math
from types import SimpleNamespace

import torch

TAIL_FLOOR = 2.0 ** -20


def top_logits(x, k, T):
    """-> values [n, k] (-inf absent), ids [n, k] (-1 absent), lse [n]"""
    n, V = x.shape
    z = x.double()
    vals, ids = torch.full((n, k), -math.inf, dtype=torch.float64), torch.full((n, k), -1, dtype=torch.int64)
    for r in range(n):
        order = sorted(range(V), key=lambda v: (-float(z[r, v]), v)) if V <= 64 else torch.sort(z[r], descending=True, stable=True).indices.tolist()
        order = [v for v in order[:k] if z[r, v] > -math.inf]
        ids[r, :len(order)] = torch.tensor(order, dtype=torch.int64)
        vals[r, :len(order)] = z[r, order]
    return vals, ids, torch.logsumexp(z / _col(T), 1)


def _col(T):
    return T.double().view(-1, 1) if isinstance(T, torch.Tensor) else T


def _logits(x):
    return x.detach().double().clone().requires_grad_(True)


def _grad(scalar, z, dead):
    (g,) = torch.autograd.grad(scalar, z)
    return torch.where(dead, 0.0, g)


def _token_terms(z, tok, T):
    ls = torch.log_softmax(z / _col(T), 1)
    logp = ls.gather(1, tok.clamp(min=0).view(-1, 1)).view(-1)
    fin = torch.isfinite(ls)
    safe = torch.where(fin, ls, 0.0)
    H = -(torch.where(fin, ls.exp(), 0.0) * safe).sum(1)
    return ls, logp, H


def _token_scale(ls, H, tok, T, g, h):
    q = ls.exp()
    lq = torch.where(q > 0, ls, 0.0).abs()
    s = q * (g.abs().view(-1, 1) + h.abs().view(-1, 1) * (lq + H.view(-1, 1) + 1.0))
    s = s.scatter_add(1, tok.clamp(min=0).view(-1, 1), g.abs().view(-1, 1))
    return (s / _col(T)).detach()


def token_logprobs(x, tok, T, d_logp=None, d_entropy=None):
    z = _logits(x)
    on = tok >= 0
    tok = torch.where(on, tok.long(), x.float().argmax(1))     # rows left out: any usable token, discarded below
    ls, logp, H = _token_terms(z, tok, T)
    out = SimpleNamespace(logp=torch.where(on, logp, 0.0).detach(), entropy=torch.where(on, H, 0.0).detach())
    if d_logp is not None:
        g = torch.where(on, d_logp.double(), 0.0)
        h = torch.where(on, d_entropy.double(), 0.0) if d_entropy is not None else torch.zeros_like(g)
        scalar = (torch.where(g != 0, logp, 0.0) * g).sum() + (torch.where(h != 0, H, 0.0) * h).sum()
        out.grad = _grad(scalar, z, torch.isinf(x) & (h != 0).view(-1, 1))
        out.scale = _token_scale(ls, H, tok, T, g, h)
    return out


def policy(x, tok, T, old, adv, ref=None, clip_low=0.2, clip_high=0.2, kl_coef=0.0, entropy_coef=0.0, weight=None):
    z = _logits(x)
    on = tok >= 0
    tok = torch.where(on, tok.long(), x.float().argmax(1))     # rows left out: any usable token, discarded below
    ls, logp, H = _token_terms(z, tok, T)
    rho = (logp - old.double()).exp()
    A = adv.double()
    loss = -torch.minimum(rho * A, rho.clamp(1 - clip_low, 1 + clip_high) * A)
    kl = torch.zeros_like(loss)
    if ref is not None:
        d = ref.double() - logp
        kl = d.exp() - d - 1
        loss = loss + kl_coef * kl
    if entropy_coef != 0.0:
        loss = loss - entropy_coef * H
    w = torch.ones_like(loss) if weight is None else weight.double()
    w = torch.where(on, w, 0.0).detach()
    loss = torch.where(on, loss, 0.0)
    out = SimpleNamespace(loss=loss.detach(), logp=torch.where(on, logp, 0.0).detach(), kl=torch.where(on, kl, 0.0).detach(),
                          entropy=torch.where(on, H, 0.0).detach())
    out.grad = _grad((loss * w).sum(), z, torch.isinf(x))
    with torch.no_grad():
        size = w.abs() * ((rho * A).abs() + (kl_coef * (1 + (ref.double() - logp).exp()) if ref is not None else 0.0))
        out.scale = _token_scale(ls.detach(), H.detach(), tok, T, size, w * entropy_coef)
        out.loss_scale = 1 + (rho * A).abs() + (kl_coef * (kl + (ref.double() - logp).abs() + 1) if ref is not None else 0.0) + abs(entropy_coef) * H
        out.kl_scale = (1 + (ref.double() - logp).exp()) if ref is not None else torch.ones_like(loss)
    return out


def distill(x, T, values, ids, lse=None, kind="forward_kl", mix=0.5, weight=None):
    n, V = x.shape
    z = _logits(x)
    here = (ids >= 0) & (values > -math.inf)
    on = here.any(1)
    at = ids.long().clamp(min=0)
    ls = torch.log_softmax(z / _col(T), 1)
    lq = torch.where(here, ls.gather(1, at), 0.0)
    inside = torch.zeros(n, V, dtype=torch.int64).scatter_add(1, at, here.long()) > 0
    rest = torch.where(inside, -math.inf, ls)
    has = torch.isfinite(rest).any(1)
    ln_rho = torch.logsumexp(torch.where(has.view(-1, 1), rest, 0.0), 1)
    ln_rho = torch.where(has, ln_rho, 0.0)
    rho = torch.where(has, ln_rho.exp(), 0.0)
    t = torch.where(here, values.double() / _col(T), -math.inf)
    t = t - (lse.double().view(-1, 1) if lse is not None else torch.logsumexp(torch.where(on.view(-1, 1), t, 0.0), 1, keepdim=True))
    lp = torch.where(here, t, 0.0)
    p, q = torch.where(here, lp.exp(), 0.0), torch.where(here, lq.exp(), 0.0)
    r = torch.zeros(n, dtype=torch.float64)
    if lse is not None:
        r = 1 - p.sum(1)
        r = torch.where(r < TAIL_FLOOR, torch.where(rho > 0, TAIL_FLOOR, 0.0), r).detach()
    ln_r = torch.where(r > 0, r, torch.ones_like(r)).log()
    if kind == "forward_kl":
        tail = torch.where(r > 0, torch.where(has, r * (ln_r - ln_rho), math.inf), 0.0)
        loss = torch.where(p > 0, p * (lp - lq), 0.0).sum(1) + tail
        g, gt = torch.where(here, -p / q, 0.0), torch.where(rho > 0, -r / rho, 0.0)
    elif kind == "reverse_kl":
        loss = torch.where(q > 0, q * (lq - lp), 0.0).sum(1) + torch.where(has, rho * (ln_rho - ln_r), 0.0)
        g, gt = torch.where(here & (q > 0), lq - lp, 0.0), torch.where(rho > 0, ln_rho - ln_r, 0.0)
    else:
        m, mt = mix * p + (1 - mix) * q, mix * r + (1 - mix) * rho
        lm, lmt = torch.where(m > 0, m, 1.0).log(), torch.where(mt > 0, mt, 1.0).log()
        loss = torch.where(p > 0, mix * p * (lp - lm), 0.0).sum(1) + torch.where(q > 0, (1 - mix) * q * (lq - lm), 0.0).sum(1)
        loss = loss + torch.where(r > 0, mix * r * (ln_r - lmt), 0.0) + torch.where(rho > 0, (1 - mix) * rho * (ln_rho - lmt), 0.0)
        g, gt = torch.where(here & (q > 0), (1 - mix) * (lq - lm), 0.0), torch.where(rho > 0, (1 - mix) * (ln_rho - lmt), 0.0)
    loss = torch.where(on, loss, 0.0)
    w = torch.ones(n, dtype=torch.float64) if weight is None else weight.double()
    w = torch.where(on, w, 0.0)
    out = SimpleNamespace(loss=loss.detach())
    finite = torch.isfinite(loss)
    out.grad = _grad((torch.where(finite, loss, 0.0) * w).sum(), z, torch.isinf(x) | ~on.view(-1, 1))
    with torch.no_grad():
        qg = torch.where(here, torch.where(q > 0, q * g.abs(), p if kind == "forward_kl" else 0.0), 0.0)
        cbar = qg.sum(1) + rho * gt.abs()
        per = ls.exp() * (gt.abs() + cbar + 1).view(-1, 1)
        per = torch.where(inside, 0.0, per).scatter_add(1, at, torch.where(here, qg + q * (cbar.view(-1, 1) + 1), 0.0))
        out.scale = per * w.abs().view(-1, 1) / _col(T)
        out.loss_scale = 1 + cbar + (p * lp.abs()).sum(1)
    return out
