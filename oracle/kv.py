"""The key/value cache held in 4 bits from its definition, in 64 bits where the format does not fix 32 (torch on the CPU).

A group x of 64: m = min x rounded down to bfloat16, s = (max x - m) r in 32 bits, r the 32-bit number nearest to 1 / 15, rounded up
to bfloat16 and at least 2^-126, c = (x - m) / s, the difference rounded to 32 bits, to the nearest whole number, ties to even; a code stands for m + s c.
"""
from __future__ import annotations

import math
from typing import NamedTuple

import torch

GROUP = 64


def _neighbour(x, direction):
    """x (32 bits) as the nearest bfloat16 in the direction, as 32 bits."""
    y = x.bfloat16()
    off = y.float() > x if direction < 0 else y.float() < x
    return torch.where(off, torch.nextafter(y, torch.full_like(y, direction * math.inf)), y).float()


def quantise(x):
    """[..., D] -> (codes uint8 [..., D/2], params bfloat16 [..., D/64, 2])"""
    x = x.float().unflatten(-1, (-1, GROUP))
    m = _neighbour(x.amin(-1), -1)
    s = _neighbour((x.amax(-1) - m) * torch.tensor(1 / 15, dtype=torch.float32), 1)
    usable = torch.isfinite(s) & torch.isfinite(m)
    s = torch.where(usable, s.clamp(min=2.0 ** -126), torch.nan)
    m = torch.where(usable, m, torch.nan)
    c = ((x - m.unsqueeze(-1)).double() / s.double().unsqueeze(-1)).round()
    c = torch.where(usable.unsqueeze(-1), c, 0.0).to(torch.uint8).flatten(-2)
    assert int(c.max()) <= 15
    return c[..., ::2] + 16 * c[..., 1::2], torch.stack([s, m], -1).bfloat16()


def values(codes, params):
    """-> [..., D] float64"""
    c = torch.stack([codes % 16, codes // 16], -1).flatten(-2).double().unflatten(-1, (-1, GROUP))
    return (params[..., 1:].double() + params[..., :1].double() * c).flatten(-2)


def tokens_of(codes, params, pages, b, n):
    """Keys and values [2, H, n, D] float64 of the first n tokens of sequence b."""
    page = codes.shape[3]
    out = [values(codes[int(pages[b, t // page]), :, :, t % page], params[int(pages[b, t // page]), :, :, t % page]) for t in range(n)]
    return torch.stack(out, 2) if n else torch.zeros(2, codes.shape[2], 0, codes.shape[4] * 2, dtype=torch.float64)


class Attention(NamedTuple):
    out: torch.Tensor       # [B, Q, HQ, D]
    lse: torch.Tensor       # [B, Q, HQ]
    weighted: torch.Tensor  # sum_t p_t s_t c_t: what a relative error of the weights enters times
    spread: torch.Tensor    # 7.5 sum_t p_t s_t: the same for codes less their middle, at the most
    reach: torch.Tensor     # max_t |v_t - out| over the tokens seen: what an error of the weights can move a result by
    size: torch.Tensor      # [B, Q, HQ] max_t of sum_d |q| (|m| + s c) scale log2(e): the size of what the scores sum
    tiny: torch.Tensor      # [B, Q, HQ] tokens seen times the largest scale among them


def attention(q, codes, params, pages, start, counts=None, scale=None, window=0, sinks=0):
    B, Q, HQ, D = q.shape
    H = codes.shape[2]
    scale = D ** -0.5 if scale is None else scale
    out, weighted, spread, reach = (torch.zeros(B, Q, HQ, D, dtype=torch.float64) for _ in range(4))
    lse = torch.full((B, Q, HQ), -math.inf, dtype=torch.float64)
    size, tiny = torch.zeros(B, Q, HQ, dtype=torch.float64), torch.zeros(B, Q, HQ, dtype=torch.float64)
    for b in range(B):
        n = Q if counts is None else max(0, min(Q, int(counts[b])))
        if n == 0:
            continue
        last = int(start[b]) + n
        page = codes.shape[3]
        ids = pages[b, : -(-last // page)].long()
        c, m = (x[ids].permute(1, 2, 0, 3, *range(4, x.dim())).flatten(2, 3)[:, :, :last] for x in (codes, params))
        kv = values(c, m)                                                             # [2, H, last, D]
        least = m[..., 1].double().repeat_interleave(GROUP, -1)
        for i in range(n):
            p = int(start[b]) + i
            t = torch.arange(last)
            see = t <= p
            if window:
                see &= (t > p - window) | (t < sinks)
            k, v, lo = kv[0][:, see], kv[1][:, see], least[:, :, see]
            x = q[b, i].double().view(H, -1, D)
            s = x @ k.transpose(1, 2) * scale
            w = s.softmax(-1)
            r = w @ v
            out[b, i], lse[b, i] = r.reshape(HQ, D), s.logsumexp(-1).reshape(HQ)
            weighted[b, i] = (w @ (v - lo[1])).reshape(HQ, D)
            spread[b, i] = 7.5 * (w @ m[1][:, see][..., 0].double().repeat_interleave(GROUP, -1)).reshape(HQ, D)
            reach[b, i] = torch.maximum(v.amax(1, keepdim=True) - r, r - v.amin(1, keepdim=True)).reshape(HQ, D)
            size[b, i] = (x.abs() @ (lo[0].abs() + (k - lo[0])).transpose(1, 2)).amax(-1).reshape(HQ) * abs(scale) / math.log(2)
            tiny[b, i] = (len(v[0]) * m[1][:, see][..., 0].double().amax((1, 2))).repeat_interleave(HQ // H)
    return Attention(out, lse, weighted, spread, reach, size, tiny)
