"""The 64-bit definitions of the 4-bit cache against plain statements of the same thing."""
import math

import pytest
import torch

from oracle import kv as O


@pytest.mark.parametrize("scale", [1.0, 1e-30, 1e30, 300.0])
def test_a_value_comes_back_within_half_a_step(scale):
    g = torch.Generator().manual_seed(3)
    x = (torch.randn(50, 128, generator=g) + torch.randn(50, 1, generator=g) * 20) * scale
    codes, params = O.quantise(x)
    assert codes.shape == (50, 64) and params.shape == (50, 2, 2)
    off = (O.values(codes, params) - x.double()).abs().unflatten(-1, (-1, 64))
    step = params[..., :1].double()
    low = params[..., 1:].double().abs()
    assert (off <= step / 2 + 2.0 ** -24 * (x.double().abs().unflatten(-1, (-1, 64)) + low)).all()
    assert (params[..., 1].double() <= x.unflatten(-1, (-1, 64)).amin(-1).double()).all()


def test_constant_and_unusable_groups():
    x = torch.zeros(5, 64)
    x[1] = 1.5
    x[2, 7] = math.nan
    x[3, 9] = -math.inf
    x[4, 0], x[4, 1] = 3e38, -3e38
    v = O.values(*O.quantise(x))
    assert torch.equal(v[:2], x[:2].double()) and v[2:].isnan().all()


def test_ties_go_to_the_even_code():
    x = torch.zeros(1, 64)
    x[0, :5] = torch.tensor([0.5, 1.5, 2.5, 7.5, 15.0])
    codes, params = O.quantise(x)
    assert params[0, 0].tolist() == [1.0, 0.0]
    assert O.values(codes, params)[0, :5].tolist() == [0.0, 2.0, 2.0, 8.0, 15.0]


def test_attention_is_softmax_over_what_is_seen():
    g = torch.Generator().manual_seed(5)
    kv = torch.randn(4, 2, 2, 16, 64, generator=g)
    codes, params = O.quantise(kv)
    pages = torch.tensor([[2, 0, 3]])
    dense = O.tokens_of(codes, params, pages, 0, 40)
    q = torch.randn(1, 3, 4, 64, generator=g)
    got = O.attention(q, codes, params, pages, torch.tensor([37]), torch.tensor([2]), window=5, sinks=2)
    for i in range(2):
        p = 37 + i
        see = [t for t in range(p + 1) if t < 2 or t > p - 5]
        for n in range(4):
            s = [float(q[0, i, n].double() @ dense[0, n // 2, t]) / 8 for t in see]
            top = max(s)
            e = [math.exp(x - top) for x in s]
            want = sum(w * dense[1, n // 2, t] for w, t in zip(e, see)) / sum(e)
            assert (got.out[0, i, n] - want).abs().max() < 1e-12
            assert abs(got.lse[0, i, n] - (top + math.log(sum(e)))) < 1e-12
    assert (got.out[0, 2] == 0).all() and (got.lse[0, 2] == -math.inf).all()
