"""What the cache's Python calls refuse before anything is launched: no device is touched."""
import pytest
import torch

import paper_2512_13194_b200 as ears
from paper_2512_13194_b200 import sampler as module


@pytest.mark.parametrize("bad", [torch.zeros(2, dtype=torch.int32), torch.zeros(3), torch.zeros(3, 1, dtype=torch.int32),
                                 torch.zeros(3, dtype=torch.int16), torch.zeros(1, dtype=torch.int32).expand(3)])
def test_a_step_with_an_unusable_start_is_refused_before_it_begins(monkeypatch, bad):
    steps = []

    def verify(*args, **kwargs):
        steps.append(args)
        return torch.tensor([4, 0, -1], dtype=torch.int32), torch.zeros(3, 6, dtype=torch.int32)

    monkeypatch.setattr(module.binding, "verify", verify)
    sampler = ears.EarsSampler(1.0, 0.1, seed=3, first_offset=7)
    target, draft, tokens = torch.zeros(3, 6, 11), torch.zeros(3, 5, 11), torch.zeros(3, 5, dtype=torch.int32)
    with pytest.raises(ValueError):
        sampler(target, draft, tokens, kv_start=bad)
    assert not steps and sampler.offset == 7 and sampler.steps == 0
    start = torch.tensor([10, 20, 30])
    sampler(target, draft, tokens, kv_start=start)
    assert start.tolist() == [15, 21, 30] and sampler.offset == 8


def test_advance_refuses_lengths_that_are_no_integers():
    start = torch.zeros(3, dtype=torch.int32)
    for bad in (torch.zeros(3), torch.zeros(3, dtype=torch.bool)):
        with pytest.raises((TypeError, ValueError)):
            ears.kv_advance(start, bad)
    with pytest.raises(ValueError):
        ears.kv_advance(start[:1].expand(3), torch.zeros(3, dtype=torch.int32))
    assert ears.kv_advance(start, torch.tensor([1, 0, -1], dtype=torch.int16)).tolist() == [2, 1, 0]
