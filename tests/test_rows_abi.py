"""Refusals of the operators on rows of logits that the host decides: no device is touched."""
import ctypes
import types

import pytest
import torch

import paper_2512_13194_b200 as ears

BUF = (ctypes.c_float * 4096)()
P = (ctypes.addressof(BUF) + 255) // 256 * 256
FAR = P + 8192


def rows(dtype=0, x=P, B=2, R=3, V=8, sb=24, sr=8, T=1.0, seq=None):
    return (dtype, x, B, R, V, sb, sr, T, seq)


def lib():
    return ears.load_library()


CALLS = {
    "top": lambda h, k=4, v=P, i=P, l=P, acc=None, st=None: lib().ears_top_logits(*h, acc, k, v, i, l, st, None),
    "token": lambda h, tok=P, out=P, H=None, saved=None, st=None: lib().ears_token_logprobs(*h, tok, out, H, saved, st, None),
    "token_backward": lambda h, tok=P, saved=P, dl=P, dh=None, g=FAR, gsb=24, gsr=8: lib().ears_token_logprobs_backward(
        *h, tok, saved, dl, dh, g, gsb, gsr, None, None),
    "token_step": lambda h, tok=P, dl=P, dh=None, out=P, H=None, g=FAR, gsb=24, gsr=8: lib().ears_token_logprobs_step(
        *h, tok, dl, dh, out, H, g, gsb, gsr, None, None),
    "policy": lambda h, tok=P, old=P, ref=None, adv=P, lo=0.2, hi=0.2, kl=0.0, ent=0.0, out=P, saved=None: lib().ears_policy_loss(
        *h, tok, old, ref, adv, lo, hi, kl, ent, out, None, None, None, saved, None, None),
    "policy_backward": lambda h, tok=P, old=P, ref=None, adv=P, lo=0.2, hi=0.2, kl=0.0, ent=0.0, saved=P, dl=P, g=FAR, gsb=24,
    gsr=8: lib().ears_policy_backward(*h, tok, old, ref, adv, lo, hi, kl, ent, saved, dl, g, gsb, gsr, None, None),
    "policy_step": lambda h, tok=P, old=P, ref=None, adv=P, lo=0.2, hi=0.2, kl=0.0, ent=0.0, w=None, out=P, g=FAR, gsb=24,
    gsr=8: lib().ears_policy_step(*h, tok, old, ref, adv, lo, hi, kl, ent, w, out, None, None, None, g, gsb, gsr, None, None),
    "distill": lambda h, k=4, v=P, i=P, l=P, kind=0, mix=0.5, out=P, saved=None: lib().ears_distill_loss(
        *h, k, v, i, l, kind, mix, out, saved, None, None),
    "distill_backward": lambda h, k=4, v=P, i=P, l=P, kind=0, mix=0.5, saved=P, dl=P, g=FAR, gsb=24, gsr=8: lib().ears_distill_backward(
        *h, k, v, i, l, kind, mix, saved, dl, g, gsb, gsr, None, None),
    "distill_step": lambda h, k=4, v=P, i=P, l=P, kind=0, mix=0.5, w=None, out=P, g=FAR, gsb=24, gsr=8: lib().ears_distill_step(
        *h, k, v, i, l, kind, mix, w, out, g, gsb, gsr, None, None),
}


@pytest.mark.parametrize("name", sorted(CALLS))
def test_rows_are_checked_by_every_entry_point(name):
    call = CALLS[name]
    assert call(rows(x=None)) == -1
    assert call(rows(dtype=5)) == -3
    assert call(rows(B=0)) == -2 and call(rows(R=0)) == -2 and call(rows(V=0)) == -2 and call(rows(V=2**30 + 1)) == -2
    assert call(rows(B=2**20, R=2**10)) == -2                    # more CTAs than a launch can hold
    assert call(rows(sb=-1)) == -2 and call(rows(sr=-8)) == -2
    assert call(rows(sb=2**62)) == -2
    for T in (0.0, -1.0, float("nan"), float("inf"), 1e-39):
        assert call(rows(T=T)) == -3
    assert call(rows(x=P + 2)) == -4 and call(rows(dtype=1, x=P + 1)) == -4
    assert call(rows(seq=P + 2)) == -4


@pytest.mark.parametrize("name", [n for n in sorted(CALLS) if "step" in n or "backward" in n])
def test_gradient_rows_are_checked(name):
    call = CALLS[name]
    assert call(rows(), g=None) == -1
    assert call(rows(), g=FAR + 2) == -4
    assert call(rows(), gsb=-24) == -2 and call(rows(), gsr=-8) == -2
    assert call(rows(), gsr=7) == -2 and call(rows(), gsb=23) == -2      # rows that overlap
    assert call(rows(), gsb=0) == -2 and call(rows(), gsr=0) == -2
    assert call(rows(sb=0), g=P, gsb=0) == -2                             # a broadcast input cannot take its gradient
    assert call(rows(), g=P + 4) == -3 and call(rows(), g=P - 4) == -3    # overlaps the logits in part
    assert call(rows(), g=P, gsb=48) == -3                                # same start, other rows


def test_operator_arguments_are_checked():
    h = rows()
    top, token, policy, distill = CALLS["top"], CALLS["token"], CALLS["policy"], CALLS["distill"]
    for bad in ("v", "i", "l"):
        assert top(h, **{bad: None}) == -1 and top(h, **{bad: P + 1}) == -4
    assert top(h, k=0) == -2 and top(h, k=129) == -2 and top(h, acc=P + 2) == -4 and top(h, st=P + 1) == -4
    assert token(h, tok=None) == -1 and token(h, out=None) == -1 and token(h, saved=P + 4) == -4 and token(h, H=P + 1) == -4
    assert CALLS["token_backward"](h, saved=None) == -1 and CALLS["token_backward"](h, dl=None) == -1
    for bad in ("tok", "old", "adv", "out"):
        assert policy(h, **{bad: None}) == -1
    assert policy(h, lo=-0.1) == -3 and policy(h, lo=1.5) == -3 and policy(h, hi=float("inf")) == -3 and policy(h, hi=-1.0) == -3
    assert policy(h, kl=0.1) == -3 and policy(h, kl=-0.1, ref=P) == -3 and policy(h, kl=float("nan"), ref=P) == -3
    assert policy(h, ent=float("inf")) == -3
    for bad in ("v", "i", "out"):
        assert distill(h, **{bad: None}) == -1
    assert distill(h, k=0) == -2 and distill(h, k=129) == -2
    assert distill(rows(V=2**20 + 1, sr=2**21, sb=2**23)) == -2
    assert distill(h, kind=3) == -3 and distill(h, kind=-1) == -3
    assert distill(h, kind=1, l=None) == -3
    for mix in (0.0, 1.0, -0.2, float("nan")):
        assert distill(h, kind=2, mix=mix) == -3
    for c in (3, 32, -1):
        assert lib().ears_set_row_cluster(c) == -3
    assert lib().ears_set_row_cluster(0) == 0


def test_binding_refuses_what_is_not_on_a_device():
    x = torch.zeros(2, 8)
    with pytest.raises(ValueError):
        ears.top_logits(x, 2)
    with pytest.raises(TypeError):
        ears.token_logprobs(x.double(), torch.zeros(2, dtype=torch.int32))
    with pytest.raises(ValueError):
        ears.distill_step(x, ears.TopLogits(x[:, :2], torch.zeros(2, 2, dtype=torch.int32), None))


def test_a_stream_of_another_device_is_refused():
    logits = types.SimpleNamespace(get_device=lambda: 1)
    stream = types.SimpleNamespace(device_index=0)
    for call in (lambda: ears.top_logits(logits, 2, stream=stream), lambda: ears.top_logits(logits=logits, k=2, stream=stream)):
        with pytest.raises(ValueError, match="stream"):
            call()


def test_the_sampler_refuses_a_teacher_that_cannot_be_kept():
    for k in (-1, 129):
        with pytest.raises(ValueError):
            ears.EarsSampler(teacher_k=k)
    assert ears.EarsSampler(teacher_k=128).teacher_k == 128
