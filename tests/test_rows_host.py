"""What the Python side of the row operators hands to the library and keeps between calls: tensors on the CPU pass for
device tensors, and a stand-in for the library records its arguments and touches none of them."""
import ctypes
import gc
import shutil
import warnings
import weakref

import pytest
import torch

import paper_2512_13194_b200 as ears
from paper_2512_13194_b200 import rows


class Library:
    """Every entry point: records (name, arguments) and succeeds."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def entry(*args):
            self.calls.append((name, args))
            return 0
        return entry

    def last(self, name):
        return [args for n, args in self.calls if n == name][-1]


class NoPlainCalls:
    """The extension module when nothing is in its plain form."""

    def __getattr__(self, name):
        return lambda *args: None


@pytest.fixture
def lib(monkeypatch):
    fake = Library()
    monkeypatch.setattr(torch.Tensor, "get_device", lambda self: 0)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    monkeypatch.setattr(rows, "load_library", lambda: fake)
    monkeypatch.setattr(rows, "_plain_calls", NoPlainCalls)
    monkeypatch.setattr(rows, "_current_device", lambda: 0)
    monkeypatch.setattr(rows, "_raw_stream", lambda index: 0)
    return fake


N, V, K = 3, 16, 4
STATUS = -2                # place of the status word among every entry point's arguments


class Inputs:
    """One call's inputs besides the logits."""

    def __init__(self):
        self.tokens = torch.zeros(N, dtype=torch.int32)
        self.f = [torch.zeros(N) for _ in range(3)]
        self.teacher = ears.TopLogits(torch.zeros(N, K), torch.arange(K, dtype=torch.int32).repeat(N, 1), torch.zeros(N))


# name of the entry points -> (differentiable call, returning what backward starts from)
LOSSES = {
    "ears_token_logprobs": lambda x, i, **kw: ears.token_logprobs(x, i.tokens, **kw),
    "ears_policy": lambda x, i, **kw: ears.policy_loss(x, i.tokens, i.f[0], i.f[1], ref_logp=i.f[2], kl_coef=0.1, **kw).loss,
    "ears_distill": lambda x, i, **kw: ears.distill_loss(x, i.teacher, **kw),
}


def leaf():
    return torch.zeros(N, V).requires_grad_(True)


@pytest.mark.parametrize("name", sorted(LOSSES))
def test_the_status_word_lives_until_the_backward_pass_is_over(lib, name):
    x, status = leaf(), torch.zeros(1, dtype=torch.int32)
    out = LOSSES[name](x, Inputs(), status=status)
    place, held = status.data_ptr(), weakref.ref(status)
    del status
    gc.collect()
    assert held() is not None                       # its memory may not be handed out again
    out.sum().backward()
    assert lib.last(name + "_backward")[STATUS] == place
    del out
    gc.collect()
    assert held() is None


@pytest.mark.parametrize("name", sorted(LOSSES))
def test_a_changed_temperature_is_noticed_by_the_backward_pass(lib, name):
    T = torch.ones(1)                                # logits [R, V] are one sequence
    out = LOSSES[name](leaf(), Inputs(), seq_temperature=T)
    T.mul_(0.9)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        out.sum().backward()
    assert not any(n == name + "_backward" for n, _ in lib.calls)
    T = torch.ones(1)
    LOSSES[name](leaf(), Inputs(), seq_temperature=T).sum().backward()
    assert lib.last(name + "_backward")[8] == T.data_ptr()


@pytest.mark.parametrize("name", sorted(LOSSES))
@pytest.mark.parametrize("copied", [False, True])
def test_nothing_of_the_logits_size_outlives_the_backward_pass(lib, monkeypatch, name, copied):
    memory, contiguous = [], torch.Tensor.contiguous

    def watched(t):
        t = contiguous(t)
        memory.append(weakref.ref(t.untyped_storage()))
        return t
    x = leaf()
    y = x.t().contiguous().t() if copied else x * 1.0          # entries of a row apart: the call works on a copy
    memory.append(weakref.ref(y.untyped_storage()))
    monkeypatch.setattr(torch.Tensor, "contiguous", watched)
    out = LOSSES[name](y, Inputs())
    assert len(memory) == 1 + copied
    if copied:
        assert memory[1]() is not None
    del y
    out.sum().backward()
    gc.collect()
    assert out.grad_fn is not None                              # the loss is still there
    assert all(m() is None for m in memory[:1 + copied])


@pytest.mark.parametrize("name", sorted(LOSSES))
def test_saved_tensor_hooks_stand_between_the_passes(lib, name):
    """What the backward call reads is what the hooks hand back, the statistics among it."""
    back = []

    def unpack(t):
        back.append(t.clone())
        return back[-1]
    x, T = leaf(), torch.ones(1)
    with torch.autograd.graph.saved_tensors_hooks(lambda t: t.detach(), unpack):
        out = LOSSES[name](x, Inputs(), seq_temperature=T)
        out.sum().backward()
    places = {t.data_ptr() for t in back}
    args = lib.last(name + "_backward")
    assert args[1] in places and args[8] in places              # logits, temperatures
    assert sum(a in places for a in args) == len(back)


ALL_CALLS = dict(LOSSES, **{
    "ears_top_logits": lambda x, i: ears.top_logits(x, K),
    "ears_token_logprobs_step": lambda x, i: ears.token_logprobs_step(x, i.tokens, i.f[0]),
    "ears_policy_step": lambda x, i: ears.policy_step(x, i.tokens, i.f[0], i.f[1]),
    "ears_distill_step": lambda x, i: ears.distill_step(x, i.teacher),
})


@pytest.mark.parametrize("name", sorted(ALL_CALLS))
def test_forward_mode_derivatives_are_refused(lib, name):
    from torch.autograd import forward_ad
    call = ALL_CALLS[name]
    with forward_ad.dual_level():
        dual = lambda t: forward_ad.make_dual(t, torch.ones_like(t))
        with pytest.raises(NotImplementedError, match="forward-mode"):
            call(dual(torch.zeros(N, V)), Inputs())
        i = Inputs()
        i.f, i.teacher = [dual(t) for t in i.f], i.teacher._replace(values=dual(i.teacher.values))
        if name not in ("ears_top_logits", "ears_token_logprobs"):      # which take integers beside the logits
            with pytest.raises(NotImplementedError, match="forward-mode"):
                call(torch.zeros(N, V), i)
            if "distill" in name:
                i = Inputs()
                i.teacher = [dual(i.teacher.values), *i.teacher[1:]]    # the list as a plain list
                with pytest.raises(NotImplementedError, match="forward-mode"):
                    call(torch.zeros(N, V), i)
        assert not lib.calls
        call(torch.zeros(N, V), Inputs())                       # no tangent: as ever
        call(dual(torch.zeros(N, V)).detach(), Inputs())
        assert lib.calls


def entries(place, n, ctype):
    """What a recorded address holds (the tensor must still be alive)."""
    return list((ctype * n).from_address(place))


WIDE = [2**32 + 5, 2**31, -2**32 - 1, 2**63 - 1, -2**63, 2**32]


@pytest.mark.parametrize("dtype", [torch.int64, torch.uint64, torch.uint32])
def test_ids_that_32_bits_cannot_hold_do_not_become_others(lib, monkeypatch, dtype):
    wide = WIDE if dtype is torch.int64 else [2**32 - 1, 2**31 + 3] + ([2**64 - 1, 2**63 + 7] if dtype is torch.uint64 else [])
    n = len(wide) + 3
    t = torch.tensor(wide + [7, 15, 0], dtype=dtype)
    x, f = torch.zeros(n, V), torch.zeros(n)
    got = []

    def entry(*args):
        got.append(entries(args[9], n, ctypes.c_int32))
        return 0
    monkeypatch.setattr(lib, "ears_token_logprobs", entry, raising=False)
    ears.token_logprobs(x, t)
    monkeypatch.setattr(lib, "ears_policy_step", entry, raising=False)
    ears.policy_step(x, t, f, f)
    monkeypatch.setattr(lib, "ears_distill_step", lambda *args: got.append(entries(args[11], n, ctypes.c_int32)) or 0, raising=False)
    ears.distill_step(x, ears.TopLogits(torch.zeros(n, 1), t.view(n, 1), None))
    assert len(got) == 3
    for ids in got:
        assert ids[-3:] == [7, 15, 0]
        for i in ids[:-3]:
            assert i < -1 or i >= 2**30                         # neither left out nor an entry of any row


def test_lengths_that_32_bits_cannot_hold(lib, monkeypatch):
    got = []
    monkeypatch.setattr(lib, "ears_top_logits", lambda *args: got.extend(entries(args[9], 3, ctypes.c_int32)) or 0, raising=False)
    ears.top_logits(torch.zeros(3, 2, V), 2, accept_len=torch.tensor([1, 2**32 + 1, -2**33 - 1]))
    assert got[0] == 1 and got[1] >= 2 and got[2] < 0


def test_ids_in_narrow_types_and_their_refusals(lib, monkeypatch):
    got = []
    monkeypatch.setattr(lib, "ears_token_logprobs", lambda *args: got.append(entries(args[9], N, ctypes.c_int32)) or 0, raising=False)
    for dtype in (torch.int8, torch.int16, torch.int64, torch.uint8):
        ears.token_logprobs(torch.zeros(N, V), torch.tensor([3, 1, 2], dtype=dtype))
    assert got == [[3, 1, 2]] * 4
    for dtype in (torch.float32, torch.bool, torch.float64):
        with pytest.raises(TypeError):
            ears.token_logprobs(torch.zeros(N, V), torch.zeros(N, dtype=dtype))


# ---- the extension module -----------------------------------------------------------------------------

@pytest.fixture
def unbound(monkeypatch):
    """No call has been made yet."""
    monkeypatch.setattr(rows, "_plain", None)
    monkeypatch.setattr(rows, "_plain_for", None)


def test_a_module_built_from_other_sources_is_built_again(tmp_path, monkeypatch):
    build = rows._build
    path = build.build_torch()
    assert not build.torch_is_stale()
    made = []

    def compile(cmd, **kw):
        made.append(cmd)
        shutil.copy(path, cmd[cmd.index("-o") + 1])
    monkeypatch.setattr(build, "TORCH_LIB", str(tmp_path / "ears_torch.so"))
    monkeypatch.setattr(build.subprocess, "run", compile)
    build.build_torch()                                          # absent
    build.build_torch()                                          # current
    assert len(made) == 1
    monkeypatch.setattr(torch, "__version__", "1.0.0")           # compiled against another torch
    assert build.torch_is_stale()
    monkeypatch.undo()
    copy = tmp_path / "csrc"
    shutil.copytree(build.CSRC, copy)
    monkeypatch.setattr(build, "CSRC", str(copy))
    assert not build.torch_is_stale()                            # whatever the files' times
    with open(copy / "ears_torch.cpp", "a") as f:
        f.write("// changed\n")
    assert build.torch_is_stale()
    (copy / "ears_torch.cpp").unlink()
    assert not build.torch_is_stale()                            # nothing to build it from


def test_without_the_module_calls_go_through_ctypes(unbound, monkeypatch):
    def no_compiler(*a, **kw):
        raise OSError("no compiler")
    monkeypatch.setattr(rows._build, "build_torch", no_compiler)
    with pytest.warns(RuntimeWarning, match="no compiler"):
        plain = rows._plain_calls()
    for name in ("top_logits", "token_logprobs", "token_logprobs_step", "policy", "distill"):
        assert getattr(plain, name)(1, 2, 3) is None             # "not in its plain form"
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        assert rows._plain_calls() is plain                      # said once


def test_a_library_of_another_version_is_not_called_through_the_module(unbound, monkeypatch):
    lib = ears.load_library()
    assert rows._plain_calls().version == lib.ears_version()

    class Other:
        def __getattr__(self, name):
            return (lambda: lib.ears_version() + 1) if name == "ears_version" else getattr(lib, name)
    monkeypatch.setattr(rows.binding, "_lib", Other())
    monkeypatch.setattr(rows, "load_library", lambda: rows.binding._lib)
    with pytest.warns(RuntimeWarning, match="version"):
        assert rows._plain_calls().policy() is None
