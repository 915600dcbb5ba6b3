"""Refusals of the 4-bit cache's operators that the host decides: no device is touched."""
import ctypes

import pytest
import torch

import paper_2512_13194_b200 as ears
from paper_2512_13194_b200.binding import KvCacheStruct

BUF = (ctypes.c_float * 8192)()
P = (ctypes.addressof(BUF) + 255) // 256 * 256


def lib():
    return ears.load_library()


def cache(codes=P, params=P, pages=4, heads=2, page_size=16, head_dim=64):
    return ctypes.byref(KvCacheStruct(codes, params, pages, heads, page_size, head_dim))


def seqs(table=P, width=3, stride=3, start=P, counts=None):
    return table, width, stride, start, counts


CALLS = {
    "write": lambda c=None, s=seqs(), B=1, Q=2, dtype=1, k=P, v=P, ks=(256, 128, 64), vs=(256, 128, 64), st=None: lib().ears_kv_write(
        dtype, c or cache(), k, v, B, Q, *ks, *vs, *s, st, None),
    "read": lambda c=None, s=seqs(), B=1, Q=2, dtype=1, k=P, v=P, st=None: lib().ears_kv_read(
        dtype, c or cache(), B, Q, *s, k, v, st, None),
    "attention": lambda c=None, s=seqs(), B=1, Q=2, dtype=1, q=P, heads=4, qs=(512, 256, 64), scale=0.125, window=0, sinks=0, out=P,
    lse=None, work=P, size=1 << 30, st=None: lib().ears_kv_attention(
        dtype, c or cache(), q, B, Q, heads, *qs, *s, scale, window, sinks, out, lse, work, size, st, None),
}


@pytest.mark.parametrize("name", sorted(CALLS))
def test_every_entry_point_checks_cache_and_positions(name):
    call = CALLS[name]
    assert call(c=cache(codes=None)) == -1 and call(c=cache(params=None)) == -1
    for bad in (dict(head_dim=32), dict(head_dim=96), dict(head_dim=0), dict(pages=0), dict(heads=0), dict(page_size=0), dict(page_size=8),
                dict(page_size=24), dict(page_size=2**21)):
        assert call(c=cache(**bad)) == -2, bad
    assert call(c=cache(codes=P + 8)) == -4 and call(c=cache(params=P + 4)) == -4
    assert call(s=seqs(table=None)) == -1 and call(s=seqs(start=None)) == -1
    assert call(s=seqs(width=0)) == -2 and call(s=seqs(stride=-1)) == -2 and call(s=seqs(width=2**28)) == -2
    assert call(B=0) == -2 and call(Q=0) == -2 and call(B=2**20, Q=2**20) == -2
    assert call(s=seqs(table=P + 2)) == -4 and call(s=seqs(start=P + 1)) == -4 and call(s=seqs(counts=P + 2)) == -4
    assert call(s=seqs(width=(2**31 - 1) // 16)) == -2        # positions and what is added to them stay in 31 bits
    assert call(c=cache(heads=2**15, page_size=2**11)) == -2   # a page of 2^32 bytes
    assert call(dtype=3) == -3 and call(dtype=-1) == -3
    assert call(st=P + 2) == -4


def test_write_and_read_check_their_tensors():
    w, r = CALLS["write"], CALLS["read"]
    assert w(k=None) == -1 and w(v=None) == -1 and r(k=None) == -1 and r(v=None) == -1
    assert w(k=P + 1) == -4 and w(dtype=0, v=P + 2) == -4 and r(k=P + 8) == -4 and r(v=P + 2) == -4
    for bad in ((-1, 128, 64), (256, -128, 64), (256, 128, -1), (2**62, 128, 64)):
        assert w(B=3, ks=bad) == -2 and w(B=3, vs=bad) == -2


def test_a_missing_cache_is_refused():
    assert lib().ears_kv_write(1, None, P, P, 1, 2, 256, 128, 64, 256, 128, 64, P, 3, 3, P, None, None, None) == -1
    assert lib().ears_kv_read(1, None, 1, 2, P, 3, 3, P, None, P, P, None, None) == -1
    assert lib().ears_kv_attention(1, None, P, 1, 2, 4, 512, 256, 64, P, 3, 3, P, None, 0.125, 0, 0, P, None, P, 1 << 30, None, None) == -1
    assert lib().ears_kv_attention_workspace_bytes(1, None, 1, 1, 4, 3, 0, 0) == 0


def test_attention_checks_its_arguments():
    a = CALLS["attention"]
    assert a(q=None) == -1 and a(out=None) == -1 and a(work=None) == -1
    assert a(dtype=0) == -3                                   # 32-bit queries
    assert a(heads=0) == -2 and a(heads=3) == -2 and a(qs=(-1, 1, 1)) == -2
    assert a(window=-1) == -3 and a(sinks=-1) == -3
    for scale in (float("nan"), float("inf"), 1e39):
        assert a(scale=scale) == -3
    assert a(q=P + 1) == -4 and a(out=P + 8) == -4 and a(lse=P + 2) == -4 and a(work=P + 64) == -4
    need = lib().ears_kv_attention_workspace_bytes
    assert need(0, cache(), 1, 1, 4, 3, 0, 0) == 0 and need(1, cache(head_dim=96), 1, 1, 4, 3, 0, 0) == 0
    assert need(1, cache(), 1, 1, 3, 3, 0, 0) == 0 and need(1, cache(), 0, 1, 4, 3, 0, 0) == 0 and need(1, cache(), 1, 1, 4, 3, -1, 0) == 0


def host_cache(D=64):
    return ears.KVCache(torch.zeros(2, 2, 1, 16, D // 2, dtype=torch.uint8), torch.zeros(2, 2, 1, 16, D // 64, 2, dtype=torch.bfloat16))


def test_binding_refuses_what_is_not_on_a_device():
    pages, start, x = torch.zeros(1, 1, dtype=torch.int32), torch.zeros(1, dtype=torch.int32), torch.zeros(1, 1, 1, 64, dtype=torch.bfloat16)
    c = host_cache()
    assert (c.page_size, c.heads, c.head_dim) == (16, 1, 64)
    for call in (lambda: ears.kv_write(c, x, x, pages, start), lambda: ears.kv_read(c, pages, start, 1),
                 lambda: ears.kv_attention(x, c, pages, start)):
        with pytest.raises(ValueError, match="CUDA"):
            call()


def test_binding_refuses_gradients_and_bad_pools():
    pages, start, x = torch.zeros(1, 1, dtype=torch.int32), torch.zeros(1, dtype=torch.int32), torch.zeros(1, 1, 1, 64, requires_grad=True)
    with pytest.raises(NotImplementedError):
        ears.kv_write(host_cache(), x, x, pages, start)
    with pytest.raises(NotImplementedError):
        ears.kv_attention(x, host_cache(), pages, start)
    with torch.autograd.forward_ad.dual_level():
        y = torch.autograd.forward_ad.make_dual(x.detach(), torch.ones_like(x))
        with pytest.raises(NotImplementedError):
            ears.kv_write(host_cache(), x.detach(), y, pages, start)
    for bad in (dict(head_dim=96), dict(page_size=24), dict(pages=0), dict(heads=0)):
        with pytest.raises(ValueError):
            ears.kv_cache(**{**dict(pages=1, heads=1, head_dim=64, page_size=16), **bad}, device="cpu")
    pool = ears.kv_cache(3, 2, 128, 32, device="cpu")
    assert pool.codes.shape == (3, 2, 2, 32, 64) and pool.params.shape == (3, 2, 2, 32, 2, 2)


def test_advance_moves_behind_what_a_step_keeps():
    start = torch.tensor([10, 0, 7], dtype=torch.int32)
    assert ears.kv_advance(start, torch.tensor([4, 0, -1], dtype=torch.int32)) is start
    assert start.tolist() == [15, 1, 7]
    with pytest.raises(ValueError):
        ears.kv_advance(start, torch.zeros(2, dtype=torch.int32))
    with pytest.raises(ValueError):
        ears.kv_advance(start.float(), torch.zeros(3, dtype=torch.int32))
