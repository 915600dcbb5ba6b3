"""The key/value cache held in 4 bits against its 64-bit definition (oracle/kv.py).

What is written and read is fixed by the format to the bit: the read value is m + s c, exact up to one rounding to 32 bits and
one to the type (s c has 12 bits), and codes, scales and minima are equal.

Attention, tolerances from the arithmetic.  In units of log2 a score is a sum of products whose absolute values add up to at
most `size` (oracle): the query's 2^-26 of its largest element (2^-26 * 64 terms of that size at worst, 2^-20 size), at most
D / 64 * 8 accumulations on tensor cores (truncating: 2^-23 each) and about ten 32-bit roundings: 2^-17.9 size at D = 256;
S_TOL = 2^-17 (size + 1), the 1 for the exponential's own 2^-22.  A relative error e in every weight moves a result by at most 2 e reach, e = ln 2
S_TOL.  A weight's rounding to half precision is 2^-11 of `weighted` for bfloat16 queries; for half-precision ones, where what it
lost is added back times the middle code, 2^-11 of `spread`, 7.5 codes either way; weights that are subnormal there are off by at most 2^-25 of 2^-6 of the largest scale, 15 codes each: 2^-27 tiny.  The sums
over up to some ten thousand tokens are in 32 bits, split over at least four warps: below 2^-14 relative of what is summed at the
worst, sqrt of that in truth; 2^-18 (weighted + |out| + reach).  Then one rounding to the type, half a step.
"""
import math

import pytest
import torch

from oracle import kv as O

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def values(shape, g):
    return torch.randn(shape, generator=g) * (torch.rand(shape[-1], generator=g) + 0.5) + torch.randn(shape[-1], generator=g)


def pool(lengths, H, D, page, seed, extra=2):
    """A pool filled with quantised values, and a page table in random order; unused entries name no page."""
    g = torch.Generator().manual_seed(seed)
    held = [-(-n // page) for n in lengths]
    total = sum(held) + extra
    codes, params = O.quantise(values((total, 2, H, page, D), g))
    order = torch.randperm(total, generator=g)
    pages = torch.full((len(lengths), max(max(held), 1)), -7, dtype=torch.int32)
    at = 0
    for b, n in enumerate(held):
        pages[b, :n] = order[at:at + n].int()
        at += n
    return codes, params, pages, g


def on_device(ears, codes, params):
    return ears.KVCache(codes.to(DEV), params.to(DEV))


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


# ---- write and read -----------------------------------------------------------------------------------

@pytest.mark.parametrize("D,H,page", [(64, 3, 16), (128, 8, 64), (128, 1, 48), (256, 2, 32)])
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("layout", ["plain", "joined", "odd", "heads_first"])
def test_write_matches_the_format_and_touches_nothing_else(ears, dtype, D, H, page, layout):
    B, Q = 3, 37
    start, counts = [0, 5, page - 1], [37, 0, 20]
    codes, params, pages, g = pool([60, 60, page + 60], H, D, page, 7)
    if layout == "joined":
        kv = values((B, Q, 2 * H, D), g).to(DT[dtype]).to(DEV)
        k, v = kv[:, :, :H], kv[:, :, H:]
    elif layout == "odd":            # starts on no 16 bytes
        kv = values((B, Q, H, 2 * D + 9), g).to(DT[dtype]).to(DEV)
        k, v = kv[..., 1:D + 1], kv[..., D + 4:2 * D + 4]
    elif layout == "heads_first":
        k, v = (values((B, H, Q, D), g).to(DT[dtype]).to(DEV).transpose(1, 2) for _ in range(2))
    else:
        k, v = (values((B, Q, H, D), g).to(DT[dtype]).to(DEV) for _ in range(2))
    cache = on_device(ears, codes, params)
    status = ints([0])
    ears.kv_write(cache, k, v, pages.to(DEV), ints(start), ints(counts), status=status)
    for kind, x in enumerate((k, v)):
        c, m = O.quantise(x.cpu())
        for b in range(B):
            for i in range(counts[b]):
                t = start[b] + i
                codes[pages[b, t // page], kind, :, t % page] = c[b, i]
                params[pages[b, t // page], kind, :, t % page] = m[b, i]
    assert torch.equal(cache.codes.cpu(), codes)
    assert torch.equal(cache.params.cpu().view(torch.int16), params.view(torch.int16))
    assert status.item() == 0


def hard_groups():
    x = torch.zeros(16, 64)
    i = torch.arange(64).float()
    x[1] = 3.25
    x[2] = -1.2345
    x[3, 5] = math.nan
    x[4, 63] = math.inf
    x[5, 0] = -math.inf
    x[6] = i * 0.25 % 15.5                       # ties in plenty
    x[7] = (i % 31) * 0.5
    x[8] = torch.where(i % 2 == 0, 3.3e38, -3.3e38)
    x[9] = i * 1e-42                             # below the normal numbers
    x[10] = 1000 + i / 64
    x[11] = -1000 - i / 64
    x[12] = torch.where(i == 9, 6e4, 0.0)
    x[13] = 3.3e38
    x[14] = -0.0
    x[15] = torch.where(i % 3 == 0, -0.0, 0.0) + torch.where(i == 1, 1e-30, 0.0)
    return x


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
def test_groups_that_are_hard_to_quantise(ears, dtype):
    x = hard_groups().to(DT[dtype]).view(1, 16, 1, 64)
    cache = ears.kv_cache(1, 1, 64, 16)
    ears.kv_write(cache, x.to(DEV), x.flip(1).to(DEV), ints([[0]]), ints([0]))
    codes, params = O.quantise(x[0, :, 0])
    for kind, order in ((0, slice(None)), (1, range(15, -1, -1))):
        want = O.values(codes, params)[order] if kind == 0 else O.values(codes, params).flip(0)
        got = O.values(cache.codes[0, kind, 0].cpu(), cache.params[0, kind, 0].cpu())
        assert torch.equal(got.nan_to_num(7e77), want.nan_to_num(7e77)), (got - want).abs().amax(-1)
    k, v = ears.kv_read(cache, ints([[0]]), ints([0]), 16, dtype=torch.float32)
    want = O.values(codes, params).float()
    assert torch.equal(k[0, :, 0].cpu().nan_to_num(7e7), want.nan_to_num(7e7)) and torch.equal(v.flip(1).nan_to_num(7e7), k.nan_to_num(7e7))


@pytest.mark.parametrize("D,H,page", [(64, 5, 16), (128, 2, 48), (256, 3, 128)])
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
def test_read(ears, dtype, D, H, page):
    lengths, start, counts = [90, 1, 200, 33], [3, 0, 160, 33], [51, 1, 40, 0]
    codes, params, pages, _ = pool(lengths, H, D, page, 9)
    k, v = ears.kv_read(on_device(ears, codes, params), pages.to(DEV), ints(start), 51, ints(counts), dtype=DT[dtype])
    assert k.shape == v.shape == (4, 51, H, D) and k.dtype == DT[dtype]
    for b in range(4):
        want = O.tokens_of(codes, params, pages, b, start[b] + counts[b])[:, :, start[b]:].transpose(1, 2).float().to(DT[dtype])
        assert torch.equal(k[b, :counts[b]].cpu(), want[0]) and torch.equal(v[b, :counts[b]].cpu(), want[1])
        assert not k[b, counts[b]:].any() and not v[b, counts[b]:].any()


def test_positions_outside_the_table_and_pages_outside_the_pool(ears):
    codes, params, pages, g = pool([40, 40, 40], 2, 64, 16, 11)
    pages[1, 1] = codes.shape[0]                 # no page of the pool
    pages[2, 0] = -1
    x = values((3, 20, 2, 64), g).bfloat16().to(DEV)
    start = [pages.shape[1] * 16 - 10, 10, -3]
    cache, status = on_device(ears, codes, params), ints([4])
    ears.kv_write(cache, x, x, pages.to(DEV), ints(start), status=status)
    assert status.item() == 5
    c, m = O.quantise(x.cpu())
    seen = torch.zeros(3, 20, dtype=torch.bool)
    for b in range(3):
        for i in range(20):
            t = start[b] + i
            if 0 <= t < pages.shape[1] * 16 and 0 <= pages[b, t // 16] < codes.shape[0]:
                seen[b, i] = True
                codes[pages[b, t // 16], :, :, t % 16] = c[b, i]
                params[pages[b, t // 16], :, :, t % 16] = m[b, i]
    assert seen.any(1).all() and not seen.all(1).any()
    assert torch.equal(cache.codes.cpu(), codes) and torch.equal(cache.params.cpu(), params)
    status.zero_()
    k, v = ears.kv_read(cache, pages.to(DEV), ints(start), 20, dtype=torch.float32, status=status)
    assert status.item() == 1
    assert torch.equal(~k.isnan().any(-1).any(-1).cpu(), seen) and torch.equal(k.isnan().all(-1).all(-1).cpu(), ~seen)
    assert torch.equal(k[seen.to(DEV)].cpu().double(), O.values(c, m)[seen])
    # and nothing is reported where such positions are left out
    status.zero_()
    ears.kv_read(cache, pages.to(DEV), ints(start), 20, ints([10, 6, 0]), status=status)
    assert status.item() == 0


# ---- attention -------------------------------------------------------------------------------------------

def close(got, want, dtype, lse=None):
    eps = torch.finfo(DT[dtype]).eps / 2
    got = got.cpu().double()
    e = 2.0 ** -17 * math.log(2) * (want.size + 1)
    rounded = want.weighted if dtype == "bf16" else want.spread
    limit = (2 * e.unsqueeze(-1) * want.reach + 2.0 ** -11 * rounded + 2.0 ** -18 * want.weighted + 2.0 ** -18 * (want.out.abs() + want.reach)
             + 2.0 ** -27 * want.tiny.unsqueeze(-1))
    limit = limit * (1 + eps) + eps * want.out.abs() + (2.0 ** -25 if dtype == "fp16" else 0.0)
    err = (got - want.out).abs()
    assert not got.isnan().any()
    assert (err <= limit).all(), (float((err / limit.clamp(min=1e-300)).max()), (err > limit).nonzero()[:4].tolist())
    if lse is not None:
        lse, empty = lse.cpu().double(), want.lse == -math.inf
        assert (lse[empty] == -math.inf).all()
        # a sum of n terms in 32 bits, and the result's own rounding
        assert ((lse - want.lse)[~empty].abs() <= (e + 2.0 ** -18 + 2.0 ** -23 * want.lse.abs())[~empty]).all()


def attend(ears, dtype, lengths, Q, group, H, D, page, counts=None, window=0, sinks=0, seed=1, scale=None, sharp=1.0, table_extra=0):
    """lengths: tokens each sequence has, its newest Q among them."""
    codes, params, pages, g = pool(lengths, H, D, page, seed)
    if table_extra:
        pages = torch.nn.functional.pad(pages, (0, table_extra), value=-1)
    start = [max(0, n - Q) for n in lengths]
    q = (torch.randn(len(lengths), Q, H * group, D, generator=g) * sharp).to(DT[dtype])
    n = [min(Q, length) for length in lengths] if counts is None else counts
    want = O.attention(q, codes, params, pages, start, n, scale, window, sinks)
    got, lse = ears.kv_attention(q.to(DEV), on_device(ears, codes, params), pages.to(DEV), ints(start), ints(n), window=window, sinks=sinks,
                                 scale=scale, lse=True)
    assert got.shape == q.shape and got.dtype == q.dtype and lse.dtype == torch.float32
    close(got, want, dtype, lse)
    for b in range(len(lengths)):
        assert not got[b, n[b]:].any()
    return got


# a table as wide as 12800 tokens and more has rows in blocks of several eights, a narrow one a block per eight
@pytest.mark.parametrize("table_extra", [0, 800])
@pytest.mark.parametrize("Q,group", [(1, 1), (1, 8), (5, 4), (3, 3), (6, 1), (2, 16), (9, 5), (1, 71), (4, 4), (7, 8)])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_attention(ears, dtype, D, Q, group, table_extra):
    attend(ears, dtype, [1, 2, 17, 64, 65, 300, 1000, 0], Q, group, 2, D, 16 if D == 64 else 48, seed=D + Q, table_extra=table_extra)


@pytest.mark.parametrize("Q,group", [(2, 8), (5, 4), (8, 4), (5, 8)])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_windows_over_many_units_of_several_eights(ears, dtype, D, Q, group):
    g = torch.Generator().manual_seed(D + Q)
    lengths = torch.randint(0, 700, (40,), generator=g).tolist()
    attend(ears, dtype, lengths, Q, group, 8, D, 64, window=401, sinks=5, seed=D)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (7, 3), (16, 16), (50, 4), (64, 33), (100, 500), (1000, 4), (5000, 0), (2**31 - 1, 0), (9, 2**31 - 1)])
def test_attention_with_a_window_and_sinks(ears, dtype, window, sinks):
    attend(ears, dtype, [3, 40, 100, 333, 900], 5, 4, 2, 64, 32, window=window, sinks=sinks, seed=window)
    attend(ears, dtype, [700, 20], 3, 2, 1, 128, 16, window=window, sinks=sinks, seed=window + 1)


@pytest.mark.parametrize("D,H,group,lengths", [(128, 1, 8, [40000]), (128, 8, 4, [9000, 3]), (64, 2, 6, [20011, 5000, 1]), (256, 1, 16, [7001])])
def test_attention_over_units_that_many_ctas_share(ears, D, H, group, lengths):
    attend(ears, "bf16", lengths, 2, group, H, D, 64, seed=3, sharp=2.0)
    attend(ears, "fp16", lengths, 1, group, H, D, 64, seed=4)


def test_attention_over_many_sequences(ears):
    g = torch.Generator().manual_seed(1)
    lengths = torch.randint(0, 90, (300,), generator=g).tolist()
    lengths[7], lengths[299] = 2500, 1200
    attend(ears, "bf16", lengths, 4, 2, 3, 64, 16, seed=5)
    attend(ears, "fp16", lengths[:130], 1, 4, 1, 128, 32, seed=6, table_extra=50)


def test_attention_of_a_long_block(ears):
    """A prompt's worth of positions: many row blocks, most of them masked in part."""
    attend(ears, "bf16", [130, 77], 130, 2, 1, 128, 16, seed=8, counts=[130, 70])
    attend(ears, "fp16", [200], 150, 3, 2, 64, 32, seed=9, window=40, sinks=3)


@pytest.mark.parametrize("scale", [0.0, -0.3, 2.0])
def test_attention_scales(ears, scale):
    attend(ears, "bf16", [50, 400], 2, 4, 2, 128, 16, scale=scale, seed=12)


def test_attention_where_sizes_differ_widely(ears):
    """Scales of values over 2^60 from token to token, keys and queries far from 1, one token that takes it all."""
    D, H, page = 128, 2, 16
    codes, params, pages, g = pool([600], H, D, page, 21)
    row = torch.randint(-30, 31, (codes.shape[0], 1, H, page, 1, 1), generator=g).double()
    params[:, 1:] = (params[:, 1:].double() * 2.0 ** row).bfloat16()
    params[:, :1] = (params[:, :1].double() * 2.0 ** -40).bfloat16()
    q = torch.randn(1, 3, 8, D, generator=g)
    q[0, 1] *= 2.0 ** -20
    q[0, 2] *= 8.0
    q = (q * 2.0 ** 40).bfloat16()
    want = O.attention(q, codes, params, pages, [597])
    got, lse = ears.kv_attention(q.to(DEV), on_device(ears, codes, params), pages.to(DEV), ints([597]), lse=True)
    close(got, want, "bf16", lse)


def poison(codes, params, keep):
    """NaN scales, infinite minima and full codes wherever no row may look."""
    bad = ~keep
    codes[bad] = 255
    params[bad] = torch.tensor([math.nan, math.inf], dtype=torch.bfloat16).expand(params[bad].shape)
    odd = bad & (torch.arange(keep.shape[-1]) % 2 == 0)
    params[odd] = torch.tensor([3e38, -3e38], dtype=torch.bfloat16).expand(params[odd].shape)


@pytest.mark.parametrize("window,sinks", [(0, 0), (37, 5)])
@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("fp16", 64), ("bf16", 256)])
def test_what_no_row_sees_does_not_matter(ears, dtype, D, window, sinks):
    H, page, Q, lengths = 2, 32, 4, [70, 5, 333, 200]
    counts = [4, 4, 2, 0]
    codes, params, pages, g = pool(lengths, H, D, page, 31)
    start = [n - Q for n in lengths]
    start[1] = 1
    q = torch.randn(4, Q, H * 4, D, generator=g).to(DT[dtype]).to(DEV)
    call = lambda: ears.kv_attention(q, on_device(ears, codes, params), pages.to(DEV), ints(start), ints(counts), window=window, sinks=sinks, lse=True)
    clean, clean_lse = call()
    keep = torch.zeros(codes.shape[0], 2, H, page, dtype=torch.bool)
    for b in range(4):
        for t in range(start[b] + counts[b] if counts[b] else 0):
            if not window or t < sinks or t > start[b] - window:
                keep[pages[b, t // page], :, :, t % page] = True
    poison(codes, params, keep)
    got, lse = call()
    assert torch.equal(got, clean) and torch.equal(lse, clean_lse) and not got.isnan().any()


def test_nan_reaches_the_rows_that_see_it_and_no_other(ears):
    D, H, page, Q = 128, 2, 16, 6
    codes, params, pages, g = pool([300, 300], H, D, page, 41)
    start = [294, 294]
    q = torch.randn(2, Q, H * 2, D, generator=g).bfloat16()
    q[1, 3, 1, 7] = math.inf
    q[1, 4, 2, 0] = math.nan
    t = 296                                       # seen by rows 2 .. 5: once in a key of head 0, once in a value of head 1
    params[pages[0, t // page], 0, 0, t % page, 1] = math.nan
    params[pages[0, t // page], 1, 1, t % page, 0] = math.nan
    got, lse = ears.kv_attention(q.to(DEV), on_device(ears, codes, params), pages.to(DEV), ints(start), lse=True)
    bad = got.isnan().any(-1).cpu()
    want = torch.zeros(2, Q, 4, dtype=torch.bool)
    want[0, 2:, :] = True
    want[1, 3, 1] = want[1, 4, 2] = True
    assert torch.equal(bad, want)
    clean = O.attention(q.nan_to_num(0, 0, 0), codes, params.nan_to_num(0, 0, 0), pages, start)
    ok = ~want
    err = (got.cpu().double() - clean.out).abs()[ok]
    assert float(err.max()) < 0.05
    # a window that has left the token behind
    got = ears.kv_attention(q[:1, 4:].to(DEV), on_device(ears, codes, params), pages[:1].to(DEV), ints([298]), window=2)
    assert not got.isnan().any()


def test_attention_where_positions_or_pages_are_unusable(ears):
    D, H, page, Q = 64, 2, 16, 3
    codes, params, pages, g = pool([100] * 5, H, D, page, 51)
    start = [97, 97, -2, pages.shape[1] * page - 2, 97]
    pages[1, 2] = 10**6                           # tokens 32 .. 47
    pages[4, 2] = -5
    q = torch.randn(5, Q, H * 2, D, generator=g).bfloat16()
    status = ints([0])
    got, lse = ears.kv_attention(q.to(DEV), on_device(ears, codes, params), pages.to(DEV), ints(start), ints([3, 3, 2, 3, 0]), lse=True, status=status)
    assert status.item() == 1
    want = O.attention(q[:1], codes, params, pages[:1], start[:1])
    close(got[:1], want, "bf16", lse[:1])
    assert got[1].isnan().all() and got[2, :2].isnan().all() and not got[2, 2].any() and got[3].isnan().all() and not got[4].any()
    assert lse[1].isnan().all() and lse[3].isnan().all() and (lse[4] == -math.inf).all()
    # behind a window the missing page is not looked for
    status.zero_()
    got, lse = ears.kv_attention(q[1:2].to(DEV), on_device(ears, codes, params), pages[1:2].to(DEV), ints([97]), window=30, sinks=20, lse=True, status=status)
    assert status.item() == 0
    pages[1, 2] = 0
    close(got, O.attention(q[1:2], codes, params, pages[1:2], [97], window=30, sinks=20), "bf16", lse)


@pytest.mark.parametrize("layout", ["joined", "odd", "heads_first"])
def test_queries_are_used_where_they_lie(ears, layout):
    D, H, Q, lengths = 128, 2, 5, [100, 33]
    codes, params, pages, g = pool(lengths, H, D, 16, 61)
    x = torch.randn(2, Q, 12, D, generator=g).bfloat16().to(DEV)
    if layout == "joined":
        q = x[:, :, 2:10]
    elif layout == "odd":
        q = torch.cat([x[:, :, :8], x[:, :, :8, :5]], -1)[..., 3:D + 3]
    else:
        q = x[:, :, :8].transpose(1, 2).contiguous().transpose(1, 2)
    cache, place = on_device(ears, codes, params), (pages.to(DEV), ints([95, 28]))
    got = ears.kv_attention(q, cache, *place)
    assert torch.equal(got, ears.kv_attention(q.contiguous(), cache, *place))


def test_integers_of_other_types_and_tables_that_are_slices(ears):
    codes, params, pages, g = pool([100, 33], 2, 64, 16, 62)
    cache = on_device(ears, codes, params)
    q = torch.randn(2, 1, 4, 64, generator=g).half().to(DEV)
    want = ears.kv_attention(q, cache, pages.to(DEV), ints([99, 32]))
    wide = torch.nn.functional.pad(pages, (3, 5)).to(DEV)
    assert torch.equal(ears.kv_attention(q, cache, wide[:, 3:-5], ints([99, 32])), want)
    assert torch.equal(ears.kv_attention(q, cache, wide.t().contiguous().t()[:, 3:-5], ints([99, 32]).long(), counts=ints([1, 1]).short()), want)
    status = ints([0])
    far = torch.tensor([99, 2**32 + 32], device=DEV)
    assert ears.kv_attention(q, cache, pages.to(DEV).long(), far, status=status)[1].isnan().all() and status.item() == 1
    for bad in (dict(start=ints([1])), dict(start=ints([1, 2]).float()), dict(pages=pages[0].to(DEV)), dict(pages=pages.to(DEV).double()),
                dict(counts=ints([[1, 1]])), dict(start=torch.tensor([1, 2])), dict(status=torch.zeros(1, device=DEV))):
        with pytest.raises((ValueError, TypeError)):
            ears.kv_attention(**{**dict(q=q, cache=cache, pages=pages.to(DEV), start=ints([99, 32])), **bad})
    for bad in (q.float(), q[:, :, :3], q[..., :32], q[:1], q[0]):
        with pytest.raises((ValueError, TypeError)):
            ears.kv_attention(bad, cache, pages.to(DEV), ints([99, 32]))
    for kw in (dict(window=-1), dict(sinks=-1), dict(window=2**31)):
        with pytest.raises((ValueError, ears.EarsError)):
            ears.kv_attention(q, cache, pages.to(DEV), ints([99, 32]), **kw)
    x = torch.zeros(2, 3, 2, 64, device=DEV)
    for k, v in ((x, x.half()), (x, x[:, :2]), (x.double(), x.double()), (x[:, :, :1], x[:, :, :1]), (x.cpu(), x)):
        with pytest.raises((ValueError, TypeError)):
            ears.kv_write(cache, k, v, pages.to(DEV), ints([0, 0]))
    with pytest.raises((ValueError, TypeError)):
        ears.kv_read(cache, pages.to(DEV), ints([0, 0]), 0)
    with pytest.raises(TypeError):
        ears.kv_read(cache, pages.to(DEV), ints([0, 0]), 2, dtype=torch.int8)
    with pytest.raises(ValueError):
        ears.kv_read(ears.KVCache(cache.codes[:, :, :, ::2], cache.params[:, :, :, ::2]), pages.to(DEV), ints([0, 0]), 2)


def test_plain_calls_need_no_conversion_and_gradients_are_refused(ears, monkeypatch):
    from paper_2512_13194_b200 import kv as module
    codes, params, pages, g = pool([100, 33], 2, 64, 16, 63)
    cache, pages, start = on_device(ears, codes, params), pages.to(DEV), ints([95, 28])
    q = torch.randn(2, 5, 4, 64, generator=g).half().to(DEV)
    k = torch.randn(2, 5, 2, 64, generator=g).to(DEV)
    want = ears.kv_attention(q, cache, pages.long(), start, scale=0.125, lse=True)          # not plain: 64-bit integers
    grads = [t.clone().requires_grad_() for t in (q, k)]
    for call in (lambda: ears.kv_attention(grads[0], cache, pages, start), lambda: ears.kv_write(cache, grads[1], k, pages, start),
                 lambda: ears.kv_write(cache, k, grads[1], pages, start)):
        with pytest.raises(NotImplementedError):
            call()

    def fail(*args):
        raise AssertionError("converted")

    monkeypatch.setattr(module, "_Call", fail)
    got = ears.kv_attention(q, cache, pages, start, lse=True)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert torch.equal(ears.kv_attention(q, cache, pages, start, lse=1)[1], want[1])
    with torch.no_grad():
        assert torch.equal(ears.kv_attention(grads[0], cache, pages, start), want[0])
    ears.kv_write(cache, k, k, pages, start, ints([5, 2]))
    assert torch.equal(*ears.kv_read(cache, pages, start, 5, ints([5, 2]), dtype=torch.float32))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = ears.kv_attention(q, cache, pages, start, window=7, sinks=1, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(out, ears.kv_attention(q, cache, pages, start, window=7, sinks=1))


def test_offsets_beyond_32_bits(ears):
    """A pool whose codes pass 2^32 bytes; what is written, read and attended to lies behind them."""
    D, H, page = 256, 8, 128
    n = (2**32 + 2**28) // (2 * H * page * D // 2)
    cache = ears.KVCache(torch.empty(n, 2, H, page, D // 2, dtype=torch.uint8, device=DEV),
                         torch.empty(n, 2, H, page, D // 64, 2, dtype=torch.bfloat16, device=DEV))
    pages = ints([[n - 1, n - 2], [0, n // 2]])
    g = torch.Generator().manual_seed(2)
    k, v = (values((2, 150, H, D), g).half().to(DEV) for _ in range(2))
    ears.kv_write(cache, k, v, pages, ints([0, 0]))
    rk, rv = ears.kv_read(cache, pages, ints([0, 0]), 150, dtype=torch.float32)
    for got, x in ((rk, k), (rv, v)):
        assert torch.equal(got.cpu().double(), O.values(*O.quantise(x.cpu())))
    q = torch.randn(2, 2, H, D, generator=g).bfloat16()
    order = [n - 1, n - 2, 0, n // 2]
    small = [torch.stack([x[i] for i in order]).cpu() for x in cache]
    want = O.attention(q, *small, torch.tensor([[0, 1], [2, 3]]), [148, 148])
    close(ears.kv_attention(q.to(DEV), cache, pages, ints([148, 148])), want, "bf16")


# ---- streams, graphs, runs of calls --------------------------------------------------------------------------

def test_same_call_same_bits_on_any_stream(ears):
    codes, params, pages, g = pool([20000, 7], 2, 128, 64, 71)
    q = torch.randn(2, 3, 8, 128, generator=g).bfloat16().to(DEV)
    cache, place = on_device(ears, codes, params), (pages.to(DEV), ints([19997, 4]))
    want = ears.kv_attention(q, cache, *place)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    got = [ears.kv_attention(q, cache, *place, stream=s) for s in streams for _ in range(4)]      # side by side
    torch.cuda.synchronize()
    assert all(torch.equal(x, want) for x in got)


def test_captured_passes_follow_their_inputs(ears):
    """Two graphs, each a write and an attention, replayed side by side with new tokens and positions."""
    H, D, page, Q = 2, 128, 16, 3
    parts = []
    for seed in (81, 82):
        codes, params, pages, g = pool([400], H, D, page, seed)
        cache, table, start = on_device(ears, codes, params), pages.to(DEV), ints([0])
        k, v = (torch.zeros(1, Q, H, D, dtype=torch.bfloat16, device=DEV) for _ in range(2))
        q = torch.zeros(1, Q, H * 4, D, dtype=torch.bfloat16, device=DEV)
        ears.kv_write(cache, k, v, table, start)
        ears.kv_attention(q, cache, table, start)
        cache.codes.copy_(codes), cache.params.copy_(params)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            ears.kv_write(cache, k, v, table, start)
            out = ears.kv_attention(q, cache, table, start)
        parts.append((codes, params, pages, g, cache, start, k, v, q, graph, out, torch.cuda.Stream()))
    for at in (0, 14, 397, 200):
        held = []
        for codes, params, pages, g, cache, start, k, v, q, graph, out, stream in parts:
            x = [torch.randn(t.shape, generator=g).bfloat16() for t in (k, v, q)]
            for t, y in zip((k, v, q), x):
                t.copy_(y)
            start.fill_(at)
            held.append(x)
        torch.cuda.synchronize()
        for part in parts:
            with torch.cuda.stream(part[-1]):
                part[-3].replay()
        torch.cuda.synchronize()
        for (codes, params, pages, g, *_, out, _), x in zip(parts, held):
            for kind in (0, 1):
                c, m = O.quantise(x[kind])
                for i in range(Q):
                    t = at + i
                    codes[pages[0, t // page], kind, :, t % page] = c[0, i]
                    params[pages[0, t // page], kind, :, t % page] = m[0, i]
            close(out, O.attention(x[2], codes, params, pages, [at]), "bf16")


@pytest.mark.parametrize("window,sinks", [(0, 0), (24, 4)])
def test_a_decoding_loop_over_the_cache(ears, window, sinks):
    """Prompt, then verification steps: each writes K + 1 tokens, attends from them, verifies, and keeps accept_len + 1.  The
    attention of every step is that of a cache which never saw a rejected token."""
    B, K, H, group, D, V, page = 3, 4, 2, 2, 64, 97, 16
    g = torch.Generator().manual_seed(91)
    embed = {n: torch.randn(V, heads, D, generator=g) for n, heads in (("k", H), ("v", H), ("q", H * group))}
    head = torch.randn(H * group * D, V, generator=g) * 0.2
    prompt = [23, 1, 40]
    text = [torch.randint(0, V, (n,), generator=g).tolist() for n in prompt]
    cache = ears.kv_cache(40, H, D, page)
    pages = torch.randperm(40, generator=g)[:36].view(3, 12).int().to(DEV)
    row = lambda name, tokens: embed[name][torch.tensor(tokens)].bfloat16()
    longest = max(prompt)
    padded = [t + [0] * (longest - len(t)) for t in text]
    ears.kv_write(cache, torch.stack([row("k", t) for t in padded]).to(DEV), torch.stack([row("v", t) for t in padded]).to(DEV), pages,
                  ints([0] * B), ints([n - 1 for n in prompt]))            # the newest token enters with the first drafts
    start = ints([n - 1 for n in prompt])
    sampler = ears.EarsSampler(0.9, 0.1, seed=5)
    kept = 0
    for step in range(6):
        drafts = torch.randint(0, V, (B, K), generator=g)
        fed = [[t[-1]] + d for t, d in zip(text, drafts.tolist())]
        k, v, q = (torch.stack([row(n, f) for f in fed]).to(DEV) for n in ("k", "v", "q"))
        before = start.clone()
        ears.kv_write(cache, k, v, pages, start)
        out = ears.kv_attention(q, cache, pages, start, window=window, sinks=sinks)
        codes, params = (torch.zeros_like(x.cpu()) for x in cache)
        for b in range(B):                                                   # a cache of this text and these drafts alone
            line = text[b][:-1] + fed[b]
            for kind, name in ((0, "k"), (1, "v")):
                c, m = O.quantise(row(name, line))
                for t in range(len(line)):
                    codes[pages[b, t // page], kind, :, t % page] = c[t]
                    params[pages[b, t // page], kind, :, t % page] = m[t]
        assert before.tolist() == [len(t) - 1 for t in text]
        close(out, O.attention(q.cpu(), codes, params, pages.cpu(), before.tolist(), window=window, sinks=sinks), "bf16")
        logits = out.float().flatten(2) @ head.to(DEV)
        draft_logits = logits[:, :K] + 0.3
        res = sampler(logits, draft_logits.contiguous(), drafts.int().to(DEV), kv_start=start)
        for b, new in enumerate(res.emitted()):
            text[b] += new
            kept += len(new)
    assert kept >= 18
