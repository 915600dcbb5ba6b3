"""The operators on rows of logits against their 64-bit definitions (oracle/rows.py).

Tolerances, from the arithmetic.  A term 2^t, t = (l - m) c: the special-function unit is off by at most
2^-22 relative; t carries three roundings (the difference, c, the product), 3 * 2^-24 |t| together, which is
ln 2 * 1.8e-7 |t| relative in the term.  Weighted by the terms themselves the mean |t| stays below
log2(V) + 2 <= 19, so a normaliser is off by at most 2.4e-7 + 2.4e-6 from its terms, plus the sum's roundings
(<= ~600 per thread in four lanes, then a tree: some tens of 2^-24 at worst, 1.3e-6): Z_TOL = 4e-6.
  logarithms (logp, lse, tails)   4e-6 absolute, plus half a step of the 32-bit result
  entropy                         W = sum 2^t t: 4e-6 (|t| + 1) on average, |t| <= 19: 6e-5 absolute
  gradient entries                each is a sum of terms of size `scale` (oracle/rows.py): the entry's own 2^t,
                                  |t| <= 40 where it still counts: 40 * 1.3e-7 + 2.4e-7 = 5.5e-6, the normaliser's
                                  4e-6 (twice where a tail mass enters), ten scalar roundings; 3e-5 scale, entropy parts
                                  6e-5.  Entries beyond |t| = 40 have 2^t < 1e-12 and their 150 * 1.3e-7 = 2e-5 relative
                                  error is inside 3e-5 scale.  Rounded once to the type: half a step, and for fp16 half a
                                  subnormal step (2^-25), for bf16 / fp32 flushed terms below 2^-126.
"""
import math

import pytest
import torch

from oracle import rows as R

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
LOG_TOL, H_TOL, G_TOL = 4e-6, 6e-5, 3e-5
HALF32 = torch.finfo(torch.float32).eps / 2
CLUSTERS = [0, 1, 2, 4, 8, 16]


@pytest.fixture(autouse=True)
def _automatic(ears):
    yield
    ears.set_row_cluster(0)


def logits(n, V, dtype, seed, scale=2.0, mask=True):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(n, V, generator=g) * scale
    x[::2, torch.randint(0, V, (1,), generator=g)] += 9.0
    if mask and V > 16:
        x[:, -(V // 16):] = -math.inf
        x[1::3, : V // 8] = -math.inf
    return x.to(DT[dtype]), g


def close(got, want, tol):
    got, want = got.detach().double().cpu(), want.double()
    inf = torch.isinf(want)
    assert torch.equal(got[inf], want[inf])
    assert not torch.isnan(got).any()
    err = (torch.where(inf, 0.0, got) - torch.where(inf, 0.0, want)).abs()
    limit = (tol if isinstance(tol, torch.Tensor) else torch.full_like(want, tol)) + HALF32 * torch.where(inf, 0.0, want).abs() * 1.0001
    assert (err <= limit).all(), (float((err - limit).max()), float(err.max()))


def close_grad(got, want, scale, tol, dtype):
    got, want = got.detach().double().cpu(), want.double()
    eps = torch.finfo(DT[dtype]).eps / 2
    tiny = {"fp32": 2.0 ** -125, "bf16": 2.0 ** -125, "fp16": 2.0 ** -25}[dtype]
    limit = tol * scale * (1 + eps) + eps * want.abs() + tiny
    err = (got - want).abs()
    assert not torch.isnan(got).any()
    bad = err > limit
    assert not bad.any(), (float((err / limit).max()), bad.nonzero()[:4].tolist())


# ---- top logits ---------------------------------------------------------------------------------

@pytest.mark.parametrize("cluster", CLUSTERS)
@pytest.mark.parametrize("V,k", [(1, 1), (5, 8), (64, 64), (257, 1), (1000, 128), (4099, 37), (33001, 64)])
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
def test_top_logits(ears, dtype, V, k, cluster):
    ears.set_row_cluster(cluster)
    x, _ = logits(5, V, dtype, 10 + V)
    T = 0.8
    top = ears.top_logits(x.to(DEV), k, T)
    v, i, lse = R.top_logits(x, k, T)
    assert torch.equal(top.ids.cpu().long(), i)
    assert torch.equal(top.values.cpu().double(), v)
    close(top.lse, lse, LOG_TOL)


PATTERNS = {
    "ascending": lambda V: torch.arange(V) / V * 20,
    "descending": lambda V: -torch.arange(V) / V * 20,
    "constant": lambda V: torch.full((V,), 1.5),
    "two_values": lambda V: (torch.arange(V) % 7 == 3).float(),
    "signed_zeros": lambda V: torch.where(torch.arange(V) % 3 == 0, -0.0, 0.0),
    "three_finite": lambda V: torch.where(torch.arange(V) % (V // 3 + 1) == 1, torch.arange(V) / V, -math.inf),
    "lowest_masks": lambda V: torch.where(torch.arange(V) % 5 == 0, torch.sin(torch.arange(V) * 1.0), torch.finfo(torch.bfloat16).min),
    "nothing_but_lowest": lambda V: torch.full((V,), float(torch.finfo(torch.bfloat16).min)),
    "extremes": lambda V: torch.where(torch.arange(V) % 2 == 0, 3.0e38, -3.0e38),
}


@pytest.mark.parametrize("cluster", [1, 4, 16])
@pytest.mark.parametrize("name", sorted(PATTERNS))
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_top_logits_orders_that_are_hard(ears, dtype, name, cluster):
    ears.set_row_cluster(cluster)
    V, k = 50021, 100
    x = PATTERNS[name](V).to(DT[dtype]).view(1, V)
    top = ears.top_logits(x.to(DEV), k, 1.0)
    v, i, lse = R.top_logits(x, k, 1.0)
    assert torch.equal(top.ids.cpu().long(), i)
    assert torch.equal(top.values.cpu().double(), v)
    # the terms' mean |t| can reach 29 (ascending rows); the sum's largest part is exact
    close(top.lse, lse, LOG_TOL * 2)


@pytest.mark.parametrize("V", [300, 1501, 2043])
@pytest.mark.parametrize("name", sorted(PATTERNS))
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
def test_top_logits_of_short_rows_in_hard_orders(ears, dtype, name, V):
    x = PATTERNS[name](V)
    if dtype == "fp16":
        x = x.clamp(-65504.0, 65504.0) if name != "three_finite" else x
    x = torch.stack([x, x.flip(0), x.roll(7)]).to(DT[dtype])
    for k in (1, 100, 128):
        top = ears.top_logits(x.to(DEV), k, 1.0)
        v, i, lse = R.top_logits(x, k, 1.0)
        assert torch.equal(top.ids.cpu().long(), i)
        assert torch.equal(top.values.cpu().double(), v)
        close(top.lse, lse, LOG_TOL * 2)


@pytest.mark.parametrize("dtype,V", [("bf16", 2100), ("bf16", 16370), ("fp16", 7001), ("fp32", 1100), ("fp32", 8181)])
def test_top_logits_of_many_rows(ears, dtype, V):
    """More rows than CTAs fit on the device at once, a few of them hard: those first and last are checked."""
    n, k = 1300, 100
    g = torch.Generator().manual_seed(V)
    x = torch.randn(n, V + 3, generator=g)
    hard = [(0, "ascending"), (1, "constant"), (2, "two_values"), (3, "three_finite"), (n - 2, "signed_zeros"), (n - 1, "descending")]
    for row, name in hard:
        x[row, 2:2 + V] = PATTERNS[name](V)
    x[5, 2:2 + V] = -math.inf
    x[7, 9] = math.nan
    x = x.to(DT[dtype])[:, 2:2 + V]
    acc = torch.full((n,), 0, dtype=torch.int32)
    acc[9] = -1
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    wide = torch.zeros(n, V + 3, dtype=DT[dtype], device=DEV)
    wide[:, 2:2 + V] = x.to(DEV)
    dev = wide[:, 2:2 + V].unsqueeze(1)
    top = ears.top_logits(dev, k, 0.9, accept_len=acc.to(DEV), status=st)
    assert int(st) == ears.DEV_INVALID_INPUT
    bad = [5, 7]
    assert torch.isnan(top.lse[bad, 0]).all() and (top.ids[bad + [9]] == -1).all() and float(top.lse[9, 0]) == -math.inf
    pick = [r for r in list(range(0, 40)) + list(range(n - 40, n)) if r not in bad + [9]]
    v, i, lse = R.top_logits(x[pick], k, 0.9)
    assert torch.equal(top.ids[pick, 0].cpu().long(), i)
    assert torch.equal(top.values[pick, 0].cpu().double(), v)
    close(top.lse[pick, 0], lse, LOG_TOL * 2)


@pytest.mark.parametrize("V", [300, 1026, 1501, 2043])
@pytest.mark.parametrize("name", sorted(PATTERNS) + ["normal"])
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
def test_top_logits_of_many_short_rows_in_hard_orders(ears, dtype, name, V):
    """As many rows as it takes for each to fall to a single warp."""
    x = PATTERNS[name](V) if name in PATTERNS else torch.randn(V, generator=torch.Generator().manual_seed(V))
    if dtype == "fp16":
        x = x.clamp(-65504.0, 65504.0) if name != "three_finite" else x
    x = torch.stack([x, x.flip(0), x.roll(7)]).to(DT[dtype])
    many = x.to(DEV).repeat(300, 1)
    for k in (2, 33, 64, 100, 128):
        top = ears.top_logits(many, k, 1.0)
        v, i, lse = R.top_logits(x, k, 1.0)
        assert torch.equal(top.ids.cpu().long().view(300, 3, k), i.expand(300, 3, k))
        assert torch.equal(top.values.cpu().double().view(300, 3, k), v.expand(300, 3, k))
        # equal rows that start at different places of a 16-byte vector are summed in a different order
        close(top.lse, lse.repeat(300), LOG_TOL * 2)


@pytest.mark.parametrize("V", [8200, 16390, 20000, 24600, 33000, 41000, 49200, 57300, 70001])
def test_steps_at_every_number_of_stages(ears, V):
    """Rows of one to nine 16 KB chunks, held whole or fetched again, by one and by two CTAs."""
    n, k = 3, 10
    x, vals, ids, lse, g = teacher_case(n, V, k, "bf16", 1.0, 80 + V)
    tok, dl = ids[:, 1].contiguous(), torch.randn(n, generator=g)
    teacher = ears.TopLogits(vals.to(DEV), ids.to(DEV), lse.to(DEV))
    o, od = R.token_logprobs(x, tok, 1.0, dl), R.distill(x, 1.0, vals, ids, lse=lse, weight=dl.abs())
    for cluster in (0, 1, 2):
        ears.set_row_cluster(cluster)
        logp, _, grad = ears.token_logprobs_step(x.to(DEV), tok.to(DEV), dl.to(DEV))
        close(logp, o.logp, LOG_TOL)
        close_grad(grad, o.grad, o.scale, G_TOL, "bf16")
        loss, grad = ears.distill_step(x.to(DEV), teacher, row_weight=dl.abs().to(DEV))
        close(loss, od.loss, od.loss_scale * (3 * LOG_TOL))
        close_grad(grad, od.grad, od.scale, G_TOL, "bf16")


@pytest.mark.parametrize("dtype,V", [("bf16", 2100), ("bf16", 8100), ("fp16", 16001), ("fp32", 1100), ("fp32", 4090), ("fp32", 8001)])
def test_many_rows_that_a_warp_streams(ears, dtype, V):
    n, k, T = 2500, 12, 1.1
    g = torch.Generator().manual_seed(V)
    wide = (torch.randn(n, V + 3, generator=g) * 2).to(DT[dtype])
    wide[:, 2 + V // 2:2 + V // 2 + 40] = -math.inf
    x = wide[:, 2:2 + V]
    dev = wide.to(DEV)[:, 2:2 + V]
    tok = torch.randint(0, V // 2, (n,), generator=g, dtype=torch.int32)
    dl, dh = torch.randn(n, generator=g), torch.randn(n, generator=g)
    tok[11], dl[13], dh[13] = -1, 0.0, 0.0
    teacher = ears.top_logits((dev.float() * 0.6).to(DT[dtype]), k, T)
    pick = list(range(20)) + list(range(n - 20, n))
    o = R.token_logprobs(x[pick], tok[pick], T, dl[pick], dh[pick])
    logp, H, grad = ears.token_logprobs_step(dev, tok.to(DEV), dl.to(DEV), dh.to(DEV), T)
    close(logp[pick], o.logp, LOG_TOL)
    close(H[pick], o.entropy, H_TOL)
    close_grad(grad[pick], o.grad, o.scale, 2 * H_TOL, dtype)
    close(ears.token_logprobs(dev, tok.to(DEV), T)[pick], o.logp, LOG_TOL)
    w = dl.abs()
    for kind in ("forward_kl", "jsd"):
        od = R.distill(x[pick], T, *(t[pick].cpu() for t in teacher[:2]), lse=teacher.lse[pick].cpu(), kind=kind, weight=w[pick])
        loss, grad = ears.distill_step(dev, teacher, T, kind=kind, row_weight=w.to(DEV))
        close(loss[pick], od.loss, od.loss_scale * (3 * LOG_TOL))
        close(ears.distill_loss(dev, teacher, T, kind=kind)[pick], od.loss, od.loss_scale * (3 * LOG_TOL))
        close_grad(grad[pick], od.grad, od.scale, G_TOL, dtype)
        leaf = dev.clone().requires_grad_(True)
        (ears.distill_loss(leaf, teacher, T, kind=kind) * w.to(DEV)).sum().backward()
        close_grad(leaf.grad[pick], od.grad, od.scale, G_TOL, dtype)
        over = wide.to(DEV)
        ears.distill_step(over[:, 2:2 + V], teacher, T, kind=kind, row_weight=w.to(DEV), out_grad=over[:, 2:2 + V])
        assert torch.equal(over[:, 2:2 + V], grad) and torch.equal(over[:, :2].cpu(), wide[:, :2]) and torch.equal(over[:, 2 + V:].cpu(), wide[:, 2 + V:])


def test_many_short_rows_and_rows_that_start_anywhere(ears):
    for dtype in ("fp32", "bf16"):
        for V in (3, 17, 700, 2030, 6001, 12001):
            n = 37 if V > 1000 else 203
            x, g = logits(n, V + 8, dtype, 60 + V, mask=False)
            for off in (0, 1, 3, 8):
                rows = x[:, off:off + V]
                dev = x.to(DEV)[:, off:off + V]
                tok = torch.randint(0, V, (n,), generator=g, dtype=torch.int32)
                dl = torch.randn(n, generator=g)
                o = R.token_logprobs(rows, tok, 0.9, dl)
                logp, _, grad = ears.token_logprobs_step(dev, tok.to(DEV), dl.to(DEV), None, 0.9)
                close(logp, o.logp, LOG_TOL)
                close_grad(grad, o.grad, o.scale, G_TOL, dtype)
                k = min(V, 5)
                top = ears.top_logits(dev, k)
                v, i, lse = R.top_logits(rows, k, 1.0)
                assert torch.equal(top.ids.cpu().long(), i)
                teacher = ears.TopLogits(v.float().to(DEV), i.to(torch.int32).to(DEV), lse.float().to(DEV))
                y = (rows.float() * 0.7).to(DT[dtype])
                wide = torch.zeros(n, V + 8, dtype=DT[dtype], device=DEV)
                wide[:, off:off + V] = y.to(DEV)
                od = R.distill(y, 1.0, v.float(), i.to(torch.int32), lse=lse.float(), kind="jsd", weight=dl.abs())
                loss, grad = ears.distill_step(wide[:, off:off + V], teacher, kind="jsd", row_weight=dl.abs().to(DEV),
                                               out_grad=wide[:, off:off + V])
                close(loss, od.loss, od.loss_scale * (3 * LOG_TOL))
                close_grad(wide[:, off:off + V], od.grad, od.scale, G_TOL, dtype)
                assert not wide[:, :off].any() and not wide[:, off + V:].any()


def test_top_logits_takes_strided_rows_and_leaves_out_what_lies_behind_a_rejection(ears):
    B, K, V, k = 6, 3, 5003, 9
    x, g = logits(B * (K + 1), V, "bf16", 3)
    x = x.view(B, K + 1, V)
    acc = torch.tensor([0, 1, 2, 3, -1, 3], dtype=torch.int32)
    T = torch.linspace(0.5, 1.5, B)
    top = ears.top_logits(x.to(DEV)[:, :K], k, accept_len=acc.to(DEV), seq_temperature=T.to(DEV))
    v, i, lse = R.top_logits(x[:, :K].reshape(B * K, V), k, T.repeat_interleave(K))
    live = (torch.arange(K)[None] <= acc[:, None]).view(-1)
    v[~live], i[~live], lse[~live] = -math.inf, -1, -math.inf
    assert torch.equal(top.ids.cpu().long().view(-1, k), i) and torch.equal(top.values.cpu().double().view(-1, k), v)
    close(top.lse.view(-1), lse, LOG_TOL)
    # rows with an odd pitch that start between 16-byte boundaries
    wide = torch.full((4, 5021), 100.0, dtype=torch.bfloat16)
    wide[:, 7:7 + 5003] = x[0]
    top = ears.top_logits(wide.to(DEV)[:, 7:7 + 5003], k)
    v, i, lse = R.top_logits(x[0], k, 1.0)
    assert torch.equal(top.ids.cpu().long(), i)
    close(top.lse, lse, LOG_TOL)


def test_unusable_rows_are_marked_and_leave_the_others_alone(ears):
    x, _ = logits(6, 3001, "fp32", 4)
    x[1, 2000], x[3, 17] = math.nan, math.inf
    x[4] = -math.inf
    clean = [0, 2, 5]
    xg = x.to(DEV)
    tok = torch.tensor([40, 41, 3001, 43, 44, -1], dtype=torch.int32, device=DEV)
    for cluster in (1, 4):
        ears.set_row_cluster(cluster)
        st = torch.zeros(1, dtype=torch.int32, device=DEV)
        top = ears.top_logits(xg, 5, status=st)
        assert int(st) == ears.DEV_INVALID_INPUT
        assert torch.isnan(top.lse[[1, 3, 4]]).all() and (top.ids[[1, 3, 4]] == -1).all()
        assert torch.equal(top.ids[clean].cpu().long(), R.top_logits(x[clean], 5, 1.0)[1])
        st.zero_()
        logp, H, grad = ears.token_logprobs_step(xg, tok, torch.ones(6, device=DEV), torch.ones(6, device=DEV), status=st)
        assert int(st) == ears.DEV_INVALID_INPUT
        for bad in (1, 2, 3, 4):
            assert torch.isnan(logp[bad]) and torch.isnan(H[bad]) and not grad[bad].any()
        assert float(logp[5]) == 0.0 and float(H[5]) == 0.0 and not grad[5].any()
        assert torch.isfinite(logp[0]) and grad[0].any()
        st.zero_()
        ears.token_logprobs(xg[:1], tok[:1], status=st)
        assert int(st) == 0
        # one temperature that cannot be used
        T = torch.tensor([1.0, 0.0, float("nan")], device=DEV)
        y = xg[[0, 2, 5]].view(3, 1, -1).contiguous()
        top = ears.top_logits(y, 5, seq_temperature=T, status=st)
        assert int(st) == ears.DEV_INVALID_INPUT and torch.isfinite(top.lse[0, 0]) and torch.isnan(top.lse[1:]).all()


# ---- token log probabilities ---------------------------------------------------------------------

@pytest.mark.parametrize("cluster", CLUSTERS)
@pytest.mark.parametrize("V", [1, 7, 1000, 4099, 40000])
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
def test_token_logprobs(ears, dtype, V, cluster):
    ears.set_row_cluster(cluster)
    n, T = 6, 0.9
    x, g = logits(n, V, dtype, 20 + V)
    tok = torch.randint(V // 8, max(V - V // 16, 1), (n,), generator=g, dtype=torch.int32)
    if n > 3 and V > 1:
        tok[3] = -1
    dl, dh = torch.randn(n, generator=g), torch.randn(n, generator=g)
    dl[5] = 0.0
    dh[5] = 0.0
    xg, tg = x.to(DEV), tok.to(DEV)
    plain = ears.token_logprobs(xg, tg, T)
    logp, H = ears.token_logprobs(xg, tg, T, entropy=True)
    o = R.token_logprobs(x, tok, T, dl, dh)
    close(plain, o.logp, LOG_TOL)
    close(logp, o.logp, LOG_TOL)
    close(H, o.entropy, H_TOL)
    l2, H2, grad = ears.token_logprobs_step(xg, tg, dl.to(DEV), dh.to(DEV), T)
    close(l2, o.logp, LOG_TOL)
    close(H2, o.entropy, H_TOL)
    close_grad(grad, o.grad, o.scale, 2 * H_TOL, dtype)
    o = R.token_logprobs(x, tok, T, dl)
    l3, none, grad = ears.token_logprobs_step(xg, tg, dl.to(DEV), None, T)
    assert none is None
    close_grad(grad, o.grad, o.scale, G_TOL, dtype)
    assert not grad[5].any()
    # written over the logits
    over = xg.clone()
    _, _, same = ears.token_logprobs_step(over, tg, dl.to(DEV), None, T, out_grad=over)
    assert same.data_ptr() == over.data_ptr() and torch.equal(over, grad)


def test_masks_of_the_lowest_value_and_extreme_rows(ears):
    V = 2051
    for dtype in ("fp32", "bf16", "fp16"):
        low = torch.finfo(DT[dtype]).min
        x = torch.full((4, V), float(low)).to(DT[dtype])
        x[1, 5:50] = torch.linspace(-1, 1, 45).to(DT[dtype])
        x[2, 7] = torch.finfo(DT[dtype]).max
        x[3] = 0.0
        tok = torch.tensor([3, 20, 7, 2050], dtype=torch.int32)
        one = torch.ones(4)
        o = R.token_logprobs(x, tok, 0.7, one, one)
        for cluster in (1, 2, 8):
            ears.set_row_cluster(cluster)
            logp, H, grad = ears.token_logprobs_step(x.to(DEV), tok.to(DEV), one.to(DEV), one.to(DEV), 0.7)
            close(logp, o.logp, LOG_TOL)
            close(H, o.entropy, H_TOL)
            close_grad(grad, o.grad, o.scale, 2 * H_TOL, dtype)


def test_a_masked_token_has_probability_zero(ears):
    x, _ = logits(2, 500, "fp32", 5)
    tok = torch.tensor([499, 100], dtype=torch.int32)
    dl = torch.ones(2)
    logp, _, grad = ears.token_logprobs_step(x.to(DEV), tok.to(DEV), dl.to(DEV))
    assert float(logp[0]) == -math.inf and math.isfinite(float(logp[1]))
    want = -torch.softmax(x[0].double(), 0)
    want[499] += 1
    close_grad(grad[:1], want.view(1, -1), want.abs().view(1, -1), G_TOL, "fp32")


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_gradients_into_strided_rows_leave_the_rest_alone(ears, dtype):
    B, Rr, V = 3, 4, 1003
    x, g = logits(B * Rr, V, dtype, 6)
    x = x.view(B, Rr, V)
    tok = torch.randint(0, 900, (B, Rr), generator=g, dtype=torch.int32)
    dl = torch.randn(B, Rr, generator=g)
    o = R.token_logprobs(x.view(-1, V), tok.view(-1), 1.0, dl.view(-1))
    for cluster in (1, 2):
        ears.set_row_cluster(cluster)
        for off, pitch in ((0, V), (3, V + 9), (8, V + 5)):      # same alignment as the logits and others
            buf = torch.full((B, Rr, pitch + 16), 7.0, dtype=DT[dtype], device=DEV)
            out = buf[:, :, off:off + V]
            ears.token_logprobs_step(x.to(DEV), tok.to(DEV), dl.to(DEV), out_grad=out)
            close_grad(out.reshape(-1, V), o.grad, o.scale, G_TOL, dtype)
            assert (buf[:, :, :off] == 7).all() and (buf[:, :, off + V:] == 7).all()
        # rows with the batch inside
        t = torch.empty(Rr, B, V, dtype=DT[dtype], device=DEV).transpose(0, 1)
        ears.token_logprobs_step(x.to(DEV), tok.to(DEV), dl.to(DEV), out_grad=t)
        close_grad(t.reshape(-1, V), o.grad, o.scale, G_TOL, dtype)


def test_offsets_beyond_32_bits(ears):
    V, far = 1000, (1 << 31) + 40
    buf = torch.empty(far + V, dtype=torch.bfloat16, device=DEV)
    x, g = logits(2, V, "bf16", 8)
    rows = torch.as_strided(buf, (2, V), (far, 1))
    rows.copy_(x.to(DEV))
    tok = torch.tensor([300, 500], dtype=torch.int32)
    dl = torch.tensor([1.0, -2.0])
    o = R.token_logprobs(x, tok, 1.0, dl)
    for cluster in (1, 4):
        ears.set_row_cluster(cluster)
        top = ears.top_logits(rows, 6)
        assert torch.equal(top.ids.cpu().long(), R.top_logits(x, 6, 1.0)[1])
        keep = rows.clone()
        logp, _, grad = ears.token_logprobs_step(rows, tok.to(DEV), dl.to(DEV), out_grad=rows)
        close(logp, o.logp, LOG_TOL)
        close_grad(rows, o.grad, o.scale, G_TOL, "bf16")
        rows.copy_(keep)


# ---- policy loss ---------------------------------------------------------------------------------

@pytest.mark.parametrize("cluster", [0, 1, 4, 16])
@pytest.mark.parametrize("kl,ent", [(0.0, 0.0), (0.1, 0.0), (0.05, 0.02), (0.0, -0.01)])
@pytest.mark.parametrize("dtype,V", [("fp32", 999), ("bf16", 4099), ("fp16", 12000)])
def test_policy(ears, dtype, V, kl, ent, cluster):
    ears.set_row_cluster(cluster)
    n, T = 12, 1.1
    x, g = logits(n, V, dtype, 30 + V)
    tok = torch.randint(V // 8, V - V // 16, (n,), generator=g, dtype=torch.int32)
    logp = R.token_logprobs(x, tok, T).logp
    old = (logp + 0.3 * torch.randn(n, generator=g)).float()
    ref = (logp + 0.4 * torch.randn(n, generator=g)).float() if kl else None
    adv, w = torch.randn(n, generator=g), torch.rand(n, generator=g)
    tok[4] = -1
    w[7] = 0.0
    kw = dict(clip_low=0.2, clip_high=0.28, kl_coef=kl, entropy_coef=ent)
    o = R.policy(x, tok, T, old, adv, ref=ref, weight=w, **kw)
    # no row close enough to a clip border for 32 bits to decide otherwise
    ratio = (logp - old.double()).exp()
    assert ((ratio - 0.8).abs() > 1e-4).all() and ((ratio - 1.28).abs() > 1e-4).all()
    d = lambda t: None if t is None else t.to(DEV)
    args = (x.to(DEV), tok.to(DEV), old.to(DEV), adv.to(DEV), T)
    terms = ears.policy_loss(*args, ref_logp=d(ref), **kw)
    step, grad = ears.policy_step(*args, ref_logp=d(ref), row_weight=w.to(DEV), **kw)
    for t in (terms, step):
        close(t.loss, o.loss, o.loss_scale * (2 * LOG_TOL) + abs(ent) * H_TOL)
        close(t.logp, o.logp, LOG_TOL)
        if ref is not None:
            close(t.kl, o.kl, o.kl_scale * LOG_TOL)
        assert (t.kl is None) == (ref is None) and (t.entropy is None) == (ent == 0.0)
        if ent:
            close(t.entropy, o.entropy, H_TOL)
    close_grad(grad, o.grad, o.scale, 2 * H_TOL if ent else G_TOL, dtype)
    assert not grad[4].any() and not grad[7].any()
    leaf = x.to(DEV).requires_grad_(True)
    t = ears.policy_loss(leaf, *args[1:], ref_logp=d(ref), **kw)
    assert not t.logp.requires_grad
    (t.loss * w.to(DEV)).sum().backward()
    close_grad(leaf.grad, o.grad, o.scale, 2 * H_TOL if ent else G_TOL, dtype)


def test_policy_rows_that_are_not_finite(ears):
    x, g = logits(5, 700, "fp32", 9)
    tok = torch.tensor([100, 699, 100, 100, 100], dtype=torch.int32)     # 699 is masked
    old = torch.zeros(5)
    ref = torch.zeros(5)
    adv = torch.ones(5)
    old[2], adv[3] = math.nan, math.inf
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    args = [t.to(DEV) for t in (x, tok, old, adv)]
    terms, grad = ears.policy_step(*args, ref_logp=ref.to(DEV), kl_coef=0.1, status=st)
    assert int(st) == ears.DEV_INVALID_INPUT
    assert torch.isnan(terms.loss[1:4]).all() and not grad[1:4].any()
    assert torch.isfinite(terms.loss[[0, 4]]).all()


# ---- distillation ---------------------------------------------------------------------------------

def teacher_case(n, V, k, dtype, T, seed, noise=0.8):
    t, g = logits(n, V, dtype, seed)
    x = (t.float() + noise * torch.randn(n, V, generator=g)).to(DT[dtype])
    vals, ids, lse = R.top_logits(t, k, T)
    return x, vals.float(), ids.to(torch.int32), lse.float(), g


@pytest.mark.parametrize("cluster", CLUSTERS)
@pytest.mark.parametrize("kind,tail", [("forward_kl", True), ("forward_kl", False), ("reverse_kl", True), ("jsd", True), ("jsd", False)])
@pytest.mark.parametrize("dtype,V,k", [("fp32", 1003, 5), ("bf16", 4099, 64), ("fp16", 33001, 128), ("bf16", 40, 1)])
def test_distill(ears, dtype, V, k, kind, tail, cluster):
    ears.set_row_cluster(cluster)
    n, T = 7, 1.2
    x, vals, ids, lse, g = teacher_case(n, V, k, dtype, T, 40 + V)
    w = torch.rand(n, generator=g)
    ids[2], vals[2] = -1, -math.inf                       # nothing listed
    if k > 3:
        ids[3, 1], vals[4, 2] = -1, -math.inf             # entries missing inside a list
    w[5] = 0.0
    kw = dict(kind=kind, mix=0.35)
    o = R.distill(x, T, vals, ids, lse=lse if tail else None, weight=w, **kw)
    teacher = ears.TopLogits(vals.to(DEV), ids.to(DEV), lse.to(DEV) if tail else None)
    loss = ears.distill_loss(x.to(DEV), teacher, T, **kw)
    l2, grad = ears.distill_step(x.to(DEV), teacher, T, row_weight=w.to(DEV), **kw)
    for l in (loss, l2):
        close(l, o.loss, o.loss_scale * (3 * LOG_TOL))
    close_grad(grad, o.grad, o.scale, G_TOL, dtype)
    assert not grad[2].any() and not grad[5].any() and float(l2[2]) == 0.0
    leaf = x.to(DEV).requires_grad_(True)
    (ears.distill_loss(leaf, teacher, T, **kw) * w.to(DEV)).sum().backward()
    close_grad(leaf.grad, o.grad, o.scale, G_TOL, dtype)
    over = x.to(DEV)
    _, same = ears.distill_step(over, teacher, T, row_weight=w.to(DEV), out_grad=over, **kw)
    assert torch.equal(over, grad)


@pytest.mark.parametrize("kind", ["forward_kl", "reverse_kl", "jsd"])
def test_distill_small_tails_keep_their_digits(ears, kind):
    """A draft whose mass outside the list is 1e-4 .. 1e-12, which 1 - sum q would not resolve."""
    n, V, k, T = 6, 5000, 8, 1.0
    g = torch.Generator().manual_seed(2)
    x = torch.randn(n, V, generator=g)
    ids = torch.stack([torch.randperm(V, generator=g)[:k] for _ in range(n)]).to(torch.int32)
    lift = torch.tensor([17.0, 20.0, 24.0, 28.0, 32.0, 36.0]).view(-1, 1)
    x.scatter_(1, ids.long(), lift + torch.randn(n, k, generator=g))
    t = torch.randn(n, V, generator=g)
    t.scatter_(1, ids.long(), 12.0 + torch.randn(n, k, generator=g))
    vals, lse = t.gather(1, ids.long()), torch.logsumexp(t.double(), 1).float()
    o = R.distill(x, T, vals, ids, lse=lse, kind=kind)
    loss, grad = ears.distill_step(x.to(DEV), ears.TopLogits(vals.to(DEV), ids.to(DEV), lse.to(DEV)), T, kind=kind)
    close(loss, o.loss, o.loss_scale * (3 * LOG_TOL))
    close_grad(grad, o.grad, o.scale, G_TOL, "fp32")


def test_distill_lists_at_the_edges(ears):
    V = 12
    x, g = logits(1, V, "fp32", 11, mask=False)
    # the whole vocabulary listed: nothing is left for the tail
    t = torch.randn(1, V, generator=g)
    vals, ids, lse = R.top_logits(t, V, 1.0)
    for kind in ("forward_kl", "reverse_kl", "jsd"):
        o = R.distill(x, 1.0, vals.float(), ids.to(torch.int32), lse=lse.float(), kind=kind)
        loss, grad = ears.distill_step(x.to(DEV), ears.TopLogits(vals.float().to(DEV), ids.to(torch.int32).to(DEV), lse.float().to(DEV)), kind=kind)
        close(loss, o.loss, o.loss_scale * (3 * LOG_TOL))
        close_grad(grad, o.grad, o.scale, G_TOL, "fp32")
    # a listed entry that the draft has masked: the forward divergence is infinite, its gradient is not
    y = x.clone()
    y[0, int(ids[0, 2])] = -math.inf
    four = ears.TopLogits(vals[:, :4].float().contiguous().to(DEV), ids[:, :4].to(torch.int32).contiguous().to(DEV), lse.float().to(DEV))
    loss, grad = ears.distill_step(y.to(DEV), four)
    assert float(loss[0]) == math.inf and torch.isfinite(grad).all()
    assert float(grad[0, int(ids[0, 2])]) < 0
    loss, grad = ears.distill_step(y.to(DEV), four, kind="jsd")
    o = R.distill(y, 1.0, four.values.cpu(), four.ids.cpu(), lse=four.lse.cpu(), kind="jsd")
    close(loss, o.loss, o.loss_scale * (3 * LOG_TOL))


def test_distill_longest_rows(ears):
    V, k, T = 1 << 20, 128, 1.0
    for dtype, cluster in (("fp32", 1), ("fp32", 0), ("bf16", 0)):
        ears.set_row_cluster(cluster)
        x, vals, ids, lse, g = teacher_case(2, V, k, dtype, T, 70)
        o = R.distill(x, T, vals, ids, lse=lse)
        teacher = ears.TopLogits(vals.to(DEV), ids.to(DEV), lse.to(DEV))
        loss, grad = ears.distill_step(x.to(DEV), teacher, T)
        for l in (loss, ears.distill_loss(x.to(DEV), teacher, T)):
            close(l, o.loss, o.loss_scale * (3 * LOG_TOL))
        close_grad(grad, o.grad, o.scale, G_TOL, dtype)


def test_distill_lists_that_cannot_be_used(ears):
    n, V, k = 6, 300, 4
    x, vals, ids, lse, g = teacher_case(n, V, k, "fp32", 1.0, 12)
    ids[0, 3] = ids[0, 1]                   # named twice
    ids[1, 0] = V
    ids[2, 0] = -2
    vals[3, 1] = math.nan
    lse[4] = math.inf
    for cluster in (1, 2):
        ears.set_row_cluster(cluster)
        st = torch.zeros(1, dtype=torch.int32, device=DEV)
        loss, grad = ears.distill_step(x.to(DEV), ears.TopLogits(vals.to(DEV), ids.to(DEV), lse.to(DEV)), status=st)
        assert int(st) == ears.DEV_INVALID_INPUT
        assert torch.isnan(loss[:5]).all() and not grad[:5].any()
        o = R.distill(x[5:], 1.0, vals[5:], ids[5:], lse=lse[5:])
        close(loss[5:], o.loss, o.loss_scale * (3 * LOG_TOL))


# ---- streams, graphs, autograd ---------------------------------------------------------------------

def test_gradients_agree_with_differences_of_the_loss(ears):
    x, vals, ids, lse, g = teacher_case(1, 64, 6, "fp32", 1.0, 13)
    x = torch.where(torch.isinf(x), -3.0, x)
    teacher = ears.TopLogits(vals.to(DEV), ids.to(DEV), lse.to(DEV))
    _, grad = ears.distill_step(x.to(DEV), teacher, kind="jsd")
    f = lambda y: float(R.distill(y, 1.0, vals, ids, lse=lse, kind="jsd").loss)
    for v in (int(ids[0, 0]), int(ids[0, 5]), 3, 40):
        hi, lo = x.double(), x.double()
        hi[0, v] += 1e-4
        lo[0, v] -= 1e-4
        assert abs((f(hi) - f(lo)) / 2e-4 - float(grad[0, v])) < 1e-6


def test_another_stream_and_side_by_side_calls(ears):
    x, g = logits(40, 30000, "bf16", 14)
    tok = torch.randint(4000, 20000, (40,), generator=g, dtype=torch.int32)
    xg, tg, dl = x.to(DEV), tok.to(DEV), torch.ones(40, device=DEV)
    want = ears.token_logprobs_step(xg, tg, dl)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    outs = []
    for _ in range(4):
        for s in streams:
            with torch.cuda.stream(s):
                outs.append(ears.token_logprobs_step(xg, tg, dl))
    explicit = ears.token_logprobs(xg, tg, stream=streams[0])
    torch.cuda.synchronize()
    assert torch.equal(explicit, want[0])
    for o in outs:
        assert torch.equal(o[0], want[0]) and torch.equal(o[2], want[2])


def test_calls_queued_behind_one_another_see_what_came_before(ears):
    """A chain in which every call reads what the one before wrote, alternating with other kernels, long and short."""
    g = torch.Generator().manual_seed(18)
    for n, V in ((3, 900), (40, 30000), (700, 5000)):
        x = torch.randn(n, V, generator=g)
        tok = torch.randint(0, V, (n,), generator=g, dtype=torch.int32).to(DEV)
        dl = torch.ones(n, device=DEV)

        def chain(sync):
            y, logps = x.to(DEV), []
            for i in range(12):
                if i % 3 == 2:
                    y.mul_(1.01)
                logp, _, grad = ears.token_logprobs_step(y, tok, dl)
                ears.token_logprobs_step(grad, tok, dl, out_grad=grad)
                y = y + grad * 0.1
                logps.append(logp)
                if sync:
                    torch.cuda.synchronize()
            return torch.stack(logps), y
        want, got = chain(True), chain(False)
        assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])


def test_captured_steps_replay_on_new_inputs(ears):
    n, V, k = 9, 20011, 16
    x, vals, ids, lse, g = teacher_case(n, V, k, "bf16", 1.0, 15)
    xg, teacher = x.to(DEV), ears.TopLogits(vals.to(DEV), ids.to(DEV), lse.to(DEV))
    tok = ids[:, 0].contiguous().to(DEV)
    dl = torch.ones(n, device=DEV)
    leaf = xg.clone().requires_grad_(True)
    alive = ears.distill_loss(leaf, teacher).sum()          # an eager graph of its own stays alive meanwhile
    run = lambda: (ears.top_logits(xg, k), ears.distill_step(xg, teacher), ears.token_logprobs_step(xg, tok, dl, dl))
    run()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        top, (loss, grad), (logp, H, g2) = run()
        with pytest.raises(RuntimeError, match="cannot be recorded"):
            ears.distill_loss(leaf, teacher)
        with pytest.raises(RuntimeError, match="cannot be recorded"):
            ears.token_logprobs(leaf, tok)
    for seed in (1, 2):
        xg.copy_((x.float() + torch.randn(n, V, generator=torch.Generator().manual_seed(seed))).to(torch.bfloat16).to(DEV))
        graph.replay()
        torch.cuda.synchronize()
        e_top, (e_loss, e_grad), (e_logp, e_H, e_g2) = run()
        for a, b in ((top.ids, e_top.ids), (top.lse, e_top.lse), (loss, e_loss), (grad, e_grad), (logp, e_logp), (H, e_H), (g2, e_g2)):
            assert torch.equal(a, b)
    alive.backward()
    assert torch.isfinite(leaf.grad).all()


def test_inputs_that_need_converting_give_the_same_results(ears):
    n, V, k = 7, 3001, 9
    x, vals, ids, lse, g = teacher_case(n, V, k, "fp32", 1.0, 17)
    xg = x.to(DEV)
    tok = ids[:, 0].contiguous().to(DEV)
    f = [torch.randn(n, generator=g).to(DEV) for _ in range(4)]
    wide = [torch.stack([t, t], 1)[:, 0] for t in f]                 # strided
    double = [t.double() for t in f]
    transposed = xg.t().contiguous().t()
    teacher = ears.TopLogits(vals.to(DEV), ids.to(DEV), lse.to(DEV))
    other = ears.TopLogits(vals.double().to(DEV), ids.long().to(DEV), lse.double().to(DEV))

    def same(a, b):
        for u, v in zip(a, b):
            assert (u is None and v is None) or torch.equal(u, v)
    for a, b in ((f, wide), (f, double)):
        for logits, t in ((xg, tok.long()), (transposed, tok)):
            same(ears.token_logprobs_step(xg, tok, a[0], a[1]), ears.token_logprobs_step(logits, t, b[0], b[1]))
            pa, ga = ears.policy_step(xg, tok, a[0], a[1], ref_logp=a[2], kl_coef=0.1, entropy_coef=0.01, row_weight=a[3])
            pb, gb = ears.policy_step(logits, t, b[0], b[1], ref_logp=b[2], kl_coef=0.1, entropy_coef=0.01, row_weight=b[3])
            same(pa + (ga,), pb + (gb,))
            same(ears.policy_loss(xg, tok, a[0], a[1], entropy=1), ears.policy_loss(logits, t, b[0], b[1], entropy=True))
            same(ears.distill_step(xg, teacher, kind="jsd", row_weight=a[3]), ears.distill_step(logits, other, kind="jsd", row_weight=b[3]))
            same([ears.distill_loss(xg, teacher)], [ears.distill_loss(logits, other)])
            same(ears.token_logprobs(xg, tok, entropy=1), ears.token_logprobs(logits, t, entropy=True))
    same(ears.top_logits(xg, 4), ears.top_logits(transposed, 4))
    same(ears.top_logits(xg, 4), [t.squeeze(0) for t in ears.top_logits(xg.unsqueeze(0), torch.tensor(4).item(), 1)])


def test_calls_that_are_refused(ears):
    x = torch.zeros(3, 50, device=DEV)
    tok, f = torch.zeros(3, dtype=torch.int32, device=DEV), torch.zeros(3, device=DEV)
    teacher = ears.top_logits(x, 4)
    for bad in (0.0, -1.0, float("nan"), float("inf")):
        with pytest.raises(ears.EarsError):
            ears.token_logprobs(x, tok, bad)
    for k in (0, 129, -3):
        with pytest.raises(ValueError):
            ears.top_logits(x, k)
    with pytest.raises(ValueError):
        ears.token_logprobs(x, tok[:2])
    with pytest.raises(ValueError):
        ears.token_logprobs(x, tok.cpu())
    with pytest.raises(TypeError):
        ears.token_logprobs(x, f)
    with pytest.raises(ValueError):
        ears.distill_loss(x, teacher, kind="no such kind")
    with pytest.raises(ears.EarsError):
        ears.distill_loss(x, teacher, kind="jsd", mix=1.0)
    with pytest.raises(ears.EarsError):
        ears.distill_loss(x, ears.TopLogits(teacher.values, teacher.ids, None), kind="reverse_kl")
    with pytest.raises(ears.EarsError):
        ears.policy_loss(x, tok, f, f, kl_coef=0.1)
    with pytest.raises(ValueError):
        ears.token_logprobs_step(x, tok, f, out_grad=torch.zeros(3, 51, device=DEV))
    with pytest.raises(ears.EarsError):                               # rows that share memory
        ears.token_logprobs_step(x, tok, f, out_grad=torch.zeros(50, device=DEV).expand(3, 50))
    with pytest.raises(ears.EarsError):                               # overlaps the logits in part
        buf = torch.zeros(200, device=DEV)
        ears.token_logprobs_step(buf[:150].view(3, 50), tok, f, out_grad=buf[50:].view(3, 50))
    with pytest.raises(ValueError):
        ears.top_logits(x[:0], 2)
    with pytest.raises(ValueError):
        ears.top_logits(x, 2, status=torch.zeros(1, device=DEV))


def test_autograd_matches_the_step_and_notices_changed_logits(ears):
    n, V = 6, 9001
    x, g = logits(n, V, "bf16", 16)
    tok = torch.randint(1200, 8000, (n,), generator=g, dtype=torch.int32).to(DEV)
    dl, dh = torch.randn(n, generator=g).to(DEV), torch.randn(n, generator=g).to(DEV)
    leaf = x.to(DEV).requires_grad_(True)
    logp, H = ears.token_logprobs(leaf, tok, entropy=True)
    torch.autograd.backward([logp, H], [dl, dh])
    _, _, grad = ears.token_logprobs_step(x.to(DEV), tok, dl, dh)
    assert torch.equal(leaf.grad, grad)
    leaf2 = x.to(DEV).requires_grad_(True)
    y = leaf2 * 1.0
    out = ears.token_logprobs(y, tok)
    with torch.no_grad():
        y.add_(1.0)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        out.sum().backward()
    old = torch.zeros(n, device=DEV)
    out = ears.policy_loss(leaf2, tok, old, dl).loss
    old.add_(1.0)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        out.sum().backward()
    # the entropy's gradient alone, and only the log probability's
    for pick in (0, 1):
        leaf.grad = None
        outs = ears.token_logprobs(leaf, tok, entropy=True)
        outs[pick].sum().backward()
        o = R.token_logprobs(x, tok.cpu(), 1.0, *((torch.ones(n), None) if pick == 0 else (torch.zeros(n), torch.ones(n))))
        close_grad(leaf.grad, o.grad, o.scale, 2 * H_TOL, "bf16")


@pytest.mark.parametrize("n", [330, 700])
@pytest.mark.parametrize("V", [3, 17, 700, 2030, 6001])
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
def test_short_rows_in_numbers(ears, dtype, V, n):
    """Rows of one round of a warp and more, more of them than SMs and than four per SM, at every kind of start."""
    x, g = logits(n, V + 3, dtype, 90 + V, mask=False)
    dev = x.to(DEV)
    tok, dl = torch.randint(0, V, (n,), generator=g, dtype=torch.int32), torch.randn(n, generator=g)
    k = min(V, 40)
    pick = list(range(12)) + list(range(n - 12, n))
    for off in (0, 1, 3):
        rows, at = x[pick][:, off:off + V], dev[:, off:off + V]
        o = R.token_logprobs(rows, tok[pick], 0.9, dl[pick])
        logp, _, grad = ears.token_logprobs_step(at, tok.to(DEV), dl.to(DEV), None, 0.9)
        close(logp[pick], o.logp, LOG_TOL)
        close_grad(grad[pick], o.grad, o.scale, G_TOL, dtype)
        close(ears.token_logprobs(at, tok.to(DEV), 0.9)[pick], o.logp, LOG_TOL)
        teacher = ears.top_logits((at.float() * 0.7).to(DT[dtype]), k)
        held = [t[pick].cpu() for t in teacher]
        od = R.distill(rows, 1.0, held[0], held[1], lse=held[2], kind="jsd", weight=dl[pick].abs())
        loss, grad = ears.distill_step(at, teacher, kind="jsd", row_weight=dl.abs().to(DEV))
        close(loss[pick], od.loss, od.loss_scale * (3 * LOG_TOL))
        close_grad(grad[pick], od.grad, od.scale, G_TOL, dtype)
        close(ears.distill_loss(at, teacher, kind="jsd")[pick], od.loss, od.loss_scale * (3 * LOG_TOL))
        leaf = at.clone().requires_grad_(True)
        (ears.distill_loss(leaf, teacher, kind="jsd") * dl.abs().to(DEV)).sum().backward()
        close_grad(leaf.grad[pick], od.grad, od.scale, G_TOL, dtype)


@pytest.mark.parametrize("convert", [False, True])
def test_a_gradient_written_over_saved_logits_is_noticed(ears, convert):
    n, V = 3, 700
    x, _ = logits(n, V, "bf16", 18)
    leaf = x.to(DEV).requires_grad_(True)
    tok = torch.zeros(n, dtype=torch.int64 if convert else torch.int32, device=DEV)   # converted tensors go through ctypes
    f = torch.ones(n, dtype=torch.float64 if convert else torch.float32, device=DEV)
    teacher = ears.top_logits(x.to(DEV), 4)
    if convert:
        teacher = teacher._replace(ids=teacher.ids.long())
    steps = (lambda y: ears.token_logprobs_step(y, tok, f, out_grad=y), lambda y: ears.policy_step(y, tok, f, f, out_grad=y),
             lambda y: ears.distill_step(y, teacher, out_grad=y))
    for step in steps:
        y = leaf * 1.0
        out = ears.token_logprobs(y, tok)
        step(y.detach())                       # shares its memory and its version with y
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            out.sum().backward()
        y = leaf * 1.0                         # the gradient handed on from where the logits were
        step(y.detach())
        leaf.grad = None
        y.backward(y.detach())
        assert torch.equal(leaf.grad, y.detach())


def test_a_round_of_drafting_and_learning(ears):
    """Verification, capture of the teacher, scoring, one distillation step and one policy step, as a program
    that trains its draft and its policy from the same rows runs them."""
    from paper_2512_13194_b200 import synth
    B, K, V, T = 10, 4, 30011, 0.9
    w, t, d, x = synth.tiny_inputs(B, K, V, "bf16", seed=77, noise=1.0, temperature=T)
    tg, dg, xg = t.to(DEV), d.to(DEV), x.to(DEV)
    s = ears.EarsSampler(temperature=T, beta=0.2, seed=5, report_logprobs=True, teacher_k=32)
    res = s(tg, dg, xg)
    base = ears.EarsSampler(temperature=T, beta=0.2, seed=5)(tg, dg, xg)
    assert torch.equal(res.tokens, base.tokens) and torch.equal(res.accept_len, base.accept_len)
    n = res.accept_len.cpu()
    emitted = res.tokens.cpu()
    o = R.token_logprobs(t.view(-1, V), emitted.view(-1), T)
    close(res.logprobs.view(-1), o.logp, LOG_TOL)
    vals, ids, lse = R.top_logits(t[:, :K].reshape(-1, V), 32, T)
    live = (torch.arange(K)[None] <= n[:, None]).view(-1)
    assert torch.equal(res.teacher.ids.cpu().view(-1, 32).long()[live], ids[live])
    assert (res.teacher.ids.cpu().view(-1, 32)[~live] == -1).all()
    count = float(live.sum())
    weight = torch.full((B, K), 1.0 / count, device=DEV)
    loss, grad = ears.distill_step(dg, res.teacher, T, row_weight=weight)
    od = R.distill(d.view(-1, V), T, res.teacher.values.cpu().view(-1, 32), res.teacher.ids.cpu().view(-1, 32),
                   lse=res.teacher.lse.cpu().view(-1), weight=weight.cpu().view(-1))
    close(loss.view(-1), od.loss, od.loss_scale * (3 * LOG_TOL))
    close_grad(grad.view(-1, V), od.grad, od.scale, G_TOL, "bf16")
    assert not grad.view(-1, V)[(~live).to(DEV)].any()
    adv = torch.randn(B, K + 1, generator=torch.Generator().manual_seed(1)).to(DEV)
    terms, pg = ears.policy_step(tg, res.tokens, res.logprobs, adv, T, ref_logp=res.logprobs, kl_coef=0.1)
    op = R.policy(t.view(-1, V), emitted.view(-1), T, res.logprobs.cpu().view(-1), adv.cpu().view(-1),
                  ref=res.logprobs.cpu().view(-1), kl_coef=0.1)
    close(terms.loss.view(-1), op.loss, op.loss_scale * (2 * LOG_TOL))
    close_grad(pg.view(-1, V), op.grad, op.scale, G_TOL, "bf16")
    # per-sequence temperatures go the same way
    Ts = torch.linspace(0.7, 1.3, B)
    s2 = ears.EarsSampler(temperature=Ts.to(DEV), beta=0.2, seed=5, report_logprobs=True, teacher_k=4)
    r2 = s2(tg, dg, xg)
    o2 = R.token_logprobs(t.view(-1, V), r2.tokens.cpu().view(-1), Ts.repeat_interleave(K + 1))
    close(r2.logprobs.view(-1), o2.logp, LOG_TOL)


@pytest.mark.parametrize("dtype,V", [("fp32", 1003), ("bf16", 9001), ("fp16", 33001)])
@pytest.mark.parametrize("cluster", [0, 1, 4])
def test_a_temperature_per_sequence_in_every_loss_step_and_backward_call(ears, dtype, V, cluster):
    ears.set_row_cluster(cluster)
    B, Rr, k = 4, 3, 9
    n = B * Rr
    Ts = torch.tensor([0.5, 0.9, 1.0, 1.7])
    T = Ts.repeat_interleave(Rr)
    x, g = logits(n, V, dtype, 200 + V)
    t = (x.float() + 0.8 * torch.randn(n, V, generator=g)).to(DT[dtype])
    tok = torch.randint(V // 8, V - V // 16, (n,), generator=g, dtype=torch.int32)
    dl, dh, w = torch.randn(n, generator=g), torch.randn(n, generator=g), torch.rand(n, generator=g)
    vals, ids, lse = R.top_logits(t, k, T)
    held = (vals.float(), ids.to(torch.int32), lse.float())
    logp = R.token_logprobs(x, tok, T).logp
    old, ref = (logp + 0.3).float(), (logp - 0.2).float()
    row = lambda a: a.view(B, Rr, *a.shape[1:]).to(DEV)
    flat = lambda a: a.reshape(n, *a.shape[2:])
    xg, tg, seq = row(x), row(tok), Ts.to(DEV)
    coefs = dict(kl_coef=0.1, entropy_coef=0.02)

    top = ears.top_logits(row(t), k, seq_temperature=seq)
    assert torch.equal(flat(top.ids).cpu(), held[1])
    close(flat(top.lse), lse, LOG_TOL)
    o = R.token_logprobs(x, tok, T, dl, dh)
    lp, H, grad = ears.token_logprobs_step(xg, tg, row(dl), row(dh), seq_temperature=seq)
    close(flat(lp), o.logp, LOG_TOL)
    close(flat(H), o.entropy, H_TOL)
    close_grad(flat(grad), o.grad, o.scale, 2 * H_TOL, dtype)
    leaf = xg.clone().requires_grad_(True)
    torch.autograd.backward(ears.token_logprobs(leaf, tg, entropy=True, seq_temperature=seq), [row(dl), row(dh)])
    close_grad(flat(leaf.grad), o.grad, o.scale, 2 * H_TOL, dtype)

    o = R.policy(x, tok, T, old, dl, ref=ref, weight=w, **coefs)
    args = (tg, row(old), row(dl))
    terms, grad = ears.policy_step(xg, *args, ref_logp=row(ref), row_weight=row(w), seq_temperature=seq, **coefs)
    close(flat(terms.loss), o.loss, o.loss_scale * (2 * LOG_TOL) + 0.02 * H_TOL)
    close_grad(flat(grad), o.grad, o.scale, 2 * H_TOL, dtype)
    leaf.grad = None
    terms = ears.policy_loss(leaf, *args, ref_logp=row(ref), seq_temperature=seq, **coefs)
    close(flat(terms.loss), o.loss, o.loss_scale * (2 * LOG_TOL) + 0.02 * H_TOL)
    (terms.loss * row(w)).sum().backward()
    close_grad(flat(leaf.grad), o.grad, o.scale, 2 * H_TOL, dtype)

    teacher = ears.TopLogits(*map(row, held))
    for kind in ("forward_kl", "reverse_kl", "jsd"):
        o = R.distill(x, T, *held[:2], lse=held[2], kind=kind, weight=w)
        loss, grad = ears.distill_step(xg, teacher, kind=kind, row_weight=row(w), seq_temperature=seq)
        close(flat(loss), o.loss, o.loss_scale * (3 * LOG_TOL))
        close_grad(flat(grad), o.grad, o.scale, G_TOL, dtype)
        leaf.grad = None
        loss = ears.distill_loss(leaf, teacher, kind=kind, seq_temperature=seq)
        close(flat(loss), o.loss, o.loss_scale * (3 * LOG_TOL))
        (loss * row(w)).sum().backward()
        close_grad(flat(leaf.grad), o.grad, o.scale, G_TOL, dtype)


@pytest.mark.parametrize("sliced", [False, True])
def test_backward_through_hooks_checkpoints_and_twice(ears, sliced):
    """Logits offloaded between the passes, recomputed, or kept for a second backward pass: the same gradient; and nothing of
    their size is left behind it."""
    from torch.utils.checkpoint import checkpoint
    B, Rr, V, k = 3, 5, 40003, 8
    x, vals, ids, lse, g = teacher_case(B * Rr, V, k, "bf16", 1.0, 19)
    base = x.view(B, Rr, V).to(DEV)
    leaf = base.clone().requires_grad_(True)
    at = (lambda t: t[:, :-1]) if sliced else (lambda t: t)
    n = at(base).shape[:2]
    row = lambda t: at(t.view(B, Rr, *t.shape[1:])).contiguous().to(DEV)
    teacher, tok, f = ears.TopLogits(row(vals.float()), row(ids.to(torch.int32)), row(lse.float())), row(ids[:, 0].to(torch.int32)), torch.ones(n, device=DEV)
    losses = (lambda y: ears.distill_loss(y, teacher, kind="jsd"), lambda y: ears.token_logprobs(y, tok),
              lambda y: ears.policy_loss(y, tok, -f, f, entropy_coef=0.01).loss)
    for loss in losses:
        def grad(run):
            leaf.grad = None
            run()
            torch.cuda.synchronize()
            return leaf.grad
        want = grad(lambda: loss(at(leaf * 1.0)).sum().backward())
        assert want.any()

        def offloaded():
            with torch.autograd.graph.save_on_cpu():
                loss(at(leaf * 1.0)).sum().backward()

        def twice():
            out = loss(at(leaf * 1.0)).sum()
            out.backward(retain_graph=True)
            first, leaf.grad = leaf.grad, None
            out.backward()
            assert torch.equal(first, leaf.grad)
            with pytest.raises(RuntimeError, match="second time"):
                out.backward()
        for run in (offloaded, twice, lambda: checkpoint(lambda y: loss(at(y * 1.0)), leaf, use_reentrant=False).sum().backward()):
            assert torch.equal(grad(run), want)
        leaf.grad = None
        torch.cuda.synchronize()
        before = torch.cuda.memory_allocated()
        out = loss(at(leaf * 1.0))
        out.sum().backward()
        leaf.grad = None
        assert torch.cuda.memory_allocated() - before < V * 2 and out.grad_fn is not None


def test_ids_beyond_32_bits_make_their_rows_unusable(ears):
    V, wide = 300, [2**32 + 5, 2**31, -2**32 - 1, -1]
    x, g = logits(5, V, "fp32", 21)
    tok = torch.tensor(wide + [100])
    for logits_ in (x.to(DEV), x.to(DEV).requires_grad_(True)):
        st = torch.zeros(1, dtype=torch.int32, device=DEV)
        logp = ears.token_logprobs(logits_, tok.to(DEV), status=st)
        assert int(st) == ears.DEV_INVALID_INPUT
        logp = logp.detach()
        assert torch.isnan(logp[:3]).all() and float(logp[3]) == 0.0
        close(logp[4:], R.token_logprobs(x[4:], tok[4:], 1.0).logp, LOG_TOL)
    ids = torch.tensor([[5, w] for w in wide + [100]])
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    loss, grad = ears.distill_step(x.to(DEV), ears.TopLogits(torch.zeros(5, 2, device=DEV), ids.to(DEV), None), status=st)
    assert int(st) == ears.DEV_INVALID_INPUT
    assert torch.isnan(loss[:3]).all() and not grad[:3].any()
    o = R.distill(x[3:], 1.0, torch.tensor([[0.0, -math.inf], [0.0, 0.0]]), ids[3:])
    close(loss[3:], o.loss, o.loss_scale * (3 * LOG_TOL))      # entry 5 of the last row is masked: infinite
    close_grad(grad[3:4], o.grad[:1], o.scale[:1], G_TOL, "fp32")
    assert torch.isfinite(grad[4]).all()


def test_plain_calls_go_through_the_module(ears):
    from paper_2512_13194_b200 import rows
    assert rows._plain_calls().__name__.endswith("ears_torch")
    out = rows._plain_calls().token_logprobs(torch.zeros(3, 50, device=DEV), torch.zeros(3, dtype=torch.int32, device=DEV), False, 1.0, None, None)
    assert out is not None and out[1] is None


def test_running_out_of_memory_is_told_as_such(ears):
    """A broadcast row has a gradient of 8 TB."""
    n = 1 << 21
    x = torch.zeros(1, 1 << 20, device=DEV).expand(n, 1 << 20)
    tok, f = torch.zeros(n, dtype=torch.int32, device=DEV), torch.zeros(n, device=DEV)
    teacher = ears.TopLogits(torch.zeros(n, 1, device=DEV), torch.zeros(n, 1, dtype=torch.int32, device=DEV), None)
    for step in (lambda t: ears.token_logprobs_step(x, t, f), lambda t: ears.policy_step(x, t, f, f), lambda t: ears.distill_step(x, teacher)):
        for t in (tok, tok.long()):                      # through the module, through ctypes
            with pytest.raises(torch.OutOfMemoryError):
                step(t)
    ears.token_logprobs(x[:3], tok[:3])


@pytest.mark.parametrize("T", [1e30, 3e38, 2e45, 1e300])
@pytest.mark.parametrize("dtype,V,n", [("fp32", 1003, 6), ("bf16", 9001, 6), ("fp16", 40, 400)])
def test_temperatures_so_high_that_32_bits_hold_nothing_of_their_inverse(ears, dtype, V, n, T):
    """Every entry that is not masked has the same probability; masked ones have none."""
    x, g = logits(n, V, dtype, 22)
    k = 5
    tok = torch.randint(V // 8 + 1, V - V // 16 - 1, (n,), generator=g, dtype=torch.int32)
    dl, dh = torch.randn(n, generator=g), torch.randn(n, generator=g)
    vals, ids, lse = R.top_logits(x, k, T)
    Ts = [(T, {})] + ([(1.0, dict(seq_temperature=torch.tensor([T], device=DEV)))] if T < 1e38 or T == 3e38 else [])
    for scalar, kw in Ts:
        exact = T if not kw else float(torch.tensor(T))
        o = R.token_logprobs(x, tok, exact, dl, dh)
        top = ears.top_logits(x.to(DEV), k, scalar, **kw)
        assert torch.equal(top.ids.cpu().long(), ids)
        close(top.lse, lse, LOG_TOL)
        logp, H, grad = ears.token_logprobs_step(x.to(DEV), tok.to(DEV), dl.to(DEV), dh.to(DEV), scalar, **kw)
        close(logp, o.logp, LOG_TOL)
        close(H, o.entropy, H_TOL)
        close_grad(grad, o.grad, o.scale, 2 * H_TOL, dtype)
        leaf = x.to(DEV).requires_grad_(True)
        torch.autograd.backward(ears.token_logprobs(leaf, tok.to(DEV), scalar, entropy=True, **kw), [dl.to(DEV), dh.to(DEV)])
        close_grad(leaf.grad, o.grad, o.scale, 2 * H_TOL, dtype)
        teacher = ears.TopLogits(vals.float().to(DEV), ids.to(torch.int32).to(DEV), lse.float().to(DEV))
        o = R.distill(x, exact, vals.float(), ids, lse=lse.float(), kind="jsd")
        loss, grad = ears.distill_step(x.to(DEV), teacher, scalar, kind="jsd", **kw)
        close(loss, o.loss, o.loss_scale * (3 * LOG_TOL))
        close_grad(grad, o.grad, o.scale, G_TOL, dtype)


@pytest.mark.parametrize("cluster", [0, 1, 4])
def test_a_kl_term_without_weight_stays_out_of_the_loss(ears, cluster):
    """ref_logp with kl_coef = 0 only reports the term: infinite where the token is masked or the reference far above, and
    neither the loss nor the gradient take notice."""
    ears.set_row_cluster(cluster)
    n, V = 6, 7001
    x, g = logits(n, V, "fp32", 23)
    tok = torch.tensor([V - 1, 2000, 2001, -1, 2002, V - 2], dtype=torch.int32)      # the first and last are masked
    adv, w = torch.randn(n, generator=g), torch.rand(n, generator=g)
    logp = R.token_logprobs(x, tok, 1.0).logp
    old = torch.where(torch.isinf(logp), -5.0, logp + 0.1).float()
    ref = torch.tensor([-3.0, 0.0, 1000.0, 0.0, -math.inf, -2.0])
    d = lambda t: t.to(DEV)
    args = (d(x), d(tok), d(old), d(adv))
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    want, gw = ears.policy_step(*args, row_weight=d(w), entropy_coef=0.01)
    assert torch.isfinite(want.loss).all()
    got, gg = ears.policy_step(*args, row_weight=d(w), entropy_coef=0.01, ref_logp=d(ref), status=st)
    assert torch.equal(got.loss, want.loss) and torch.equal(got.logp, want.logp) and torch.equal(gg, gw) and int(st) == 0
    o = R.policy(x, tok, 1.0, old, adv, entropy_coef=0.01, weight=w)
    close(got.loss, o.loss, o.loss_scale * (2 * LOG_TOL) + 0.01 * H_TOL)
    delta = ref[1].double() - logp[1]
    kl = torch.tensor([math.inf, float(delta.exp() - delta - 1), math.inf, 0.0, math.inf, math.inf], dtype=torch.float64)
    close(got.kl, kl, LOG_TOL * (1 + float(delta.exp())))
    leaf = d(x).requires_grad_(True)
    terms = ears.policy_loss(leaf, *args[1:], entropy_coef=0.01, ref_logp=d(ref), status=st)
    (terms.loss * d(w)).sum().backward()
    assert int(st) == 0
    close_grad(leaf.grad, o.grad, o.scale, 2 * H_TOL, "fp32")


def test_the_same_call_gives_the_same_bits(ears):
    """Over every form that rows may take: many short rows, few, middling, long, split."""
    g = torch.Generator().manual_seed(24)
    for n, V, dtype in ((20, 700, "bf16"), (700, 700, "fp32"), (3000, 6000, "bf16"), (40, 33001, "fp16"), (3, 128256, "bf16")):
        x = (torch.randn(n, V + 3, generator=g) * 2).to(DT[dtype]).to(DEV)
        k = 12
        f, tok = torch.randn(n, generator=g).to(DEV), torch.randint(0, V, (n,), generator=g, dtype=torch.int32).to(DEV)

        def run(at):
            teacher = ears.top_logits(at, k)
            yield from teacher
            yield from ears.token_logprobs(at, tok, entropy=True)
            yield from ears.token_logprobs_step(at, tok, f, f)
            yield from ears.distill_step(at * 0.5, teacher, kind="jsd")
        for at in (x[:, :V], x[:, 1:V + 1]):
            first = list(run(at))
            for _ in range(3):
                for a, b in zip(first, run(at)):
                    assert torch.equal(a, b)


def test_ids_of_64_bits_go_through_the_module(ears):
    from paper_2512_13194_b200 import rows
    n, V, k = 6, 900, 5
    x, g = logits(2 * n, V, "bf16", 25)
    x3 = x.view(2, n, V).to(DEV)
    tok = torch.randint(V // 8, V - V // 16, (2, n), generator=g).to(DEV)
    f = torch.randn(2, n, generator=g).to(DEV)
    acc = torch.tensor([2, -1], device=DEV)
    narrow = lambda t: t.to(torch.int32)
    teacher = ears.top_logits(x3, k)
    plain = rows._plain_calls()
    for of in (lambda i: plain.token_logprobs(x3, i(tok), True, 1.0, None, None), lambda i: plain.top_logits(x3, i(acc), k, 1.0, None, None),
               lambda i: plain.token_logprobs_step(x3, i(tok), f, None, None, 1.0, None, None),
               lambda i: plain.policy(x3, i(tok), f, None, f, 0.2, 0.2, 0.0, 0.0, False, True, None, None, 1.0, None, None),
               lambda i: plain.distill(x3, teacher.values, i(teacher.ids.long()), teacher.lse, 2, 0.5, True, None, None, 1.0, None, None)):
        wide, small = of(lambda t: t), of(narrow)
        assert wide is not None and len(wide) == len(small)
        for a, b in zip(wide, small):
            assert (a is None and b is None) or torch.equal(a, b)
    assert plain.token_logprobs(x3, tok.t(), True, 1.0, None, None) is None


def test_tokens_of_every_integer_type(ears):
    x, g = logits(4, 100, "fp32", 26)
    tok = torch.tensor([20, 50, 93, 13], dtype=torch.int32)
    want = ears.token_logprobs(x.to(DEV), tok.to(DEV))
    for dtype in (torch.int8, torch.uint8, torch.int16, torch.int64, torch.uint16, torch.uint32, torch.uint64):
        assert torch.equal(ears.token_logprobs(x.to(DEV), tok.to(dtype).to(DEV)), want)
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    far = torch.tensor([2**64 - 1, 2**63 + 7, 2**32, 13], dtype=torch.uint64)
    logp = ears.token_logprobs(x.to(DEV), far.to(DEV), status=st)
    assert torch.isnan(logp[:3]).all() and torch.equal(logp[3], want[3]) and int(st) == ears.DEV_INVALID_INPUT
