"""Attention over the 4-bit cache where values' scales, minima and weights differ by powers of two, and where parameters are not finite.

Tolerances as in test_gpu_kv.py, but for two terms.  A relative error e in every weight moves a result by at most 2 e drift with drift =
sum_t p_t |v_t - out| (not the farthest token's distance).  Where a block has a row's tokens to itself, its 32 lanes of a row add n / 32
weights each, one after the other: (n / 32) 2^-24 relative where all roundings go one way, as they do for equal weights beside a large one; and its
four warps add n / 64 products each of 16 tokens, which truncate, 2^-23 each: n 2^-29 both, beside test_gpu_kv.py's 2^-18.  Products P s that
half precision holds as subnormals are off by 2^-12 of the row's and group's sum of them, times up to 15 codes: 2^-11 spread, spread = 7.5 sum_t p_t s_t
of that row and group; for half-precision queries, 7.5 codes either way, half of that.  Nothing goes by the largest scale of a token that weighs
nothing, of another group, or of a token that the row does not see.
"""
import math

import pytest
import torch

from oracle import kv as O

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"bf16": torch.bfloat16, "fp16": torch.float16}


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def pool(n, D, page, seed, keys=0.0):
    """One sequence of n tokens, one head: keys that are zero but for their minimum in dimensions 0 .. 63, values with scales
    between 1/2 and 3/2 and minima about 0, pages in random order."""
    g = torch.Generator().manual_seed(seed)
    held = -(-n // page)
    codes = torch.randint(0, 256, (held, 2, 1, page, D // 2), generator=g, dtype=torch.uint8)
    params = torch.stack([torch.rand(held, 2, 1, page, D // 64, generator=g) + 0.5, torch.randn(held, 2, 1, page, D // 64, generator=g)], -1)
    codes[:, 0] = 0
    params[:, 0, ..., 1] = 0.0
    pages = torch.randperm(held, generator=g)
    score = torch.as_tensor(keys, dtype=torch.float32).expand(n)
    t = torch.arange(n)
    params[pages[t // page], 0, 0, t % page, 0, 1] = score
    return codes, params.bfloat16(), pages.int()[None], g


def place(pages, t, page):
    return int(pages[0, t // page]), t % page


def expect(q, codes, params, pages, start, dtype, scale=1.0):
    """Results, log-sum-exps and tolerances of the rows of one sequence with one key head, in 64 bits."""
    Q, HQ, D = q.shape[1:]
    page = codes.shape[3]
    last = start + Q
    ids = pages[0, : -(-last // page)].long()
    c, m = (x[ids].permute(1, 2, 0, 3, *range(4, x.dim())).flatten(2, 3)[:, 0, :last] for x in (codes, params))
    k, v = O.values(c, m)
    s, lo = (m[1][..., j].double().repeat_interleave(64, -1) for j in (0, 1))
    reach_k = m[0][..., 1].double().abs().repeat_interleave(64, -1) + (k - m[0][..., 1].double().repeat_interleave(64, -1))
    out, limit = (torch.zeros(Q, HQ, D, dtype=torch.float64) for _ in range(2))
    lse, lse_limit = (torch.zeros(Q, HQ, dtype=torch.float64) for _ in range(2))
    for i in range(Q):
        n = start + i + 1
        for h in range(HQ):
            x = q[0, i, h].double()
            sc = k[:n] @ x * scale
            p = sc.softmax(0)
            out[i, h], lse[i, h] = p @ v[:n], sc.logsumexp(0)
            size = float((reach_k[:n] @ x.abs()).max()) * abs(scale) / math.log(2)
            e = 2.0 ** -17 * math.log(2) * (size + 1)
            drift = p @ (v[:n] - out[i, h]).abs()
            weighted, spread = p @ (v[:n] - lo[:n]), 7.5 * (p @ s[:n])
            limit[i, h] = (2 * e * drift + 2.0 ** -11 * (weighted if dtype == "bf16" else spread) + 2.0 ** (-11 if dtype == "bf16" else -12) * spread
                           + (2.0 ** -18 + n * 2.0 ** -29) * (p @ v[:n].abs() + weighted + out[i, h].abs()))
            lse_limit[i, h] = e + 2.0 ** -18 + n * 2.0 ** -29 + 2.0 ** -23 * abs(float(lse[i, h]))
    eps = torch.finfo(DT[dtype]).eps / 2
    return out, limit * (1 + eps) + eps * out.abs() + (2.0 ** -25 if dtype == "fp16" else 0.0), lse, lse_limit


def call(ears, q, codes, params, pages, start, copies, table_extra=0):
    """The call for ``copies`` sequences that are one and the same: with as many as here a unit's tokens stay with one block or two."""
    table = torch.nn.functional.pad(pages, (0, table_extra), value=-1).to(DEV).expand(copies, -1)
    return ears.kv_attention(q.to(DEV).expand(copies, -1, -1, -1), ears.KVCache(codes.to(DEV), params.to(DEV)), table, ints([start] * copies), scale=1.0,
                             lse=True)


def check(ears, q, codes, params, pages, start, dtype, rows=slice(None), table_extra=0, copies=(1, 450)):
    out, limit, want_lse, lse_limit = (x.to(DEV) for x in expect(q, codes, params, pages, start, dtype))
    for n in copies:
        got, lse = (x[:, rows].double() for x in call(ears, q, codes, params, pages, start, n, table_extra))
        assert got.isfinite().all()
        worst = float(((got - out[rows]).abs() / limit[rows]).max())
        assert worst <= 1, worst
        assert ((lse - want_lse[rows]).abs() <= lse_limit[rows]).all()


def ask(Q, HQ, D, dtype):
    q = torch.zeros(1, Q, HQ, D)
    q[..., 0] = 1.0
    return q.to(DT[dtype])


# ---- weights times scales over a wide range -------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("n,R", [(32768, 4096.0), (131072, 1024.0), (131072, 2.0 ** 20)])
def test_a_token_of_no_weight_with_large_values(ears, dtype, n, R):
    """The first token has half of the weight, one (of the same warp's) has values R times the others' and weighs e^-60."""
    g = torch.Generator().manual_seed(n)
    keys = torch.randn(n, generator=g) * 0.5
    far = n // 3 // 64 * 64
    keys[0], keys[far] = math.log(n), -60.0
    codes, params, pages, _ = pool(n, 128, 64, 5, keys)
    at = place(pages, far, 64)
    params[at[0], 1, 0, at[1]] = (params[at[0], 1, 0, at[1]].float() * R).bfloat16()
    check(ears, ask(1, 3, 128, dtype), codes, params, pages, n - 1, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("n,D,R", [(131072, 128, 1024.0), (9000, 128, 2.0 ** 14), (9000, 64 * 4, 2.0 ** 20), (700, 128, 2.0 ** 40)])
def test_groups_of_a_head_far_apart(ears, dtype, n, D, R):
    if dtype == "fp16":
        R = min(R, 2.0 ** 20)
    g = torch.Generator().manual_seed(n)
    keys = torch.randn(n, generator=g) * 2.0
    keys[0] = math.log(n)
    codes, params, pages, _ = pool(n, D, 64, 6, keys)
    params[:, 1, ..., 1:, :] = (params[:, 1, ..., 1:, :].float() / R).bfloat16()
    if D > 128:
        params[:, 1, ..., 2, :] = (params[:, 1, ..., 2, :].float() / 64).bfloat16()
    check(ears, ask(1, 4, D, dtype), codes, params, pages, n - 1, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("D,heads,table_extra", [(64, 2, 0), (128, 3, 0), (128, 5, 6000), (256, 4, 6000), (64, 8, 12000), (128, 8, 0)])
def test_a_later_draft_with_large_values(ears, dtype, D, heads, table_extra):
    """Rows that do not see it are as exact as without it."""
    n, Q = 1500, 4
    g = torch.Generator().manual_seed(D)
    keys = torch.randn(n, generator=g)
    keys[3] = 8.0
    keys[n - 1] = -40.0
    codes, params, pages, _ = pool(n, D, 16, 7, keys)
    at = place(pages, n - 1, 16)
    params[at[0], 1, 0, at[1]] = torch.tensor([2.0 ** 60, -(2.0 ** 61)], dtype=torch.bfloat16)
    check(ears, ask(Q, heads, D, dtype), codes, params, pages, n - Q, dtype, rows=slice(0, Q - 1), table_extra=table_extra)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("D,share", [(64, 2.0 ** -3), (128, 2.0 ** -6), (256, 2.0 ** -9)])
def test_a_million_tokens_beside_one_that_has_nearly_all_weight(ears, dtype, D, share):
    """... and no values to speak of: the result is what the others' small weights make."""
    n = 2 ** 20 if D < 256 else 2 ** 18
    keys = torch.full((n,), -12.0)
    keys[0] = float(torch.tensor(-12.0 + math.log(n / share)).bfloat16())
    codes, params, pages, _ = pool(n, D, 128, 8, keys)
    at = place(pages, 0, 128)
    params[at[0], 1, 0, at[1]] = torch.tensor([2.0 ** -30, 0.0], dtype=torch.bfloat16)
    check(ears, ask(1, 1, D, dtype), codes, params, pages, n - 1, dtype)


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("n", [40, 700, 5000])
def test_scores_that_rise_through_the_sequence(ears, D, n):
    """The running maximum is raised again and again, by little and by much, while scales fall and rise."""
    g = torch.Generator().manual_seed(n + D)
    keys = torch.linspace(-300, 100, n) + 3 * torch.randn(n, generator=g)
    codes, params, pages, _ = pool(n, D, 16, 9, keys)
    t = torch.arange(n)
    size = 2.0 ** (30 * torch.sin(t * 0.01))
    ids, slot = pages[0].long()[t // 16], t % 16
    params[ids, 1, 0, slot] = (params[ids, 1, 0, slot].float() * size[:, None, None]).bfloat16()
    q = ask(3, 4, D, "bf16")
    q[0, 1] *= 0.25
    q[0, :, 2] *= -0.5
    q[0, :, 3] *= 0.0
    check(ears, q, codes, params, pages, n - 3, "bf16")


# ---- values near the ends of the type -------------------------------------------------------------------

@pytest.mark.parametrize("D,heads,table_extra", [(64, 2, 0), (128, 2, 0), (256, 2, 0), (128, 20, 40000), (256, 16, 40000)])
@pytest.mark.parametrize("size,n", [(2.0 ** 122, 3000), (2.0 ** 100, 3000), (2.0 ** -60, 3000), (2.0 ** -86, 3000), (2.0 ** 122, 20000)])
def test_large_and_small_values(ears, D, heads, table_extra, size, n):
    """Up to 2^127 and down to 2^-86; half of the weight on the first tokens, so that sums of weights are far above 1."""
    g = torch.Generator().manual_seed(n)
    keys = torch.randn(n, generator=g) * 0.25
    codes, params, pages, _ = pool(n, D, 64, 10, keys)
    params[:, 1] = (params[:, 1].clamp(-2, 2).float() * size).bfloat16()
    check(ears, ask(1, heads, D, "bf16"), codes, params, pages, n - 1, "bf16", table_extra=table_extra)


@pytest.mark.parametrize("D,heads", [(64, 2), (128, 5), (256, 8)])
@pytest.mark.parametrize("at", [0, 5, 1000])
def test_a_token_without_any_weight_beside_tiny_values(ears, D, heads, at):
    """Its scale times the power of two that the others' take would pass 2^127."""
    n = 2000
    keys = torch.zeros(n)
    keys[at] = -1000.0
    codes, params, pages, g = pool(n, D, 16, 14, keys)
    params[:, 1] = (params[:, 1].float() * 2.0 ** -80).bfloat16()
    slot = place(pages, at, 16)
    params[slot[0], 1, 0, slot[1]] = torch.tensor([2.0 ** 100, 1.0], dtype=torch.bfloat16)
    check(ears, ask(1, heads, D, "bf16"), codes, params, pages, n - 1, "bf16")


@pytest.mark.parametrize("D", [64, 128])
def test_constant_groups(ears, D):
    """Scales of 2^-126, all that counts is in the minima, beside tokens of ordinary groups."""
    n = 2000
    codes, params, pages, g = pool(n, D, 16, 11, 0.0)
    flat = torch.rand(codes.shape[0], 16, generator=g) < 0.7
    params[:, 1, 0, :, 0][flat] = torch.tensor([2.0 ** -126, -3.25], dtype=torch.bfloat16)
    codes[:, 1, 0, :, :32][flat] = 0
    check(ears, ask(2, 2, D, "bf16"), codes, params, pages, n - 2, "bf16")


# ---- parameters that are not finite ----------------------------------------------------------------------

@pytest.mark.parametrize("table_extra", [0, 3000])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("token", [10, 200, 296, 298])
@pytest.mark.parametrize("what", ["scale", "minimum", "both", "infinite scale", "infinite minimum"])
def test_a_nan_in_one_group_of_values_takes_the_whole_row(ears, D, token, what, table_extra):
    """Wherever the token stands, in a part that all rows see or in one that only some do."""
    n, Q, page = 300, 5, 16
    codes, params, pages, g = pool(n, D, page, 12, torch.randn(n, generator=torch.Generator().manual_seed(1)))
    at = place(pages, token, page)
    bad = {"scale": (math.nan, 0.5), "minimum": (0.5, math.nan), "both": (math.nan, math.nan), "infinite scale": (math.inf, 0.5),
           "infinite minimum": (0.5, -math.inf)}[what]
    params[at[0], 1, 0, at[1], D // 64 - 1] = torch.tensor(bad, dtype=torch.bfloat16)
    for heads, copies in ((1, 1), (6, 1), (1, 450), (6, 450)):
        got, lse = call(ears, ask(Q, heads, D, "bf16"), codes, params, pages, n - Q, copies, table_extra)
        first = max(0, token - (n - Q))                     # rows from here on see it
        assert got[:, first:].isnan().all() and lse[:, first:].isnan().all()
        assert got[:, :first].isfinite().all() and lse[:, :first].isfinite().all()


# ---- rows per block ---------------------------------------------------------------------------------------

def eights_per_block(ears, D, H, B, Q, group, tokens, window=0, sinks=0):
    """As the workspace shows: two parts of a block's rows for every resident CTA, three per SM with one eight of up to 128 dimensions, else two (for calls
    that fill them)."""
    import ctypes
    from paper_2512_13194_b200.binding import KvCacheStruct
    cache = KvCacheStruct(256, 256, 10, H, 64, D)          # nothing is read
    need = ears.load_library().ears_kv_attention_workspace_bytes(1, ctypes.byref(cache), B, Q, H * group, -(-tokens // 64), window, sinks)
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    for nt in (1, 2, 3, 4):
        grid = sms * (3 if nt == 1 and D <= 128 else 2)
        if 0 <= need - grid * (16 + 2 * nt * 8 * (8 + 4 * D)) < 3 * 256:
            return nt
    return need


def test_rows_per_block_go_by_all_blocks_chunks(ears):
    for D in (64, 128, 256):
        assert eights_per_block(ears, D, 8, 1, 5, 4, 16000) == 1                # 3 eights, 13.5 chunks per SM
        assert eights_per_block(ears, D, 8, 1, 33, 8, 2000) == 1                # 33 eights of 1.7
        for B, Q, tokens in ((1, 33, 4000), (1, 33, 18900), (12, 33, 1000), (4, 66, 2000)):
            assert eights_per_block(ears, D, 8, B, Q, 8, tokens) in (2, 3, 4)
    assert eights_per_block(ears, 128, 8, 128, 5, 4, 9001) == 3
    assert eights_per_block(ears, 64, 8, 32, 8, 8, 20000, 1024, 4) == 4
    assert eights_per_block(ears, 64, 8, 1, 5, 4, 131072) == 3                  # the table's width counts
    assert eights_per_block(ears, 64, 8, 1, 5, 4, 131072, 4000, 4) == 1         # but no more of it than a window shows


# ---- gradients ---------------------------------------------------------------------------------------------

def test_a_cache_that_requires_a_gradient_is_refused(ears):
    from torch.autograd import forward_ad
    codes, params, pages, g = pool(40, 64, 16, 13)
    plain = ears.KVCache(codes.to(DEV), params.to(DEV))
    k, q = torch.randn(1, 3, 1, 64, generator=g).to(DEV), ask(3, 2, 64, "bf16").to(DEV)
    at = (pages.to(DEV), ints([20]))
    want = ears.kv_attention(q, plain, *at)

    def calls(cache):
        return (lambda: ears.kv_attention(q, cache, *at), lambda: ears.kv_read(cache, *at, 3), lambda: ears.kv_write(cache, k, k, *at),
                lambda: ears.kv_attention(q, cache, at[0].long(), at[1]))

    cache = ears.KVCache(plain.codes, plain.params.clone().requires_grad_())
    for call in calls(cache):
        with pytest.raises(NotImplementedError):
            call()
    with torch.no_grad():
        assert torch.equal(ears.kv_attention(q, cache, *at), want)
        ears.kv_write(cache, k, k, *at)
        assert torch.equal(*ears.kv_read(cache, *at, 3))
    with forward_ad.dual_level():
        for call in calls(ears.KVCache(plain.codes, forward_ad.make_dual(plain.params, torch.ones_like(plain.params)))):
            with pytest.raises(NotImplementedError):
                call()
