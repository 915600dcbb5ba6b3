"""A key/value cache held in 4 bits, beside the verification step: the forward pass whose logits a step verifies writes K+1
tokens per sequence into the cache, its attention reads it, and the step's accepted lengths say how many of them stay.

Three operators: ``write`` (quantising tokens into the cache's pages, here with the block read back), ``read`` (a range of every
sequence as values) and ``attention`` of the newest positions over the cache, full or with a sliding window and first tokens
that stay visible.  ``own = False`` computes them in elementary torch operations in 32 bits.

The cache: ``codes`` uint8 [P, 2, H, page, D/2] (keys, values; two codes a byte, the even one in the low half), ``params`` bfloat16
[P, 2, H, page, D/64, 2] with the scale s and the minimum m of 64 values: a code c stands for m + s c.  Token t of sequence b lies
in page ``pages[b, t // page]`` at place ``t % page``.  Position i of a call is token ``start[b] + i``, for i < counts[b].
Quantising a group x: m = min(x) rounded down to bfloat16, s = (max(x) - m) / 15 in 32 bits rounded up to it (2^-126 at least),
c = (x - m) / s, the difference rounded to 32 bits, to the nearest whole number and to the even one of two.
"""
import math

import torch

own = False

GROUP = 64
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
BYTES = {"bf16": 2, "fp16": 2, "fp32": 4}


def listed():
    return [
        # one sequence with K = 4 drafts: the smallest verification step, bound by latency
        dict(name="attention_one_sequence", op="attention", dtype="bf16", B=1, Q=5, HQ=32, H=8, D=128, page=64, longest=1000, shortest=1000, window=0, sinks=0),
        # a small batch with K = 5, of uneven lengths
        dict(name="attention_small_batch", op="attention", dtype="bf16", B=8, Q=6, HQ=32, H=8, D=128, page=32, longest=4096, shortest=37, window=0, sinks=0),
        # ordinary decoding: single tokens of a serving batch
        dict(name="attention_single_tokens", op="attention", dtype="bf16", B=64, Q=1, HQ=64, H=8, D=128, page=64, longest=8192, shortest=6000, window=0, sinks=0),
        # a serving batch's verification step, K = 4, lengths from a few tokens to long ones
        dict(name="attention_large_batch", op="attention", dtype="bf16", B=128, Q=5, HQ=32, H=8, D=128, page=16, longest=9001, shortest=5, window=0, sinks=0),
        # layers with a window: K = 7, narrow heads, fp16
        dict(name="attention_window", op="attention", dtype="fp16", B=32, Q=8, HQ=64, H=8, D=64, page=64, longest=20000, shortest=700, window=1024, sinks=4),
        # one long context, wide heads, single token
        dict(name="attention_long_context", op="attention", dtype="bf16", B=1, Q=1, HQ=16, H=4, D=256, page=128, longest=131071, shortest=131071, window=0, sinks=0),
        # what a step appends: K + 1 = 6 tokens for 8 sequences
        dict(name="write_step", op="write", dtype="bf16", B=8, Q=6, H=8, D=128, page=64, longest=4000, shortest=30),
        # prompts of uneven lengths
        dict(name="write_prompts", op="write", dtype="bf16", B=4, Q=4097, H=8, D=128, page=64, longest=200, shortest=0),
        # an fp32 model's prompt, narrow heads
        dict(name="write_fp32", op="write", dtype="fp32", B=3, Q=1111, H=12, D=64, page=16, longest=90, shortest=0),
        # a short range of every sequence
        dict(name="read_blocks", op="read", dtype="fp16", B=16, Q=33, H=4, D=256, page=32, longest=900, shortest=0),
        # a long shared prefix as values, for an operator that wants them so
        dict(name="read_prefix", op="read", dtype="bf16", B=1, Q=65003, H=8, D=128, page=64, longest=0, shortest=0),
    ]


def _spread(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["attention", "attention", "write", "read"])
    D, H, page = rng.choice([64, 128, 128, 256]), rng.choice([1, 2, 4, 8, 8, 12]), rng.choice([16, 32, 48, 64, 128])
    if op == "attention":
        dtype, heads = rng.choice(["bf16", "bf16", "fp16"]), rng.choice([1, 3, 4, 8])
        Q, longest = rng.choice([1, 1, 2, 4, 5, 6, 8, rng.randint(9, 33)]), _spread(rng, 20, 131072)
        room = 4.0e8 / (H * D * longest) * min(1.0, 40 / (Q * heads))          # no more than the largest listed case
        B = max(1, min(_spread(rng, 1, 256), int(room)))
        window = rng.choice([0, 0, 0, _spread(rng, 16, 8192)])
        sinks = rng.choice([0, 1, 4, rng.randint(5, 90)]) if window else 0
        return dict(op=op, dtype=dtype, B=B, Q=Q, HQ=H * heads, H=H, D=D, page=page, longest=longest,
                    shortest=rng.choice([longest, max(1, longest // 2), 1]), window=window, sinks=sinks)
    dtype, tokens = rng.choice(["bf16", "fp16", "fp32"]), _spread(rng, 1, 12000)
    B = max(1, min(tokens, _spread(rng, 1, 200)))
    longest = _spread(rng, 1, 4000)
    return dict(op=op, dtype=dtype, B=B, Q=max(1, tokens // B), H=H, D=D, page=page, longest=longest, shortest=rng.choice([longest, longest // 3, 0]))


# ---- inputs ----------------------------------------------------------------------------------------------------------

def _lengths(case, generator):
    """Tokens that each sequence has in the cache before the call, the first of them the longest."""
    low, high = case["shortest"], case["longest"]
    start = torch.randint(low, high + 1, (case["B"],), generator=generator)
    start[0] = high
    return start


def _values(shape, generator, device):
    """Keys or values as layers write them: spread differently, and about another mean, in each of the last dimension's channels."""
    D = shape[-1]
    spread = torch.rand(D, generator=generator, device=device) + 0.5
    mean = torch.randn(D, generator=generator, device=device)
    return torch.randn(shape, generator=generator, device=device) * spread + mean


def prepare(case, seed):
    host, g = torch.Generator().manual_seed(seed), torch.Generator(device="cuda").manual_seed(seed)
    B, Q, H, D, page = case["B"], case["Q"], case["H"], case["D"], case["page"]
    attention = case["op"] == "attention"
    # attention's newest Q tokens are in the cache already; of the blocks that are written or read some end early
    start = _lengths(case, host)
    if attention:
        start = (start - Q).clamp(min=0)
    counts = torch.full((B,), Q)
    if Q > 1 and B > 1:
        counts[1:] = torch.randint(Q // 2 if not attention else Q - 1, Q + 1, (B - 1,), generator=host)
    held = (start + Q + page - 1) // page
    width, total = int(held.max()), int(held.sum())
    order = torch.randperm(total + 3, generator=host)[:total]
    pages = torch.zeros(B, width, dtype=torch.int64)
    pages[torch.arange(width)[None, :] < held[:, None]] = order
    codes = torch.empty(total + 3, 2, H, page, D // 2, dtype=torch.uint8, device="cuda")
    params = torch.empty(total + 3, 2, H, page, D // GROUP, 2, dtype=torch.bfloat16, device="cuda")
    part = max(1, (1 << 26) // (2 * H * page * D))
    for i in range(0, total + 3, part):
        x = _values((min(part, total + 3 - i), 2, H, page, D), g, "cuda")
        codes[i:i + part], params[i:i + part] = _quantised(x)
    state = dict(case=case, codes=codes, params=params, pages=pages.int().cuda(), start=start.int().cuda(), counts=counts.int().cuda())
    dtype = TYPES[case["dtype"]]
    if attention:
        state["q"] = (torch.randn(B, Q, case["HQ"], D, generator=g, device="cuda") * 1.5).to(dtype)
    elif case["op"] == "write":
        # keys and values lie side by side, as one product with the joined weights leaves them
        kv = torch.cat([_values((B, Q, H, D), g, "cuda") for _ in range(2)], dim=2).to(dtype)
        state["k"], state["v"] = kv[:, :, :H], kv[:, :, H:]
    return state


# ---- the plain form ---------------------------------------------------------------------------------------------------

def _down(x):
    """To bfloat16 and, where that is inexact, to the smaller one; as 32-bit values."""
    bits = x.contiguous().view(torch.int32)
    cut = bits & -65536
    return torch.where((bits < 0) & (bits != cut), cut + 65536, cut).view(torch.float32)


def _quantised(x):
    """x [..., D] -> codes [..., D/2] uint8, params [..., D/64, 2] bfloat16"""
    x = x.float().unflatten(-1, (-1, GROUP))
    m = _down(x.amin(-1))
    s = (-_down(-((x.amax(-1) - m) / 15))).clamp(min=2.0 ** -126)
    fine = s.isfinite()
    s, m = torch.where(fine, s, math.nan), torch.where(fine, m, math.nan)
    # the quotient stands next to a border between two codes: 64 bits
    c = ((x - m[..., None]).double() / s[..., None].double()).round().nan_to_num(0.0).clamp(0, 15).to(torch.uint8).flatten(-2)
    return c[..., 0::2] | c[..., 1::2] << 4, torch.stack([s, m], -1).bfloat16()


def _valued(codes, params):
    c = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).float().unflatten(-1, (-1, GROUP))
    p = params.float()
    return (p[..., 1:] + p[..., :1] * c).flatten(-2)


def _places(s, count):
    """Page and place [B, n] of the positions start + 0 .. n-1, and which of them are within ``count`` [B]."""
    B, page = s["pages"].shape[0], s["case"]["page"]
    i = torch.arange(s["case"]["Q"], device="cuda")[None, :]
    t = (s["start"].long()[:, None] + i).clamp(max=s["pages"].shape[1] * page - 1)
    return s["pages"].long().gather(1, t // page), t % page, (i < count[:, None]).expand(B, -1)


def _plain_write(s):
    page, place, real = _places(s, s["counts"])
    x = torch.stack([s["k"], s["v"]], 2)                                    # [B, Q, 2, H, D]
    codes, params = _quantised(x[real])
    s["codes"][page[real], :, :, place[real]] = codes
    s["params"][page[real], :, :, place[real]] = params
    return _plain_read(s, torch.float32)


def _plain_read(s, dtype):
    page, place, real = _places(s, s["counts"])
    x = _valued(s["codes"][page, :, :, place], s["params"][page, :, :, place])
    x = torch.where(real[:, :, None, None, None], x, 0.0).to(dtype)
    return x[:, :, 0].contiguous(), x[:, :, 1].contiguous()


def _seen(case, start, counts, n):
    """Which of the tokens 0 .. n-1 each position sees, [B, Q, n]."""
    i = torch.arange(case["Q"], device=start.device)
    p, t = (start.long()[:, None] + i)[:, :, None], torch.arange(n, device=start.device)
    seen = (t <= p) & (i < counts[:, None])[:, :, None]
    if case["window"]:
        seen &= (t > p - case["window"]) | (t < case["sinks"])
    return seen


def _plain_attention(s):
    case, q = s["case"], s["q"]
    B, Q, H, D = case["B"], case["Q"], case["H"], case["D"]
    pages = s["pages"].long()
    kv = _valued(s["codes"][pages], s["params"][pages]).permute(2, 0, 3, 1, 4, 5).flatten(3, 4)     # [2, B, H, tokens, D]
    seen = _seen(case, s["start"], s["counts"], kv.shape[3])[:, None, :, None, :]                   # [B, 1, Q, 1, tokens]
    rows = q.float().unflatten(2, (H, -1)).permute(0, 2, 1, 3, 4)                                   # [B, H, Q, heads, D]
    x = (rows.flatten(2, 3) @ kv[0].transpose(-1, -2)).unflatten(2, (Q, -1)) / math.sqrt(D)
    x = torch.where(seen, x, -math.inf)
    e = torch.exp(x - x.amax(-1, keepdim=True).clamp(min=torch.finfo(torch.float32).min))
    total = e.sum(-1, keepdim=True)
    out = (e.flatten(2, 3) @ kv[1]).unflatten(2, (Q, -1)) / torch.where(total > 0, total, 1.0)
    return out.permute(0, 2, 1, 3, 4).flatten(2, 3).to(q.dtype)


def run(state):
    case = state["case"]
    if own:
        import paper_2512_13194_b200 as ears
        cache, place = ears.KVCache(state["codes"], state["params"]), (state["pages"], state["start"])
        if case["op"] == "attention":
            return ears.kv_attention(state["q"], cache, *place, state["counts"], window=case["window"], sinks=case["sinks"])
        if case["op"] == "write":
            ears.kv_write(cache, state["k"], state["v"], *place, state["counts"])
            return ears.kv_read(cache, *place, case["Q"], state["counts"], dtype=torch.float32)
        return ears.kv_read(cache, *place, case["Q"], state["counts"], dtype=TYPES[case["dtype"]])
    if case["op"] == "attention":
        return _plain_attention(state)
    return _plain_write(state) if case["op"] == "write" else _plain_read(state, TYPES[case["dtype"]])


# ---- what a pass cannot do without --------------------------------------------------------------------------------------

def work(case):
    """Lengths are drawn with the inputs: their mean stands here, (longest + shortest) / 2 beside the one longest."""
    B, Q, H, D, e = case["B"], case["Q"], case["H"], case["D"], BYTES[case["dtype"]]
    held = D / 2 + D / GROUP * 4                                       # bytes of a token's keys, or values, in one head
    mean = (case["longest"] + (B - 1) * (case["longest"] + case["shortest"]) / 2) / B
    if case["op"] == "attention":
        tokens = max(mean, Q)
        if case["window"]:
            tokens = min(tokens, case["window"] + case["sinks"] + Q)
        return {"bytes": B * (tokens * H * 2 * held + 2 * Q * case["HQ"] * D * e), "flops": 4.0 * B * Q * case["HQ"] * D * tokens}
    tokens = (Q + (B - 1) * Q * 0.75) if Q > 1 else B                # a block is full, or between half full and full
    if case["op"] == "write":                                        # the elements, the codes twice, the values of the whole block
        return {"bytes": 2 * H * (tokens * (D * e + 2 * held) + B * Q * D * 4), "flops": 2.0 * tokens * H * D * 8}
    return {"bytes": 2 * H * (tokens * held + B * Q * D * e), "flops": 2.0 * tokens * H * D * 2}


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------------

def _token_values(codes, params):
    """[2, H, n, D/2], [2, H, n, D/64, 2] -> [2, H, n, D] in 64 bits"""
    out = torch.empty(*codes.shape[:-1], codes.shape[-1] * 2, dtype=torch.float64, device=codes.device)
    out[..., 0::2] = codes.remainder(16).double()
    out[..., 1::2] = codes.div(16, rounding_mode="floor").double()
    s, m = (params[..., k].double().repeat_interleave(GROUP, -1) for k in (0, 1))
    return out * s + m


def _sequence(s, b, n):
    """Codes and params of the first n tokens of sequence b."""
    page = s["case"]["page"]
    held = s["pages"][b, :-(-n // page)].long()
    return tuple(s[k][held].transpose(0, 1).transpose(1, 2).flatten(2, 3)[:, :, :n] for k in ("codes", "params"))


def _group_values(x):
    """The values that the cache holds for x [..., 64]; the steps whose rounding the format fixes are taken in 32 bits."""
    x = x.float()
    low, high = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
    m = low.bfloat16()
    m = torch.where(m.float() > low, torch.nextafter(m, torch.full_like(m, -math.inf)), m).float()
    wide = (high - m) / 15.0
    s = wide.bfloat16()
    s = torch.where(s.float() < wide, torch.nextafter(s, torch.full_like(s, math.inf)), s).double().clamp(min=2.0 ** -126)
    c = ((x - m).double() / s).round()
    return m.double() + s * c


def exact(case, seed):
    s = prepare(case, seed)
    B, Q, H, D = case["B"], case["Q"], case["H"], case["D"]
    starts, counts = s["start"].tolist(), s["counts"].tolist()
    if case["op"] != "attention":
        out = torch.zeros(2, B, Q, H, D, dtype=torch.float64, device="cuda")
        for b in range(B):
            n = counts[b]
            if case["op"] == "write":
                for k, name in enumerate(("k", "v")):
                    out[k, b, :n] = _group_values(s[name][b, :n].unflatten(-1, (-1, GROUP))).flatten(-2)
            else:
                codes, params = _sequence(s, b, starts[b] + n)
                out[:, b, :n] = _token_values(codes[:, :, starts[b]:], params[:, :, starts[b]:]).transpose(1, 2)
        return out[0], out[1]
    out = torch.zeros(B, Q, case["HQ"], D, dtype=torch.float64, device="cuda")
    for b in range(B):
        n = counts[b]
        k, v = _token_values(*_sequence(s, b, starts[b] + n))
        t = torch.arange(starts[b] + n, device="cuda")
        for i in range(n):
            p = starts[b] + i
            see = t <= p
            if case["window"]:
                see = see & ((t > p - case["window"]) | (t < case["sinks"]))
            q = s["q"][b, i].double().view(H, -1, D)
            w = (q @ k.transpose(-1, -2) * D ** -0.5).masked_fill(~see, -math.inf).softmax(-1)
            out[b, i] = (w @ v).reshape(case["HQ"], D)
    return out
