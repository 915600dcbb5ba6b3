"""The logit-row operators beside the verification step: what is measured, and on what.

  top_logits       a teacher's k largest logits of every row, with the row's log normaliser
  token_logprobs   log probability (and entropy) of one token per row, forward and training step
  distill          divergence of a draft row from a teacher's top logits, forward and training step
  policy           clipped policy loss with a KL term and an entropy bonus, forward and training step

`run` computes them with elementary torch operations in 32 bits (row scalars in 64), or, when
`own` is true, through the package's entry points.  `exact` restates the definitions in 64 bits and
takes gradients by differentiating them.
"""
import math

import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
TAIL_FLOOR = 2.0 ** -20     # tail mass that a 32-bit log normaliser still resolves


# ---- cases ------------------------------------------------------------------------------------

def listed():
    return [
        # a draft model's four proposals of one sequence: the best few ids for a log
        dict(name="top_one_sequence", op="top", B=1, R=4, V=32000, k=8, dtype="fp32", T=1.0, live=False),
        # teacher lists captured from the target rows of a verification batch, live positions only
        dict(name="top_capture_batch", op="top", B=32, R=7, V=128256, k=64, dtype="bf16", T=1.0, live=True),
        # the same for a large batch with long lists
        dict(name="top_capture_large", op="top", B=128, R=4, V=152064, k=128, dtype="bf16", T=0.9, live=False),
        # log probabilities of the tokens one verification step emitted (-1 behind the last one)
        dict(name="score_emitted", op="token", B=8, R=6, V=32000, dtype="bf16", T=0.7, entropy=False, train=False, absent=0.4),
        # scoring of a whole batch under a reference model, with the entropy
        dict(name="score_long_rows", op="token", B=512, R=4, V=256000, dtype="fp32", T=1.2, entropy=True, train=False, absent=0.0),
        # next-token training of a draft model: known weights, gradient in one call
        dict(name="token_train", op="token", B=8, R=256, V=128256, dtype="bf16", T=1.0, entropy=False, train=True, absent=0.1),
        # the draft's divergence watched during serving
        dict(name="distill_watch", op="distill", B=8, R=5, V=32000, k=16, dtype="bf16", T=1.0, kind="forward_kl", mix=0.5,
             tail=True, train=False, absent=0.3),
        # distillation step over a few thousand captured positions
        dict(name="distill_train", op="distill", B=292, R=7, V=128256, k=64, dtype="bf16", T=1.0, kind="forward_kl", mix=0.5,
             tail=True, train=True, absent=0.1),
        # 32-bit logits and the symmetric divergence
        dict(name="distill_train_long_rows", op="distill", B=512, R=3, V=256000, k=32, dtype="fp32", T=1.2, kind="jsd", mix=0.5,
             tail=True, train=True, absent=0.0),
        # odd vocabulary, short list, mode-seeking divergence
        dict(name="distill_train_odd_rows", op="distill", B=37, R=5, V=33001, k=20, dtype="fp16", T=0.9, kind="reverse_kl", mix=0.5,
             tail=True, train=True, absent=0.2),
        # one short response
        dict(name="policy_one_response", op="policy", B=1, R=24, V=32000, dtype="bf16", T=1.0, kl=0.05, ent=0.0, ref=True,
             train=True, absent=0.0),
        # a training batch of responses
        dict(name="policy_train", op="policy", B=16, R=256, V=152064, dtype="bf16", T=1.0, kl=0.02, ent=0.01, ref=True,
             train=True, absent=0.15),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["top", "token", "distill", "policy"])
    dtype = rng.choice(["fp32", "bf16", "bf16", "fp16"])
    V = _spread(rng, 600, 262144)
    train = op == "policy" or (op != "top" and rng.random() < 0.7)
    budget = 2.3e9 / (V * (4 if dtype == "fp32" else 2) * (2 if train else 1))   # bytes of the largest listed cases
    if op == "top":
        budget *= 0.08
    R = rng.randint(1, 8) if op in ("top", "distill") else _spread(rng, 1, 256)
    B = _spread(rng, 1, 1024)
    while B * R > budget and B > 1:
        B = (B + 1) // 2
    while B * R > budget and R > 1:
        R = (R + 1) // 2
    case = dict(op=op, B=B, R=R, V=V, dtype=dtype, T=round(rng.uniform(0.6, 1.4), 2))
    if op == "top":
        case.update(k=rng.randint(1, 128), live=rng.random() < 0.5)
    elif op == "token":
        case.update(entropy=rng.random() < 0.5, train=train, absent=rng.choice([0.0, 0.3]))
    elif op == "distill":
        kind = rng.choice(["forward_kl", "reverse_kl", "jsd"])
        case.update(k=rng.randint(1, 128), kind=kind, mix=round(rng.uniform(0.1, 0.9), 2),
                    tail=kind == "reverse_kl" or rng.random() < 0.7, train=train, absent=rng.choice([0.0, 0.3]))
    else:
        case.update(kl=rng.choice([0.0, 0.05]), ent=rng.choice([0.0, 0.01]), ref=True, train=True, absent=rng.choice([0.0, 0.3]))
    return case


# ---- inputs -----------------------------------------------------------------------------------

def _rows(gen, n, V, dtype, device):
    """Logit rows as a language model leaves them: gaussian with a scale per row, one entry of half
    the rows far above the others, the last columns (padding of the vocabulary) masked."""
    out = torch.empty((n, V), dtype=dtype, device=device)
    step = max(1, (1 << 27) // V)
    for a in range(0, n, step):
        m = min(step, n - a)
        scale = 1.0 + 2.0 * torch.rand((m, 1), generator=gen, device=device)
        x = torch.randn((m, V), generator=gen, device=device) * scale
        peak = torch.randint(0, V, (m, 1), generator=gen, device=device)
        boost = torch.where(torch.rand((m, 1), generator=gen, device=device) < 0.5, 4.0, 16.0)
        x.scatter_add_(1, peak, boost)
        out[a:a + m] = x.to(dtype)
    if V >= 1000:
        out[:, V - V // 200:] = -math.inf
    return out


def _noisy(gen, x, sigma):
    """The same rows as another model sees them."""
    out = torch.empty_like(x)
    step = max(1, (1 << 27) // x.shape[1])
    for a in range(0, x.shape[0], step):
        y = x[a:a + step].float()
        out[a:a + step] = (y + sigma * torch.randn(y.shape, generator=gen, device=x.device)).to(x.dtype)
    return out


def _log_z(x, T):
    """fp64 log normalisers of the rows of x at temperature T."""
    out = torch.empty(x.shape[0], dtype=torch.float64, device=x.device)
    step = max(1, (1 << 26) // x.shape[1])
    for a in range(0, x.shape[0], step):
        out[a:a + step] = torch.logsumexp(x[a:a + step].double() / T, 1)
    return out


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed * 7919 + 17)
    op, B, R, V, T = case["op"], case["B"], case["R"], case["V"], case["T"]
    dtype = DTYPES[case["dtype"]]
    n = B * R
    state = dict(case=case)
    if op == "top":
        # target rows of a verification step: R positions of R + 1 rows
        x = _rows(gen, B * (R + 1), V, dtype, dev).view(B, R + 1, V)
        state["logits"] = x[:, :R]
        state["accept_len"] = torch.randint(0, R + 1, (B,), generator=gen, device=dev, dtype=torch.int32) if case["live"] else None
        return state
    absent = torch.rand((B, R), generator=gen, device=dev) < case["absent"]
    if op == "distill":
        teacher = _rows(gen, n, V, dtype, dev)
        k = min(case["k"], V)
        student = _noisy(gen, teacher, 0.7)
        val, idx = torch.topk(teacher.float(), k, dim=1)
        idx = torch.where(torch.isinf(val), -1, idx)
        gone = absent.view(n, 1)
        state.update(logits=student.view(B, R, V),
                     values=torch.where(gone, -math.inf, val).view(B, R, k).contiguous(),
                     ids=torch.where(gone, -1, idx).to(torch.int32).view(B, R, k).contiguous(),
                     lse=_log_z(teacher, T).float().view(B, R) if case["tail"] else None,
                     weight=torch.rand((B, R), generator=gen, device=dev) / n)
        return state
    x = _rows(gen, n, V, dtype, dev)
    # tokens as they are sampled: mostly from the row's head
    noise = torch.empty((n, V), dtype=torch.float32, device=dev) if n * V < (1 << 29) else None
    if noise is not None:
        noise.exponential_(generator=gen)
        tok = (x.float() / T - noise.log_()).argmax(1)
        del noise
    else:
        tok = torch.cat([(r.float() / T - torch.empty(r.shape, device=dev).exponential_(generator=gen).log_()).argmax(1)
                         for r in x.split(max(1, (1 << 27) // V))])
    state["logits"] = x.view(B, R, V)
    state["tokens"] = torch.where(absent, -1, tok.view(B, R)).to(torch.int32)
    if op == "token":
        state["d_logp"] = -torch.rand((B, R), generator=gen, device=dev) / n
        state["d_entropy"] = 0.01 * torch.randn((B, R), generator=gen, device=dev) / n if case["entropy"] else None
        return state
    logp = (x.gather(1, tok.view(n, 1)).double().view(n) / T - _log_z(x, T)).view(B, R)
    state["old_logp"] = (logp + 0.15 * torch.randn((B, R), generator=gen, device=dev)).float()
    state["ref_logp"] = (logp + 0.3 * torch.randn((B, R), generator=gen, device=dev)).float() if case["ref"] else None
    state["advantage"] = torch.randn((B, 1), generator=gen, device=dev).expand(B, R).contiguous()
    state["weight"] = torch.full((B, R), 1.0 / n, device=dev)
    return state


CLIP_LOW, CLIP_HIGH = 0.2, 0.28


# ---- the operators in their plain form -----------------------------------------------------------

def _softmax_parts(x, T):
    """-> e = exp((x - m) / T), m [n, 1], z [n] (32 bits)"""
    m = x.max(1, keepdim=True).values
    e = ((x - m) / T).exp_()
    return e, m, e.sum(1)


def _plain_top(s):
    c = s["case"]
    B, R, V = s["logits"].shape
    k, T = c["k"], c["T"]
    x = s["logits"].reshape(B * R, V).float() + 0.0
    bits = x.view(torch.int32).long()
    order = torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits)            # same order as the values
    keys = order * (1 << 31) + (V - 1 - torch.arange(V, device=x.device))  # equal values: lowest index first
    kk = min(k, V)
    idx = torch.topk(keys, kk, dim=1, sorted=True).indices
    val = x.gather(1, idx)
    idx = torch.where(torch.isinf(val), -1, idx)
    if kk < k:
        val = torch.cat([val, torch.full((B * R, k - kk), -math.inf, device=x.device)], 1)
        idx = torch.cat([idx, torch.full((B * R, k - kk), -1, device=x.device)], 1)
    _, m, z = _softmax_parts(x, T)
    lse = m.view(-1).double() / T + z.double().log()
    if s["accept_len"] is not None:
        live = (torch.arange(R, device=x.device)[None, :] <= s["accept_len"][:, None]).view(-1, 1)
        val = torch.where(live, val, -math.inf)
        idx = torch.where(live, idx, -1)
        lse = torch.where(live.view(-1), lse, -math.inf)
    return val.view(B, R, k), idx.to(torch.int32).view(B, R, k), lse.float().view(B, R)


def _plain_token_parts(x, tok, T, entropy):
    """fp64 per row: logp, log z, entropy (or None); and e, z in 32 bits"""
    e, m, z = _softmax_parts(x, T)
    lt = x.gather(1, tok.clamp(min=0).view(-1, 1)).double().view(-1)
    log_z = z.double().log()
    logp = (lt - m.view(-1).double()) / T - log_z
    H = None
    if entropy:
        w = (e * ((x - m) / T).clamp(min=-1e30)).sum(1)
        H = log_z - w.double() / z.double()
    return e, m, z, logp, log_z, H


def _plain_token_grad(x, e, m, z, log_z, H, tok, T, g_logp, g_ent, dtype):
    """g_logp d logp / dx + g_ent d H / dx"""
    a = (-g_logp / z.double()).float().view(-1, 1)
    if g_ent is None:
        grad = e * a
    else:
        b = (-g_ent / z.double())
        a = (a.view(-1).double() + b * (H - log_z)).float().view(-1, 1)
        grad = e * (a + b.float().view(-1, 1) * ((x - m) / T).clamp(min=-1e30))
    grad.scatter_add_(1, tok.clamp(min=0).view(-1, 1), g_logp.float().view(-1, 1))
    grad /= T
    grad[tok < 0] = 0.0
    return grad.to(dtype)


def _plain_token(s):
    c = s["case"]
    B, R, V = s["logits"].shape
    T = c["T"]
    x, tok = s["logits"].reshape(B * R, V).float(), s["tokens"].view(-1).long()
    e, m, z, logp, log_z, H = _plain_token_parts(x, tok, T, c["entropy"])
    gone = tok < 0
    out = [torch.where(gone, 0.0, logp).float().view(B, R)]
    if c["entropy"]:
        out.append(torch.where(gone, 0.0, H).float().view(B, R))
    if c["train"]:
        g_ent = s["d_entropy"].view(-1).double() if c["entropy"] else None
        out.append(_plain_token_grad(x, e, m, z, log_z, H, tok, T, s["d_logp"].view(-1).double(), g_ent,
                                     s["logits"].dtype).view(B, R, V))
    return out


def _plain_policy(s):
    c = s["case"]
    B, R, V = s["logits"].shape
    T, n = c["T"], B * R
    x, tok = s["logits"].reshape(n, V).float(), s["tokens"].view(-1).long()
    e, m, z, logp, log_z, H = _plain_token_parts(x, tok, T, c["ent"] != 0.0)
    gone = tok < 0
    A = s["advantage"].view(-1).double()
    ratio = (logp - s["old_logp"].view(-1).double()).exp()
    plain, clipped = ratio * A, ratio.clamp(1.0 - CLIP_LOW, 1.0 + CLIP_HIGH) * A
    loss = -torch.minimum(plain, clipped)
    g = torch.where(plain <= clipped, -plain, 0.0)
    d = s["ref_logp"].view(-1).double() - logp
    kl = d.exp() - d - 1.0
    loss = loss + c["kl"] * kl
    g = g + c["kl"] * (1.0 - d.exp())
    g_ent = None
    w = s["weight"].view(-1).double()
    if H is not None:
        loss = loss - c["ent"] * H
        g_ent = -c["ent"] * w
    out = [torch.where(gone, 0.0, loss).float().view(B, R), torch.where(gone, 0.0, logp).float().view(B, R),
           torch.where(gone, 0.0, kl).float().view(B, R)]
    if H is not None:
        out.append(torch.where(gone, 0.0, H).float().view(B, R))
    out.append(_plain_token_grad(x, e, m, z, log_z, H, tok, T, g * w, g_ent, s["logits"].dtype).view(B, R, V))
    return out


def _plain_distill(s):
    c = s["case"]
    B, R, V = s["logits"].shape
    T, n, k, kind, mix = c["T"], B * R, s["ids"].shape[2], c["kind"], c["mix"]
    x = s["logits"].reshape(n, V).float()
    ids = s["ids"].view(n, k).long()
    here = ids >= 0
    gone = ~here.any(1)
    at = ids.clamp(min=0)
    e, m, z = _softmax_parts(x, T)
    xs = x.gather(1, at).double()
    es = torch.where(here, ((xs - m.double()) / T).exp(), 0.0)
    hits = torch.zeros((n, V), dtype=torch.bool, device=x.device)
    hits.scatter_(1, torch.where(here, at, at[:, :1]), True)          # absent entries repeat a present one
    tail_e = torch.where(hits, 0.0, e).sum(1).double()
    Z = tail_e + es.sum(1)
    log_q = torch.where(here, (xs - m.double()) / T - Z.log().view(-1, 1), 0.0)
    q = es / Z.view(-1, 1)
    rho = tail_e / Z
    val = torch.where(here, s["values"].view(n, k).double() / T, -math.inf)
    L = s["lse"].view(-1, 1).double() if s["lse"] is not None else torch.logsumexp(val, 1, keepdim=True)
    log_p = torch.where(here, val - L, 0.0)
    p = torch.where(here, (val - L).exp(), 0.0)
    if s["lse"] is not None:
        r = 1.0 - p.sum(1)
        r = torch.where(r < TAIL_FLOOR, torch.where(rho > 0, TAIL_FLOOR, 0.0), r)
    else:
        r = torch.zeros_like(rho)
    log_rho, log_r = rho.log(), r.log()
    if kind == "forward_kl":
        terms, tail = p * (log_p - log_q), torch.where(r > 0, r * (log_r - log_rho), 0.0)
        total = p.sum(1) + r
        gs = q * total.view(-1, 1) - p                                # q (g - c)
        gt = rho * total - r
    elif kind == "reverse_kl":
        terms, tail = q * (log_q - log_p), torch.where(rho > 0, rho * (log_rho - log_r), 0.0)
        cst = terms.sum(1) + tail
        gs = q * (log_q - log_p - cst.view(-1, 1))
        gt = torch.where(rho > 0, rho * (log_rho - log_r - cst), 0.0)
    else:
        mid, mid_t = mix * p + (1 - mix) * q, mix * r + (1 - mix) * rho
        kq = torch.where(here, log_q - mid.log(), 0.0)
        kq_t = torch.where(rho > 0, log_rho - mid_t.log(), 0.0)
        terms = mix * torch.where(here, p * (log_p - mid.log()), 0.0) + (1 - mix) * q * kq
        tail = mix * torch.where(r > 0, r * (log_r - mid_t.log()), 0.0) + (1 - mix) * rho * kq_t
        cst = (1 - mix) * ((q * kq).sum(1) + rho * kq_t)
        gs = q * ((1 - mix) * kq - cst.view(-1, 1))
        gt = rho * ((1 - mix) * kq_t - cst)
    loss = torch.where(gone, 0.0, terms.sum(1) + tail)
    out = [loss.float().view(B, R)]
    if c["train"]:
        w = torch.where(gone, 0.0, s["weight"].view(-1).double()) / T
        scale = torch.where(tail_e > 0, w * gt / tail_e, 0.0)
        scale = torch.where(gone, 0.0, scale)
        grad = e * scale.float().view(-1, 1)
        gs = torch.where(gone.view(-1, 1), 0.0, w.view(-1, 1) * gs).float()
        # absent entries repeat the first present one, with its value
        first = here.int().argmax(1, keepdim=True)
        grad.scatter_(1, torch.where(here, at, at.gather(1, first)), torch.where(here, gs, gs.gather(1, first)))
        out.append(grad.to(s["logits"].dtype).view(B, R, V))
    return out


# ---- one pass -------------------------------------------------------------------------------------

def _own_run(s):
    import paper_2512_13194_b200 as ears
    c = s["case"]
    op, T = c["op"], c["T"]
    if op == "top":
        top = ears.top_logits(s["logits"], c["k"], T, accept_len=s["accept_len"])
        return top.values, top.ids, top.lse
    if op == "token":
        if c["train"]:
            logp, entropy, grad = ears.token_logprobs_step(s["logits"], s["tokens"], s["d_logp"], s["d_entropy"], T)
            return [logp, grad] if entropy is None else [logp, entropy, grad]
        if c["entropy"]:
            return list(ears.token_logprobs(s["logits"], s["tokens"], T, entropy=True))
        return [ears.token_logprobs(s["logits"], s["tokens"], T)]
    if op == "distill":
        teacher = ears.TopLogits(s["values"], s["ids"], s["lse"])
        if c["train"]:
            return list(ears.distill_step(s["logits"], teacher, T, kind=c["kind"], mix=c["mix"], row_weight=s["weight"]))
        return [ears.distill_loss(s["logits"], teacher, T, kind=c["kind"], mix=c["mix"])]
    terms, grad = ears.policy_step(s["logits"], s["tokens"], s["old_logp"], s["advantage"], T, ref_logp=s["ref_logp"],
                                   clip_low=CLIP_LOW, clip_high=CLIP_HIGH, kl_coef=c["kl"], entropy_coef=c["ent"],
                                   row_weight=s["weight"])
    out = [terms.loss, terms.logp, terms.kl]
    if c["ent"] != 0.0:
        out.append(terms.entropy)
    return out + [grad]


def run(state):
    if own:
        return _own_run(state)
    with torch.no_grad():
        return {"top": _plain_top, "token": _plain_token, "distill": _plain_distill, "policy": _plain_policy}[state["case"]["op"]](state)


def work(case):
    n, V = case["B"] * case["R"], case["V"]
    size = 4 if case["dtype"] == "fp32" else 2
    if case["op"] == "top":
        rows, R = n, case["R"]
        if case["live"]:                                    # position j counts when j <= accept_len, uniform in 0..R
            rows = case["B"] * sum(min(R, a + 1) for a in range(R + 1)) / (R + 1)
        return {"bytes": rows * V * size + n * (8 * case["k"] + 4), "flops": 4.0 * rows * V}
    live = n * (1.0 - case["absent"])
    per_row = 12 if case["op"] == "token" else (8 * case["k"] + 12 if case["op"] == "distill" else 32)
    bytes_, flops = live * V * size + n * per_row, 4.0 * live * V
    if case["train"]:
        bytes_ += n * V * size
        flops += 4.0 * live * V
    return {"bytes": bytes_, "flops": flops}


# ---- the definitions in 64 bits --------------------------------------------------------------------

def _exact_top(s):
    c = s["case"]
    B, R, V = s["logits"].shape
    k = c["k"]
    values = torch.full((B, R, k), -math.inf, dtype=torch.float64)
    ids = torch.full((B, R, k), -1, dtype=torch.int64)
    lse = torch.full((B, R), -math.inf, dtype=torch.float64)
    for b in range(B):
        stop = R if s["accept_len"] is None else min(R, int(s["accept_len"][b]) + 1)
        for j in range(stop):
            row = s["logits"][b, j].double()
            val, idx = torch.sort(row, descending=True, stable=True)
            cnt = min(k, int((val > -math.inf).sum()))
            values[b, j, :cnt] = val[:cnt].cpu()
            ids[b, j, :cnt] = idx[:cnt].cpu()
            lse[b, j] = float(torch.logsumexp(row / c["T"], 0))
    return values, ids, lse


def _exact_token_terms(s, a, z, entropy):
    """Differentiable log probabilities (and entropies) of the rows a .. of the 64-bit logits z."""
    ls = torch.log_softmax(z / s["case"]["T"], 1)
    tok = s["tokens"].reshape(-1)[a:a + z.shape[0]].long()
    logp = ls.gather(1, tok.clamp(min=0)[:, None])[:, 0]
    H = None
    if entropy:
        finite = torch.isfinite(ls)
        H = -(torch.where(finite, ls.exp(), 0.0) * torch.where(finite, ls, 0.0)).sum(1)
    return logp, H, tok >= 0


def _exact_rows(s, terms, train):
    """terms(a, z) -> (outputs [m], weighted scalar); gathers outputs and d scalar / d z over all rows."""
    B, R, V = s["logits"].shape
    x = s["logits"].reshape(B * R, V)
    step = max(1, (1 << 26) // V)
    outs, grads = None, []
    for a in range(0, B * R, step):
        z = x[a:a + step].double()
        dead = torch.isinf(z)
        z = z.requires_grad_(train)
        o, scalar = terms(a, z)
        outs = [[] for _ in o] if outs is None else outs
        for lst, t in zip(outs, o):
            lst.append(t.detach())
        if train:
            (g,) = torch.autograd.grad(scalar, z)
            grads.append(torch.where(dead, 0.0, g))
    res = [torch.cat(l).view(B, R) for l in outs]
    if train:
        res.append(torch.cat(grads).view(B, R, V))
    return res


def _exact_token(s):
    c = s["case"]

    def terms(a, z):
        logp, H, on = _exact_token_terms(s, a, z, c["entropy"])
        cut = slice(a, a + z.shape[0])
        out = [torch.where(on, logp, 0.0)]
        scalar = (out[0] * s["d_logp"].reshape(-1)[cut].double()).sum()
        if c["entropy"]:
            out.append(torch.where(on, H, 0.0))
            scalar = scalar + (out[1] * s["d_entropy"].reshape(-1)[cut].double()).sum()
        return out, scalar
    return _exact_rows(s, terms, c["train"])


def _exact_policy(s):
    c = s["case"]

    def terms(a, z):
        cut = slice(a, a + z.shape[0])
        logp, H, on = _exact_token_terms(s, a, z, c["ent"] != 0.0)
        old, ref, adv, w = (s[key].reshape(-1)[cut].double() for key in ("old_logp", "ref_logp", "advantage", "weight"))
        ratio = torch.exp(logp - old)
        loss = -torch.minimum(ratio * adv, torch.clamp(ratio, 1 - CLIP_LOW, 1 + CLIP_HIGH) * adv)
        kl = torch.exp(ref - logp) - (ref - logp) - 1
        loss = loss + c["kl"] * kl
        if H is not None:
            loss = loss - c["ent"] * H
        out = [torch.where(on, loss, 0.0), torch.where(on, logp, 0.0), torch.where(on, kl, 0.0)]
        if H is not None:
            out.append(torch.where(on, H, 0.0))
        return out, (out[0] * w).sum()
    return _exact_rows(s, terms, True)


def _exact_distill(s):
    c = s["case"]
    T, kind, mix = c["T"], c["kind"], c["mix"]
    k = s["ids"].shape[2]

    def terms(a, z):
        m = z.shape[0]
        ids = s["ids"].reshape(-1, k)[a:a + m].long()
        here = ids >= 0
        on = here.any(1)
        ls = torch.log_softmax(z / T, 1)
        log_q = torch.where(here, ls.gather(1, ids.clamp(min=0)), 0.0)
        listed_cols = torch.zeros(z.shape, dtype=torch.float64, device=z.device)
        listed_cols.scatter_add_(1, ids.clamp(min=0), here.double())
        rest = torch.where(listed_cols > 0, -math.inf, ls)
        log_rho = torch.logsumexp(rest, 1)
        has_rest = torch.isfinite(log_rho)
        log_rho = torch.where(has_rest, log_rho, 0.0)
        rho = torch.where(has_rest, log_rho.exp(), 0.0)
        t = torch.where(here, s["values"].reshape(-1, k)[a:a + m].double() / T, -math.inf)
        if s["lse"] is not None:
            t = t - s["lse"].reshape(-1)[a:a + m, None].double()
            r = 1 - t.exp().sum(1)
            r = torch.where(r < TAIL_FLOOR, torch.where(has_rest, TAIL_FLOOR, 0.0), r)
        else:
            t = torch.log_softmax(t, 1)
            r = torch.zeros(m, dtype=torch.float64, device=z.device)
        log_p = torch.where(here, t, 0.0)
        one, zero = torch.ones_like(r), torch.zeros_like(r)
        log_r = torch.where(r > 0, r, one).log()
        p, q = torch.where(here, log_p.exp(), 0.0), torch.where(here, log_q.exp(), 0.0)
        both = (r > 0) & has_rest
        if kind == "forward_kl":
            loss = (p * (log_p - log_q)).sum(1) + torch.where(r > 0, torch.where(both, r * (log_r - log_rho), math.inf), zero)
        elif kind == "reverse_kl":
            loss = (q * (log_q - log_p)).sum(1) + torch.where(has_rest, rho * (log_rho - log_r), zero)
        else:
            log_mid = torch.where(here, torch.logaddexp(log_p + math.log(mix), log_q + math.log(1 - mix)), 0.0)
            mid = mix * r + (1 - mix) * rho
            log_mid_t = torch.where(mid > 0, mid, one).log()
            loss = (mix * p * (log_p - log_mid) + (1 - mix) * q * (log_q - log_mid)).sum(1)
            loss = loss + mix * r * (log_r - log_mid_t) + (1 - mix) * rho * (log_rho - log_mid_t)
        loss = torch.where(on, loss, 0.0)
        return [loss], (loss * s["weight"].reshape(-1)[a:a + m].double()).sum()

    # rows without a list leave NaN behind in their discarded branch
    out = _exact_rows(s, terms, c["train"])
    if c["train"]:
        off = ~(s["ids"] >= 0).any(2)
        out[1][off] = 0.0
    return out


def exact(case, seed):
    s = prepare(case, seed)
    return {"top": _exact_top, "token": _exact_token, "distill": _exact_distill, "policy": _exact_policy}[case["op"]](s)
