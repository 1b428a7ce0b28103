"""The rollout-record operators as measurable cases.

An engine that brings its own probabilities and random numbers verifies the
drafted tokens with ``verify_probs``; a rollout keeps the target's largest
logits of each position (``top_logits``) instead of whole rows; and the draft
heads are trained on those lists (``distill_loss_fwd_bwd``).  The listed cases
are these calls from a single request to the large batch, drawn cases spread
over the same ranges.
"""

import math

import torch

own = False

MAX_ELEMS = 4096 * 3 * 151936  # logits of the largest listed case


def listed():
    return [
        # one request's decoding step: the four target rows' lists, where latency counts
        dict(name="top one request", op="top", N=1, K=4, V=151936, dtype="bf16", M=64, T=1.0),
        # the record of a rollout engine's decoding batch
        dict(name="top rollout batch", op="top", N=256, K=4, V=151936, dtype="bf16", M=64, T=1.0),
        # the lists of a whole training batch from the target's forward pass
        dict(name="top training batch", op="top", N=4096, K=3, V=151936, dtype="bf16", M=128, T=1.0),
        # float32 logits of an odd vocabulary (rows that no vector load is aligned to), long lists
        dict(name="top float32 odd rows", op="top", N=96, K=1, V=100003, dtype="f32", M=200, T=0.7),
        # a small fine-tuning step: few positions, where launches count
        dict(name="distill small step", op="distill", N=8, K=3, V=151936, dtype="bf16", M=64, T=1.0, tail=True,
             grad="f32", empty=0, kind="forward"),
        # the training step: lists with the mass outside them as one more outcome
        dict(name="distill training step", op="distill", N=4096, K=3, V=151936, dtype="bf16", M=64, T=1.0, tail=True,
             grad="f32", empty=0, kind="forward"),
        # bfloat16 gradients for the head's products, a padded batch (one position in four has no list)
        dict(name="distill padded bf16 gradient", op="distill", N=2000, K=3, V=151936, dtype="bf16", M=128, T=2.0,
             tail=False, grad="bf16", empty=4, kind="forward"),
        # float32 logits of an odd vocabulary, short lists
        dict(name="distill float32 odd rows", op="distill", N=300, K=2, V=100003, dtype="f32", M=20, T=1.0,
             tail=False, grad="f32", empty=0, kind="ce"),
        # the loss alone, on held-out positions of a larger vocabulary
        dict(name="distill evaluation", op="distill", N=1000, K=3, V=262144, dtype="bf16", M=256, T=1.0, tail=True,
             grad=None, empty=0, kind="forward"),
        # one request's decoding step: latency of the smallest call
        dict(name="verify probs one request", op="verify", B=1, K=3, V=151936, dtype="f32", draft=True, ragged=False,
             overlap=False),
        # a rollout batch with the acceptance overlaps it logs
        dict(name="verify probs main batch", op="verify", B=256, K=3, V=151936, dtype="f32", draft=True,
             ragged=False, overlap=True),
        # the large decoding batch with its own number of drafts in every row
        dict(name="verify probs ragged batch", op="verify", B=1000, K=4, V=262144, dtype="bf16", draft=True,
             ragged=True, overlap=False),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("top", "distill", "distill", "verify", "verify"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    V = _log_uniform(rng, 32000, 262144)
    step = rng.choice((64, 64, 8, 1))  # padded vocabularies mostly, ragged ones among them
    V = V // step * step if step > 1 else V | 1
    K = rng.choice((1, 2, 3, 3, 4, 5))
    if op == "verify":
        dtype = rng.choice(("bf16", "f32", "f32"))
        most = MAX_ELEMS // (2 * V * (2 * K + 1))
        return dict(op=op, B=_log_uniform(rng, 1, max(1, min(1024, most))), K=K, V=V, dtype=dtype,
                    draft=rng.random() < 0.75, ragged=rng.random() < 0.4, overlap=rng.random() < 0.5)
    most = MAX_ELEMS // (K * V * (1 if dtype == "bf16" else 2))
    N = _log_uniform(rng, 1, max(1, min(4096, most)))
    M = _log_uniform(rng, 1, 256)
    T = rng.choice((1.0, 1.0, 0.7, 2.0))
    if op == "top":
        return dict(op=op, N=N, K=K, V=V, dtype=dtype, M=M, T=T)
    return dict(op=op, N=N, K=K, V=V, dtype=dtype, M=M, T=T, tail=rng.random() < 0.6,
                grad=rng.choice(("f32", "f32", None) + (("bf16",) if dtype == "bf16" else ("f32",))),
                empty=rng.choice((0, 0, 3)), kind=rng.choice(("forward", "forward", "ce")))


def _type(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _rows_per_chunk(V):
    return max(1, (1 << 25) // V)


def _logit_rows(g, n, V):
    """Rows of logits from flat to peaked, as the positions of a text have them."""
    z = torch.randn((n, V), device="cuda", generator=g)
    return z.mul_(torch.empty((n, 1), device="cuda").uniform_(1.5, 4.5, generator=g))


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 9973 + 5)
    op, V, K, ty = case["op"], case["V"], case["K"], _type(case["dtype"])
    s = dict(case=dict(case))
    if op == "verify":
        B = case["B"]
        p = torch.empty((B, K + 1, V), dtype=ty, device="cuda")
        q = torch.empty((B, K, V), dtype=ty, device="cuda") if case["draft"] else None
        ids = torch.empty((B, K), dtype=torch.int32, device="cuda")
        step = max(1, _rows_per_chunk(V) // (K + 1))
        for b in range(0, B, step):
            n = min(step, B - b)
            z = _logit_rows(g, n * (K + 1), V).view(n, K + 1, V)
            p[b:b + n] = torch.softmax(z, -1)
            # a draft head's distribution: the target's with noise (about three tokens in four are accepted)
            d = z[:, :K].add_(torch.randn((n, K, V), device="cuda", generator=g), alpha=0.6)
            d = torch.softmax(d, -1)
            if q is not None:
                q[b:b + n] = d
                d = d.div_(torch.empty_like(d).exponential_(generator=g))  # one draw from the draft
            ids[b:b + n] = d.argmax(-1).to(torch.int32)
        s.update(target=p, draft=q, ids=ids, u=torch.rand((B, K), device="cuda", generator=g),
                 us=torch.rand(B, device="cuda", generator=g), lens=None)
        if case["ragged"]:
            s["lens"] = torch.randint(0, K + 1, (B,), device="cuda", generator=g, dtype=torch.int32)
        return s
    N, M, T = case["N"], case["M"], case["T"]
    z = torch.empty((N * K, V), dtype=ty, device="cuda")
    if op == "distill":
        ids = torch.empty((N * K, M), dtype=torch.int32, device="cuda")
        val = torch.empty((N * K, M), dtype=torch.float32, device="cuda")
        lz = torch.empty(N * K, dtype=torch.float32, device="cuda")
    step = _rows_per_chunk(V)
    for r in range(0, N * K, step):
        n = min(step, N * K - r)
        t = _logit_rows(g, n, V)
        if op == "distill":
            # the teacher's list from its stored logits, and a student some way from it
            st = t.to(ty).float()
            v, i = torch.topk(st, M, dim=-1)
            ids[r:r + n], val[r:r + n] = i.to(torch.int32), v
            lz[r:r + n] = torch.logsumexp(st / T, -1)
            t = t.add_(torch.randn((n, V), device="cuda", generator=g), alpha=0.8)
        z[r:r + n] = t
    s["logits"] = z.view(N, K, V)
    if op == "distill":
        ids, lz = ids.view(N, K, M), lz.view(N, K)
        if case["empty"]:
            ids[::case["empty"]] = -1  # padding: positions without a list
        s.update(ids=ids, values=val.view(N, K, M), logz=lz if case["tail"] else None)
    return s


def run(state):
    c = state["case"]
    if own:
        from paper_2606_12370_amd import binding
        if c["op"] == "top":
            return binding.top_logits(state["logits"], c["M"], c["T"])
        if c["op"] == "distill":
            return binding.distill_loss_fwd_bwd(
                state["logits"], state["ids"], state["values"], state["logz"], temperature=c["T"], kind=c["kind"],
                scale=1.0 / c["N"], want_grad=c["grad"] is not None,
                grad_dtype=None if c["grad"] is None else _type(c["grad"]))
        return binding.verify_probs(state["target"], state["draft"], state["ids"], state["u"], state["us"],
                                    draft_lens=state["lens"], want_overlap=c["overlap"])
    if c["op"] == "top":
        return _plain_top(state["logits"], c["M"], c["T"])
    if c["op"] == "distill":
        return _plain_distill(state, c)
    return _plain_verify(state, c)


# ---- plain forms --------------------------------------------------------------

def _plain_top(logits, M, T):
    """Largest first, ties to the lowest index: one 64-bit key per logit, its
    order in the high half and the reversed index in the low half."""
    N, K, V = logits.shape
    rows = logits.reshape(N * K, V)
    R = N * K
    ids = torch.empty((R, M), dtype=torch.int32, device=rows.device)
    values = torch.empty((R, M), dtype=torch.float32, device=rows.device)
    logz = torch.empty(R, dtype=torch.float32, device=rows.device)
    back = (1 << 32) - 1 - torch.arange(V, device=rows.device)
    for r in range(0, R, 2048):  # 64-bit keys of a whole training batch would take most of the memory
        x = rows[r:r + 2048].float() + 0.0  # one zero
        bits = x.view(torch.int32)
        key = (bits ^ ((bits >> 31) & 0x7fffffff)).long()
        key = torch.topk(key * (1 << 32) + back, min(M, V), dim=-1).values
        i = (1 << 32) - 1 - (key & ((1 << 32) - 1))
        v = torch.gather(x, 1, i)
        ids[r:r + 2048] = -1
        values[r:r + 2048] = -math.inf
        ids[r:r + 2048, :v.shape[1]] = torch.where(v > -math.inf, i, -1).to(torch.int32)
        values[r:r + 2048, :v.shape[1]] = v
        x = x / T
        m = x.amax(-1, keepdim=True)
        logz[r:r + 2048] = m[:, 0] + (x - m).exp().sum(-1).log()
    return dict(ids=ids.view(N, K, M), values=values.view(N, K, M), logz=logz.view(N, K))


TAIL_MIN = 2.0 ** -18  # a smaller mass outside the list is below what a float32 log Z resolves


def _plain_distill(s, c):
    z, ids, T = s["logits"], s["ids"].long(), c["T"]
    N, K, V = z.shape
    used = ids >= 0
    at = ids.clamp(min=0)
    # the teacher's few probabilities, in 64 bits (the tail is a difference)
    a = torch.where(used, s["values"].double() / T, -math.inf)
    if s["logz"] is None:
        m = a.amax(-1, keepdim=True)
        m = torch.where(m > -math.inf, m, 0.0)
        lse = m + (a - m).exp().sum(-1, keepdim=True).log()
        lp = torch.where(used, a - lse, -math.inf)
        tail = torch.zeros((N, K), dtype=torch.float64, device=z.device)
    else:
        lp = a - s["logz"].double()[..., None]
        tail = 1.0 - lp.exp().sum(-1)
        tail = torch.where(tail > TAIL_MIN, tail, 0.0)
    p = lp.exp()
    any_used = used.any(-1)
    tail = torch.where(any_used, tail, 0.0)
    mass = p.sum(-1)
    # the student's distribution
    x = z.float() / T
    x = x - x.amax(-1, keepdim=True)
    e = x.exp()
    E = e.sum(-1, keepdim=True)
    lq = torch.gather(x, 2, at).double() - E.double().log()
    live = p > 0
    L = -torch.where(live, p * torch.where(live, lq, 0.0), 0.0).sum(-1)
    if c["kind"] == "forward":
        L = L + torch.where(live, p * torch.where(live, lp, 0.0), 0.0).sum(-1)
    tail32 = tail.float()[..., None]
    coef = None
    if s["logz"] is not None:
        listed = torch.zeros((N, K, V + 1), dtype=torch.bool, device=z.device)
        listed.scatter_(2, torch.where(used, at, V), True)
        Et = torch.where(listed[..., :V], 0.0, e).sum(-1, keepdim=True)
        lqt = (Et / E).double().log()[..., 0]
        has = tail > 0
        t1 = -lqt
        if c["kind"] == "forward":
            t1 = t1 + torch.where(has, tail, 1.0).log()
        L = L + torch.where(has, tail * torch.where(has, t1, 0.0), 0.0)
        # off the list q_v (W + r - r / q_tail)
        coef = torch.where(listed[..., :V], 0.0, torch.where(tail32 > 0, tail32 * (E / Et), 0.0))
    loss = (L.sum() / (N * K)).float().reshape(1)
    grad = None
    if c["grad"] is not None:
        f = (mass + tail).float()[..., None]
        g = e / E * (f if coef is None else f - coef)
        g.scatter_add_(2, at, torch.where(used, -p, 0.0).float())
        grad = g.mul_(1.0 / (N * K * T)).to(_type(c["grad"]))
    return loss, L.float(), grad


def _plain_verify(s, c):
    p, q, ids = s["target"], s["draft"], s["ids"].long()
    B, K1, V = p.shape
    K = K1 - 1
    dev = p.device
    lens = torch.full((B,), K, device=dev) if s["lens"] is None else s["lens"].long()
    step = torch.arange(K, device=dev)[None]
    on = step < lens[:, None]
    px = torch.gather(p[:, :K], 2, ids[..., None])[..., 0].double()
    qx = torch.ones_like(px) if q is None else torch.gather(q, 2, ids[..., None])[..., 0].double()
    ok = on & (s["u"].double() * qx < px)  # exact: 24-bit factors in 64 bits
    n = ok.long().cumprod(-1).sum(-1)
    b = torch.arange(B, device=dev)
    r = p[b, n].double()
    pn = r
    rejected = (n < lens)[:, None]
    at = n.clamp(max=K - 1)
    if q is None:
        v = torch.arange(V, device=dev)[None]
        r = torch.where(rejected & (v == ids[b, at][:, None]), 0.0, r)
    else:
        r = (r - torch.where(rejected, q[b, at].double(), 0.0)).clamp(min=0.0)
    cum = r.cumsum(-1)
    none = cum[:, -1:] <= 0.0
    cum = torch.where(none, pn.cumsum(-1), cum)
    tok = (cum <= s["us"].double()[:, None] * cum[:, -1:]).sum(-1)
    slots = torch.arange(K + 1, device=dev)[None]
    emitted = torch.cat([ids, ids[:, :1]], 1)
    emitted = torch.where(slots < n[:, None], emitted, -1)
    emitted = torch.where(slots == n[:, None], tok[:, None], emitted).to(torch.int32)
    out = dict(accept_len=n.to(torch.int32), emitted=emitted)
    if c["overlap"]:
        ov = px if q is None else torch.minimum(p[:, :K], q).sum(-1, dtype=torch.float64)
        out["overlap"] = torch.where(on, ov, 0.0).float()
    return out


# ---- what a pass cannot do without ----------------------------------------------

ACCEPT = 0.76  # of the drafted tokens (noise of 0.6 on the logits: 2 Phi(-0.3))


def work(case):
    V, K = case["V"], case["K"]
    e = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "top":
        rows = case["N"] * K
        # per logit the widening, maximum, exponential, sum and comparison
        return dict(bytes=rows * (V * e + 8 * case["M"] + 4), flops=5 * rows * V)
    if case["op"] == "distill":
        N = case["N"]
        rows = N * K
        live = rows - ((N + case["empty"] - 1) // case["empty"] * K if case["empty"] else 0)
        g = {"f32": 4, "bf16": 2, None: 0}[case["grad"]]
        b = live * V * e + rows * V * g + rows * case["M"] * 8 + rows * 4 * (2 if case["tail"] else 1) + 4
        return dict(bytes=b, flops=live * V * (8 if g else 4))
    B = case["B"]
    steps = K / 2 if case["ragged"] else K
    if case["overlap"] and case["draft"]:
        rows = 2 * steps + ACCEPT ** steps  # all pairs, and the bonus row where every draft passes
    else:
        # the emitting step: its pair, or the bonus row alone
        rows = 1 + (1 - ACCEPT ** steps if case["draft"] else 0)
    return dict(bytes=int(B * rows * V * e) + B * (16 * K + 16), flops=int(B * rows * V * 2))


# ---- 64-bit values ----------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"top": _exact_top, "distill": _exact_distill, "verify": _exact_verify}[case["op"]](case, s)


def _exact_top(c, s):
    N, K, V = s["logits"].shape
    rows = s["logits"].reshape(N * K, V)
    M = min(c["M"], V)
    ids, values, logz = [], [], []
    for r in range(0, N * K, 64):
        v, i = rows[r:r + 64].double().sort(dim=-1, descending=True, stable=True)
        ids.append(torch.where(v[:, :M].isinf(), -1, i[:, :M]).to(torch.int32))
        values.append(v[:, :M].clone())
        logz.append(torch.logsumexp(v / c["T"], -1))
    return dict(ids=torch.cat(ids).view(N, K, M), values=torch.cat(values).view(N, K, M),
                logz=torch.cat(logz).view(N, K))


def _exact_distill(c, s):
    z, T = s["logits"], c["T"]
    N, K, V = z.shape
    per = torch.zeros((N, K), dtype=torch.float64, device=z.device)
    grad = None
    if c["grad"] is not None:
        if N * K * V > MAX_ELEMS:
            return None
        grad = torch.zeros((N, K, V), dtype=torch.float64, device=z.device)
    step = max(1, (1 << 25) // (K * V))
    for n in range(0, N, step):
        lq = torch.log_softmax(z[n:n + step].double() / T, -1)
        ids = s["ids"][n:n + step].long()
        t = torch.where(ids >= 0, s["values"][n:n + step].double() / T, -torch.inf)
        lp = torch.log_softmax(t, -1) if s["logz"] is None else t - s["logz"][n:n + step].double()[..., None]
        lp = torch.where(ids >= 0, lp, -torch.inf)
        p = lp.exp()
        P = torch.zeros_like(lq)
        P.scatter_add_(-1, ids.clamp(min=0), p)
        L = -torch.xlogy(p, 1.0).sum(-1)
        lqi = lq.gather(-1, ids.clamp(min=0))
        L = L - torch.where(p > 0, p * lqi, 0.0).sum(-1)
        W = p.sum(-1)
        r = torch.zeros_like(W)
        q = lq.exp()
        off = torch.zeros_like(q)
        if s["logz"] is not None:
            r = 1.0 - W
            r = torch.where((r > TAIL_MIN) & (ids >= 0).any(-1), r, 0.0)
            hit = torch.zeros_like(q).scatter_add_(-1, ids.clamp(min=0), (ids >= 0).double())
            off = torch.where(hit > 0, 0.0, q)
            qt = off.sum(-1)
            L = L - torch.where(r > 0, r * qt.log(), 0.0)
            off = off * torch.where(r > 0, r / qt, 0.0)[..., None]
        if c["kind"] == "forward":
            L = L + torch.xlogy(p, p).sum(-1) + torch.xlogy(r, r)
        per[n:n + step] = L
        if grad is not None:
            grad[n:n + step] = (q * (W + r)[..., None] - P - off) / (N * K * T)
    return per.sum().reshape(1) / (N * K), per, grad


def _exact_verify(c, s):
    p, q, ids, u, us = s["target"], s["draft"], s["ids"], s["u"], s["us"]
    B, K = ids.shape
    acc = torch.zeros(B, dtype=torch.int32, device=p.device)
    em = torch.full((B, K + 1), -1, dtype=torch.int32, device=p.device)
    ov = torch.zeros((B, K), dtype=torch.float64, device=p.device)
    lens = [K] * B if s["lens"] is None else s["lens"].tolist()
    host_ids, host_u = ids.tolist(), u.tolist()
    for b in range(B):
        pd = p[b].double()
        n = 0
        px = [float(v) for v in pd[torch.arange(K, device=p.device), ids[b].long()]]
        qx = [1.0] * K if q is None else [float(v) for v in q[b].double()[torch.arange(K, device=p.device),
                                                                          ids[b].long()]]
        while n < lens[b] and host_u[b][n] * qx[n] < px[n]:
            em[b, n] = host_ids[b][n]
            n += 1
        acc[b] = n
        r = pd[n].clone()
        if n < lens[b]:
            if q is None:
                r[host_ids[b][n]] = 0.0
            else:
                r = torch.relu(r - q[b, n].double())
        if float(r.sum()) <= 0.0:
            r = pd[n]
        cum = torch.cumsum(r, 0)
        em[b, n] = torch.searchsorted(cum, us[b].double() * cum[-1:], right=True)[0].to(torch.int32)
        if c["overlap"]:
            for i in range(lens[b]):
                ov[b, i] = px[i] if q is None else torch.minimum(pd[i], q[b, i].double()).sum()
    out = dict(accept_len=acc, emitted=em)
    if c["overlap"]:
        out["overlap"] = ov
    return out
