"""Inputs and comparisons shared by the CPU and GPU tests of the rollout calls."""

import numpy as np
import torch

from oracle.rollout import distill_ref, top_ref, verify_probs_ref

U = 2.0 ** -24  # half a step of float32, relative
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
LOWEST = {torch.float32: torch.finfo(torch.float32).min, torch.bfloat16: torch.finfo(torch.bfloat16).min}


def f64(t):
    return t.detach().double().cpu().numpy()


def check_top(out, logits, M, T, want_logz=True):
    """Lists exact.  log Z: each exponential is off by the roundings of the
    difference, of the scale and of the product, 2^-24 |d| / T each, and its own
    (2 2^-24); a float32 sum of 32 by 31 2^-24 more; then one rounding."""
    V = logits.shape[-1]
    z = f64(logits).reshape(-1, V)
    Tn = np.asarray(T, dtype=np.float64)
    if Tn.ndim:
        Tn = np.repeat(Tn, z.shape[0] // len(Tn))
    ref = top_ref(z, M, Tn)
    assert np.array_equal(out["ids"].cpu().numpy().reshape(-1, M), ref["ids"])
    assert np.array_equal(f64(out["values"]).reshape(-1, M), ref["values"], equal_nan=True)
    if not want_logz:
        assert "logz" not in out
        return ref
    lz = f64(out["logz"]).reshape(-1)
    # (a row of the lowest float32 at T = 1/2 has log Z near -6.8e38, which rounds to -inf in float32)
    with np.errstate(over="ignore"):
        ref32 = ref["logz"].astype(np.float32)
    fin = np.isfinite(ref32)
    assert np.array_equal(lz[~fin], ref32[~fin], equal_nan=True)
    err = np.abs(lz[fin] - ref["logz"][fin])
    lim = (U * (33 + 3 * ref["spread"]) + U * np.abs(ref["logz"]))[fin]
    assert np.all(err <= lim), (err.max(), lim.min())
    return ref


def check_distill(got, z, ids, values, logz, T, kind, scale=1.0):
    """Errors within what the oracle counts in units of 2^-24, plus one rounding
    of each output (and float32's smallest normal number)."""
    loss, per, grad = got
    T = float(np.float32(T))
    scale = float(np.float32(scale))
    ref = distill_ref(f64(z), ids.cpu().numpy(), f64(values), None if logz is None else f64(logz), T, kind, scale)
    R = ref["per_step"]
    tiny = 2.0 ** -126

    def close(a, b, lim):
        same = (a == b) | (np.isnan(a) & np.isnan(b))
        with np.errstate(invalid="ignore"):
            ok = same | (np.abs(a - b) <= lim)
        assert np.all(ok), (int((~ok).sum()), a[~ok][:3], b[~ok][:3], np.broadcast_to(lim, a.shape)[~ok][:3])

    step_lim = U * ref["step_err"] + U * np.abs(R) + tiny
    if per is not None:
        close(f64(per), R, step_lim)
    if loss is not None:
        close(f64(loss), np.array([ref["loss"]]),
              abs(scale) * (U * ref["step_err"]).mean(axis=1).sum() + U * abs(ref["loss"]) + tiny)
    if grad is not None:
        close(f64(grad), ref["grad"], U * ref["grad_err"] + HALF[grad.dtype] * np.abs(ref["grad"])
              + tiny * (1 + ref["grad_unit"][..., None]))
    return ref


def check_probs(out, p, q, ids, u, us, lens=None):
    """Tokens exact; overlaps to one rounding of a float64 sum."""
    K = p.shape[1] - 1
    ref = verify_probs_ref(f64(p), None if q is None else f64(q), ids.cpu().numpy(), f64(u), f64(us),
                           None if lens is None else lens.cpu().numpy())
    assert ref["margin"].min() > 1e-13, "a uniform of these inputs lies on a step of the cumulative sum"
    assert np.array_equal(out["accept_len"].cpu().numpy(), ref["accept_len"])
    assert np.array_equal(out["emitted"].cpu().numpy(), ref["emitted"])
    if "overlap" in out and K:
        o = f64(out["overlap"])
        assert np.array_equal(np.isnan(o), np.isnan(ref["overlap"]))
        assert np.all(np.abs(np.nan_to_num(o - ref["overlap"])) <= (U + 1e-12) * np.abs(np.nan_to_num(ref["overlap"])) + 2.0 ** -149)
    return ref


def logit_rows(shape, dtype, seed, device="cuda", spread=3.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * spread).to(dtype).to(device)


def lists(N, K, V, M, seed, T=1.0, device="cuda", near=None):
    """A teacher's lists and log Z from random rows (distinct ids)."""
    g = torch.Generator().manual_seed(seed)
    t = torch.randn((N, K, V), generator=g) * 3.0 if near is None else near
    m = min(M, V)
    v, i = torch.topk(t, m, dim=-1)
    ids = torch.full((N, K, M), -1, dtype=torch.int32)
    val = torch.full((N, K, M), -torch.inf)
    ids[..., :m], val[..., :m] = i.to(torch.int32), v
    lz = torch.logsumexp(t.double() / T, -1).float()
    return ids.to(device), val.to(device), lz.to(device)


def probs(B, K, V, dtype, seed, device="cuda", noise=0.6, draft=True):
    """Target and draft probabilities, draft tokens drawn from the draft, uniforms."""
    g = torch.Generator().manual_seed(seed)
    z = torch.randn((B, K + 1, V), generator=g) * 2.5
    d = z[:, :K] + noise * torch.randn((B, K, V), generator=g)
    p = torch.softmax(z, -1)
    q = torch.softmax(d, -1)
    ids = (q / torch.empty_like(q).exponential_(generator=g)).argmax(-1).to(torch.int32) if K else \
        torch.zeros((B, 0), dtype=torch.int32)
    u = torch.rand((B, K), generator=g)
    us = torch.rand(B, generator=g)
    q = q.to(dtype).to(device) if draft else None
    return p.to(dtype).to(device), q, ids.to(device), u.to(device), us.to(device)
