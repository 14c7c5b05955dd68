"""The vocabulary operators' definitions in 64 bits (numpy, a row at a time),
and their inputs and tolerances.

Tolerances, from the arithmetic (u = 2^-24, fp32's rounding unit):
  log probabilities: (x - max) / T takes three roundings, 3 u |z|; the sum of
    exponentials is off by its terms' 4 u + 2 u |z| (weighted by p) and by one
    rounding per addition of the longest chain, at most 160 u; so 1e-5 absolute
    and 1e-6 of the value.
  entropy: a sum of like-signed terms with those errors: 1e-5 of it and 1e-5.
  gradients: p to 2e-5 of itself, at a target 1 - p to 4e-7 more; entropy terms
    p (logp + H) to 2e-5 of p (|logp| + H + 1).  bf16 results: one rounding more,
    2^-8 of the value.
  losses: T^2 times the errors of log q and log p, 2e-5, and 1e-5 of the value.
"""
import math

import numpy as np
import torch

from paper_2502_10940_gb300 import cola

TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}


# ------------------------------------------------------------- definitions
def softmax_stats(z):
    """Maximum, log of the sum of exp(z - maximum), and probabilities of one row;
    zeros where it is all -inf.  (The two are kept apart: a maximum of 1e38
    would swallow the logarithm.)"""
    m = z.max()
    if m == -np.inf:
        return m, 0.0, np.zeros_like(z)
    with np.errstate(invalid="ignore", over="ignore"):
        e = np.exp(z - m)
        s = e.sum()
        return m, np.log(s), e / s


def log_softmax(z, m, logs):
    return np.full(len(z), -np.inf) if m == -np.inf else (z - m) - logs


def _xlogx(p, logp):
    return np.where(p > 0, p * np.where(p > 0, logp, 0.0), p * 0.0)


def logprob_row(x, y, T, g=0.0, h=0.0, k=0):
    V = len(x)
    with np.errstate(invalid="ignore"):
        z = x / T
        m, logs, p = softmax_stats(z)
        logp = log_softmax(z, m, logs)
        H = -_xlogx(p, logp).sum() if m != -np.inf else 0.0
        there = 0 <= y < V
        g = g if there else 0.0
        dx = np.zeros(V)
        if (g != 0 or h != 0) and m != -np.inf:
            dx = -g * p - h * (_xlogx(p, logp) + p * H)
            if there:
                dx[y] += g
            dx /= T
    # largest first, NaN above all, ties to the lower id
    order = np.lexsort((np.arange(V), -np.where(np.isnan(x), 0, x), ~np.isnan(x)))[:k]
    return dict(logp=logp[y] if there else 0.0, entropy=H, top_ids=order, top_logp=logp[order], dlogits=dx, p=p, logp_all=logp)


def distill_row(x, ids, vals, lse_t, T, Tt, rest, w=0.0):
    V = len(x)
    with np.errstate(invalid="ignore", divide="ignore"):
        z = x / T
        m, logs, p = softmax_stats(z)
        logp = log_softmax(z, m, logs)
        ok = (ids >= 0) & (ids < V)
        ids, u = ids[ok], vals[ok] / Tt
        if rest:
            q = np.exp(u - lse_t)
        else:
            q = softmax_stats(u)[2] if len(u) else u
        out = np.ones(V, bool)
        out[ids] = False
        has_rest = bool(rest and out.any() and (np.isnan(x[out]).any() or x[out].max() > -np.inf))
        mr, logr, rp = softmax_stats(z[out]) if out.any() else (-np.inf, 0.0, z[:0])
        qr = max(0.0, 1.0 - q.sum()) if has_rest else 0.0
        loss = 0.0
        for qk, lp in zip(q, logp[ids]):
            if qk > 0 or qk != qk:
                loss += qk * (math.log(qk) - lp) if qk > 0 else qk
        if qr > 0:
            loss += qr * (math.log(qr) - ((mr - m) + (logr - logs)))
        dx = np.zeros(V)
        if w != 0 and m != -np.inf:
            Q = q.sum() + qr
            dx = Q * p
            dx[ids] -= q
            dx[out] -= qr * rp
            dx *= w * T
    within = np.zeros(V)
    within[out] = rp
    return dict(loss=T * T * loss, dlogits=dx, p=p, rest=within)


# ------------------------------------------------------------------ inputs
def place(x, dtype, layout="dense", fill=4096.0):
    """x [n x V] (float64 numpy) on the GPU in one of the layouts; returns the view."""
    n, V = x.shape
    pitch, shift = {"dense": (V, 0), "padded": ((V + 63) // 64 * 64 + 64, 0), "odd": (V + 3, 0), "shifted": (V + 5, 3)}[layout]
    buf = torch.full((n * pitch + 8,), fill, dtype=TORCH[dtype], device="cuda")
    view = torch.as_strided(buf, (n, V), (pitch, 1), shift)
    view.copy_(torch.from_numpy(x))
    return view


def like(view, fill=float("nan"), shift=0):
    """An output of the view's shape and pitch, everything set to fill."""
    n, V = view.shape
    buf = torch.full((n * view.stride(0) + 8,), fill, dtype=view.dtype, device="cuda")
    return torch.as_strided(buf, (n, V), (view.stride(0), 1), shift), buf


def rounded(x, dtype):
    """x as the values the type holds."""
    return torch.from_numpy(np.asarray(x)).to(TORCH[dtype]).double().numpy()


def logits(rng, n, V, dtype, scale=2.0):
    x = rng.standard_normal((n, V)) * scale
    for i in range(n):
        at = rng.integers(0, V, size=min(V, 4))
        x[i, at] += rng.uniform(2.0, 9.0, size=len(at))
    return rounded(x, dtype)


def host(t):
    return None if t is None else t.detach().cpu().double().numpy()


# -------------------------------------------------------------- comparisons
def same_nonfinite(name, got, ref):
    assert np.array_equal(np.isnan(got), np.isnan(ref)), (name, got, ref)
    inf = np.isinf(ref)
    assert np.array_equal(np.isinf(got), inf) and np.array_equal(got[inf], ref[inf]), (name, got, ref)


def check(name, got, ref, tol):
    got = np.asarray(got, np.float64)
    with np.errstate(over="ignore"):   # results are fp32: beyond its range they are infinite
        ref = np.where(np.isinf(np.asarray(ref, np.float64).astype(np.float32)), np.asarray(ref).astype(np.float32), ref)
    same_nonfinite(name, got, ref)
    ok = np.isfinite(ref)
    tol = np.broadcast_to(np.asarray(tol, np.float64), ref.shape)
    far = np.abs(got[ok] - ref[ok]) - tol[ok]
    assert far.size == 0 or far.max() <= 0, f"{name}: over its tolerance by {far.max():.3e}"


def logp_tol(ref):
    return 1e-5 + 1e-6 * np.abs(np.where(np.isfinite(ref), ref, 0))


def grad_tol(ref, base, dtype):
    return base + (2.0 ** -8 * np.abs(np.where(np.isfinite(ref), ref, 0)) if dtype == "bf16" else 0.0) + 1e-37


def check_logprob_grad(got, r, y, g, h, T, dtype):
    p = np.where(np.isfinite(r["p"]), r["p"], 0)
    L = np.abs(np.where(np.isfinite(r["logp_all"]), r["logp_all"], 0))
    H = r["entropy"] if np.isfinite(r["entropy"]) else 0.0
    base = (abs(g) * 2e-5 * p + abs(h) * 2e-5 * p * (L + H + 1)) / T
    if 0 <= y < len(p):
        base[y] += abs(g) * 4e-7 / T
    check("dlogits", got, r["dlogits"], grad_tol(r["dlogits"], base, dtype))


def check_distill_grad(got, r, ids, w, T, dtype):
    # outside the list: the rate Q - q_R / p_R times p is (sum q - sum p) times the
    # softmax over the rest, the difference off by at most 4e-6 of a whole (3 u |u_k|
    # and 3 u |z_k| in exponents weighted by q and p), the softmax by 2e-5 of itself
    base = abs(w) * T * 4e-6 * np.nan_to_num(r["rest"]) + 2e-5 * np.abs(np.nan_to_num(r["dlogits"]))
    ids = ids[(ids >= 0) & (ids < len(base))]
    base[ids] += abs(w) * T * 2e-5
    check("dlogits", got, r["dlogits"], grad_tol(r["dlogits"], base, dtype))


def loss_tol(ref, T):
    return T * T * 2e-5 + 1e-5 * np.abs(np.where(np.isfinite(ref), ref, 0))


# -------------------------------------------------------------- both at once
def run_logprob(x, targets, dtype, T, k, g=None, h=None, layout="dense", place_like=None):
    """fwd, bwd and step on the same rows; every output on the host, the
    backward's and the step's gradients both."""
    n, V = x.shape
    X = place(x, dtype, layout)
    pitch = X.stride(0)
    d = cola.vocab_desc(n, V, ld=pitch, ld_grad=pitch, dtype=dtype, temperature=T, k=k)
    f = lambda *s: torch.full(s, float("nan"), device="cuda")   # noqa: E731
    tg = torch.as_tensor(targets, dtype=torch.int64, device="cuda")
    o = dict(logp=f(n), entropy=f(n), stats=f(n, 4), top_ids=None, top_logp=None)
    if k:
        o["top_ids"] = torch.full((n, k), -7, dtype=torch.int64, device="cuda")
        o["top_logp"] = f(n, k)
    cola.cola_token_logprob_fwd(d, X, tg, o["logp"], o["entropy"], o["top_ids"], o["top_logp"], o["stats"])
    if g is not None or h is not None:
        up = [None if v is None else torch.as_tensor(v, dtype=torch.float32, device="cuda") for v in (g, h)]
        shift = X.storage_offset() if layout != "shifted" else 1   # shifted: another offset than the logits'
        o["bwd"], b1 = like(X, shift=shift)
        cola.cola_token_logprob_bwd(d, X, tg, o["stats"], up[0], up[1], o["bwd"])
        o["step"], b2 = like(X, shift=shift)
        o["logp2"], o["entropy2"] = f(n), f(n)
        cola.cola_token_logprob_step(d, X, tg, up[0], up[1], o["logp2"], o["entropy2"], o["step"])
        torch.cuda.synchronize()
        for b in (b1, b2):   # nothing outside the rows
            t = b.clone()
            torch.as_strided(t, (n, V), (pitch, 1), shift).fill_(float("nan"))
            assert bool(torch.isnan(t).all())
    return {key: None if t is None else t.cpu().numpy() if t.dtype == torch.int64 else host(t) for key, t in o.items()}


def run_distill(x, ids, vals, lse, dtype, T, Tt, rest, w, layout="dense"):
    n, V = x.shape
    X = place(x, dtype, layout)
    pitch = X.stride(0)
    k = ids.shape[1]
    d = cola.vocab_desc(n, V, ld=pitch, ld_grad=pitch, dtype=dtype, temperature=T, k=k, rest=rest, teacher_temperature=Tt)
    f = lambda *s: torch.full(s, float("nan"), device="cuda")   # noqa: E731
    I = torch.as_tensor(ids, dtype=torch.int64, device="cuda")
    U = torch.as_tensor(vals, dtype=torch.float32, device="cuda")
    L = None if lse is None else torch.as_tensor(lse, dtype=torch.float32, device="cuda")
    W = torch.as_tensor(w, dtype=torch.float32, device="cuda")
    o = dict(loss=f(n), loss2=f(n), stats=f(n, 4))
    cola.cola_topk_distill_fwd(d, X, I, U, L, o["loss"], o["stats"])
    shift = X.storage_offset() if layout != "shifted" else 1
    o["bwd"], b1 = like(X, shift=shift)
    cola.cola_topk_distill_bwd(d, X, I, U, L, o["stats"], W, o["bwd"])
    o["step"], b2 = like(X, shift=shift)
    cola.cola_topk_distill_step(d, X, I, U, L, W, o["loss2"], o["step"])
    torch.cuda.synchronize()
    for b in (b1, b2):
        t = b.clone()
        torch.as_strided(t, (n, V), (pitch, 1), shift).fill_(float("nan"))
        assert bool(torch.isnan(t).all())
    return {key: host(t) for key, t in o.items()}


def teacher(rng, x, k, Tt, noise=1.0):
    """A teacher's k most likely tokens of each row, their logits in fp32, and
    its log sum exp at temperature Tt (-inf students included)."""
    t = x * 0.9 + rng.standard_normal(x.shape) * noise
    ids = np.argsort(-t, axis=1, kind="stable")[:, :k]
    vals = np.take_along_axis(t, ids, 1).astype(np.float32)
    m = t.max(1)
    m0 = np.where(np.isfinite(m), m, 0)
    with np.errstate(divide="ignore"):
        lse = (m0 / Tt + np.log(np.exp((t - m0[:, None]) / Tt).sum(1))).astype(np.float32)
    return ids, vals, lse
