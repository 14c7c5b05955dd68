"""Gradients whose row pitch is not the logits': rows of one call that lie on
16-byte boundaries alike and otherwise, of every kernel that stores them."""
import numpy as np
import pytest
import torch

import vocab_helpers as H
from paper_2502_10940_gb300 import cola

pytestmark = pytest.mark.gpu

# rows of a warp, of four warps, of several tiles, of a cluster
SHAPES = [(9, 517), (9, 5003), (700, 9001), (3, 90001)]
# what the gradient's pitch has more than the logits': a whole number of 16-byte blocks, odd and even ones
MORE = [8, 1, 2, 4, 7]


def _gradient(n, V, pitch, dtype):
    """Rows at a pitch, NaN everywhere, and whether nothing but the rows was stored to."""
    buf = torch.full((n * pitch + 8,), float("nan"), dtype=H.TORCH[dtype], device="cuda")
    view = torch.as_strided(buf, (n, V), (pitch, 1), 0)

    def rows_alone():
        t = buf.clone()
        torch.as_strided(t, (n, V), (pitch, 1), 0).fill_(float("nan"))
        return bool(torch.isnan(t).all())

    return view, rows_alone


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("more", MORE)
@pytest.mark.parametrize("n,V", SHAPES)
def test_log_probabilities(n, V, more, dtype):
    rng = np.random.default_rng(V + more)
    x = H.logits(rng, n, V, dtype)
    x[1, ::2] = -np.inf
    x[2, V // 2:] = float(torch.finfo(H.TORCH[dtype]).min)
    t = rng.integers(0, V, n)
    t[1] = 1
    g, h = (rng.standard_normal(n).astype(np.float32) for _ in range(2))
    X, T = H.place(x, dtype), 1.5
    f = lambda a, dt=torch.float32: torch.as_tensor(a, dtype=dt, device="cuda")   # noqa: E731
    G, E, tg = f(g), f(h), f(t, torch.int64)
    stats, logp, ent = (torch.empty(s, device="cuda") for s in ((n, 4), (n,), (n,)))
    d = cola.vocab_desc(n, V, ld=V, ld_grad=V + more, dtype=dtype, temperature=T)
    cola.cola_token_logprob_fwd(d, X, tg, logp, None, None, None, stats)
    for dent in (None, E):
        bwd, alone1 = _gradient(n, V, V + more, dtype)
        step, alone2 = _gradient(n, V, V + more, dtype)
        cola.cola_token_logprob_bwd(d, X, tg, stats, G, dent, bwd)
        cola.cola_token_logprob_step(d, X, tg, G, dent, logp, ent, step)
        assert alone1() and alone2()
        a, b = H.host(bwd), H.host(step)
        for i in range(n):
            hi = float(h[i]) if dent is not None else 0.0
            r = H.logprob_row(x[i], t[i], T, float(g[i]), hi)
            for got in (a[i], b[i]):
                H.check_logprob_grad(got, r, t[i], float(g[i]), hi, T, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("more", MORE)
@pytest.mark.parametrize("n,V", SHAPES)
def test_distillation(n, V, more, dtype):
    rng = np.random.default_rng(V + more)
    k, T = 20, 1.5
    x = H.logits(rng, n, V, dtype)
    ids, vals, lse = H.teacher(rng, x, k, T)
    x[1, np.setdiff1d(np.arange(V), ids[1])[::2]] = -np.inf
    x[2, np.setdiff1d(np.arange(V), ids[2])] = float(torch.finfo(H.TORCH[dtype]).min)
    w = rng.standard_normal(n).astype(np.float32)
    X = H.place(x, dtype)
    f = lambda a, dt=torch.float32: torch.as_tensor(a, dtype=dt, device="cuda")   # noqa: E731
    I, U, W = f(ids, torch.int64), f(vals), f(w)
    loss, stats = torch.empty(n, device="cuda"), torch.empty((n, 4), device="cuda")
    for rest in (False, True):
        Z = f(lse) if rest else None
        d = cola.vocab_desc(n, V, ld=V, ld_grad=V + more, dtype=dtype, temperature=T, k=k, rest=rest, teacher_temperature=T)
        bwd, alone1 = _gradient(n, V, V + more, dtype)
        step, alone2 = _gradient(n, V, V + more, dtype)
        cola.cola_topk_distill_fwd(d, X, I, U, Z, loss, stats)
        cola.cola_topk_distill_bwd(d, X, I, U, Z, stats, W, bwd)
        cola.cola_topk_distill_step(d, X, I, U, Z, W, loss, step)
        assert alone1() and alone2()
        a, b = H.host(bwd), H.host(step)
        for i in range(n):
            r = H.distill_row(x[i], ids[i], vals[i].astype(np.float64), float(lse[i]) if rest else 0.0, T, T, rest, float(w[i]))
            for got in (a[i], b[i]):
                H.check_distill_grad(got, r, ids[i], float(w[i]), T, dtype)
