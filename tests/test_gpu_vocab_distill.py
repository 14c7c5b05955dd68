"""Distillation from a teacher's top logits and its gradient against the 64-bit
definition, both ways of counting the teacher's mass, at the sizes, lists,
masks and layouts where they can go wrong."""
import numpy as np
import pytest
import torch

import vocab_helpers as H
from paper_2502_10940_gb300 import cola

pytestmark = pytest.mark.gpu


def compare(x, ids, vals, lse, dtype, T, Tt, rest, w, layout="dense"):
    n, V = x.shape
    o = H.run_distill(x, ids, vals, lse, dtype, T, Tt, rest, w, layout)
    for i in range(n):
        wi = float(np.float32(w[i]))
        r = H.distill_row(x[i], ids[i], vals[i].astype(np.float64), 0.0 if lse is None else float(lse[i]), T, Tt, rest, wi)
        for key in ("loss", "loss2"):
            H.check(key, o[key][i:i + 1], [r["loss"]], H.loss_tol(np.array([r["loss"]]), T))
        for key in ("bwd", "step"):
            H.check_distill_grad(o[key][i], r, ids[i], wi, T, dtype)
    return o


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,V,k", [(1, 1, 1), (2, 2, 1), (3, 9, 9), (4, 300, 7), (2, 300, 256), (3, 4099, 33), (2, 33001, 64),
                                   (1, 131072, 128), (2, 200003, 1)])
def test_sizes(n, V, k, dtype, rest):
    rng = np.random.default_rng(V + k)
    x = H.logits(rng, n, V, dtype)
    ids, vals, lse = H.teacher(rng, x, k, 2.0)
    compare(x, ids, vals, lse if rest else None, dtype, 2.0, 2.0, rest, rng.standard_normal(n))


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["padded", "odd", "shifted"])
@pytest.mark.parametrize("V", [33, 5003, 70001])
def test_layouts(V, layout, dtype, rest):
    rng = np.random.default_rng(V)
    x = H.logits(rng, 3, V, dtype)
    ids, vals, lse = H.teacher(rng, x, 17, 1.0)
    compare(x, ids, vals, lse if rest else None, dtype, 1.0, 1.0, rest, rng.standard_normal(3), layout)


@pytest.mark.parametrize("rest", [False, True])
def test_lists(rest):
    """Absent entries, an empty list, ids outside the vocabulary, entries of
    probability 0, first and last tokens, lists in any order."""
    rng = np.random.default_rng(2)
    n, V, k = 7, 3001, 12
    x = H.logits(rng, n, V, "f32")
    ids, vals, lse = H.teacher(rng, x, k, 1.0)
    ids[0, 5:] = -1
    ids[1, :] = -1
    ids[2, ::2] = V + np.arange(6) * 1000
    ids[3, 3] = 2 ** 40
    vals[4, 6:] = -np.inf
    vals[5, :] = -np.inf
    keep = rng.permutation(k)
    ids[6], vals[6] = ids[6, keep], vals[6, keep]
    ids[6, 0], ids[6, 1] = 0, V - 1
    compare(x, ids, vals, lse if rest else None, "f32", 1.0, 1.0, rest, rng.standard_normal(n))


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [40, 6007, 50021])
def test_masks(V, dtype, rest):
    rng = np.random.default_rng(V)
    low = float(torch.finfo(H.TORCH[dtype]).min)
    n, k = 7, 8
    x = H.logits(rng, n, V, dtype)
    ids, vals, lse = H.teacher(rng, x, k, 1.0)
    outside = [np.setdiff1d(np.arange(V), ids[i]) for i in range(n)]
    x[0, outside[0][::2]] = -np.inf              # half of the rest banned
    x[1, outside[1]] = -np.inf                   # all of the rest banned: it is left out
    x[2, ids[2, 3]] = -np.inf                    # the student bans a token of the list: infinite loss
    x[3, :] = -np.inf                            # the student bans everything
    x[4, outside[4]] = low                       # the rest at the type's lowest value
    x[5, :] = low
    x[6, outside[6][::3]] = low
    compare(x, ids, vals, lse if rest else None, dtype, 1.0, 1.0, rest, np.ones(n))


@pytest.mark.parametrize("rest", [False, True])
def test_not_finite_and_zero_weights(rest):
    rng = np.random.default_rng(4)
    n, V, k = 6, 2003, 6
    x = H.logits(rng, n, V, "f32")
    ids, vals, lse = H.teacher(rng, x, k, 1.0)
    out = np.setdiff1d(np.arange(V), ids)[7]
    x[0, ids[0, 2]] = np.nan
    x[1, out] = np.nan
    x[2, out] = np.inf
    x[3, ids[3, 0]] = np.inf
    x[4, out] = np.nan                           # weight 0: no gradient whatever the row holds
    w = np.array([1.0, 1.0, 1.0, 1.0, 0.0, 0.0])
    o = compare(x, ids, vals, lse if rest else None, "f32", 1.0, 1.0, rest, w)
    assert not o["step"][4:].any() and not o["bwd"][4:].any()


def test_confident_and_close_students():
    """The rest's probability down to 1e-30 and losses down to 1e-6 keep their
    digits: neither 1 - sum p nor terms that cancel are formed."""
    rng = np.random.default_rng(9)
    n, V, k = 4, 5003, 4
    x = rng.standard_normal((n, V)) * 0.5
    x[:, :k] += np.array([5.0, 20.0, 40.0, 70.0])[:, None]
    x = H.rounded(x, "f32")
    ids = np.tile(np.arange(k), (n, 1))
    vals = (x[:, :k] + rng.standard_normal((n, k)) * 1e-2).astype(np.float32)
    z = x.copy()
    z[:, :k] = vals
    lse = np.array([sum(H.softmax_stats(z[i])[:2]) for i in range(n)], np.float32)
    o = H.run_distill(x, ids, vals, lse, "f32", 1.0, 1.0, True, np.ones(n))
    for i in range(n):
        r = H.distill_row(x[i], ids[i], vals[i].astype(np.float64), float(lse[i]), 1.0, 1.0, True, 1.0)
        # sum q is off by 1e-6 (the exponents' and lse's rounding), the ratio q / p by 3e-6 of itself
        assert abs(o["loss"][i] - r["loss"]) <= 2e-6 + 2e-3 * r["loss"], (i, o["loss"][i], r["loss"])


def test_top_alternatives_feed_the_distillation():
    """The forward over a teacher's logits gives the list, both ways."""
    rng = np.random.default_rng(10)
    n, V, k, T = 5, 9001, 20, 2.0
    t, x = H.logits(rng, n, V, "bf16"), H.logits(rng, n, V, "bf16")
    Tt = H.place(t, "bf16")
    d = cola.vocab_desc(n, V, temperature=T, k=k)
    ids, lp = torch.empty((n, k), dtype=torch.int64, device="cuda"), torch.empty((n, k), device="cuda")
    cola.cola_token_logprob_fwd(d, Tt, None, None, None, ids, lp, None)
    for rest in (False, True):
        compare(x, ids.cpu().numpy(), lp.cpu().numpy(), None, "bf16", T, 1.0, rest, np.ones(n))


@pytest.mark.parametrize("rest", [False, True])
def test_gradient_against_differences(rest):
    """Central differences of the 64-bit loss (as for the log probabilities)."""
    rng = np.random.default_rng(11)
    V, k, T, e = 37, 5, 2.0, 1e-5
    x = H.logits(rng, 1, V, "f32")
    ids, vals, lse = H.teacher(rng, x, k, T)
    w = 0.75
    o = H.run_distill(x, ids, vals, lse if rest else None, "f32", T, T, rest, [w])

    def f(v):
        return w * H.distill_row(v, ids[0], vals[0].astype(np.float64), float(lse[0]), T, T, rest)["loss"]

    for j in range(V):
        a, b = x[0].copy(), x[0].copy()
        a[j] += e
        b[j] -= e
        num = (f(a) - f(b)) / (2 * e)
        for key in ("bwd", "step"):
            assert abs(o[key][0, j] - num) <= 3e-5 * abs(num) + 4e-5, (j, o[key][0, j], num)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [777, 20000, 90001])
def test_in_place_repeats_and_streams(V, dtype):
    rng = np.random.default_rng(V)
    n, k = 40, 30
    x = H.logits(rng, n, V, dtype)
    ids, vals, lse = H.teacher(rng, x, k, 1.0)
    X = H.place(x, dtype)
    I, U, L = torch.as_tensor(ids, device="cuda"), torch.as_tensor(vals, device="cuda"), torch.as_tensor(lse, device="cuda")
    w = torch.randn(n, device="cuda")
    d = cola.vocab_desc(n, V, dtype=dtype, k=k, rest=True)
    loss, stats, out, out2 = torch.empty(n, device="cuda"), torch.empty((n, 4), device="cuda"), torch.empty_like(X), torch.empty_like(X)
    cola.cola_topk_distill_step(d, X, I, U, L, w, loss, out)
    loss1 = loss.clone()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        cola.cola_topk_distill_step(d, X, I, U, L, w, loss, out2)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(out, out2) and torch.equal(loss, loss1)
    Y = X.clone()
    cola.cola_topk_distill_step(d, Y, I, U, L, w, loss, Y)
    assert torch.equal(out, Y) and torch.equal(loss, loss1)
    cola.cola_topk_distill_fwd(d, X, I, U, L, loss, stats)
    cola.cola_topk_distill_bwd(d, X, I, U, L, stats, w, out)
    cola.cola_topk_distill_bwd(d, X, I, U, L, stats, w, X)
    assert torch.equal(X, out)


def test_trace():
    X, I, U = torch.randn((2, 100), device="cuda"), torch.zeros((2, 1), dtype=torch.int64, device="cuda"), torch.zeros((2, 1), device="cuda")
    loss = torch.empty(2, device="cuda")
    with cola.Trace(4) as tr:
        cola.cola_topk_distill_fwd(cola.vocab_desc(2, 100, dtype="f32", k=1), X, I, U, None, loss, None)
    assert [r[0] for r in tr.records()] == ["topk_distill"]
    ref = -torch.log_softmax(X.double(), 1)[:, 0]
    assert (loss.double() - ref).abs().max().item() <= 2e-5


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_largest_vocabulary(dtype, rest):
    rng = np.random.default_rng(13)
    V = 1 << 20
    x = H.logits(rng, 1, V, dtype)
    ids, vals, lse = H.teacher(rng, x, 256, 1.0)
    compare(x, ids, vals, lse if rest else None, dtype, 1.0, 1.0, rest, [0.5])


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,V,k", [(2600, 700, 200), (2600, 700, 9), (1500, 5003, 64), (1300, 20011, 40), (40, 600, 200)])
def test_many_rows(n, V, k, dtype, rest):
    """More rows than CTAs run at once, by the definition on the GPU in 64 bits."""
    g = torch.Generator(device="cuda")
    g.manual_seed(n + V + k)
    T = 1.5
    x = (torch.randn((n, V), generator=g, device="cuda") * 2).to(H.TORCH[dtype])
    t = x.float() * 0.9 + torch.randn((n, V), generator=g, device="cuda")
    top = torch.topk(t, k, dim=1)
    ids, vals = top.indices.contiguous(), top.values.contiguous()
    lse = torch.logsumexp(t / T, 1) if rest else None
    w = torch.randn(n, generator=g, device="cuda")
    d = cola.vocab_desc(n, V, dtype=dtype, temperature=T, k=k, rest=rest, teacher_temperature=T)
    loss, loss2, stats, dx, dx2 = (torch.full(s, float("nan"), device="cuda") for s in ((n,), (n,), (n, 4), (n, V), (n, V)))
    dx, dx2 = dx.to(x.dtype), dx2.to(x.dtype)
    cola.cola_topk_distill_fwd(d, x, ids, vals, lse, loss, stats)
    cola.cola_topk_distill_bwd(d, x, ids, vals, lse, stats, w, dx)
    cola.cola_topk_distill_step(d, x, ids, vals, lse, w, loss2, dx2)
    assert torch.equal(loss, loss2)
    lp = torch.log_softmax(x.double() / T, 1)
    u = vals.double() / T
    q = (u - lse.double()[:, None]).exp() if rest else torch.softmax(u, 1)
    logq = u - lse.double()[:, None] if rest else torch.log_softmax(u, 1)
    out = torch.ones_like(lp).scatter_(1, ids, 0.0)
    kl = (q * (logq - lp.gather(1, ids))).sum(1)
    want = torch.zeros_like(lp).scatter_(1, ids, q)
    lpr = torch.logsumexp(torch.where(out > 0, lp, -torch.inf), 1)
    r = (lp - lpr[:, None]).exp() * out
    if rest:
        qr = (1 - q.sum(1)).clamp(min=0.0)
        kl = kl + torch.where(qr > 0, qr * (qr.clamp(min=1e-300).log() - lpr), 0.0)
        want = want + qr[:, None] * r
    ref = w.double()[:, None] * T * (want.sum(1, keepdim=True) * lp.exp() - want)
    ref_loss = T * T * kl
    assert bool(((loss.double() - ref_loss).abs() <= T * T * 2e-5 + 1e-5 * ref_loss.abs()).all())
    # as in check_distill_grad
    tol = w.double().abs()[:, None] * T * (4e-6 * r + 2e-5 * (1 - out)) + (2e-5 + (2.0 ** -8 if dtype == "bf16" else 0.0)) * ref.abs() + 1e-37
    for got in (dx, dx2):
        assert bool(((got.double() - ref).abs() <= tol).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["dense", "odd", "shifted"])
@pytest.mark.parametrize("V,k,rest", [(5003, 200, True), (9001, 40, True), (19003, 90, False)])
def test_many_rows_of_middle_length(V, k, rest, layout, dtype):
    """Rows of several tiles of one CTA of four warps, masks among them."""
    rng = np.random.default_rng(V + k)
    n = 640
    x = H.logits(rng, n, V, dtype)
    ids, vals, lse = H.teacher(rng, x, k, 1.5)
    x[3, V // 2:] = -np.inf
    x[4] = -np.inf
    x[5, : V // 2] = float(torch.finfo(H.TORCH[dtype]).min)
    w = rng.standard_normal(n)
    w[9] = 0.0
    compare(x, ids, vals, lse if rest else None, dtype, 1.5, 1.5, rest, w, layout)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [300, 3001, 40007])
def test_listed_tokens_that_only_the_student_finds_likely(V, dtype):
    """Teacher's probabilities down to the least above 0 and beyond, the rest
    counted: such an entry costs the student's probability and no more."""
    rng = np.random.default_rng(V)
    unlikely = np.array([-80.0, -85.0, -87.5, -90.0, -100.0, -102.5, -103.5, -110.0])
    n, k = len(unlikely) + 1, 3
    x = H.rounded(rng.standard_normal((n, V)), dtype)
    ids = np.tile(np.array([V // 3, V - 1, 0]), (n, 1))
    x[:, ids[0, 0]] = 14.0                                           # nearly all of the student's probability
    x[:, ids[0, 1]] = np.linspace(4.0, 12.0, n)
    vals = np.tile(np.array([0.0, -30.0, -1.0], np.float32), (n, 1))
    vals[:-1, 0] = unlikely
    vals[-1] = -100.0                                                # a padded list
    compare(H.rounded(x, dtype), ids, vals, np.zeros(n, np.float32), dtype, 1.0, 1.0, True, np.ones(n))


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("dtype,n,V,k", [("bf16", 1300, 32000, 64), ("bf16", 700, 21000, 200), ("f32", 700, 11000, 200),
                                         ("bf16", 300, 200000, 40)])
def test_losses_of_passes_that_share_rows_differently(dtype, n, V, k, rest):
    """Rows that the forward and the step give to other numbers of threads or
    CTAs: sums in another order, so losses within the tolerance of one another and
    of the definition (where rows are shared alike they are the same bits:
    test_many_rows)."""
    g = torch.Generator(device="cuda")
    g.manual_seed(n + V + k)
    T = 1.5
    x = (torch.randn((n, V), generator=g, device="cuda") * 2).to(H.TORCH[dtype])
    t = x.float() * 0.9 + torch.randn((n, V), generator=g, device="cuda")
    top = torch.topk(t, k, dim=1)
    ids, vals = top.indices.contiguous(), top.values.contiguous()
    lse = torch.logsumexp(t / T, 1) if rest else None
    w = torch.randn(n, generator=g, device="cuda")
    d = cola.vocab_desc(n, V, dtype=dtype, temperature=T, k=k, rest=rest, teacher_temperature=T)
    loss, loss2, dx = torch.empty(n, device="cuda"), torch.empty(n, device="cuda"), torch.empty_like(x)
    cola.cola_topk_distill_fwd(d, x, ids, vals, lse, loss, None)
    cola.cola_topk_distill_step(d, x, ids, vals, lse, w, loss2, dx)
    u = vals.double() / T
    logq = u - lse.double()[:, None] if rest else torch.log_softmax(u, 1)
    q = logq.exp()
    for i in range(0, n, 100):
        s = slice(i, min(n, i + 100))
        lp = torch.log_softmax(x[s].double() / T, 1)
        ref = (q[s] * (logq[s] - lp.gather(1, ids[s]))).sum(1)
        if rest:
            qr = (1 - q[s].sum(1)).clamp(min=0.0)
            ref += qr * (qr.clamp(min=1e-300).log() - torch.logsumexp(lp.scatter(1, ids[s], -torch.inf), 1))
        ref *= T * T
        tol = T * T * 2e-5 + 1e-5 * ref.abs()   # H.loss_tol
        for a in (loss[s].double(), loss2[s].double()):
            assert bool(((a - ref).abs() <= tol).all())
        assert bool(((loss[s].double() - loss2[s].double()).abs() <= tol).all())
