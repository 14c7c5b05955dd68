"""Log probabilities of given tokens, entropy, top alternatives and their
gradients against the 64-bit definitions, where they can go wrong: small, odd
and large vocabularies, pitches and offsets that leave rows unaligned, masks,
ties, values that are not finite, in-place gradients, other streams and graphs."""
import numpy as np
import pytest
import torch

import vocab_helpers as H
from paper_2502_10940_gb300 import cola

pytestmark = pytest.mark.gpu


def compare(x, targets, dtype, T, k, g, h, layout="dense"):
    n, V = x.shape
    o = H.run_logprob(x, targets, dtype, T, k, g, h, layout)
    for i in range(n):
        gi, hi = float(np.float32(g[i])) if g is not None else 0.0, float(np.float32(h[i])) if h is not None else 0.0
        r = H.logprob_row(x[i], targets[i], T, gi, hi, k)
        for key in ("logp", "logp2"):
            if key in o:
                H.check(key, o[key][i:i + 1], [r["logp"]], H.logp_tol(np.array([r["logp"]])))
        for key in ("entropy", "entropy2"):
            if key in o:
                H.check(key, o[key][i:i + 1], [r["entropy"]], 1e-5 + 1e-5 * abs(np.nan_to_num(r["entropy"])))
        if k:
            assert np.array_equal(o["top_ids"][i], r["top_ids"]), (i, o["top_ids"][i], r["top_ids"])
            H.check("top_logp", o["top_logp"][i], r["top_logp"], H.logp_tol(r["top_logp"]))
        for key in ("bwd", "step"):
            if key in o:
                H.check_logprob_grad(o[key][i], r, targets[i], gi if 0 <= targets[i] < V else 0.0, hi, T, dtype)
    return o


SIZES = [(1, 1), (3, 2), (4, 7), (2, 31), (5, 257), (3, 1000), (2, 4099), (2, 33001), (1, 131072), (2, 200003)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,V", SIZES)
def test_sizes(n, V, dtype):
    rng = np.random.default_rng(n * 1000 + V)
    x = H.logits(rng, n, V, dtype)
    t = rng.integers(0, V, n)
    compare(x, t, dtype, 0.75, min(V, 20), rng.standard_normal(n), rng.standard_normal(n))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["padded", "odd", "shifted"])
@pytest.mark.parametrize("V", [5, 517, 5003, 70001])
def test_layouts(V, layout, dtype):
    rng = np.random.default_rng(V)
    x = H.logits(rng, 4, V, dtype)
    t = np.array([0, V - 1, V // 2, 1])
    compare(x, t, dtype, 2.0, min(V, 5), rng.standard_normal(4), None, layout)
    compare(x, t, dtype, 2.0, 0, None, rng.standard_normal(4), layout)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [37, 3001, 40007])
def test_masks(V, dtype):
    rng = np.random.default_rng(V)
    low = float(torch.finfo(H.TORCH[dtype]).min)
    x = H.logits(rng, 9, V, dtype)
    x[0, rng.random(V) < 0.5] = -np.inf          # half banned
    x[1, :] = -np.inf                            # everything banned
    x[2, :] = -np.inf
    x[2, V // 3] = 1.5                           # one token left
    x[3, rng.random(V) < 0.5] = low              # masked by the type's lowest value
    x[4, :] = low                                # all of them: uniform
    x[5, :-1] = low                              # one left beside lowest values
    x[6, : V // 2] = -np.inf
    x[6, V // 2:] = low
    x[7, 0] = -np.inf
    x[8, -1] = -np.inf
    t = np.array([int(np.flatnonzero(np.isfinite(x[0]))[0]), 2, V // 3, 5, 7, V - 1, V - 2, 0, V - 1])
    k = min(V, 30)
    for T in (0.5, 1.0, 3.0):
        compare(x, t, dtype, T, k, rng.standard_normal(9), rng.standard_normal(9))


def test_targets_outside_the_vocabulary_and_zero_weights():
    rng = np.random.default_rng(3)
    n, V = 6, 1001
    x = H.logits(rng, n, V, "f32")
    x[4, 5] = np.nan                             # ignored row: gradient 0 although it holds a NaN
    x[5, 5] = np.inf
    t = np.array([-100, V, -1, 2 ** 40, -100, 3])
    g = np.array([1.0, 1.0, 1.0, 1.0, 1.0, 0.0])
    o = compare(x, t, "f32", 1.0, 3, g, None)
    assert not o["step"].any() and not o["bwd"].any() and not o["logp"][:5].any()
    assert np.isnan(o["logp"][5])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [9, 2003, 40007])
def test_not_finite(V, dtype):
    rng = np.random.default_rng(V)
    x = H.logits(rng, 5, V, dtype)
    x[0, V // 2] = np.nan
    x[1, :] = np.nan
    x[2, 1] = np.inf
    x[3, 0] = np.nan
    x[3, V - 1] = np.nan
    x[3, 2] = np.inf
    x[4, 3:] = -np.inf
    x[4, 1] = np.nan
    compare(x, np.array([0, 1, 1, 4, 2]), dtype, 1.0, min(V, 8), np.ones(5), np.ones(5))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("k", [1, 2, 17, 64, 255, 256])
@pytest.mark.parametrize("V", [256, 1500, 33001, 150001])
def test_top_orders(V, k, dtype):
    """Orders in which the largest are not spread evenly, and ties."""
    rng = np.random.default_rng(V + k)
    j = np.arange(V)
    rows = [np.zeros(V),                                             # every token alike
            -j / 64.0, j / 64.0,                                     # falling, rising
            np.where(j % 4096 < 8, 5.0 + j / 1e4, -1.0),             # the largest in the same few columns
            np.where(j < V // 2, 1.0, 2.0),                          # half of them tied for the top
            np.round(rng.standard_normal(V) * 4) / 4,                # many ties
            np.where(rng.random(V) < 0.5, 0.0, -0.0),                # both zeros
            np.where(j == V - 1, 3.0, -np.inf),
            rng.permutation(V) / 100.0]
    x = H.rounded(np.stack(rows), dtype)
    compare(x, np.arange(len(rows)), dtype, 1.0, k, None, None)


@pytest.mark.parametrize("T", [1e-4, 0.01, 1.0, 50.0, 1e4])
def test_temperatures(T):
    rng = np.random.default_rng(5)
    # values whose scaled rounding stays within the tolerance: z = x / T of a few units
    x = H.rounded(rng.standard_normal((3, 2001)) * 3 * T, "f32")
    compare(x, rng.integers(0, 2001, 3), "f32", float(np.float32(T)), 4, rng.standard_normal(3) * T, rng.standard_normal(3) * T)


def test_large_logits():
    """Logits far from 0 lose nothing: only their distances enter."""
    rng = np.random.default_rng(6)
    x = H.rounded(rng.standard_normal((2, 3001)) + 60000.0, "f32")
    compare(x, [5, 6], "f32", 1.0, 10, [1.0, 2.0], [0.5, 0.1])


def test_rows_past_32_bit_offsets():
    rng = np.random.default_rng(7)
    V, pitch, n = 5000, (1 << 30) + 8, 3
    x = H.logits(rng, n, V, "bf16")
    buf = torch.empty(2 * pitch + V, dtype=torch.bfloat16, device="cuda")
    X = torch.as_strided(buf, (n, V), (pitch, 1))
    X.copy_(torch.from_numpy(x))
    t = torch.tensor([1, 2, 3], device="cuda")
    g = torch.tensor([1.0, 1.0, 1.0], device="cuda")
    logp, ids, lp = torch.empty(n, device="cuda"), torch.empty((n, 4), dtype=torch.int64, device="cuda"), torch.empty((n, 4), device="cuda")
    d = cola.vocab_desc(n, V, ld=pitch, ld_grad=pitch, k=4)
    cola.cola_token_logprob_fwd(d, X, t, logp, None, ids, lp, None)
    cola.cola_token_logprob_step(d, X, t, g, None, logp, None, X)
    for i in range(n):
        r = H.logprob_row(x[i], i + 1, 1.0, 1.0, 0.0, 4)
        assert np.array_equal(ids[i].cpu().numpy(), r["top_ids"])
        H.check("logp", [logp[i].item()], [r["logp"]], 1e-5 + 1e-6 * abs(r["logp"]))
        H.check_logprob_grad(H.host(X[i]), r, i + 1, 1.0, 0.0, 1.0, "bf16")


@pytest.mark.parametrize("V", [777, 20000, 90001])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_in_place(V, dtype):
    rng = np.random.default_rng(V)
    n = 7
    x = H.logits(rng, n, V, dtype)
    X, t = H.place(x, dtype), torch.as_tensor(rng.integers(0, V, n), device="cuda")
    g, h = torch.randn(n, device="cuda"), torch.randn(n, device="cuda")
    d = cola.vocab_desc(n, V, dtype=dtype, temperature=1.5)
    logp, ent, stats, out = torch.empty(n, device="cuda"), torch.empty(n, device="cuda"), torch.empty((n, 4), device="cuda"), torch.empty_like(X)
    cola.cola_token_logprob_step(d, X, t, g, h, logp, ent, out)
    logp1 = logp.clone()
    Y = H.place(x, dtype)
    cola.cola_token_logprob_step(d, Y, t, g, h, logp, ent, Y)
    assert torch.equal(Y, out) and torch.equal(logp, logp1)
    cola.cola_token_logprob_fwd(d, X, t, logp, None, None, None, stats)
    cola.cola_token_logprob_bwd(d, X, t, stats, g, h, out)
    cola.cola_token_logprob_bwd(d, X, t, stats, g, h, X)
    assert torch.equal(X, out)


def test_gradient_against_differences():
    """The gradient of sum g logp + h H against central differences of the
    64-bit definition: step 1e-5, error 1e-10 / 6 times a third derivative of at
    most 10, and 1e-16 / 1e-5 of rounding, far below the gradient's tolerance."""
    rng = np.random.default_rng(8)
    V, T, e = 41, 1.3, 1e-5
    T = float(np.float32(T))
    x = H.logits(rng, 1, V, "f32")
    g, h, y = 0.7, -0.4, 11
    g, h = float(np.float32(g)), float(np.float32(h))
    o = H.run_logprob(x, [y], "f32", T, 0, [g], [h])

    def f(v):
        r = H.logprob_row(v, y, T)
        return g * r["logp"] + h * r["entropy"]

    for j in range(V):
        a, b = x[0].copy(), x[0].copy()
        a[j] += e
        b[j] -= e
        num = (f(a) - f(b)) / (2 * e)
        for key in ("bwd", "step"):
            assert abs(o[key][0, j] - num) <= 2e-5 * abs(num) + 4e-6, (j, o[key][0, j], num)


def test_many_rows_streams_graphs_and_repeats():
    """More rows than CTAs run at once; another stream; a replayed graph; the
    same bits every time."""
    n, V, k = 3001, 3203, 12
    X = torch.randn((n, V), device="cuda").to(torch.bfloat16)
    t = torch.randint(0, V, (n,), device="cuda")
    d = cola.vocab_desc(n, V, k=k)
    outs = []

    def call():
        o = (torch.empty(n, device="cuda"), torch.empty(n, device="cuda"), torch.empty((n, k), dtype=torch.int64, device="cuda"),
             torch.empty((n, k), device="cuda"))
        cola.cola_token_logprob_fwd(d, X, t, o[0], o[1], o[2], o[3], None)
        return o

    outs.append(call())
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        outs.append(call())
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs.append(call())
    graph.replay()
    torch.cuda.synchronize()
    for o in outs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(o, outs[0]))
    z = X.double()
    lp = z - torch.logsumexp(z, 1, keepdim=True)
    assert (outs[0][0].double() - lp.gather(1, t[:, None])[:, 0]).abs().max().item() <= 1e-5 + 1e-6 * 20
    best = torch.sort(z, dim=1, descending=True, stable=True).indices[:, :k]
    assert torch.equal(outs[0][2], best)


def test_optional_outputs_and_trace():
    V = 1000
    X = torch.randn((2, V), device="cuda")
    d = cola.vocab_desc(2, V, dtype="f32")
    ent = torch.empty(2, device="cuda")
    with cola.Trace(4) as tr:
        cola.cola_token_logprob_fwd(d, X, None, None, ent, None, None, None)
    assert [r[0] for r in tr.records()] == ["token_logprob"]
    p = torch.softmax(X.double(), 1)
    assert (ent.double() + (p * p.log()).sum(1)).abs().max().item() <= 1e-4


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V,k", [(8200, 1), (9001, 20), (20011, 64), (33000, 128), (40009, 7)])
def test_many_long_rows(V, k, dtype):
    """Rows enough for the kernel that ranks one row while it reads the next,
    every awkward order and mask among them."""
    g = torch.Generator(device="cuda")
    g.manual_seed(V + k)
    n = 2500
    low = torch.finfo(H.TORCH[dtype]).min
    x = torch.randn((n, V), generator=g, device="cuda") * 3
    j = torch.arange(V, device="cuda", dtype=torch.float32)
    special = [torch.zeros(V, device="cuda"), -j / 64, j / 64, torch.where(j % 4096 < 8, 5 + j / 1e4, -1.0),
               torch.where(j < V // 2, 1.0, 2.0), torch.round(x[0]), torch.full((V,), -torch.inf, device="cuda"),
               torch.where(j == V - 1, 3.0, -torch.inf), torch.where(j % 997 == 5, x[1], -torch.inf),
               torch.full((V,), low, device="cuda"), torch.where(j < 3, x[2], low), torch.where(j < V - 2, -torch.inf, low),
               torch.where(j % 2 == 0, 1.5, x[3].clamp(max=1.0)), torch.where(j % 50 == 0, 4.0, 0.0)]
    for i, row in enumerate(special):
        x[100 + 37 * i] = row
    x = x.to(H.TORCH[dtype])
    bad = [7, 1999, 2480]
    x[bad[0], V // 2] = torch.nan
    x[bad[1], :] = torch.nan
    x[bad[2], 11] = torch.inf
    t = torch.randint(0, V, (n,), generator=g, device="cuda")
    d = cola.vocab_desc(n, V, dtype=dtype, temperature=0.75, k=k)
    f = lambda *s: torch.full(s, -7.0, device="cuda")   # noqa: E731
    logp, ent, top, stats = f(n), f(n), f(n, k), f(n, 4)
    ids = torch.full((n, k), -7, dtype=torch.int64, device="cuda")
    cola.cola_token_logprob_fwd(d, x, t, logp, ent, ids, top, stats)
    z = x.double()
    order = torch.where(torch.isnan(z), torch.inf, z)   # the one row with both holds its NaN alone
    best = torch.sort(order, dim=1, descending=True, stable=True).indices[:, :k]
    assert torch.equal(ids, best)
    m = z.amax(1, keepdim=True)
    m = torch.where(m == -torch.inf, 0.0, m)
    w = (z - m) / 0.75
    s = w.exp().sum(1, keepdim=True)
    logs = torch.where(s == 0, 0.0, s.log())
    lp = w - logs
    p = lp.exp()
    H_ref = -torch.where(p == 0, 0.0, p * lp).sum(1)

    def near(a, b, tol):
        b = torch.where(b.float().isinf(), b.float().double(), b)
        assert torch.equal(torch.isnan(a), torch.isnan(b)) and torch.equal(torch.isinf(a), torch.isinf(b))
        ok = torch.isfinite(b)
        assert bool(((a[ok].double() - b[ok]).abs() <= 1e-5 + tol * b[ok].abs()).all())

    near(logp, lp.gather(1, t[:, None])[:, 0], 1e-6)
    near(top, lp.gather(1, best), 1e-6)
    near(ent, torch.where(s[:, 0] == 0, 0.0, H_ref), 1e-5)
    again = torch.empty_like(top)
    cola.cola_token_logprob_fwd(d, x, t, logp, None, ids, again, None)
    assert torch.equal(again.nan_to_num(5.0), top.nan_to_num(5.0)) and torch.equal(ids, best)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_largest_vocabulary(dtype):
    rng = np.random.default_rng(12)
    V = 1 << 20
    x = H.logits(rng, 2, V, dtype)
    compare(x, [3, V - 1], dtype, 1.0, 256, [1.0, -0.5], [0.25, 0.5])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V,k", [(250, 250), (640, 17), (1000, 200), (2290, 149), (3333, 256)])
def test_many_short_rows_with_long_lists(V, k, dtype):
    """k near or beyond the threads that hold a row, ties and masks among them."""
    rng = np.random.default_rng(V + k)
    x = H.logits(rng, 300, V, dtype)
    x[7] = 0.0
    x[8, k:] = -np.inf
    x[9, 3:] = -np.inf
    x[10] = np.round(x[10])
    x[11] = np.arange(V) / 64.0
    x[12, V // 2] = np.nan
    x[13, : k + 1] = np.nan
    x[14] = np.where(np.arange(V) % 3 == 0, 1.0, -np.inf)
    x = H.rounded(x, dtype)
    compare(x, rng.integers(0, V, 300), dtype, 1.5, k, None, None)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V,k", [(600, 20), (1500, 40), (2003, 100), (5003, 20), (5003, 100), (7001, 256), (20011, 100), (33001, 5)])
def test_order_around_zero(V, k, dtype):
    """Subnormal logits of both signs, beside zeros of both."""
    rng = np.random.default_rng(V + k)
    unit = 2.0 ** (-133 if dtype == "bf16" else -149)                # the least above 0
    few = np.zeros(V)
    few[rng.permutation(V)[: k // 2]] = 1.0
    rows = [rng.integers(-100, 100, V), -rng.integers(1, 120, V), rng.integers(-120, 3, V), few - rng.integers(1, 90, V) * (few == 0),
            2 * few - 3]
    if dtype == "f32":
        rows += [-rng.integers(1, 0x10000, V), rng.integers(-0x30000, 0x100, V), -rng.integers(0x7000, 0x18000, V)]
    x = np.stack(rows).astype(np.float64) * unit
    x[0, ::5] = -0.0
    compare(x, np.arange(len(rows)), dtype, 1.0, k, None, None)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["dense", "odd", "shifted"])
@pytest.mark.parametrize("V", [5003, 9001, 19003])
def test_many_rows_of_middle_length(V, layout, dtype):
    """Rows of several tiles of one CTA of four warps, masks among them, with gradients."""
    rng = np.random.default_rng(V)
    n = 640
    x = H.logits(rng, n, V, dtype)
    x[3, V // 2:] = -np.inf
    x[4] = -np.inf
    x[5, : V // 2] = float(torch.finfo(H.TORCH[dtype]).min)
    t = rng.integers(0, V, n)
    t[3], t[8] = 7, -1
    g, h = rng.standard_normal(n), rng.standard_normal(n)
    g[9] = h[9] = 0.0
    compare(x, t, dtype, 1.5, 0, g, h, layout)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V,k", [(700, 100), (2003, 20), (2003, 200), (3500, 256), (5003, 64), (5003, 100), (8000, 256),
                                 (20011, 30), (33001, 200)])
def test_top_with_many_infinities(V, k, dtype):
    """More +inf than the list has entries, scattered, alone and beside NaNs:
    the bound stays where the infinities reach it."""
    rng = np.random.default_rng(V + k)
    count = [k, k + k // 8 + 2, k + k // 8 + 3, 2 * k, V // 2, V - 1, V]
    x = rng.standard_normal((2 * len(count) + 1, V))
    for i, c in enumerate(count):
        x[i, rng.permutation(V)[:c]] = np.inf
        x[len(count) + i] = x[i]
        x[len(count) + i, rng.permutation(V)[:3]] = np.nan
    x[-1, rng.permutation(V)[: 2 * k]] = np.nan
    x = H.rounded(x, dtype)
    compare(x, np.arange(len(x)), dtype, 1.0, k, None, None)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V,k", [(5003, 100), (3500, 256), (6007, 65), (5003, 30)])
def test_many_rows_of_a_few_thousand_tokens(V, k, dtype):
    """The same awkward rows where four warps hold a row."""
    test_many_long_rows(V, k, dtype)
