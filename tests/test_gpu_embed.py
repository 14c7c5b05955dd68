"""Token embedding and its gradient against the definitions in 64 bits, where
they can go wrong: one token and many, tables of one row and of the largest,
widths that end within eight columns, pitches, ids of no token, one token named
by all, workspaces full of old values, accumulated gradients, other streams and
graphs.

Tolerances (u = 2^-24): the lookup's product is rounded to fp32 and then to the
result's type, so u and, for bf16, 2^-8 of the value.  A sum of m rows takes m
additions at most, each off by u of a partial sum, which is at most the sum of
the absolute values; scaling takes one rounding more: (m + 2) u scale sum |dX|,
and the type's rounding; accumulated, one of the old value's magnitude.
"""
import numpy as np
import pytest
import torch

from paper_2502_10940_gb300 import cola

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF = {"bf16": 2.0 ** -8, "f32": U}   # half a step of the type, of the value


def pitch_of(d, pad):
    return (d + 7) // 8 * 8 + (64 if pad else 0)


def rows(x, dtype, pad=False, fill=float("nan")):
    """x on the GPU at a pitch that is a multiple of 8; the view and its buffer,
    whose other elements are `fill`.  (fp32: on 16-byte boundaries, and padded
    on no 32-byte ones.)"""
    n, d = x.shape
    ld = pitch_of(d, pad)
    buf = torch.full((n * ld + 16,), fill, dtype=TORCH[dtype], device="cuda")
    view = torch.as_strided(buf, (n, d), (ld, 1), 4 if pad and dtype == "f32" else 8)
    view.copy_(torch.as_tensor(x).to("cuda"))
    return view, buf


def untouched(view, buf):
    """Everything of the buffer outside the view is still NaN."""
    t = buf.clone()
    torch.as_strided(t, view.shape, view.stride(), view.storage_offset()).fill_(float("nan"))
    assert bool(torch.isnan(t).all())


def host(t):
    return t.double().cpu().numpy()


def tokens(rng, n, vocab, kind):
    if kind == "same":
        return np.full(n, vocab - 1)
    if kind == "none":
        return np.where(rng.random(n) < 0.5, -1, vocab)
    ids = np.minimum((rng.pareto(1.0, n) * 2).astype(np.int64), vocab - 1) if kind == "zipf" else rng.integers(0, vocab, n)
    if kind == "rising":
        ids = np.sort(ids)
    if n > 3:   # some of no token
        ids[rng.random(n) < 0.1] = rng.choice([-100, -1, vocab, 2 ** 40, -2 ** 40, 2 ** 32])
    return ids


def forward(ids, vocab, d, t_e, t_x, scale=1.0, pad=False):
    rng = np.random.default_rng(len(ids) + d)
    E, _ = rows(rng.standard_normal((vocab, d)), t_e, pad)
    X, buf = rows(np.full((len(ids), d), np.nan), t_x, pad)
    I = torch.as_tensor(ids, dtype=torch.int64, device="cuda")
    m = cola.embed_desc(len(ids), vocab, d, ld_e=E.stride(0), ld_x=X.stride(0), ld_de=pitch_of(d, pad), scale=scale,
                        dtype_e=t_e, dtype_x=t_x)
    cola.cola_embed_fwd(m, E, I, X)
    untouched(X, buf)
    there = (ids >= 0) & (ids < vocab)
    ref = np.where(there[:, None], host(E)[np.where(there, ids, 0)] * np.float32(scale).astype(np.float64), 0.0)
    assert (np.abs(host(X) - ref) <= (U + HALF[t_x]) * np.abs(ref)).all()
    assert not host(X)[~there].any()


def backward(ids, vocab, d, t_x, t_de, scale=1.0, pad=False, accumulate=False, seed=0, dX=None):
    rng = np.random.default_rng(seed + len(ids) + d)
    n = len(ids)
    dX, _ = rows(rng.standard_normal((n, d)) if dX is None else dX, t_x, pad)
    old = rng.standard_normal((vocab, d)).astype(np.float32) if accumulate else np.full((vocab, d), np.nan, np.float32)
    dE, buf = rows(old, t_de, pad)
    I = torch.as_tensor(ids, dtype=torch.int64, device="cuda")
    m = cola.embed_desc(n, vocab, d, ld_e=pitch_of(d, pad), ld_x=dX.stride(0), ld_de=dE.stride(0), scale=scale, dtype_x=t_x,
                        dtype_de=t_de, accumulate=accumulate)
    ws = cola.embed_workspace(m)
    ws[256:].fill_(0xff)
    cola.cola_embed_bwd(m, I, dX, dE, ws)
    first = dE.clone()
    untouched(dE, buf)
    dE.copy_(torch.as_tensor(old).to("cuda"))
    cola.cola_embed_bwd(m, I, dX, dE, ws)   # over its own leftovers: the same bits
    assert torch.equal(first, dE)
    there = (ids >= 0) & (ids < vocab)
    x = host(dX)[there]
    s = float(np.float32(scale))
    ref, mag, m_rows = np.zeros((vocab, d)), np.zeros((vocab, d)), np.zeros(vocab)
    np.add.at(ref, ids[there], x)
    np.add.at(mag, ids[there], np.abs(x))
    np.add.at(m_rows, ids[there], 1)
    ref *= s
    tol = (m_rows[:, None] + 2) * U * abs(s) * mag
    if accumulate:
        ref += old
        tol += U * (np.abs(old) + np.abs(ref)) * (m_rows[:, None] > 0)
    else:
        tol += HALF[t_de] * np.abs(ref) + HALF[t_de] * tol
    got = host(first)
    far = np.abs(got - ref) - tol
    assert far.max() <= 0, (far.max(), np.unravel_index(far.argmax(), far.shape))
    return first


TYPES = [("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32"), ("f32", "f32")]


@pytest.mark.parametrize("t_e,t_x", TYPES)
@pytest.mark.parametrize("n,vocab,d", [(1, 1, 1), (1, 5, 8), (2, 3, 7), (33, 1000, 100), (5, 50021, 2056), (300, 37, 513), (4097, 129, 64)])
def test_lookup(n, vocab, d, t_e, t_x):
    rng = np.random.default_rng(n)
    forward(tokens(rng, n, vocab, "uniform"), vocab, d, t_e, t_x)
    forward(tokens(rng, n, vocab, "zipf"), vocab, d, t_e, t_x, scale=d ** 0.5, pad=True)
    forward(tokens(rng, n, vocab, "none"), vocab, d, t_e, t_x)


@pytest.mark.parametrize("t_e,t_x", TYPES)
@pytest.mark.parametrize("pad", [False, True])
def test_lookup_of_many(pad, t_e, t_x):
    """An X of 75 to 150 MB, which is stored past L2."""
    forward(tokens(np.random.default_rng(7), 30011, 901, "zipf"), 901, 1251, t_e, t_x, scale=0.3, pad=pad)
    forward(tokens(np.random.default_rng(8), 30011, 901, "uniform"), 901, 1248, t_e, t_x, pad=pad)


@pytest.mark.parametrize("t_e,t_x", TYPES)
def test_lookup_copies_what_is_not_finite(t_e, t_x):
    E, _ = rows(np.array([[np.nan, np.inf, -np.inf, 0.0, -0.0, 1e-40, 3.0, 2.0], [1.0] * 8]), t_e)
    X, _ = rows(np.zeros((3, 8)), t_x)
    m = cola.embed_desc(3, 2, 8, scale=0.5, dtype_e=t_e, dtype_x=t_x, ld_x=X.stride(0), ld_e=E.stride(0))
    cola.cola_embed_fwd(m, E, torch.tensor([0, 1, -1], device="cuda"), X)
    ref = (E.float() * 0.5).to(TORCH[t_x])
    assert torch.equal(torch.nan_to_num(X[:2].float(), nan=7.0), torch.nan_to_num(ref.float(), nan=7.0))
    assert not X[2].any()


@pytest.mark.parametrize("t_x,t_de", TYPES)
@pytest.mark.parametrize("n,vocab,d", [(40, 3000, 64), (500, 20, 136), (9000, 700, 72)])
def test_gradient_padded(n, vocab, d, t_x, t_de):
    backward(tokens(np.random.default_rng(n), n, vocab, "zipf"), vocab, d, t_x, t_de, pad=True)


@pytest.mark.parametrize("t_x,t_de", TYPES)
@pytest.mark.parametrize("n,vocab,d", [(1, 1, 1), (1, 9, 8), (2, 2, 7), (7, 1000, 12), (33, 1000, 100), (255, 50021, 64), (300, 37, 513),
                                       (1025, 1024, 264), (4096, 1025, 64), (4097, 32000, 128)])
@pytest.mark.parametrize("kind", ["uniform", "zipf", "same", "none", "rising"])
def test_gradient(n, vocab, d, kind, t_x, t_de):
    rng = np.random.default_rng(n + vocab)
    backward(tokens(rng, n, vocab, kind), vocab, d, t_x, t_de)


@pytest.mark.parametrize("n,vocab,d,kind", [(40000, 32000, 72, "zipf"), (40000, 300, 40, "same"), (300001, 50021, 16, "zipf"),
                                            (300001, 50021, 9, "rising"), (70000, 1 << 20, 8, "uniform"), (5000, 1 << 20, 8, "zipf"),
                                            (20000, 700, 2056, "zipf"), (9000, 5, 8192, "uniform"), (8192, 40000, 24, "zipf"),
                                            (8193, 40000, 24, "zipf"), (2500001, 50021, 8, "zipf"), (2200001, 1000, 8, "same"),
                                            (3, 70, 200003, "uniform"), (65536, 1 << 20, 8, "same")])
def test_gradient_of_many(n, vocab, d, kind):
    rng = np.random.default_rng(n)
    backward(tokens(rng, n, vocab, kind), vocab, d, "bf16", "f32")


@pytest.mark.parametrize("t_x,t_de", TYPES)
@pytest.mark.parametrize("n,vocab,d", [(2048, 1000, 64), (2049, 1000, 64), (2048, 700, 512), (2048, 700, 520), (2048, 700, 256), (2047, 2, 33),
                                       (513, 2, 1030), (256, 1, 40), (257, 1, 40), (1500, 1 << 20, 8), (2, 305, 200001), (100, 304, 4104)])
@pytest.mark.parametrize("kind", ["zipf", "same"])
def test_gradient_in_one_launch(n, vocab, d, kind, t_x, t_de):
    """Where a call is one launch or just no longer: by tokens and by bytes; few
    and many tokens of a row, rows of one CTA and of all."""
    rng = np.random.default_rng(n + d)
    backward(tokens(rng, n, vocab, kind), vocab, d, t_x, t_de, scale=0.75)


@pytest.mark.parametrize("kind", ["zipf", "same", "none"])
@pytest.mark.parametrize("n,vocab,d", [(2048, 500, 64), (600, 3, 1001), (300, 5000, 700), (2048, 500, 513)])
def test_accumulated_in_one_launch(n, vocab, d, kind):
    backward(tokens(np.random.default_rng(n), n, vocab, kind), vocab, d, "bf16", "f32", scale=1.5, accumulate=True)


@pytest.mark.parametrize("t_x", ["bf16", "f32"])
@pytest.mark.parametrize("n,vocab,d,kind", [(1, 3, 5, "uniform"), (100, 50, 33, "zipf"), (5000, 700, 136, "same"), (5000, 9000, 136, "zipf"),
                                            (64, 64, 64, "none")])
def test_accumulated(n, vocab, d, kind, t_x):
    rng = np.random.default_rng(n)
    backward(tokens(rng, n, vocab, kind), vocab, d, t_x, "f32", scale=1.5, pad=True, accumulate=True)


@pytest.mark.parametrize("d", [100, 520])
def test_scaled_and_pitched(d):
    rng = np.random.default_rng(d)
    for t_x, t_de in TYPES:
        backward(tokens(rng, 777, 333, "zipf"), 333, d, t_x, t_de, scale=-d ** 0.5, pad=True)
        backward(tokens(rng, 777, 333, "zipf"), 333, d, t_x, t_de, scale=0.0)


def test_rows_of_no_token_are_not_read():
    """What stands in dX behind ids of no token does not matter; NaN and inf of
    a token's rows reach that token alone."""
    ids = np.array([3, -1, 3, 9, 100, 4])
    x = np.ones((6, 40))
    x[1], x[4] = np.nan, np.inf
    x[3, 7], x[5, 8] = np.nan, np.inf
    dX, _ = rows(x, "bf16")
    dE, _ = rows(np.zeros((10, 40)), "f32")
    m = cola.embed_desc(6, 10, 40, ld_x=dX.stride(0), ld_de=dE.stride(0), dtype_de="f32")
    cola.cola_embed_bwd(m, torch.as_tensor(ids, device="cuda"), dX, dE, cola.embed_workspace(m))
    ref = np.zeros((10, 40))
    ref[3], ref[9], ref[4] = 2.0, 1.0, 1.0
    ref[9, 7], ref[4, 8] = np.nan, np.inf
    assert np.array_equal(host(dE), ref, equal_nan=True)


def test_gradient_against_differences():
    """sum(X * W) moves with E as dE (dX = W) says."""
    rng = np.random.default_rng(5)
    n, vocab, d, scale = 50, 13, 24, 3.0
    ids = tokens(rng, n, vocab, "zipf")
    I = torch.as_tensor(ids, dtype=torch.int64, device="cuda")
    W, _ = rows(rng.integers(-4, 5, (n, d)).astype(float), "f32")
    E, _ = rows(rng.integers(-4, 5, (vocab, d)).astype(float), "f32")
    m = cola.embed_desc(n, vocab, d, scale=scale, dtype_e="f32", dtype_x="f32", dtype_de="f32")
    dE, X = torch.empty((vocab, d), device="cuda"), torch.empty((n, d), device="cuda")
    cola.cola_embed_bwd(m, I, W, dE, cola.embed_workspace(m))

    def value():
        cola.cola_embed_fwd(m, E, I, X)
        return float((X.double() * W.double()).sum())

    base = value()
    for v, c in ((0, 0), (1, 23), (12, 5), (3, 8)):
        E[v, c] += 2.0
        assert value() - base == 2.0 * float(dE[v, c])   # whole numbers: exact
        E[v, c] -= 2.0


@pytest.mark.parametrize("n", [700, 3000, 9000])
def test_streams_and_graphs(n):
    """On another stream, and captured and replayed with other tokens, which
    leave other rows without any; two captured graphs share a workspace."""
    rng = np.random.default_rng(1)
    vocab, d = 5000, 136
    m = cola.embed_desc(n, vocab, d, dtype_de="f32")
    ws = cola.embed_workspace(m)
    I = torch.zeros(n, dtype=torch.int64, device="cuda")
    E = torch.randn((vocab, d), device="cuda").to(torch.bfloat16)
    X, dE = torch.empty((n, d), dtype=torch.bfloat16, device="cuda"), torch.empty((vocab, d), device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        cola.cola_embed_fwd(m, E, I, X)
        cola.cola_embed_bwd(m, I, X, dE, ws)
    torch.cuda.current_stream().wait_stream(side)
    g1, g2 = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g1):
        cola.cola_embed_fwd(m, E, I, X)
        cola.cola_embed_bwd(m, I, X, dE, ws)
    dE2 = torch.empty_like(dE)
    with torch.cuda.graph(g2):
        cola.cola_embed_bwd(m, I, X, dE2, ws)
    for kind in ("zipf", "uniform", "none", "same"):
        ids = tokens(rng, n, vocab, kind)
        I.copy_(torch.as_tensor(ids))
        X.fill_(float("nan")), dE.fill_(float("nan")), dE2.fill_(float("nan"))
        g1.replay()
        g2.replay()
        there = (ids >= 0) & (ids < vocab)
        ref, count = np.zeros((vocab, d)), np.bincount(ids[there], minlength=vocab)
        np.add.at(ref, ids[there], host(E)[ids[there]])
        assert (np.abs(host(dE) - ref) <= (count[:, None] + 2) * U * np.abs(ref)).all()
        assert torch.equal(dE, dE2)


def test_two_streams_at_once():
    """Two gradients that may run together, each with its own workspace, again and
    again: their launches overlap the ones before and behind them."""
    rng = np.random.default_rng(12)
    jobs = []
    for n, vocab, d in ((5000, 3000, 264), (20000, 9000, 264)):
        ids = tokens(rng, n, vocab, "zipf")
        m = cola.embed_desc(n, vocab, d, dtype_de="f32")
        dX = torch.as_tensor(rng.standard_normal((n, d)), device="cuda").to(torch.bfloat16)
        jobs.append((m, torch.as_tensor(ids, dtype=torch.int64, device="cuda"), dX, cola.embed_workspace(m),
                     torch.cuda.Stream(), [torch.full((vocab, d), float("nan"), device="cuda") for _ in range(6)], ids))
    torch.cuda.synchronize()
    for i in range(6):
        for m, I, dX, ws, s, dEs, _ in jobs:
            with torch.cuda.stream(s):
                cola.cola_embed_bwd(m, I, dX, dEs[i], ws)
    torch.cuda.synchronize()
    for m, I, dX, ws, s, dEs, ids in jobs:
        assert all(torch.equal(dEs[0], e) for e in dEs[1:])
        there = (ids >= 0) & (ids < m.vocab)
        ref, mag, count = np.zeros((m.vocab, m.d)), np.zeros((m.vocab, m.d)), np.bincount(ids[there], minlength=m.vocab)
        np.add.at(ref, ids[there], host(dX)[there])
        np.add.at(mag, ids[there], np.abs(host(dX)[there]))
        assert (np.abs(host(dEs[0]) - ref) <= (count[:, None] + 2) * U * mag).all()


def test_traced_launches():
    m = cola.embed_desc(5000, 300, 64)
    I = torch.zeros(5000, dtype=torch.int64, device="cuda")
    E = torch.zeros((300, 64), dtype=torch.bfloat16, device="cuda")
    X = torch.empty((5000, 64), dtype=torch.bfloat16, device="cuda")
    ws = cola.embed_workspace(m)
    with cola.Trace(8) as t:
        cola.cola_embed_fwd(m, E, I, X)
        cola.cola_embed_bwd(m, I, X, E, ws)
    assert [r[0] for r in t.records()] == ["embed", "embed_sort", "embed_sum", "embed_join"]
    assert cola.cola_check_status(ws) == (0, 0)
    for n, want in ((2048, ["embed_sum"]), (2049, ["embed_sort", "embed_sum", "embed_join"])):
        m = cola.embed_desc(n, 300, 64)
        with cola.Trace(8) as t:
            cola.cola_embed_bwd(m, I[:n], X[:n], E, ws)
        assert [r[0] for r in t.records()] == want


def test_short_workspace():
    m = cola.embed_desc(500, 300, 64)
    I = torch.zeros(500, dtype=torch.int64, device="cuda")
    X = torch.empty((500, 64), dtype=torch.bfloat16, device="cuda")
    ws = cola.embed_workspace(m)
    with pytest.raises(cola.ColaError, match="WORKSPACE"):
        cola.cola_embed_bwd(m, I, X, X, ws[:-256])


@pytest.mark.parametrize("t_x", ["bf16", "f32"])
@pytest.mark.parametrize("vocab,d", [(32000, 4096), (32000, 512), (50021, 1000), (300, 64), (1 << 20, 8), (5, 1 << 20)])
def test_workspace_sizes_grow_with_the_tokens(vocab, d, t_x):
    """Up to 20000 tokens, on both sides of later steps of the chunks and of the
    sort's CTAs, and at the limit."""
    some = set(range(1, 20000)) | {int(1.013 ** k) for k in range(1, 1490)} | {65536 * k + j for k in range(1, 70) for j in (-1, 0, 1)}
    last = 0
    for n in sorted(some | {(1 << 28) - 1}):
        if n >= 1 << 28 or n * (d // 8) > 1 << 38:
            break
        size = cola.cola_embed_workspace_size(cola.embed_desc(n, vocab, d, dtype_x=t_x))
        assert size >= last, n
        last = size


@pytest.mark.parametrize("n,most,vocab,d", [(7000, 8192, 3000, 4096), (7295, 7296, 500, 4096), (2500, 30000, 9000, 1024), (8192, 8193, 2000, 72),
                                            (65536, 65537, 3000, 8), (260000, 270000, 70000, 16), (9, 5000, 40, 2056)])
def test_few_tokens_in_the_workspace_of_more(n, most, vocab, d):
    ids = torch.as_tensor(tokens(np.random.default_rng(n), n, vocab, "zipf"), dtype=torch.int64, device="cuda")
    dX = torch.randn((n, d), device="cuda").to(torch.bfloat16)
    m = cola.embed_desc(n, vocab, d)
    own, other = (torch.full((vocab, d), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    cola.cola_embed_bwd(m, ids, dX, own, cola.embed_workspace(m))
    cola.cola_embed_bwd(m, ids, dX, other, cola.embed_workspace(cola.embed_desc(most, vocab, d)))
    assert not bool(torch.isnan(own).any()) and torch.equal(own, other)


@pytest.mark.parametrize("t_x", ["bf16", "f32"])
@pytest.mark.parametrize("n,vocab,d,kind", [(20000, 9000, 136, "zipf"), (40000, 300, 40, "same"), (9000, 50021, 33, "uniform"),
                                            (30000, 700, 1003, "zipf"), (8193, 70, 64, "none"), (70000, 1 << 20, 8, "rising"),
                                            (2200001, 1000, 8, "zipf"), (2100001, 50021, 7, "zipf")])
def test_accumulated_of_many(n, vocab, d, kind, t_x):
    """Digit by digit sorted: one pass and two, rounds that come again, sums that
    cross many chunks; rows of no token stay as they were."""
    backward(tokens(np.random.default_rng(n), n, vocab, kind), vocab, d, t_x, "f32", scale=1.5, pad=True, accumulate=True)
