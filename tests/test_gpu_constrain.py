"""Constraints on logits and the gradient through them against the definitions
in 64 bits, where they can go wrong: vocabularies of one token and the largest,
rows off 16-byte boundaries, histories of no token and long ones, one token
named by a whole history, masks that leave a row nothing, biases that name a
token twice, values that are not finite, results over their inputs, other
streams and graphs.

Tolerances (u = 2^-24, fp32's half step): an adjusted logit takes a product or
quotient, a product and two differences, and a sum of its biases, each off by u
of what it forms: 5 u (|x| max(r, 1/r) + f c + p) + (entries + 2) u sum |bias|;
and the result's type rounds once, bf16 by 2^-8 of the value.  A gradient takes
one rounding to fp32 and the type's.  All else is equal bit for bit.
"""
import numpy as np
import pytest
import torch

import vocab_helpers as H
from paper_2502_10940_gb300 import cola

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {"bf16": 2.0 ** -8, "f32": U}


def limits(rng, n, V, width, biases=0, masks=0, zero=False):
    """Constraints of every kind (numpy), with ids of no token among them."""
    ids = np.minimum((rng.pareto(0.8, (n, width)) * 3).astype(np.int64), V + 2)
    ids[rng.random((n, width)) < 0.05] = -1
    c = dict(history=ids, history_len=rng.integers(0, width + 1, n), repetition=rng.uniform(0.8, 1.5, n).astype(np.float32),
             frequency=rng.uniform(-0.2, 0.7, n).astype(np.float32), presence=rng.uniform(-0.2, 0.7, n).astype(np.float32))
    c["prompt_len"] = (c["history_len"] * rng.random(n)).astype(np.int64)
    if biases:
        c["bias_ids"] = rng.integers(-1, V + 1, (n, biases))
        c["bias"] = (rng.standard_normal((n, biases)) * 5).astype(np.float32)
    if masks:
        share = rng.choice([0.0, 0.01, 0.5, 0.99, 1.0], masks)
        bits = rng.random((masks, (V + 31) // 32, 32)) < share[:, None, None]
        c["masks"] = (bits.astype(np.int64) << np.arange(32)).sum(-1).astype(np.uint32).astype(np.int32)
        c["mask_of"] = rng.integers(-1, masks + 1, n)
    return c


def on_gpu(c):
    t = {k: torch.as_tensor(v, device="cuda") for k, v in c.items()}
    return cola.constraints(t.pop("history", None), t.pop("history_len", None), t.pop("prompt_len", None), **t)


def row(c, i, V):
    """One row's factors, penalties, biases and mask in 64 bits."""
    h = c["history"][i] if "history" in c else np.zeros(0, np.int64)
    n = len(h) if "history_len" not in c else min(max(int(c["history_len"][i]), 0), len(h))
    prompt = max(int(c["prompt_len"][i]), 0) if "prompt_len" in c else 0
    count = lambda ids: np.bincount(ids[(ids >= 0) & (ids < V)], minlength=V)   # noqa: E731
    get = lambda k, d: float(c[k][i]) if k in c else d   # noqa: E731
    o = dict(seen=count(h[:n]) > 0, times=count(h[prompt:n]), r=get("repetition", 1.0), f=get("frequency", 0.0),
             p=get("presence", 0.0), bias=np.zeros(V), size=np.zeros(V), entries=np.zeros(V), allowed=np.ones(V, bool))
    if "bias" in c:
        ids, b = c["bias_ids"][i], c["bias"][i].astype(np.float64)
        ok = (ids >= 0) & (ids < V)
        for k, v in (("bias", b), ("size", np.abs(b)), ("entries", np.ones(len(b)))):
            np.add.at(o[k], ids[ok], v[ok])
    if "masks" in c:
        m = int(c["mask_of"][i]) if "mask_of" in c else i
        if 0 <= m < len(c["masks"]):
            o["allowed"] = (c["masks"][m].astype(np.uint32)[:, None] >> np.arange(32) & 1).reshape(-1)[:V].astype(bool)
    return o


def check_row(name, got, ref, tol, exact):
    H.same_nonfinite(name, got, ref)
    ok = np.isfinite(ref)
    far = np.where(exact, 0.0, tol)[ok]
    assert (np.abs(got[ok] - ref[ok]) <= far).all(), (name, np.abs(got[ok] - ref[ok]).max())


def check_fwd(x, c, dtype, got):
    for i in range(len(x)):
        V = x.shape[1]
        o = row(c, i, V)
        with np.errstate(invalid="ignore", over="ignore"):
            big = np.abs(x[i]) * max(o["r"], 1 / o["r"])
            y = np.where(o["seen"], np.where(x[i] > 0, x[i] / o["r"], x[i] * o["r"]), x[i])
            y = np.where(o["times"] > 0, y - o["f"] * o["times"] - o["p"], y)
            y = np.where(o["entries"] > 0, y + o["bias"], y)
            y = np.where(o["allowed"], y, -np.inf)
            tol = 5 * U * (big + abs(o["f"]) * o["times"] + abs(o["p"])) + (o["entries"] + 2) * U * o["size"]
            tol = tol * (1 + HALF[dtype]) + HALF[dtype] * np.abs(y)
            # beyond the type's range (its lowest value times a penalty) rounding gives infinities
            y = np.where(np.isinf(H.rounded(y, dtype)), H.rounded(y, dtype), y)
        changed = (o["seen"] & (o["r"] != 1)) | (o["times"] > 0) | (o["entries"] > 0)
        check_row(f"row {i}", got[i], y, tol, ~changed)


def check_bwd(x, g, c, dtype, got):
    for i in range(len(x)):
        o = row(c, i, x.shape[1])
        with np.errstate(invalid="ignore"):
            y = np.where(o["seen"], np.where(x[i] > 0, g[i] / o["r"], g[i] * o["r"]), g[i])
            y = np.where(o["allowed"], y, 0.0)
            check_row(f"row {i}", got[i], y, (U + HALF[dtype]) * np.abs(y), ~o["seen"])


def whole(buf, view):
    t = buf.clone()
    torch.as_strided(t, view.shape, view.stride(), view.storage_offset()).fill_(float("nan"))
    assert bool(torch.isnan(t).all())


def run(x, g, c, dtype, layout="dense"):
    """Forward and backward, each into other memory and over its inputs."""
    n, V = x.shape
    X, G = H.place(x, dtype, layout), H.place(g, dtype, layout)
    pitch = X.stride(0)
    d = cola.vocab_desc(n, V, ld=pitch, ld_grad=pitch, dtype=dtype)
    C = on_gpu(c)
    shifts = [0, X.storage_offset()] if layout != "shifted" else [1, 3]
    for shift in shifts:
        out, b1 = H.like(X, shift=shift)
        dl, b2 = H.like(X, shift=shift)
        cola.cola_constrain_logits_fwd(d, C, X, out)
        cola.cola_constrain_logits_bwd(d, C, X, G, dl)
        whole(b1, out), whole(b2, dl)
        check_fwd(x, c, dtype, H.host(out))
        check_bwd(x, g, c, dtype, H.host(dl))
    over, g_over = H.place(x, dtype, layout), H.place(g, dtype, layout)
    cola.cola_constrain_logits_bwd(d, C, over, g_over, g_over)     # over the upstream gradient
    assert same_bits(g_over, dl)
    cola.cola_constrain_logits_bwd(d, C, over, G, over)            # over the logits
    assert same_bits(over, dl)
    over = H.place(x, dtype, layout)
    cola.cola_constrain_logits_fwd(d, C, over, over)
    assert same_bits(over, out)
    return out


def same_bits(a, b):
    i = torch.int16 if a.dtype == torch.bfloat16 else torch.int32
    return torch.equal(a.contiguous().view(i), b.contiguous().view(i))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,V,width", [(1, 1, 1), (3, 2, 5), (4, 7, 3), (2, 31, 40), (2, 33, 100), (5, 257, 64), (3, 1000, 5000), (2, 4099, 1),
                                       (2, 33001, 700), (1, 131072, 3000), (2, 200003, 300), (1, 1 << 20, 1000), (700, 100, 20),
                                       (40, 5003, 300), (25, 40007, 2000), (200, 601, 5000), (2, 3001, 70000)])
def test_sizes(n, V, width, dtype):
    rng = np.random.default_rng(V + n)
    x, g = H.logits(rng, n, V, dtype), H.rounded(rng.standard_normal((n, V)), dtype)
    run(x, g, limits(rng, n, V, width, biases=min(V, 7), masks=2), dtype)
    run(x, g, limits(rng, n, V, width), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["padded", "odd", "shifted"])
@pytest.mark.parametrize("V", [5, 517, 5003, 70001])
def test_layouts(V, layout, dtype):
    rng = np.random.default_rng(V)
    x, g = H.logits(rng, 4, V, dtype), H.rounded(rng.standard_normal((4, V)), dtype)
    run(x, g, limits(rng, 4, V, 50, biases=3, masks=3), dtype, layout)
    run(x, g, limits(rng, 4, V, 50, biases=3), dtype, layout)


@pytest.mark.parametrize("kind", ["nothing", "history", "repetition", "frequency", "biases", "masks", "own masks"])
def test_one_kind_at_a_time(kind):
    rng = np.random.default_rng(7)
    n, V = 5, 3001
    x, g = H.logits(rng, n, V, "bf16"), H.rounded(rng.standard_normal((n, V)), "bf16")
    c = limits(rng, n, V, 200, biases=5, masks=n)
    keep = {"nothing": [], "history": ["history"], "repetition": ["history", "history_len", "repetition"],
            "frequency": ["history", "prompt_len", "frequency"], "biases": ["bias_ids", "bias"], "masks": ["masks", "mask_of"],
            "own masks": ["masks"]}[kind]
    run(x, g, {k: c[k] for k in keep}, "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [37, 3001, 40007])
def test_masks(V, dtype):
    """Rows that are left nothing, one token (the first, the last), all; logits
    of -inf and of the type's lowest value, NaN and inf in masked places."""
    rng = np.random.default_rng(V)
    n = 8
    x, g = H.logits(rng, n, V, dtype), H.rounded(rng.standard_normal((n, V)), dtype)
    x[4, ::3], x[5, ::2], x[6, 1], x[7, 2] = -np.inf, float(torch.finfo(H.TORCH[dtype]).min), np.nan, np.inf
    g[6, 3], g[7, 4] = np.nan, np.inf
    bits = np.zeros((n, (V + 31) // 32 * 32), np.int64)
    bits[1, 0] = bits[2, V - 1] = bits[3] = bits[4] = 1
    bits[5, V // 2] = 1
    bits[0, V:] = bits[2, V:] = 1             # bits behind the vocabulary
    words = (bits.reshape(n, -1, 32) << np.arange(32)).sum(-1).astype(np.uint32).astype(np.int32)
    c = limits(rng, n, V, 60, biases=4)
    c["bias_ids"][2], c["bias_ids"][5] = V - 1, V // 2
    run(x, g, dict(c, masks=words), dtype)                                              # 6 and 7: banned NaN and inf
    run(x, g, dict(c, masks=words, mask_of=np.array([3, 0, 2, 1, 5, 4, 99, -1])), dtype)   # and allowed


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_histories(dtype):
    """One token over and over, prompts that are all, none or more than all of
    it, lengths below 0 and beyond the room, every token once."""
    rng = np.random.default_rng(3)
    n, V, width = 9, 1500, 4000
    x, g = H.logits(rng, n, V, dtype), H.rounded(rng.standard_normal((n, V)), dtype)
    x[8, :4] = [0.0, -0.0, np.inf, -np.inf]
    c = limits(rng, n, V, width)
    c["history"][0] = 17
    c["history"][1] = np.arange(width) % V
    c["history"][8] = np.arange(width) % 4
    c["history_len"] = np.array([width, width, 10, 10, 0, -5, width + 7, 2 ** 40, width])
    c["prompt_len"] = np.array([0, V, 10, 3, 0, 3, width, -9, 2 ** 40])
    run(x, g, c, dtype)
    run(x, g, {k: v for k, v in c.items() if k not in ("history_len", "prompt_len")}, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,V,width,layout", [(19, 5003, 4096, "dense"), (20, 5003, 4096, "dense"), (20, 5003, 4097, "dense"),
                                              (24, 70001, 4096, "padded"), (21, 33000, 1, "shifted"), (77, 501, 4096, "odd"),
                                              (304, 1003, 33, "dense"), (305, 1003, 33, "dense"), (609, 37, 300, "shifted"),
                                              (77, 66001, 4097, "shifted"), (77, 2003, 16384, "dense"), (77, 2003, 16385, "odd"),
                                              (76, 2003, 5000, "dense"), (400, 37, 5000, "padded")])
def test_many_rows(n, V, width, layout, dtype):
    """Rows on 256 and 512 threads, whose counts go by the tokens' places in the list: one
    token over and over, every token once, nothing behind the prompt."""
    rng = np.random.default_rng(n + V)
    x, g = H.logits(rng, n, V, dtype), H.rounded(rng.standard_normal((n, V)), dtype)
    c = limits(rng, n, V, width, biases=5, masks=3)
    c["history"][0], c["history"][1] = V - 1, np.arange(width) % V
    c["history"][2] = V - 1 - np.arange(width) % V
    c["history_len"][:4] = width
    c["prompt_len"][:4] = [0, 0, 1, width]
    run(x, g, c, dtype, layout)
    run(x, g, {k: v for k, v in c.items() if not k.startswith("bias") and k != "repetition"}, dtype, layout)


@pytest.mark.parametrize("width", [65535, 65536, 70001])
def test_one_token_more_often_than_16_bits_count(width):
    rng = np.random.default_rng(width)
    n, V = 2, 501
    x, g = H.logits(rng, n, V, "f32"), H.rounded(rng.standard_normal((n, V)), "f32")
    c = limits(rng, n, V, width)
    c["history"][0], c["history"][1] = 7, 500
    c["history_len"], c["prompt_len"] = np.full(n, width), np.array([0, 3])
    run(x, g, c, "f32")


@pytest.mark.parametrize("n", [2, 30])
def test_two_streams_at_once(n):
    """Two calls that may run together, each with its own rows."""
    rng = np.random.default_rng(n)
    V = 30011
    jobs = []
    for k in range(2):
        x, c = H.logits(rng, n, V, "bf16"), limits(rng, n, V, 700, biases=4, masks=3)
        jobs.append((x, c, on_gpu(c), H.place(x, "bf16"), torch.cuda.Stream()))
    outs = [torch.empty_like(j[3]) for j in jobs]
    torch.cuda.synchronize()
    for _ in range(5):
        for (x, c, C, X, s), out in zip(jobs, outs):
            with torch.cuda.stream(s):
                cola.cola_constrain_logits_fwd(cola.vocab_desc(n, V), C, X, out)
    torch.cuda.synchronize()
    for (x, c, C, X, s), out in zip(jobs, outs):
        check_fwd(x, c, "bf16", H.host(out))


@pytest.mark.parametrize("biases", [1, 300, 1024])
def test_biases_that_name_a_token_again(biases):
    rng = np.random.default_rng(biases)
    n, V = 3, 9001
    x, g = H.logits(rng, n, V, "f32"), H.rounded(rng.standard_normal((n, V)), "f32")
    c = limits(rng, n, V, 30, biases=biases)
    c["bias_ids"][0] = 5
    c["bias_ids"][1] = rng.integers(0, 20, biases)
    c["bias"][2, 0] = -np.inf
    a = run(x, g, c, "f32")
    assert same_bits(a, run(x, g, c, "f32"))   # sums of a token's entries in their order


@pytest.mark.parametrize("n", [2, 25])
@pytest.mark.parametrize("V,biases", [(60001, 1000), (5003, 300), (700, 300), (97, 333)])
def test_few_and_many_tokens_biased_again(V, biases, n):
    rng = np.random.default_rng(V + n)
    x, g = H.logits(rng, n, V, "f32"), H.rounded(rng.standard_normal((n, V)), "f32")
    c = limits(rng, n, V, 60, biases=biases, masks=2)
    c["bias_ids"][0, -1] = c["bias_ids"][0, 0]
    run(x, g, c, "f32")


def test_strided_histories_and_masks():
    rng = np.random.default_rng(11)
    n, V = 4, 2000
    x = H.logits(rng, n, V, "bf16")
    c = limits(rng, n, V, 33, masks=3)
    wide = torch.full((n, 50), 1, dtype=torch.int64, device="cuda")
    wide[:, 5:38] = torch.as_tensor(c["history"], device="cuda")
    words = torch.full((3, 90), -1, dtype=torch.int32, device="cuda")
    words[:, 3:66] = torch.as_tensor(c["masks"], device="cuda")
    t = {k: torch.as_tensor(v, device="cuda") for k, v in c.items()}
    C = cola.constraints(wide[:, 5:38], repetition=t["repetition"], frequency=t["frequency"], masks=words[:, 3:66], mask_of=t["mask_of"])
    X = H.place(x, "bf16")
    out = torch.empty_like(X)
    cola.cola_constrain_logits_fwd(cola.vocab_desc(n, V), C, X, out)
    check_fwd(x, {k: c[k] for k in ("history", "repetition", "frequency", "masks", "mask_of")}, "bf16", H.host(out))


def test_gradient_against_differences():
    """sum(out * w) moves with a logit as the gradient says (fp32, steps within
    the logit's sign)."""
    rng = np.random.default_rng(2)
    n, V = 2, 300
    x, w = H.logits(rng, n, V, "f32"), H.rounded(rng.standard_normal((n, V)), "f32")
    c = limits(rng, n, V, 80, biases=5)
    c["frequency"][:] = c["presence"][:] = 0
    C, X, W = on_gpu(c), H.place(x, "f32"), H.place(w, "f32")
    d = cola.vocab_desc(n, V, dtype="f32")
    out, dl = torch.empty_like(X), torch.empty_like(X)
    cola.cola_constrain_logits_bwd(d, C, X, W, dl)
    up = torch.where(X.abs() < 0.5, 0.0, 0.25 * X.abs())
    cola.cola_constrain_logits_fwd(d, C, X + up, out)
    high = out.double()
    cola.cola_constrain_logits_fwd(d, C, X - up, out)
    got = (high - out.double()) * W.double()
    want = dl.double() * ((X + up).double() - (X - up).double())
    # two adjusted logits, each off by a few u of |x| r + |bias|
    size = 4 * X.double().abs() + torch.as_tensor(np.abs(c["bias"]).sum(1), device="cuda")[:, None]
    assert bool(((got - want).abs() <= 16 * U * size * W.double().abs()).all())


def test_streams_and_graphs():
    """On another stream, and captured and replayed with other histories, masks
    and logits."""
    rng = np.random.default_rng(9)
    n, V = 6, 20011
    c = limits(rng, n, V, 90, biases=6, masks=2)
    t = {k: torch.as_tensor(v, device="cuda") for k, v in c.items()}
    a = dict(t)
    C = cola.constraints(a.pop("history"), a.pop("history_len"), a.pop("prompt_len"), **a)
    X = H.place(H.logits(rng, n, V, "bf16"), "bf16")
    out = torch.empty_like(X)
    d = cola.vocab_desc(n, V)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        cola.cola_constrain_logits_fwd(d, C, X, out)
    torch.cuda.current_stream().wait_stream(side)
    check_fwd(H.host(X), c, "bf16", H.host(out))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cola.cola_constrain_logits_fwd(d, C, X, out)
    for _ in range(2):
        c = limits(rng, n, V, 90, biases=6, masks=2)
        for k, v in c.items():
            t[k].copy_(torch.as_tensor(v))
        X.copy_(torch.from_numpy(H.logits(rng, n, V, "bf16")))
        graph.replay()
        check_fwd(H.host(X), c, "bf16", H.host(out))


def test_traced_launches():
    rng = np.random.default_rng(1)
    C = on_gpu(limits(rng, 2, 100, 9))
    X = H.place(H.logits(rng, 2, 100, "f32"), "f32")
    with cola.Trace(4) as t:
        cola.cola_constrain_logits_fwd(cola.vocab_desc(2, 100, dtype="f32"), C, X, X)
        cola.cola_constrain_logits_bwd(cola.vocab_desc(2, 100, dtype="f32"), C, X, X, torch.empty_like(X))
    assert [r[0] for r in t.records()] == ["constrain", "constrain"]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,V", [(1, 1), (3, 5003), (90, 1001)])
def test_histories_of_no_ids(n, V, dtype):
    """The first token of a sequence without a prompt: penalties of no token."""
    rng = np.random.default_rng(n)
    x, g = H.logits(rng, n, V, dtype), H.rounded(rng.standard_normal((n, V)), dtype)
    c = limits(rng, n, V, 0, biases=3, masks=2)
    run(x, g, c, dtype)
    run(x, g, {k: v for k, v in c.items() if k in ("history", "repetition", "presence")}, dtype, "odd")
    room = torch.zeros((n, 7), dtype=torch.int64, device="cuda")
    C = cola.constraints(room[:, :0], repetition=torch.full((n,), 2.0, device="cuda"))
    X = H.place(x, dtype)
    out = torch.empty_like(X)
    cola.cola_constrain_logits_fwd(cola.vocab_desc(n, V, dtype=dtype), C, X, out)
    assert same_bits(X, out)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,V", [(1, 33), (90, 1001)])
def test_no_masks(n, V, dtype):
    """A batch none of whose rows has a grammar."""
    rng = np.random.default_rng(n + 1)
    x, g = H.logits(rng, n, V, dtype), H.rounded(rng.standard_normal((n, V)), dtype)
    c = limits(rng, n, V, 40, biases=3)
    run(x, g, dict(c, masks=np.zeros((0, (V + 31) // 32), np.int32), mask_of=rng.integers(-1, 2, n)), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shift", [0, 1, 2, 5])
@pytest.mark.parametrize("n,V", [(1, 7), (3, 1001), (2, 40003), (400, 517)])
def test_other_logits_keep_their_bits(n, V, shift, dtype):
    """Every bit pattern, the NaNs' signs and payloads among them, wherever a row begins."""
    rng = np.random.default_rng(V)
    ints, width = (torch.int16, 16) if dtype == "bf16" else (torch.int32, 32)
    bits = rng.integers(0, 1 << width, (n, V))
    nan = 0x7f81 + rng.integers(0, 127, (n, V)) | rng.integers(0, 2, (n, V)) << 15
    bits = np.where(rng.random((n, V)) < 0.3, nan << width - 16, bits)
    bits = torch.as_tensor(np.where(bits >= 1 << width - 1, bits - (1 << width), bits), device="cuda").to(ints)
    X = bits.view(H.TORCH[dtype])
    history = torch.as_tensor(rng.integers(0, V, (n, 3)), device="cuda")
    named = torch.zeros((n, V), dtype=torch.bool, device="cuda").scatter_(1, history, True)
    C = cola.constraints(history, repetition=torch.full((n,), 2.0, device="cuda"))
    out, _ = H.like(X, shift=shift)
    cola.cola_constrain_logits_fwd(cola.vocab_desc(n, V, dtype=dtype), C, X, out)
    assert torch.equal(out.contiguous().view(ints)[~named], bits[~named])
