"""The operators at the vocabulary's two ends with the others, as programs run
them: a training step with a tied embedding, decoding under constraints by a
captured step, a policy gradient through the constraints, and the example that
does the first two.  Each operator is checked on the values that the one before
it gave, by its own definition and tolerance."""
import importlib.util
import os

import numpy as np
import pytest
import torch

import vocab_helpers as H
from paper_2502_10940_gb300 import cola
from test_gpu_constrain import check_bwd, check_fwd, limits, on_gpu

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def _example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "tied.py")
    spec = importlib.util.spec_from_file_location("example_tied", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_training_step_with_a_tied_embedding():
    """The example's step: the lookup bit for bit, the lookup's gradient on top of
    the output embedding's; all of it against autograd in 64 bits (normwise: five
    tensors rounded to bf16 between the loss and E, each 2^-9 of its norm at
    most, and the layer's own tolerance 5e-3)."""
    ex = _example()
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    n, vocab, dim, rank = 700, 1000, 136, 64
    model = ex.Model(vocab, dim, rank, g)
    s = model.plan(n)
    ids = torch.randint(0, 60, (n,), generator=g, device="cuda") ** 2 % vocab
    targets = torch.randint(0, vocab, (n,), generator=g, device="cuda")
    ids[::11] = -1                                   # padding: no token, and ignored
    targets[::11] = -100
    loss = model.step(s, ids, targets)
    w = model.weights()
    there = ids >= 0
    X = torch.where(there[:, None], w[0][ids.clamp(min=0)].float() * model.scale, 0.0).to(torch.bfloat16)
    assert torch.equal(s["X"], X)
    # the lookup's gradient apart, and what it was added to
    dh_dx = torch.zeros((vocab, dim), device="cuda")
    alone = cola.embed_desc(n, vocab, dim, scale=model.scale, dtype_de="f32")
    total = s["dX"]                                  # (the layer's part; the residual's is added in the step)
    cola.cola_embed_bwd(alone, ids, total, dh_dx, s["embed_ws"])
    ref, mag, rows = np.zeros((vocab, dim)), np.zeros((vocab, dim)), np.bincount(ids[there].cpu().numpy(), minlength=vocab)
    x = H.host(total)[there.cpu().numpy()]
    np.add.at(ref, ids[there].cpu().numpy(), x)
    np.add.at(mag, ids[there].cpu().numpy(), np.abs(x))
    sc = float(np.float32(model.scale))
    assert (np.abs(H.host(dh_dx) - sc * ref) <= (rows[:, None] + 2) * U * sc * mag).all()

    P = [t.double().requires_grad_() for t in w]
    E, A, B = P
    x64 = torch.where(there[:, None], E[ids.clamp(min=0)] * model.scale, 0.0)
    h = x64 + torch.nn.functional.silu(x64 @ A.T) @ B.T
    logp = torch.log_softmax(h @ E.T, 1)
    ok = targets >= 0
    want = -(logp.gather(1, targets.clamp(min=0)[:, None])[:, 0] * ok).sum() / n
    want.backward()
    assert abs(loss.item() - want.item()) <= 1e-2 * want.item()
    for name, got, p in zip("EAB", model.grads, P):
        rel = ((got.double() - p.grad).norm() / p.grad.norm()).item()
        assert rel <= 5e-3 + 5 * 2.0 ** -9, (name, rel)


def test_accumulation_over_micro_batches():
    """A batch cut in four gives the whole batch's gradient (sums of the same rows
    in another order)."""
    rng = np.random.default_rng(4)
    n, vocab, d = 1000, 200, 72
    ids = torch.as_tensor(np.minimum((rng.pareto(1.0, 4 * n) * 2).astype(np.int64), vocab), device="cuda")   # vocab: no token
    dX = torch.as_tensor(rng.standard_normal((4 * n, d)), device="cuda").to(torch.bfloat16)
    whole, parts = torch.empty((vocab, d), device="cuda"), torch.full((vocab, d), float("nan"), device="cuda")
    m = cola.embed_desc(4 * n, vocab, d, dtype_de="f32")
    cola.cola_embed_bwd(m, ids, dX, whole, cola.embed_workspace(m))
    ws = cola.embed_workspace(cola.embed_desc(n, vocab, d, dtype_de="f32"))
    for i in range(4):
        m = cola.embed_desc(n, vocab, d, dtype_de="f32", accumulate=i > 0)
        cola.cola_embed_bwd(m, ids[i * n:(i + 1) * n], dX[i * n:(i + 1) * n], parts, ws)
    i = ids.cpu().numpy()
    mag, rows = np.zeros((vocab + 1, d)), np.bincount(i, minlength=vocab + 1)[:vocab]
    np.add.at(mag, i, np.abs(H.host(dX)))
    assert (np.abs(H.host(whole) - H.host(parts)) <= 2 * (rows[:, None] + 8) * U * mag[:vocab]).all()


def test_decoding_under_constraints():
    """Each captured step's token is the likeliest of the constrained logits that
    the plain definition gives for the history so far."""
    rng = np.random.default_rng(8)
    n, V, steps = 5, 3001, 12
    c = limits(rng, n, V, 6 + steps, biases=4, masks=n)
    c["masks"][:, :] = -1                                    # everything, but for a third of the tokens
    c["masks"][:, ::3] = 0
    c["mask_of"] = np.array([0, 1, -1, 3, 4])
    c["history_len"] = np.full(n, 6)
    c["prompt_len"] = np.array([0, 3, 6, 2, 6])
    t = {k: torch.as_tensor(v, device="cuda") for k, v in c.items()}
    a = dict(t)
    C = cola.constraints(a.pop("history"), a.pop("history_len"), a.pop("prompt_len"), **a)
    d = cola.vocab_desc(n, V, k=1)
    source = H.place(H.logits(rng, n, V, "bf16"), "bf16")
    logits, best, logp = torch.empty_like(source), torch.empty((n, 1), dtype=torch.int64, device="cuda"), torch.empty((n, 1), device="cuda")

    def token():
        logits.copy_(source)
        cola.cola_constrain_logits_fwd(d, C, logits, logits)
        cola.cola_token_logprob_fwd(d, logits, None, None, None, best, logp, None)
        t["history"].scatter_(1, t["history_len"][:, None], best)
        t["history_len"].add_(1)

    graph = torch.cuda.CUDAGraph()
    token()
    t["history"].copy_(torch.as_tensor(c["history"]))
    t["history_len"].copy_(torch.as_tensor(c["history_len"]))
    with torch.cuda.graph(graph):
        token()
    for _ in range(steps):
        graph.replay()
        got = H.host(logits)
        check_fwd(H.host(source), c, "bf16", got)
        assert np.array_equal(best[:, 0].cpu().numpy(), got.argmax(1))
        lse = np.log(np.exp(got - got.max(1, keepdims=True)).sum(1))
        assert np.abs(logp[:, 0].cpu().numpy() + lse).max() <= 1e-5
        for i in range(n):
            c["history"][i, c["history_len"][i]] = got[i].argmax()
        c["history_len"] += 1
        assert np.array_equal(t["history"].cpu().numpy(), c["history"])


def test_policy_gradient_through_constraints():
    """Constrained logits, the policy gradient at them in place, and it at the
    model's logits."""
    rng = np.random.default_rng(6)
    n, V = 6, 2003
    x = H.logits(rng, n, V, "f32")
    c = limits(rng, n, V, 120, biases=5, masks=3)
    C, X = on_gpu(c), H.place(x, "f32")
    d = cola.vocab_desc(n, V, dtype="f32")
    out = torch.empty_like(X)
    cola.cola_constrain_logits_fwd(d, C, X, out)
    y = H.host(out)
    targets = np.array([int(np.flatnonzero(np.isfinite(r))[-1]) if np.isfinite(r).any() else -1 for r in y])
    g, h = rng.standard_normal(n).astype(np.float32), rng.standard_normal(n).astype(np.float32) * 0.1
    up = [torch.as_tensor(v, device="cuda") for v in (g, h)]
    cola.cola_token_logprob_step(d, out, torch.as_tensor(targets, device="cuda"), up[0], up[1], None, None, out)
    dy = H.host(out)
    for i in range(n):
        gi = float(g[i]) if targets[i] >= 0 else 0.0
        H.check_logprob_grad(dy[i], H.logprob_row(y[i], targets[i], 1.0, gi, float(h[i])), targets[i], gi, float(h[i]), 1.0, "f32")
    cola.cola_constrain_logits_bwd(d, C, X, out, out)
    check_bwd(x, dy, c, "f32", H.host(out))


def test_example_runs():
    lines = []
    r = _example().main(tokens=512, dim=64, vocab=700, rank=64, steps=3, sequences=5, length=9, log=lines.append)
    assert len(r["loss"]) == 2 and all(np.isfinite(r["loss"]))
    assert r["text"].shape == (5, 9) and bool(r["allowed"][r["text"]].all()) and bool((r["logp"] <= 0).all())
    assert len(lines) == 3
