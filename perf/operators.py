"""Measured cases of the vocabulary operators: what a program that pre-trains,
distils, scores or serves a CoLA model does with its rows of vocabulary
logits, [n x vocab], one row per token.

  score    log probability of one given token per row, the row's entropy and
           its k most likely tokens (cola_token_logprob_fwd)
  ce       pre-training or policy step: log probabilities and entropy with the
           gradient at the logits in one call, the upstream gradients being
           known (cola_token_logprob_step)
  policy   the gradient alone, from saved row statistics and upstream
           gradients that depended on the log probabilities
           (cola_token_logprob_bwd)
  eval     distillation loss against a teacher's k most likely tokens
           (cola_topk_distill_fwd)
  distil   that loss with its gradient in one call (cola_topk_distill_step)
  late     its gradient alone, from saved statistics (cola_topk_distill_bwd)

For a row x, temperature T:  logp_j = x_j / T - log sum exp(x / T),  p = exp(logp),
H = - sum p logp;  the gradient of g logp_y + h H is
(1/T) (g (onehot_y - p) - h p (logp + H)).  A target outside the vocabulary is
ignored.  Distillation: teacher probabilities q over its k tokens, either
renormalised over them or with one more entry, the rest of the vocabulary;
L = T^2 KL(q || p).

Logits are N(0, 2^2) with eight raised tokens per row, as a trained model's
rows have few likely tokens; "masked" sets one in 128 to -inf, as banned
tokens and padded vocabularies are.
"""
import math

import torch

own = False
F32 = torch.float32
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _case(kind, n, vocab, dtype="bf16", k=0, T=1.0, *, entropy=True, rest=False, masked=False, pad=False, graph=False, **name):
    return dict(name, kind=kind, n=n, vocab=vocab, dtype=dtype, k=k, T=T, entropy=entropy, rest=rest, masked=masked,
                pad=pad, graph=graph)


def listed():
    return [
        # serving, one user: the sampled token's log probability and 20
        # alternatives, replayed with the decode step's graph
        _case("score", 1, 128000, k=20, T=0.75, graph=True, name="score_n1_top20"),
        # serving, one token for each of 32 sequences, 5 alternatives
        _case("score", 32, 32000, k=5, graph=True, name="score_n32_top5"),
        # scoring a prompt, odd vocabulary with banned tokens, rows unaligned
        _case("score", 509, 50021, masked=True, name="score_prompt_n509"),
        # evaluation over fp32 logits: log probability and the best token
        _case("score", 4096, 32000, "f32", k=1, entropy=False, name="score_eval_f32"),
        # a teacher's list for distillation at temperature 2
        _case("score", 8192, 32000, k=64, T=2.0, entropy=False, name="teacher_top64"),
        # pre-training cross entropy, 128 x 256 tokens, some of them padding
        _case("ce", 32768, 32000, entropy=False, name="ce_step_n32768"),
        # policy gradient with an entropy bonus, fp32 logits, odd vocabulary
        _case("policy", 4096, 65537, "f32", name="policy_bwd_f32"),
        # distillation, one short micro-batch
        _case("distil", 256, 32000, k=16, T=2.0, name="distil_n256_top16"),
        # distillation step with the rest of the vocabulary as an entry
        _case("distil", 16384, 32000, k=64, T=2.0, rest=True, name="distil_step_top64"),
        # the same over fp32 logits, odd sizes, banned tokens
        _case("distil", 2047, 50021, "f32", k=50, rest=True, masked=True, name="distil_odd_f32"),
        # held-out distillation loss over a wide vocabulary and a long list
        _case("eval", 4096, 200000, k=128, T=1.5, name="eval_wide_top128"),
        # the gradient of a loss whose weights came later
        _case("late", 8192, 65536, k=32, T=2.0, rest=True, name="late_bwd_top32"),
    ]


MAX_BYTES = 4.25e9   # of one drawn pass: no more than the largest listed case


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["score", "score", "ce", "policy", "eval", "distil", "distil", "late"])
    vocab = _log_int(rng, 250, 262144)
    pick = rng.random()
    vocab = vocab // 64 * 64 if pick < 0.3 and vocab >= 64 else vocab // 8 * 8 if pick < 0.5 else vocab
    dtype = rng.choice(["bf16", "bf16", "f32"])
    k = 0
    if kind in ("eval", "distil", "late") or (kind == "score" and rng.random() < 0.75):
        k = min(vocab, _log_int(rng, 1, 256))
    case = _case(kind, _log_int(rng, 1, 32768), vocab, dtype, k, rng.choice([0.5, 0.75, 1.0, 1.0, 1.5, 2.0, 4.0]),
                 entropy=rng.random() < 0.6, rest=rng.random() < 0.5, masked=rng.random() < 0.3, pad=rng.random() < 0.3)
    while work(case)["bytes"] > MAX_BYTES:
        case["n"] = int(case["n"] * 0.7)
    case["graph"] = kind == "score" and case["n"] <= 64 and rng.random() < 0.5
    return case


def _gradient(case):
    return case["kind"] in ("ce", "policy", "distil", "late")


def work(case):
    n, v, k = case["n"], case["vocab"], case["k"]
    e = 2 if case["dtype"] == "bf16" else 4
    each = v * e * (2 if _gradient(case) else 1)
    if case["kind"] in ("score", "ce", "policy"):
        each += 8 + 12 * k + 4 * (1 + case["entropy"]) * (2 if case["kind"] == "ce" else 1)
        each += 16 if case["kind"] == "policy" else 0
    else:
        each += 12 * k + 4 * case["rest"] + (8 if case["kind"] == "distil" else 4)
        each += 16 if case["kind"] == "late" else 0
    # a difference, a product, an exponential and a sum per logit, two more
    # with the entropy; the gradient takes an exponential and a product again
    ops = {"policy": 0, "late": 0}.get(case["kind"], 6 if case["entropy"] else 4) + (4 if _gradient(case) else 0)
    return {"bytes": float(n) * each, "flops": float(n) * v * ops}


# ------------------------------------------------------------------ inputs
PAD_VALUE = 4096.0   # in the columns between vocab and the pitch


def _empty(n, vocab, dtype, pad):
    ld = (vocab + 63) // 64 * 64 if pad else vocab
    return torch.empty((n, ld), dtype=dtype, device="cuda")[:, :vocab]


def _inputs(case, seed):
    n, v, k, T, kind = case["n"], case["vocab"], case["k"], case["T"], case["kind"]
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    at = dict(generator=g, device="cuda")
    logits = _empty(n, v, TYPES[case["dtype"]], case["pad"])
    if logits.stride(0) > v:
        torch.as_strided(logits, (n, logits.stride(0) - v), (logits.stride(0), 1), v).fill_(PAD_VALUE)
    s = {"case": case, "logits": logits}
    s["targets"] = torch.empty(n, dtype=torch.int64, device="cuda")
    teacher = kind in ("eval", "distil", "late")
    if teacher:
        s["t_ids"] = torch.empty((n, k), dtype=torch.int64, device="cuda")
        s["t_vals"] = torch.empty((n, k), device="cuda")
        s["t_lse"] = torch.empty(n, device="cuda") if case["rest"] else None
    step = max(1, (1 << 27) // v)
    for i in range(0, n, step):
        j = min(n, i + step)
        x = torch.randn((j - i, v), **at).mul_(2.0)
        # one in each eighth of the vocabulary
        raised = torch.randint(0, v // 8, (j - i, 8), **at) + torch.arange(8, device="cuda") * (v // 8)
        up = torch.linspace(4.0, 11.0, 8, device="cuda") + torch.randn((j - i, 8), **at)
        x.scatter_(1, raised, up)
        pick = torch.randint(0, 8, (j - i, 1), **at)
        s["targets"][i:j] = raised.gather(1, pick)[:, 0]
        banned = None
        if case["masked"]:
            banned = torch.rand((j - i, v), **at) < 1 / 128
            banned.scatter_(1, raised, False)
            x.masked_fill_(banned, -math.inf)
        if teacher:
            t = x * 0.9 + torch.randn((j - i, v), **at)
            top = torch.topk(t, k, dim=1)
            s["t_ids"][i:j], s["t_vals"][i:j] = top.indices, top.values
            if case["rest"]:
                s["t_lse"][i:j] = torch.logsumexp(t / T, dim=1)
            del t
        logits[i:j].copy_(x)
        del x, banned
    if kind == "ce":
        # one token in ten is padding and ignored
        pad = torch.rand(n, **at) < 0.1
        s["targets"][pad] = -100
        s["dlogp"] = torch.full((n,), -1.0 / n, device="cuda")
        s["dentropy"] = torch.full((n,), 0.01 / n, device="cuda") if case["entropy"] else None
    elif kind == "policy":
        s["dlogp"] = torch.randn(n, **at) / n
        s["dentropy"] = torch.randn(n, **at) / n if case["entropy"] else None
    elif teacher:
        # the mean over the batch, one token in ten left out
        s["dloss"] = torch.where(torch.rand(n, **at) < 0.1, 0.0, 1.0 / n).to(F32)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    n, v, k, kind = case["n"], case["vocab"], case["k"], case["kind"]
    vec = lambda *shape, dtype=F32: torch.empty((n,) + shape, dtype=dtype, device="cuda")   # noqa: E731
    s["logp"], s["entropy"], s["loss"] = vec(), vec() if case["entropy"] else None, vec()
    s["top_ids"], s["top_logp"] = (vec(k, dtype=torch.int64), vec(k)) if kind == "score" and k else (None, None)
    s["dlogits"] = _empty(n, v, s["logits"].dtype, case["pad"]) if _gradient(case) else None
    if kind in ("policy", "late"):
        # what the forward saved: {max, log sum, entropy, 0} of each row, and
        # {max, log sum} of the row and of its tokens outside the list
        s["stats"] = torch.zeros((n, 4), device="cuda")
        step = max(1, (1 << 27) // v)
        for i in range(0, n, step):
            j = min(n, i + step)
            x = s["logits"][i:j].to(F32)
            s["stats"][i:j, 0], s["stats"][i:j, 1], e, d = _statistics(x, case["T"])
            if kind == "policy":
                s["stats"][i:j, 2] = _entropy(s["stats"][i:j, 1], e, d)
            else:
                _, _, rest = _lists(s["t_ids"][i:j], v)
                s["stats"][i:j, 2], s["stats"][i:j, 3], _, _ = _statistics(torch.where(rest, x, -math.inf), case["T"])
    if case["graph"]:
        _pass(s)
        torch.cuda.synchronize()
        s["graph"] = torch.cuda.CUDAGraph()
        with torch.cuda.graph(s["graph"]):
            s["out"] = _pass(s)
    return s


def run(state):
    if "graph" in state:
        state["graph"].replay()
        return state["out"]
    return _pass(state)


def _pass(s):
    return _own(s) if own else _plain(s)


# ------------------------------------------------------- the framework's way
def _own(s):
    from paper_2502_10940_gb300 import cola

    case, kind = s["case"], s["case"]["kind"]
    d = s.get("desc")
    if d is None:
        grad = s["dlogits"].stride(0) if s["dlogits"] is not None else 0
        d = s["desc"] = cola.vocab_desc(case["n"], case["vocab"], ld=s["logits"].stride(0), ld_grad=grad,
                                        dtype=case["dtype"], temperature=case["T"], k=case["k"], rest=case["rest"],
                                        teacher_temperature=case["T"])
    x = s["logits"]
    if kind == "score":
        cola.cola_token_logprob_fwd(d, x, s["targets"], s["logp"], s["entropy"], s["top_ids"], s["top_logp"], None)
        return {"logp": s["logp"], "entropy": s["entropy"], "top_ids": s["top_ids"], "top_logp": s["top_logp"]}
    if kind == "ce":
        cola.cola_token_logprob_step(d, x, s["targets"], s["dlogp"], s["dentropy"], s["logp"], s["entropy"], s["dlogits"])
        return {"logp": s["logp"], "entropy": s["entropy"], "dlogits": s["dlogits"]}
    if kind == "policy":
        cola.cola_token_logprob_bwd(d, x, s["targets"], s["stats"], s["dlogp"], s["dentropy"], s["dlogits"])
        return {"dlogits": s["dlogits"]}
    if kind == "eval":
        cola.cola_topk_distill_fwd(d, x, s["t_ids"], s["t_vals"], s["t_lse"], s["loss"], None)
        return {"loss": s["loss"]}
    if kind == "distil":
        cola.cola_topk_distill_step(d, x, s["t_ids"], s["t_vals"], s["t_lse"], s["dloss"], s["loss"], s["dlogits"])
        return {"loss": s["loss"], "dlogits": s["dlogits"]}
    cola.cola_topk_distill_bwd(d, x, s["t_ids"], s["t_vals"], s["t_lse"], s["stats"], s["dloss"], s["dlogits"])
    return {"dlogits": s["dlogits"]}


# -------------------------------------------------------------- plain forms
def _statistics(x, T):
    """m = max x, log sum exp((x - m) / T), exp((x - m) / T) and (x - m) / T.
    A row of nothing but -inf: m = -inf, the sum's logarithm 0, no exponentials."""
    m = x.amax(dim=1)
    d = (x - torch.where(m == -math.inf, 0.0, m)[:, None]) / T
    e = torch.exp(d)
    return m, torch.where(m == -math.inf, 0.0, torch.log(e.sum(dim=1))), e, d


def _entropy(logs, e, d):
    """log s - sum p (x - m) / T, where p = 0 counts as 0."""
    return logs - torch.where(e == 0, 0.0, e * d).sum(dim=1) * torch.exp(-logs)


def _lists(ids, vocab):
    """Which entries are tokens, the ids with 0 in the others' place, and the
    rest of the vocabulary."""
    there = (ids >= 0) & (ids < vocab)
    safe = torch.where(there, ids, 0)
    hits = torch.zeros((ids.shape[0], vocab), dtype=torch.int32, device=ids.device)
    hits.scatter_add_(1, safe, there.to(torch.int32))
    return there, safe, hits == 0


def _top(x, k):
    """The k largest of each row, ties to the lowest id, NaN above all: by one
    whole number per logit that orders the value first and the id second."""
    bits = (x + 0.0).view(torch.int32).to(torch.int64)
    value = torch.where(bits >= 0, bits, -2147483648 - bits - 1)
    value = torch.where(torch.isnan(x), 2147483647, value)
    key = value * 4294967296 + (4294967295 - torch.arange(x.shape[1], device=x.device))
    return 4294967295 - (torch.topk(key, k, dim=1).values & 4294967295)


def _plain_logprob(s, gradient, stats=None):
    case = s["case"]
    x, T, v = s["logits"].to(F32), case["T"], case["vocab"]
    if stats is None:
        m, logs, e, d = _statistics(x, T)
        H = _entropy(logs, e, d)
    else:
        m, logs, H = stats[:, 0], stats[:, 1], stats[:, 2]
        d = (x - torch.where(m == -math.inf, 0.0, m)[:, None]) / T
    logp = d - logs[:, None]
    there = (s["targets"] >= 0) & (s["targets"] < v)
    y = torch.where(there, s["targets"], 0)[:, None]
    out = {}
    if stats is None:
        out["logp"] = torch.where(there, logp.gather(1, y)[:, 0], 0.0)
        out["entropy"] = torch.where(m == -math.inf, 0.0, H) if case["entropy"] else None
    if case["kind"] == "score":
        out["top_ids"] = out["top_logp"] = None
        if case["k"]:
            out["top_ids"] = _top(x, case["k"])
            out["top_logp"] = logp.gather(1, out["top_ids"])
    if gradient:
        p = torch.exp(logp)
        g = torch.where(there, s["dlogp"], 0.0)
        dx = -g[:, None] * p
        live = (g != 0) & (m != -math.inf)
        if s["dentropy"] is not None:
            dx -= s["dentropy"][:, None] * torch.where(p == 0, 0.0, p * (logp + H[:, None]))
            live = ((g != 0) | (s["dentropy"] != 0)) & (m != -math.inf)
        dx.scatter_add_(1, y, g[:, None])
        out["dlogits"] = torch.where(live[:, None], dx / T, 0.0).to(s["logits"].dtype)
    return out


def _plain_distill(s, gradient, stats=None):
    case = s["case"]
    x, T, v = s["logits"].to(F32), case["T"], case["vocab"]
    there, ids, rest = _lists(s["t_ids"], v)
    u = s["t_vals"] / T
    if case["rest"]:
        q = torch.where(there, torch.exp(u - s["t_lse"][:, None]), 0.0)
        logq = u - s["t_lse"][:, None]
    else:
        u = torch.where(there, u, -math.inf)
        um, ulogs, ue, ud = _statistics(u, T=1.0)
        logq = ud - ulogs[:, None]
        q = torch.where(there, torch.exp(logq), 0.0)
    if stats is None:
        m, logs, _, _ = _statistics(x, T)
        mr, logr, er, dr = _statistics(torch.where(rest, x, -math.inf), T)
    else:
        m, logs, mr, logr = stats.unbind(1)
        dr = (torch.where(rest, x, -math.inf) - torch.where(mr == -math.inf, 0.0, mr)[:, None]) / T
    m0 = torch.where(m == -math.inf, 0.0, m)
    logp = (x.gather(1, ids) - m0[:, None]) / T - logs[:, None]
    logpr = (mr - m0) / T + logr - logs
    p = torch.where(there, torch.exp(logp), 0.0)
    qr = torch.zeros_like(m)
    if case["rest"]:
        qr = torch.where(mr == -math.inf, 0.0, (1 - q.sum(dim=1)).clamp(min=0.0))
    entry = qr > 0
    out = {}
    if stats is None:
        plain = torch.where(q > 0, q * (logq - logp), 0.0 * q).sum(dim=1)
        whole = torch.where(q > 0, q * _excess(logq - logp), p).sum(dim=1)
        whole += qr * _excess(torch.log1p(-torch.where(entry, q.sum(dim=1), 0.0)) - torch.where(entry, logpr, 0.0))
        out["loss"] = T * T * torch.where(entry, whole, plain)
    if gradient:
        w, Q = s["dloss"], torch.where(entry, 1.0, q.sum(dim=1))
        pr = torch.exp(logpr)
        rate = torch.where(entry, (q - p).sum(dim=1), Q * pr)
        dx = (w * T * rate)[:, None] * torch.exp(dr - logr[:, None])
        at = torch.where(there, (w * T)[:, None] * (Q[:, None] * p - q), 0.0)
        dx.scatter_add_(1, ids, at)
        out["dlogits"] = torch.where(((w != 0) & (m != -math.inf))[:, None], dx, 0.0).to(s["logits"].dtype)
    return out


def _excess(r):
    """r + exp(-r) - 1 >= 0.  Where q and p both sum to 1, KL(q || p) is the sum
    of q excess(log q / p): no terms of both signs that nearly cancel."""
    near = r * r * (0.5 - r * (1 / 6 - r * (1 / 24 - r * (1 / 120 - r * (1 / 720 - r / 5040)))))
    return torch.where(r.abs() < 0.3, near, r + torch.expm1(-r))


def _plain(s):
    kind = s["case"]["kind"]
    if kind in ("score", "ce", "policy"):
        return _plain_logprob(s, kind != "score", s["stats"] if kind == "policy" else None)
    return _plain_distill(s, kind != "eval", s["stats"] if kind == "late" else None)


# ------------------------------------------------------------------- exact
def exact(case, seed):
    """By the definitions, in 64 bits, a few rows at a time."""
    s = _inputs(case, seed)
    n, v, T, kind = case["n"], case["vocab"], case["T"], case["kind"]
    parts = []
    step = max(1, (1 << 26) // v)
    for i in range(0, n, step):
        r = slice(i, min(n, i + step))
        z = s["logits"][r].double() / T
        lp = z - torch.logsumexp(z, dim=1, keepdim=True)
        p = lp.exp()
        o = {}
        if kind in ("score", "ce", "policy"):
            H = -torch.special.xlogy(p, p).sum(dim=1)
            y = s["targets"][r]
            used = (y >= 0) & (y < v)
            if kind != "policy":
                o["logp"] = torch.where(used, lp.gather(1, y.clamp(0, v - 1)[:, None])[:, 0], 0.0)
                o["entropy"] = H if case["entropy"] else None
            if kind == "score":
                o["top_ids"] = o["top_logp"] = None
                if case["k"]:
                    best = torch.sort(s["logits"][r].double(), dim=1, descending=True, stable=True).indices[:, :case["k"]]
                    o["top_ids"], o["top_logp"] = best, lp.gather(1, best)
            else:
                g = torch.where(used, s["dlogp"][r].double(), 0.0)
                hit = torch.arange(v, device="cuda")[None, :] == y[:, None]
                dx = g[:, None] * (hit.double() - p)
                if s["dentropy"] is not None:
                    dx -= s["dentropy"][r].double()[:, None] * (torch.special.xlogy(p, p) + p * H[:, None])
                o["dlogits"] = dx / T
        else:
            ids, t = s["t_ids"][r], s["t_vals"][r].double() / T
            used = (ids >= 0) & (ids < v)
            if case["rest"]:
                q = torch.where(used, (t - s["t_lse"][r].double()[:, None]).exp(), 0.0)
            else:
                q = torch.softmax(torch.where(used, t, -math.inf), dim=1)
            outside = torch.ones_like(p).scatter_(1, ids.clamp(0, v - 1), 0.0)
            if not bool(used.all()):
                return None
            qr = (1 - q.sum(dim=1)).clamp(min=0.0) if case["rest"] else torch.zeros_like(q[:, 0])
            lpr = torch.logsumexp(torch.where(outside > 0, lp, -math.inf), dim=1)
            qr = torch.where(lpr == -math.inf, 0.0, qr)
            if kind != "late":
                kl = (torch.special.xlogy(q, q) - torch.where(q > 0, q * lp.gather(1, ids), 0.0)).sum(dim=1)
                kl += torch.special.xlogy(qr, qr) - torch.where(qr > 0, qr * lpr, 0.0)
                o["loss"] = T * T * kl
            if kind != "eval":
                whole = q.sum(dim=1) + qr
                want = torch.zeros_like(p).scatter_add_(1, ids, q)
                want += (lp - lpr[:, None]).exp() * outside * qr[:, None]
                o["dlogits"] = (s["dloss"][r].double() * T)[:, None] * (whole[:, None] * p - want)
        parts.append(o)
    return {key: None if parts[0][key] is None else torch.cat([o[key] for o in parts]) for key in parts[0]}
