"""Measured cases of the operators at the vocabulary's two ends that stand
beside its log probabilities and distillation: how token ids become the first
layer's input, what the embedding table learns from it, and what a server
imposes on logits before a token is taken from them.

  embed    X = scale E[ids], the input of the first block (cola_embed_fwd)
  grad     dE of it: for each token of the vocabulary the sum of dX over the
           rows that named it, overwritten or accumulated (cola_embed_bwd)
  limit    penalties for tokens that occurred, biases and grammar masks on
           rows of logits (cola_constrain_logits_fwd)
  policy   the gradient through those (cola_constrain_logits_bwd)

Ids outside the vocabulary name no token: their rows of X are 0, their rows of
dX unused.  Constraints, in this order, for a logit x of a token that occurs c
times in the row's history after its prompt:
  x > 0 ? x / repetition : x repetition    where the whole history has it
  x - frequency c - presence [c > 0] + the sum of its entries among the biases
  -inf where the row's mask has a 0 bit for it.
The gradient is that of the first line, and 0 where masked.

Token frequencies follow a Zipf law; ids in its order, as byte-pair vocabularies
have them, or "mixed".
"""
import math

import torch

own = False
F32 = torch.float32
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _embed(kind, n, vocab, d, types, *, scale=1.0, padding=0.0, pad=False, mixed=False, micro=0, graph=False, **name):
    """types: of E (embed) or dE (grad), and of X or dX."""
    return dict(name, kind=kind, n=n, vocab=vocab, d=d, types=types, scale=scale, padding=padding, pad=pad, mixed=mixed,
                micro=micro, graph=graph)


def _limit(kind, n, vocab, dtype, history, *, biases=0, masks=0.0, pad=False, mixed=False, graph=False, **name):
    """masks: the share of rows that have one."""
    return dict(name, kind=kind, n=n, vocab=vocab, dtype=dtype, history=history, biases=biases, masks=masks, pad=pad,
                mixed=mixed, graph=graph)


def listed():
    return [
        # serving, the next token of each of 32 sequences, replayed with the
        # decode step's graph
        _embed("embed", 32, 32000, 4096, "bf16 bf16", graph=True, name="embed_decode_n32"),
        # pre-training, 128 x 256 tokens
        _embed("embed", 32768, 32000, 2048, "bf16 bf16", name="embed_step_n32768"),
        # fp32 master table, scaled by the root of an odd width, some padding
        _embed("embed", 8191, 50021, 1000, "f32 bf16", scale=1000 ** 0.5, padding=0.1, pad=True, name="embed_scaled_f32"),
        # fine-tuning: four short micro-batches into one fp32 gradient
        _embed("grad", 2048, 32000, 512, "f32 bf16", micro=4, padding=0.1, name="grad_micro_f32"),
        # pre-training, 128 x 256 tokens
        _embed("grad", 32768, 32000, 2048, "bf16 bf16", name="grad_step_n32768"),
        # odd sizes, a scaled embedding, fp32 gradient
        _embed("grad", 8191, 50021, 1000, "f32 f32", scale=1000 ** 0.5, padding=0.1, pad=True, mixed=True, name="grad_odd_f32"),
        # pre-training, 512 x 256 tokens of the widest model
        _embed("grad", 131072, 32000, 4096, "bf16 bf16", name="grad_step_n131072"),
        # serving, one user: penalties over a long answer, a few biases
        _limit("limit", 1, 128000, "bf16", 2048, biases=20, graph=True, name="limit_n1"),
        # serving, 32 users over fp32 logits of an odd vocabulary, long
        # histories, half of the rows under a grammar
        _limit("limit", 32, 50021, "f32", 32768, biases=8, masks=0.5, mixed=True, name="limit_n32_long"),
        # serving, a large batch, a quarter of it under a grammar
        _limit("limit", 256, 128000, "bf16", 4096, biases=20, masks=0.25, name="limit_n256"),
        # policy gradient of answers that were sampled under constraints
        _limit("policy", 4096, 32000, "bf16", 1024, masks=0.25, name="policy_n4096"),
        # the same of one prompt over fp32 logits, odd sizes
        _limit("policy", 509, 50021, "f32", 4096, masks=0.5, pad=True, mixed=True, name="policy_odd_f32"),
    ]


MAX_BYTES = 1.3e9   # of one drawn pass: no more than the largest listed case


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["embed", "embed", "grad", "grad", "grad", "limit", "limit", "limit", "policy"])
    vocab = _log_int(rng, 250, 262144)
    vocab = vocab // 64 * 64 if rng.random() < 0.4 and vocab >= 64 else vocab
    pad, mixed = rng.random() < 0.3, rng.random() < 0.5
    if kind in ("embed", "grad"):
        d = _log_int(rng, 64, 8192)
        d = d // 64 * 64 if rng.random() < 0.6 else d
        micro = rng.randint(1, 4) if kind == "grad" and rng.random() < 0.3 else 0
        types = ("f32" if micro else rng.choice(["bf16", "bf16", "f32"])) + " " + rng.choice(["bf16", "bf16", "f32"])
        case = _embed(kind, _log_int(rng, 1, 131072), vocab, d, types, scale=rng.choice([1.0, 1.0, d ** 0.5]),
                      padding=rng.choice([0.0, 0.1]), pad=pad, mixed=mixed, micro=micro)
    else:
        case = _limit(kind, _log_int(rng, 1, 4096), vocab, rng.choice(["bf16", "bf16", "f32"]), _log_int(rng, 1, 32768),
                      biases=rng.choice([0, 1, 20, 300]) if kind == "limit" else 0, masks=rng.choice([0.0, 0.25, 1.0]), pad=pad,
                      mixed=mixed)
    while work(case)["bytes"] > MAX_BYTES:
        key = "n" if case["n"] > 1 else "vocab"
        case[key] = max(1, int(case[key] * 0.7))
    case["graph"] = case["n"] <= 64 and kind in ("embed", "limit") and rng.random() < 0.5
    return case


def _frequencies(vocab):
    w = (torch.arange(vocab, dtype=torch.float64) + 3.0) ** -1.05
    return w / w.sum()


def _distinct(case):
    """The tokens that n draws are expected to name."""
    n = case["n"] * (1 - case["padding"])
    return float((1 - torch.exp(n * torch.log1p(-_frequencies(case["vocab"]).clamp(max=1 - 1e-9)))).sum())


def work(case):
    n, v = case["n"], case["vocab"]
    if case["kind"] in ("embed", "grad"):
        d, (e, x) = case["d"], (2 if t == "bf16" else 4 for t in case["types"].split())
        if case["kind"] == "embed":
            return {"bytes": 8.0 * n + _distinct(case) * d * e + float(n) * d * x, "flops": float(n) * d}
        passes = max(1, case["micro"])
        each = n * (8.0 + d * x * (1 - case["padding"])) + (_distinct(case) * d * e * 2 if case["micro"] else 0)
        return {"bytes": passes * each + float(v) * d * e, "flops": float(passes) * n * d}
    e = 2 if case["dtype"] == "bf16" else 4
    # half of the masks leave little, half ban little
    read = 1 - 0.5 * case["masks"]
    each = v * e * (1 + read) + case["masks"] * v / 8 + 8 * 0.75 * case["history"] + 12 * case["biases"] + 28
    return {"bytes": float(n) * each, "flops": float(n) * v}


# ------------------------------------------------------------------ inputs
PAD_VALUE = 4096.0   # in the columns between a row's width and its pitch


def _rows(n, width, dtype, pad, unit):
    """n rows at a pitch that is a multiple of `unit`, `pad`ded further or not."""
    ld = -(-width // unit) * unit
    ld = -(-ld // 64) * 64 + 64 if pad else ld
    buf = torch.full((n, ld), PAD_VALUE, dtype=dtype, device="cuda")
    return buf[:, :width]


def _tokens(case, shape, at):
    """Token ids by the Zipf law."""
    total = torch.cumsum(_frequencies(case["vocab"]).cuda(), 0)
    ids = torch.searchsorted(total, torch.rand(shape, dtype=torch.float64, **at)).clamp_(max=case["vocab"] - 1)
    if case["mixed"]:
        ids = torch.randperm(case["vocab"], **at)[ids]
    return ids


def _embed_inputs(case, at):
    n, v, d, kind = case["n"], case["vocab"], case["d"], case["kind"]
    t_e, t_x = (TYPES[t] for t in case["types"].split())
    s = {"case": case, "E": None, "dX": None, "X": None, "dE": None}
    shape = (max(1, case["micro"]), n)
    ids = _tokens(case, shape, at)
    # padding: at the ends of sequences, told by ids of no token
    ids = torch.where(torch.rand(shape, **at) < case["padding"], -100, ids)
    s["ids"] = ids if case["micro"] else ids[0]
    if kind == "embed":
        s["E"] = _rows(v, d, t_e, case["pad"], 8)
        s["E"].copy_(torch.randn((v, d), **at) * d ** -0.5)
        s["X"] = _rows(n, d, t_x, case["pad"], 8)
    else:
        s["dX"] = [_rows(n, d, t_x, case["pad"], 8) for _ in range(shape[0])]
        for m in s["dX"]:
            m.copy_(torch.randn((n, d), **at) * (torch.rand((n, 1), **at) + 0.5))
        s["dE"] = _rows(v, d, t_e, case["pad"], 8)
    return s


def _limit_inputs(case, at):
    n, v, h, kind = case["n"], case["vocab"], case["history"], case["kind"]
    s = {"case": case, "bias_ids": None, "bias": None, "masks": None, "mask_of": None, "dout": None, "dlogits": None, "out": None}
    s["logits"] = _rows(n, v, TYPES[case["dtype"]], case["pad"], 1)
    s["logits"].copy_(torch.randn((n, v), **at).mul_(2.0))
    s["history"] = _tokens(case, (n, h), at)
    # between half and all of the longest; the prompt a third of it or so
    s["history_len"] = torch.randint((h + 1) // 2, h + 1, (n,), **at)
    s["prompt_len"] = (s["history_len"] * torch.rand(n, **at) * 0.66).to(torch.int64)
    uniform = lambda lo, hi: torch.rand(n, **at) * (hi - lo) + lo   # noqa: E731
    s["repetition"], s["frequency"], s["presence"] = uniform(1.0, 1.3), uniform(0.0, 0.5), uniform(0.0, 0.5)
    if case["biases"]:
        s["bias_ids"] = torch.randint(0, v, (n, case["biases"]), **at)
        s["bias"] = torch.randn((n, case["biases"]), **at) * 4
    if case["masks"]:
        # a grammar's states in turn: few tokens allowed, few banned
        count = max(1, round(n * case["masks"]))
        s["masks"] = torch.empty((count, (v + 31) // 32), dtype=torch.int32, device="cuda")
        for i in range(0, count, 256):
            some = s["masks"][i:i + 256]
            share = torch.where(torch.arange(i, i + len(some), device="cuda") % 2 == 0, 0.004, 0.95)
            bits = torch.rand((len(some), some.shape[1], 32), **at) < share[:, None, None]
            some.copy_((bits.to(torch.int64) << torch.arange(32, device="cuda")).sum(-1).to(torch.int32))
        s["mask_of"] = torch.full((n,), -1, dtype=torch.int64, device="cuda")
        s["mask_of"][torch.randperm(n, **at)[:count]] = torch.arange(count, device="cuda")
    like = lambda: _rows(n, v, TYPES[case["dtype"]], case["pad"], 1)   # noqa: E731
    if kind == "limit":
        s["out"] = like()
    else:
        s["dout"], s["dlogits"] = like(), like()
        s["dout"].copy_(torch.randn((n, v), **at) / n)
    return s


def _inputs(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    at = dict(generator=g, device="cuda")
    return _embed_inputs(case, at) if case["kind"] in ("embed", "grad") else _limit_inputs(case, at)


def prepare(case, seed):
    s = _inputs(case, seed)
    if case["graph"]:
        _pass(s)
        torch.cuda.synchronize()
        s["graph"] = torch.cuda.CUDAGraph()
        with torch.cuda.graph(s["graph"]):
            s["result"] = _pass(s)
    return s


def run(state):
    if "graph" in state:
        state["graph"].replay()
        return state["result"]
    return _pass(state)


def _pass(s):
    return _own(s) if own else _plain(s)


# ------------------------------------------------------- the framework's way
def _own(s):
    from paper_2502_10940_gb300 import cola

    case, kind = s["case"], s["case"]["kind"]
    if kind in ("embed", "grad"):
        if "desc" not in s:
            t_e, t_x = case["types"].split()
            pitch = lambda t: t.stride(0) if t is not None else 0   # noqa: E731
            s["desc"] = cola.embed_desc(case["n"], case["vocab"], case["d"], ld_e=pitch(s["E"]),
                                        ld_x=pitch(s["X"] if kind == "embed" else s["dX"][0]), ld_de=pitch(s["dE"]),
                                        scale=case["scale"], dtype_e=t_e, dtype_x=t_x, dtype_de=t_e)
            s["ws"] = cola.embed_workspace(s["desc"]) if kind == "grad" else None
        if kind == "embed":
            cola.cola_embed_fwd(s["desc"], s["E"], s["ids"], s["X"])
            return {"X": s["X"]}
        s["desc"].accumulate = 0   # the first micro-batch overwrites, the others add
        for ids, dX in zip(s["ids"] if case["micro"] else [s["ids"]], s["dX"]):
            cola.cola_embed_bwd(s["desc"], ids, dX, s["dE"], s["ws"])
            s["desc"].accumulate = 1
        return {"dE": s["dE"]}
    if "desc" not in s:
        result = s["out"] if kind == "limit" else s["dlogits"]
        s["desc"] = cola.vocab_desc(case["n"], case["vocab"], ld=s["logits"].stride(0), ld_grad=result.stride(0),
                                    dtype=case["dtype"])
        s["limits"] = cola.constraints(s["history"], s["history_len"], s["prompt_len"], repetition=s["repetition"],
                                       frequency=s["frequency"], presence=s["presence"], bias_ids=s["bias_ids"],
                                       bias=s["bias"], masks=s["masks"], mask_of=s["mask_of"])
    if kind == "limit":
        cola.cola_constrain_logits_fwd(s["desc"], s["limits"], s["logits"], s["out"])
        return {"out": s["out"]}
    cola.cola_constrain_logits_bwd(s["desc"], s["limits"], s["logits"], s["dout"], s["dlogits"])
    return {"dlogits": s["dlogits"]}


# -------------------------------------------------------------- plain forms
def _plain_embed(s):
    case, ids = s["case"], s["ids"].reshape(-1)
    v, d = case["vocab"], case["d"]
    there = (ids >= 0) & (ids < v)
    if case["kind"] == "embed":
        x = s["E"].index_select(0, torch.where(there, ids, 0)).to(F32) * case["scale"]
        return {"X": torch.where(there[:, None], x, 0.0).to(s["X"].dtype)}
    dX = torch.cat(s["dX"]) if case["micro"] else s["dX"][0]
    total = torch.zeros((v + 1, d), device=ids.device)          # ids of no token: the row behind the last
    total.index_add_(0, torch.where(there, ids, v), dX.to(F32))
    return {"dE": (total[:v] * case["scale"]).to(s["dE"].dtype)}


def _banned(s):
    """Where the rows' masks have a 0 bit, or None."""
    if s["masks"] is None:
        return None
    at = torch.arange(s["case"]["vocab"], device="cuda")
    has = (s["mask_of"] >= 0) & (s["mask_of"] < len(s["masks"]))
    words = s["masks"].index_select(0, torch.where(has, s["mask_of"], 0))
    allowed = (words.index_select(1, at // 32) >> (at % 32).to(torch.int32)) & 1
    return has[:, None] & (allowed == 0)


def _occurrences(s, first):
    """How often each token occurs in each row's history from `first` on."""
    n, v, h = s["case"]["n"], s["case"]["vocab"], s["case"]["history"]
    at = torch.arange(h, device="cuda")[None, :]
    count = (at >= first[:, None]) & (at < s["history_len"][:, None])
    return torch.zeros((n, v), device="cuda").scatter_add_(1, s["history"], count.to(F32))


def _plain_limit(s):
    case = s["case"]
    x = s["logits"].to(F32)
    seen = _occurrences(s, torch.zeros_like(s["prompt_len"])) > 0
    r = s["repetition"][:, None]
    banned = _banned(s)
    if case["kind"] == "policy":
        g = s["dout"].to(F32)
        g = torch.where(seen, torch.where(x > 0, g / r, g * r), g)
        g = g if banned is None else torch.where(banned, 0.0, g)
        return {"dlogits": g.to(s["dlogits"].dtype)}
    x = torch.where(seen, torch.where(x > 0, x / r, x * r), x)
    count = _occurrences(s, s["prompt_len"])
    x = x - s["frequency"][:, None] * count - s["presence"][:, None] * (count > 0)
    if case["biases"]:
        x = x + torch.zeros_like(x).scatter_add_(1, s["bias_ids"], s["bias"])
    x = x if banned is None else torch.where(banned, -math.inf, x)
    return {"out": x.to(s["out"].dtype)}


def _plain(s):
    return _plain_embed(s) if s["case"]["kind"] in ("embed", "grad") else _plain_limit(s)


# ------------------------------------------------------------------- exact
def exact(case, seed):
    """By the definitions, in 64 bits: sums by token, logits a row at a time."""
    s = _inputs(case, seed)
    n, v, kind = case["n"], case["vocab"], case["kind"]
    if kind == "embed":
        X = torch.zeros(s["X"].shape, dtype=torch.float64, device="cuda")
        used = s["ids"] >= 0
        X[used] = s["E"][s["ids"][used]].double() * case["scale"]
        return {"X": X}
    if kind == "grad":
        dE = torch.zeros(s["dE"].shape, dtype=torch.float64, device="cuda")
        for ids, dX in zip(s["ids"].view(-1, n), s["dX"]):
            used = ids >= 0
            dE.index_put_((ids[used],), dX[used].double(), accumulate=True)
        return {"dE": dE.mul_(case["scale"])}
    rows = []
    length, prompt = s["history_len"].tolist(), s["prompt_len"].tolist()
    mask_of = s["mask_of"].tolist() if s["mask_of"] is not None else [-1] * n
    shifts = torch.arange(32, device="cuda")
    for i in range(n):
        x = s["logits"][i].double()
        whole = torch.bincount(s["history"][i, :length[i]], minlength=v)
        answer = torch.bincount(s["history"][i, prompt[i]:length[i]], minlength=v)
        r = s["repetition"][i].double()
        factor = torch.where(whole > 0, torch.where(x > 0, 1 / r, r), 1.0)
        if kind == "limit":
            y = x * factor - answer * s["frequency"][i].double() - answer.clamp(max=1) * s["presence"][i].double()
            if case["biases"]:
                y.index_put_((s["bias_ids"][i],), s["bias"][i].double(), accumulate=True)
        else:
            y = s["dout"][i].double() * factor
        if mask_of[i] >= 0:
            bits = (s["masks"][mask_of[i]].to(torch.int64)[:, None] >> shifts & 1).reshape(-1)[:v]
            y[bits == 0] = -math.inf if kind == "limit" else 0.0
        rows.append(y)
    return {"out" if kind == "limit" else "dlogits": torch.stack(rows)}
