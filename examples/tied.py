#!/usr/bin/env python3
"""A model with a tied embedding around one CoLA layer: trained on a made-up
language, then asked for text under constraints.  The layer, the vocabulary
operators at both ends and the embedding together, as programs have them.

  train     X = scale E[ids] (cola_embed_fwd), h = X + B sigma(A x) (cola_fwd),
            logits = h E^T
            -> cola_token_logprob_step: cross entropy and its gradient, over the logits
            -> cola_bwd: dA, dB, dX;  dE = dlogits^T h, then cola_embed_bwd adds the
               lookup's gradient to it
  generate  a token of each sequence at a time: cola_constrain_logits_fwd in place
            (penalties for what the sequence has, a grammar's mask),
            cola_token_logprob_fwd for the likeliest token, cola_embed_fwd of it;
            one step captured in a CUDA graph

The products with E are plain matrix products of the caller.  The language: the
next token is a fixed permutation of the last, or any token one time in four.

    python examples/tied.py [--tokens N] [--dim D] [--vocab V] [--rank R] [--steps S] [--sequences B] [--length L]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2502_10940_gb300 import cola   # noqa: E402

BF = dict(dtype=torch.bfloat16, device="cuda")


class Model:
    """fp32 parameters E [vocab x dim], A [rank x dim], B [dim x rank], and their gradients."""

    def __init__(self, vocab, dim, rank, g):
        rnd = lambda *s, std: torch.randn(s, generator=g, device="cuda").mul_(std)   # noqa: E731
        self.vocab, self.dim, self.rank, self.scale = vocab, dim, rank, dim ** 0.5
        self.params = [rnd(vocab, dim, std=dim ** -0.5), rnd(rank, dim, std=dim ** -0.5), rnd(dim, rank, std=0.5 * rank ** -0.5)]
        self.grads = [torch.zeros_like(p) for p in self.params]

    def plan(self, n):
        """What a call on n tokens needs."""
        s = dict(n=n, embed=cola.embed_desc(n, self.vocab, self.dim, scale=self.scale, dtype_de="f32", accumulate=True),
                 layer=cola.desc(n, self.dim, self.dim, self.rank, sigma="silu", mode="cola_m", wgrad_fp32=True),
                 rows=cola.vocab_desc(n, self.vocab), X=torch.empty((n, self.dim), **BF), Y=torch.empty((n, self.dim), **BF),
                 Z=torch.empty((n, self.rank), **BF), dX=torch.empty((n, self.dim), **BF))
        s["layer_ws"], s["embed_ws"] = cola.workspace(s["layer"]), cola.embed_workspace(s["embed"])
        return s

    def weights(self):
        return [p.to(torch.bfloat16) for p in self.params]

    def forward(self, s, w, ids):
        """The last activation and its logits."""
        cola.cola_embed_fwd(s["embed"], w[0], ids, s["X"])
        cola.cola_fwd(s["layer"], s["X"], w[1], w[2], s["Y"], s["Z"], None, s["layer_ws"])
        h = s["X"] + s["Y"]
        return h, torch.matmul(h, w[0].T)

    def step(self, s, ids, targets):
        """Mean loss of the tokens; the gradients are overwritten."""
        w = self.weights()
        h, logits = self.forward(s, w, ids)
        logp, up = torch.empty(s["n"], device="cuda"), torch.full((s["n"],), -1.0 / s["n"], device="cuda")
        cola.cola_token_logprob_step(s["rows"], logits, targets, up, None, logp, None, logits)   # now their gradient
        dh = torch.matmul(logits, w[0])
        for g in self.grads[1:]:
            g.zero_()
        cola.cola_bwd(s["layer"], s["X"], w[1], w[2], dh, s["Z"], None, s["dX"], self.grads[1], self.grads[2], s["layer_ws"])
        self.grads[0].copy_(torch.matmul(logits.T, h))
        cola.cola_embed_bwd(s["embed"], ids, s["dX"] + dh, self.grads[0], s["embed_ws"])
        return -logp.mean()


def generate(model, sequences, length, allowed, g):
    """`length` tokens for each of `sequences`, the likeliest of those that `allowed`
    [vocab] leaves under penalties; the tokens and their log probabilities."""
    s, w = model.plan(sequences), model.weights()
    mask = torch.zeros(-(-model.vocab // 32) * 32, dtype=torch.int64, device="cuda")
    mask[:model.vocab] = allowed
    words = (mask.view(-1, 32) << torch.arange(32, device="cuda")).sum(1).to(torch.int32)[None, :]
    history = torch.full((sequences, length + 1), -1, dtype=torch.int64, device="cuda")   # ids of no token: not there yet
    history[:, 0] = torch.randint(0, model.vocab, (sequences,), generator=g, device="cuda")
    per_row = lambda v: torch.full((sequences,), v, device="cuda")   # noqa: E731
    limits = cola.constraints(history, repetition=per_row(1.2), frequency=per_row(0.3), presence=per_row(0.2), masks=words,
                              mask_of=torch.zeros(sequences, dtype=torch.int64, device="cuda"))
    rows = cola.vocab_desc(sequences, model.vocab, k=1)
    best, logp = torch.empty((sequences, 1), dtype=torch.int64, device="cuda"), torch.empty((sequences, 1), device="cuda")
    last, at = history[:, 0].clone(), torch.ones(1, dtype=torch.int64, device="cuda")
    logps = torch.zeros((sequences, length + 1), device="cuda")

    def token():
        _, logits = model.forward(s, w, last)
        cola.cola_constrain_logits_fwd(rows, limits, logits, logits)
        cola.cola_token_logprob_fwd(rows, logits, None, None, None, best, logp, None)
        last.copy_(best[:, 0])
        history.index_copy_(1, at, best)
        logps.index_copy_(1, at, logp)
        at.add_(1)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        token()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        token()
    for _ in range(length - 1):
        graph.replay()
    return history[:, 1:], logps[:, 1:]


def main(tokens=4096, dim=256, vocab=4096, rank=128, steps=100, sequences=16, length=24, lr=4e-3, seed=0, log=print):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    model = Model(vocab, dim, rank, g)
    for p, d in zip(model.params, model.grads):
        p.grad = d
    adam = torch.optim.Adam(model.params, lr=lr)
    follows = torch.randperm(vocab, generator=g, device="cuda")
    s = model.plan(tokens)
    losses = []
    for step in range(steps):
        ids = torch.randint(0, vocab, (tokens,), generator=g, device="cuda")
        any_one = torch.randint(0, vocab, (tokens,), generator=g, device="cuda")
        targets = torch.where(torch.rand(tokens, generator=g, device="cuda") < 0.25, any_one, follows[ids])
        loss = model.step(s, ids, targets)
        adam.step()
        if step % 20 == 0 or step == steps - 1:
            losses.append(loss.item())
            log(f"step {step:4d}  loss {losses[-1]:.4f}")
    for ws in (s["layer_ws"], s["embed_ws"]):
        status, code = cola.cola_check_status(ws)
        if status:
            raise RuntimeError(f"device status {status} code {code}")
    allowed = torch.rand(vocab, generator=g, device="cuda") < 0.9
    text, logp = generate(model, sequences, length, allowed, g)
    log(f"{sequences} sequences of {length} tokens, mean log p {logp.mean().item():.3f}, all allowed: {bool(allowed[text].all())}")
    return {"loss": losses, "text": text, "logp": logp, "allowed": allowed}


if __name__ == "__main__":
    p = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    for name, default in (("tokens", 4096), ("dim", 256), ("vocab", 4096), ("rank", 128), ("steps", 100), ("sequences", 16), ("length", 24)):
        p.add_argument(f"--{name}", type=int, default=default)
    main(**vars(p.parse_args()))
