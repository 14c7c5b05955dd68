#!/usr/bin/env python3
"""Distils a full-rank projection into a CoLA layer through the vocabulary: the
layer calls and the vocabulary operators together, as a training program has
them.

  teacher   Y = X W^T, logits = Y E^T (E: the output embedding, full-rank, shared)
            -> cola_token_logprob_fwd: its k most likely tokens per row and their
               log probabilities at temperature T, once
  student   h = B sigma(A x) (cola_fwd), logits = h E^T
            -> cola_topk_distill_step: loss and its gradient, over the logits in place
            -> dh = dlogits E, cola_bwd: dA, dB
  check     cola_token_logprob_fwd over the student's logits: log probability of the
            teacher's best token, entropy, and how often the two agree on it

The products with E and W are plain matrix products of the caller.

    python examples/distill.py [--tokens N] [--dim D] [--vocab V] [--rank R] [--top K] [--temperature T] [--steps S]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2502_10940_gb300 import cola   # noqa: E402


def main(tokens=4096, dim=512, vocab=32000, rank=128, top=32, temperature=2.0, steps=60, lr=2e-3, seed=0, log=print):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    bf = dict(dtype=torch.bfloat16, device="cuda")
    rnd = lambda *s, std=1.0: torch.randn(s, generator=g, device="cuda").mul_(std).to(torch.bfloat16)   # noqa: E731
    X, E, W = rnd(tokens, dim), rnd(vocab, dim, std=3.0 * dim ** -0.5), rnd(dim, dim, std=dim ** -0.5)

    # the teacher's list, taken once
    per_row = lambda *s, dtype=torch.float32: torch.empty((tokens,) + s, dtype=dtype, device="cuda")   # noqa: E731
    ids, logq = per_row(top, dtype=torch.int64), per_row(top)
    v = cola.vocab_desc(tokens, vocab, temperature=temperature, k=top, rest=True)
    cola.cola_token_logprob_fwd(v, torch.matmul(torch.matmul(X, W.T), E.T), None, None, None, ids, logq, None)
    best = ids[:, 0].contiguous()

    # the student: one CoLA layer, fp32 master factors
    A = rnd(rank, dim, std=dim ** -0.5).float().requires_grad_()
    B = rnd(dim, rank, std=rank ** -0.5).float().requires_grad_()
    adam = torch.optim.Adam([A, B], lr=lr)
    d = cola.desc(tokens, dim, dim, rank, sigma="silu", mode="cola_m", wgrad_fp32=True)
    ws = cola.workspace(d)
    Y, Z, dX = torch.empty((tokens, dim), **bf), torch.empty((tokens, rank), **bf), torch.empty((tokens, dim), **bf)
    loss, weight = per_row(), torch.full((tokens,), 1.0 / tokens, device="cuda")
    history = []
    for step in range(steps):
        Ab, Bb = A.detach().to(torch.bfloat16), B.detach().to(torch.bfloat16)
        cola.cola_fwd(d, X, Ab, Bb, Y, Z, None, ws)
        logits = torch.matmul(Y, E.T)
        cola.cola_topk_distill_step(v, logits, ids, logq, None, weight, loss, logits)   # logits become their gradient
        A.grad, B.grad = torch.zeros_like(A), torch.zeros_like(B)
        cola.cola_bwd(d, X, Ab, Bb, torch.matmul(logits, E), Z, None, dX, A.grad, B.grad, ws)
        adam.step()
        if step % 10 == 0 or step == steps - 1:
            history.append(loss.mean().item())
            log(f"step {step:4d}  loss {history[-1]:.4f}")
    status, code = cola.cola_check_status(ws)
    if status:
        raise RuntimeError(f"device status {status} code {code}")

    # what the student answers
    cola.cola_fwd(d, X, A.detach().to(torch.bfloat16), B.detach().to(torch.bfloat16), Y, Z, None, ws)
    logp, entropy, mine, mine_logp = per_row(), per_row(), per_row(1, dtype=torch.int64), per_row(1)
    cola.cola_token_logprob_fwd(cola.vocab_desc(tokens, vocab, k=1), torch.matmul(Y, E.T), best, logp, entropy, mine, mine_logp,
                                None)
    agree = (mine[:, 0] == best).float().mean().item()
    log(f"log p of the teacher's best token {logp.mean().item():.3f}, entropy {entropy.mean().item():.3f}, "
        f"agreement {agree:.1%}")
    return {"loss": history, "logp": logp.mean().item(), "agreement": agree}


if __name__ == "__main__":
    p = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    p.add_argument("--tokens", type=int, default=4096)
    p.add_argument("--dim", type=int, default=512)
    p.add_argument("--vocab", type=int, default=32000)
    p.add_argument("--rank", type=int, default=128)
    p.add_argument("--top", type=int, default=32)
    p.add_argument("--temperature", type=float, default=2.0)
    p.add_argument("--steps", type=int, default=60)
    main(**vars(p.parse_args()))
