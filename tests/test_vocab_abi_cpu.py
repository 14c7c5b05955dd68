"""Refusals of the vocabulary entry points, before any device is touched."""
import ctypes

import pytest

from test_abi_cpu import FAKE, L  # noqa: F401


def _desc(L, **kw):   # noqa: F811
    args = dict(n=4, vocab=100, k=0)
    args.update(kw)
    return L.vocab_desc(**args)


CALLS = {   # name: arguments after the descriptor that pass every check (k = 5 where a list is given)
    "cola_token_logprob_fwd": (0, [FAKE] * 4 + [None, None, FAKE]),
    "cola_token_logprob_bwd": (0, [FAKE] * 6),
    "cola_token_logprob_step": (0, [FAKE] * 7),
    "cola_topk_distill_fwd": (5, [FAKE] * 6),
    "cola_topk_distill_bwd": (5, [FAKE] * 7),
    "cola_topk_distill_step": (5, [FAKE] * 7),
}


def _call(L, name, d, args):   # noqa: F811
    return getattr(L.lib(), name)(ctypes.byref(d) if d is not None else None, *args, None)


def test_desc_layout(L):   # noqa: F811
    assert ctypes.sizeof(L.cola_vocab_desc_t) == 4 * 8 + 6 * 4


@pytest.mark.parametrize("name", sorted(CALLS))
@pytest.mark.parametrize("kw,code", [
    (dict(n=0), 1), (dict(n=-1), 1), (dict(vocab=0), 1), (dict(ld=99), 1), (dict(ld_grad=-1), 1), (dict(ld_grad=99), 1),
    (dict(dtype="f16"), 1), (dict(dtype=7), 1), (dict(temperature=0.0), 1), (dict(temperature=-1.0), 1),
    (dict(temperature=float("nan")), 1), (dict(temperature=float("inf")), 1), (dict(temperature=1e-5), 1),
    (dict(teacher_temperature=0.0), 1), (dict(k=-1), 1), (dict(k=101), 1),
    (dict(vocab=(1 << 20) + 1), 3), (dict(vocab=1000, k=257), 3), (dict(n=1 << 28), 3), (dict(ld=1 << 31), 3),
])
def test_bad_descriptors(L, name, kw, code):   # noqa: F811
    k, args = CALLS[name]
    d = _desc(L, **{"k": k, **kw})
    assert _call(L, name, d, args) == code


@pytest.mark.parametrize("name", sorted(CALLS))
def test_missing_descriptor_reserved_and_rest(L, name):   # noqa: F811
    k, args = CALLS[name]
    assert _call(L, name, None, args) == 1
    d = _desc(L, k=k)
    d.reserved = 1
    assert _call(L, name, d, args) == 1
    d = _desc(L, k=k)
    d.rest = 2
    assert _call(L, name, d, args) == 1


# position: what a null there gives (1: refused, None: allowed), and the byte
# offset that is refused as misaligned
@pytest.mark.parametrize("name,nulls,offsets", [
    # logits, targets, logp, entropy, top_ids, top_logp, stats
    ("cola_token_logprob_fwd", [0, 1, 2], {0: 1, 1: 4, 2: 2, 3: 2, 6: 8}),
    # logits, targets, stats, dlogp, dentropy, dlogits
    ("cola_token_logprob_bwd", [0, 1, 2, 5], {0: 1, 1: 4, 2: 4, 3: 1, 4: 2, 5: 1}),
    # logits, targets, dlogp, dentropy, logp, entropy, dlogits
    ("cola_token_logprob_step", [0, 1, 6], {0: 1, 1: 4, 2: 2, 3: 2, 4: 2, 5: 2, 6: 1}),
    # logits, t_ids, t_vals, t_lse, loss, stats
    ("cola_topk_distill_fwd", [0, 1, 2, 4], {0: 1, 1: 4, 2: 2, 3: 2, 4: 2, 5: 4}),
    # logits, t_ids, t_vals, t_lse, stats, dloss, dlogits
    ("cola_topk_distill_bwd", [0, 1, 2, 4, 5, 6], {0: 1, 1: 4, 2: 2, 3: 2, 4: 4, 5: 2, 6: 1}),
    # logits, t_ids, t_vals, t_lse, dloss, loss, dlogits
    ("cola_topk_distill_step", [0, 1, 2, 4, 5, 6], {0: 1, 1: 4, 2: 2, 3: 2, 4: 2, 5: 2, 6: 1}),
])
def test_pointers(L, name, nulls, offsets):   # noqa: F811
    k, args = CALLS[name]
    d = _desc(L, k=k)
    for i in nulls:
        a = list(args)
        a[i] = None
        assert _call(L, name, d, a) == 1, i
    for i, off in offsets.items():
        a = list(args)
        a[i] = FAKE + off
        assert _call(L, name, d, a) == 2, i


def test_lists_go_with_k(L):   # noqa: F811
    f = "cola_token_logprob_fwd"
    none = [FAKE, None, None, None, None, None, None]
    assert _call(L, f, _desc(L), none) == 1                                            # nothing wanted
    assert _call(L, f, _desc(L, k=3), [FAKE] * 4 + [None, None, None]) == 1             # k without a list
    assert _call(L, f, _desc(L, k=0), [FAKE] * 7) == 1                                 # a list without k
    assert _call(L, f, _desc(L, k=3), [FAKE] * 5 + [None, None]) == 1                   # ids without log probabilities
    assert _call(L, f, _desc(L, k=3), [FAKE] * 4 + [FAKE + 4, FAKE, None]) == 2
    for g in ("cola_topk_distill_fwd", "cola_topk_distill_bwd", "cola_topk_distill_step"):
        assert _call(L, g, _desc(L, k=0), CALLS[g][1]) == 1                             # a teacher without entries
    # a backward without any upstream gradient
    assert _call(L, "cola_token_logprob_bwd", _desc(L), [FAKE, FAKE, FAKE, None, None, FAKE]) == 1
    assert _call(L, "cola_token_logprob_step", _desc(L), [FAKE, FAKE, None, None, FAKE, FAKE, FAKE]) == 1


def test_binding_raises(L):   # noqa: F811
    with pytest.raises(L.ColaError, match="cola_token_logprob_fwd"):
        L.cola_token_logprob_fwd(_desc(L, vocab=0), FAKE, FAKE, FAKE, None, None, None, None, stream=0)


# the last values that pass (what comes next is that the logits are misaligned) and the first that do not
@pytest.mark.parametrize("name", sorted(CALLS))
@pytest.mark.parametrize("kw,code", [
    (dict(n=(1 << 28) - 1), 2), (dict(n=1 << 28), 3),
    (dict(ld=(1 << 31) - 256), 2), (dict(ld=(1 << 31) - 255), 3),
    (dict(ld_grad=(1 << 31) - 256), 2), (dict(ld_grad=(1 << 31) - 255), 3),
    (dict(vocab=1 << 20), 2), (dict(vocab=(1 << 20) + 1), 3),
    (dict(vocab=1000, k=256), 2), (dict(vocab=1000, k=257), 3),
    (dict(temperature=1e-4), 2), (dict(temperature=1e4), 2), (dict(temperature=1.001e4), 1),
    (dict(teacher_temperature=1e-4), 2), (dict(teacher_temperature=1e4), 2), (dict(teacher_temperature=1.001e4), 1),
])
def test_edges_of_the_limits(L, name, kw, code):   # noqa: F811
    k, args = CALLS[name]
    d = _desc(L, **{"k": k, **kw})
    assert _call(L, name, d, [FAKE + 1] + args[1:]) == code
