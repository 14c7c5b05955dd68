"""Refusals of the embedding's and the constraints' entry points, before any
device is touched, and the layouts of their descriptors."""
import ctypes

import pytest
import torch

from test_abi_cpu import FAKE, L  # noqa: F401


# ------------------------------------------------------------------ embedding
def _embed(L, name, d, args):   # noqa: F811
    d = ctypes.byref(d) if d is not None else None
    if name == "cola_embed_workspace_size":
        return L.lib().cola_embed_workspace_size(d, *args)
    return getattr(L.lib(), name)(d, *args, None)


EMBED = {   # arguments after the descriptor that pass every check but the device's
    "cola_embed_fwd": [FAKE] * 3,
    "cola_embed_workspace_size": [ctypes.byref(ctypes.c_size_t(0))],
    "cola_embed_bwd": [FAKE] * 4 + [1 << 40],
}


def test_layouts(L):   # noqa: F811
    assert ctypes.sizeof(L.cola_embed_desc_t) == 6 * 8 + 6 * 4
    assert ctypes.sizeof(L.cola_constraints_t) == 10 * 8 + 4 * 8 + 2 * 4


@pytest.mark.parametrize("name", sorted(EMBED))
@pytest.mark.parametrize("kw,code", [
    (dict(n=0), 1), (dict(n=-1), 1), (dict(vocab=0), 1), (dict(d=0), 1), (dict(d=-8), 1), (dict(ld_e=-64), 1), (dict(ld_x=-64), 1),
    (dict(ld_de=-64), 1), (dict(scale=float("nan")), 1),
    (dict(scale=float("inf")), 1), (dict(dtype_e="f16"), 1), (dict(dtype_x=7), 1), (dict(dtype_de=-2), 1), (dict(accumulate=True), 1),
    (dict(vocab=(1 << 20) + 1), 3), (dict(n=1 << 28), 3), (dict(d=(1 << 20) + 8), 3), (dict(n=(1 << 28) - 1, d=1 << 20), 3),
])
def test_bad_embed_descriptors(L, name, kw, code):   # noqa: F811
    assert _embed(L, name, L.embed_desc(**{**dict(n=4, vocab=100, d=64), **kw}), EMBED[name]) == code


# each call goes by the pitches of what it reads and writes
@pytest.mark.parametrize("name,used", [("cola_embed_fwd", ("ld_e", "ld_x")), ("cola_embed_bwd", ("ld_x", "ld_de"))])
@pytest.mark.parametrize("d,ld,code", [(64, 56, 1), (64, 68, 1), (60, 0, 1), (60, 60, 1), (60, 56, 1), (64, 1 << 31, 3)])
def test_embed_pitches(L, name, used, d, ld, code):   # noqa: F811
    for which in ("ld_e", "ld_x", "ld_de"):
        kw = dict(ld_e=64, ld_x=64, ld_de=64)
        kw[which] = ld
        args = list(EMBED[name])
        args[0] = FAKE + 4     # what comes next is that the first pointer is misaligned
        assert _embed(L, name, L.embed_desc(4, 100, d, **kw), args) == (code if which in used else 2), which


@pytest.mark.parametrize("name", sorted(EMBED))
def test_embed_reserved_and_missing(L, name):   # noqa: F811
    assert _embed(L, name, None, EMBED[name]) == 1
    for field, value in (("reserved", 1), ("accumulate", 2), ("accumulate", -1)):
        d = L.embed_desc(4, 100, 64, dtype_de="f32")
        setattr(d, field, value)
        assert _embed(L, name, d, EMBED[name]) == 1


def test_embed_pointers(L):   # noqa: F811
    d = L.embed_desc(4, 100, 64)
    for name, offsets in (("cola_embed_fwd", (8, 4, 8)), ("cola_embed_bwd", (4, 8, 8, 128))):   # E, ids, X; ids, dX, dE, ws
        for i, off in enumerate(offsets):
            for value, code in ((None, 1), (FAKE + off, 2)):
                a = list(EMBED[name])
                a[i] = value
                assert _embed(L, name, d, a) == code, (name, i)
    assert L.lib().cola_embed_workspace_size(ctypes.byref(d), None) == 1


# the last values that pass (what comes next is that the ids are misaligned) and the first that do not
@pytest.mark.parametrize("kw,code", [
    (dict(n=(1 << 28) - 1), 2), (dict(n=1 << 28), 3), (dict(vocab=1 << 20), 2), (dict(vocab=(1 << 20) + 1), 3), (dict(d=1 << 20), 2),
    (dict(ld_x=(1 << 31) - 256), 2), (dict(ld_x=(1 << 31) - 248), 3), (dict(d=61, ld_e=64, ld_x=64, ld_de=72), 2),
    (dict(accumulate=True, dtype_de="f32"), 2),
])
def test_edges_of_the_embed_limits(L, kw, code):   # noqa: F811
    d = L.embed_desc(**{**dict(n=4, vocab=100, d=64), **kw})
    assert _embed(L, "cola_embed_fwd", d, [FAKE, FAKE + 4, FAKE]) == code
    assert _embed(L, "cola_embed_bwd", d, [FAKE + 4, FAKE, FAKE, FAKE, 1 << 40]) == code


# ---------------------------------------------------------------- constraints
CONSTRAIN = {"cola_constrain_logits_fwd": 2, "cola_constrain_logits_bwd": 3}   # pointers after the constraints


def _limits(L, **kw):   # noqa: F811
    c = L.constraints()
    full = dict(history=FAKE, history_len=FAKE, prompt_len=FAKE, repetition=FAKE, frequency=FAKE, presence=FAKE, bias_ids=FAKE,
                bias=FAKE, masks=FAKE, mask_of=FAKE, history_width=10, n_masks=2, n_bias=3)
    for k, v in {**full, **kw}.items():
        setattr(c, k, v)
    return c


def _constrain(L, name, d, c, args):   # noqa: F811
    ref = lambda s: ctypes.byref(s) if s is not None else None   # noqa: E731
    return getattr(L.lib(), name)(ref(d), ref(c), *args, None)


@pytest.mark.parametrize("name", sorted(CONSTRAIN))
@pytest.mark.parametrize("kw,code", [
    (dict(history=None), 1), (dict(history_width=0), 1), (dict(history_width=-1), 1), (dict(ld_history=9), 1), (dict(ld_history=-9), 1),
    (dict(bias=None), 1), (dict(bias_ids=None), 1), (dict(n_bias=0), 1), (dict(n_bias=-1), 1), (dict(n_masks=0), 1), (dict(n_masks=-1), 1),
    (dict(masks=None), 1), (dict(ld_masks=3), 1), (dict(ld_masks=-4), 1), (dict(mask_of=None, n_masks=3), 1), (dict(reserved=1), 1),
    (dict(n_bias=1025), 3), (dict(history_width=1 << 28), 3), (dict(ld_history=1 << 31), 3), (dict(ld_masks=1 << 31), 3),
    (dict(history=FAKE + 4), 2), (dict(history_len=FAKE + 4), 2), (dict(prompt_len=FAKE + 4), 2), (dict(bias_ids=FAKE + 4), 2),
    (dict(mask_of=FAKE + 4), 2), (dict(repetition=FAKE + 2), 2), (dict(frequency=FAKE + 2), 2), (dict(presence=FAKE + 2), 2),
    (dict(bias=FAKE + 2), 2), (dict(masks=FAKE + 2), 2),
])
def test_bad_constraints(L, name, kw, code):   # noqa: F811
    assert _constrain(L, name, L.vocab_desc(4, 100), _limits(L, **kw), [FAKE, FAKE + 64, FAKE + 128][:CONSTRAIN[name]]) == code


@pytest.mark.parametrize("name", sorted(CONSTRAIN))
@pytest.mark.parametrize("kw,code", [
    (dict(n=0), 1), (dict(vocab=0), 1), (dict(ld=99), 1), (dict(ld_grad=99), 1), (dict(dtype="f16"), 1), (dict(temperature=0.0), 1),
    (dict(vocab=(1 << 20) + 1), 3), (dict(n=1 << 28), 3), (dict(ld=1 << 31), 3), (dict(ld_grad=1 << 31), 3),
])
def test_bad_logit_descriptors(L, name, kw, code):   # noqa: F811
    d = L.vocab_desc(**{**dict(n=4, vocab=100), **kw})
    assert _constrain(L, name, d, _limits(L, mask_of=FAKE, ld_masks=1 << 20), [FAKE] * CONSTRAIN[name]) == code


@pytest.mark.parametrize("name", sorted(CONSTRAIN))
def test_constrain_pointers(L, name):   # noqa: F811
    d, c, count = L.vocab_desc(4, 100), _limits(L), CONSTRAIN[name]
    assert _constrain(L, name, None, c, [FAKE] * count) == 1
    assert _constrain(L, name, d, None, [FAKE] * count) == 1
    for i in range(count):
        for value, code in ((None, 1), (FAKE + 1, 2)):
            a = [FAKE] * count
            a[i] = value
            assert _constrain(L, name, d, c, a) == code, i
    # results over the logits go by one pitch
    d = L.vocab_desc(4, 100, ld=104, ld_grad=112)
    assert _constrain(L, name, d, c, [FAKE] * count) == 1
    # a gradient without a repetition penalty needs no logits: what comes next is a misaligned gradient
    if count == 3:
        d = L.vocab_desc(4, 100)
        assert _constrain(L, name, d, _limits(L, repetition=None), [None, FAKE, FAKE + 1]) == 2


def test_the_builder_checks_types(L):   # noqa: F811
    ids = torch.zeros((2, 5), dtype=torch.int64)
    for kw in (dict(history=ids.int()), dict(history=ids[0]), dict(history=ids, history_len=torch.zeros(2)),
               dict(history=ids, repetition=torch.ones(2, dtype=torch.float64)), dict(masks=ids), dict(bias_ids=ids, bias=torch.zeros(2, 4)),
               dict(bias_ids=ids[:, ::2], bias=torch.zeros(2, 3)), dict(history=ids.t()), dict(bias=torch.zeros(2, 5)),
               dict(history=ids[:1].expand(3, 5)), dict(masks=torch.zeros((1, 4), dtype=torch.int32).expand(2, 4)),
               dict(history=ids, repetition=torch.ones(1).expand(2)), dict(history=ids, repetition=torch.ones(3)),
               dict(history=ids, masks=torch.zeros((3, 4), dtype=torch.int32), mask_of=torch.zeros(3, dtype=torch.int64))):
        with pytest.raises(ValueError):
            L.constraints(**kw)
    with pytest.raises(ValueError, match="2 rows for 3"):
        L.cola_constrain_logits_fwd(L.vocab_desc(3, 10), L.constraints(ids), FAKE, FAKE, stream=0)
    c = L.constraints(ids[:1].expand(1, 5), masks=torch.zeros((1, 4), dtype=torch.int32)[:, :3])
    assert (c.history_width, c.ld_history, c.ld_masks) == (5, 0, 0)
    c = L.constraints(ids[:, 1:4], masks=torch.zeros((3, 9), dtype=torch.int32)[:, :4], mask_of=torch.zeros(2, dtype=torch.int64))
    assert (c.history_width, c.ld_history, c.n_masks, c.ld_masks, c.n_bias) == (3, 5, 3, 9, 0)


def test_bindings_raise(L):   # noqa: F811
    with pytest.raises(L.ColaError, match="cola_embed_fwd"):
        L.cola_embed_fwd(L.embed_desc(0, 1, 8), FAKE, FAKE, FAKE, stream=0)
    with pytest.raises(L.ColaError, match="cola_constrain_logits_fwd"):
        L.cola_constrain_logits_fwd(L.vocab_desc(0, 1), L.constraints(), FAKE, FAKE, stream=0)


# a call compares the masks' words with the vocabulary: of one mask, whose pitch says nothing, and of a view narrower than its pitch
@pytest.mark.parametrize("name", sorted(CONSTRAIN))
@pytest.mark.parametrize("vocab,have,need", [(32000, 1, 1000), (32000, 999, 1000), (33, 1, 2), (97, 0, 4)])
def test_masks_narrower_than_the_vocabulary(L, name, vocab, have, need):   # noqa: F811
    call, args = getattr(L, name), [FAKE] * CONSTRAIN[name]
    which = torch.zeros(2, dtype=torch.int64)
    for masks, rows in ((torch.zeros((1, have), dtype=torch.int32), 1), (torch.zeros((2, 2000), dtype=torch.int32)[:, :have], 2),
                        (torch.zeros((1, 2000), dtype=torch.int32)[:, :have], 1)):
        with pytest.raises(ValueError, match=f"masks of {have} words for a vocabulary of {vocab}, which takes {need}"):
            call(L.vocab_desc(rows, vocab), L.constraints(masks=masks, mask_of=which[:rows]), *args, stream=0)


# one that is wide enough passes that check (what comes next is that the tensors are the host's)
@pytest.mark.parametrize("vocab,have", [(32000, 1000), (33, 2), (32, 1), (32, 2)])
def test_tensors_of_the_host(L, vocab, have):   # noqa: F811
    d, args = L.vocab_desc(1, vocab), [FAKE, FAKE]
    one = torch.ones(1)
    for kw, name in ((dict(masks=torch.zeros((1, have), dtype=torch.int32)), "masks"),
                     (dict(history=torch.zeros((1, 4), dtype=torch.int64), repetition=one), "history, repetition"),
                     (dict(bias_ids=torch.zeros((1, 2), dtype=torch.int64), bias=torch.ones((1, 2))), "bias_ids, bias")):
        with pytest.raises(ValueError, match=f"{name}: on the host"):
            L.cola_constrain_logits_fwd(d, L.constraints(**kw), *args, stream=0)


# rows without ids (an empty tensor's pointer is NULL) have no named token; a width without ids stays refused
@pytest.mark.parametrize("name", sorted(CONSTRAIN))
@pytest.mark.parametrize("ld", [0, 5])
def test_histories_of_no_ids(L, name, ld):   # noqa: F811
    d, args = L.vocab_desc(4, 100), [FAKE] * CONSTRAIN[name]
    of = lambda width: _limits(L, history=None, history_width=width, ld_history=ld, bias=FAKE + 2)   # noqa: E731
    assert _constrain(L, name, d, of(0), args) == 2      # what comes next is that the biases are misaligned
    assert _constrain(L, name, d, of(1), args) == 1
    ids, r = torch.zeros((2, 5), dtype=torch.int64), torch.ones(2)
    for none in (ids[:, :0], torch.zeros((2, 0), dtype=torch.int64)):
        c = L.constraints(none, torch.zeros(2, dtype=torch.int64), repetition=r)
        assert (c.history, c.history_width, c.repetition) == (None, 0, r.data_ptr())
    for kw in (dict(repetition=r), dict(history_len=ids[:, 0].clone()), dict(presence=r), dict(frequency=r)):
        with pytest.raises(ValueError, match="without a history"):
            L.constraints(**kw)


def test_gradient_of_no_ids_still_takes_the_logits(L):   # noqa: F811
    d, args = L.vocab_desc(4, 100), [None, FAKE, FAKE]
    assert _constrain(L, "cola_constrain_logits_bwd", d, _limits(L, history=None, history_width=0), args) == 1


# no masks (an empty tensor's pointer is NULL): mask_of names none for any row
@pytest.mark.parametrize("name", sorted(CONSTRAIN))
def test_no_masks(L, name):   # noqa: F811
    d, args = L.vocab_desc(4, 100), [FAKE] * CONSTRAIN[name]
    of = lambda **kw: _limits(L, masks=None, mask_of=FAKE + 4, **kw)   # noqa: E731
    assert _constrain(L, name, d, of(n_masks=0), args) == 2      # what comes next is that mask_of is misaligned
    assert _constrain(L, name, d, of(n_masks=1), args) == 1
    which = torch.zeros(2, dtype=torch.int64)
    for none in (torch.zeros((0, 4), dtype=torch.int32), torch.empty_strided((0, 4), (0, 0), dtype=torch.int32)):
        c = L.constraints(masks=none, mask_of=which)
        assert (c.masks, c.n_masks, c.mask_of, c.rows) == (None, 0, which.data_ptr(), 2)
    with pytest.raises(ValueError, match="without masks"):
        L.constraints(mask_of=which)
    with pytest.raises(ValueError, match="on the host"):         # no masks are not too narrow
        L.cola_constrain_logits_fwd(L.vocab_desc(2, 100), L.constraints(masks=torch.zeros((0, 0), dtype=torch.int32), mask_of=which), FAKE,
                                    FAKE, stream=0)
