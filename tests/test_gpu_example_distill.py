"""The example that distils a full-rank projection into a CoLA layer: the layer
calls and the vocabulary operators together, on few tokens; the loss falls and
the student comes to agree with the teacher."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu


def _example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "distill.py")
    spec = importlib.util.spec_from_file_location("example_distill", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_distillation_learns():
    lines = []
    r = _example().main(tokens=512, dim=256, vocab=5003, rank=128, top=16, steps=60, log=lines.append)
    assert r["loss"][-1] < 0.5 * r["loss"][0], lines
    assert r["agreement"] > 50 / 5003, lines   # far above chance
