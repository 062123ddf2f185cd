"""The training example: stages, compressed boundaries, loss over the vocabulary and optimiser steps
together; the loss falls, and the 8-bit states train as the fp32 ones do."""

import importlib.util
import math
import os

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_the_example_learns():
    import __graft_entry__ as g

    g.build()
    spec = importlib.util.spec_from_file_location("train_stages", os.path.join(ROOT, "examples", "train_stages.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    last = {}
    for bits in (32, 8):
        losses = example.train(steps=120, vocab=300, width=64, stages=3, blocks=1, batch=8, length=48, topk=30,
                               state_bits=bits, log=None)
        assert bool(losses.isfinite().all())
        # the first batch knows nothing; a word's four successors leave log 4
        assert abs(float(losses[0]) - math.log(300)) < 1.0
        last[bits] = float(losses[-20:].mean())
        assert last[bits] < 0.75 * math.log(300), last
    assert abs(last[8] - last[32]) < 0.15 * last[32], last
