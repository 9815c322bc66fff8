"""The example that quantises a layer, fits it to a teacher's top logits and serves single tokens."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "distill_mx4.py")


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("distill_mx4", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_loss_falls_and_tokens_agree(example):
    losses, agree = example.run(steps=60, rows=128, vocab=500)
    assert losses[-1] < 0.5 * losses[0]
    assert agree > 0.5


def test_two_component_master_keeps_small_updates(example):
    """At a step size whose updates are below half a unit in a binary16 weight's last place the
    second component is what moves the weight."""
    one, _ = example.run(steps=40, rows=128, vocab=500, master=1, lr=0.01, nc=3)
    two, _ = example.run(steps=40, rows=128, vocab=500, master=2, lr=0.01, nc=3)
    assert two[-1] <= one[-1]
