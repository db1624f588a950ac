"""The operators at a model's output end together, as a trainer and a receiver use
them: the loss falls, and the receiver answers from its patched codes."""
import importlib.util
import os

import pytest

from paper_2602_03839_amd import pulse

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "head_loop.py")


def example():
    spec = importlib.util.spec_from_file_location("head_loop", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("form", [pulse.MXFP4, pulse.FP8_E4M3])
def test_loop_learns_and_the_receiver_follows(form):
    log = example().run(form, steps=30)
    # 2,048 entries: ln 2048 = 7.6 at the start
    assert log[0]["loss"] > 6.5 and log[-1]["loss"] < 0.7 * log[0]["loss"], log
    assert all(0 < r["sent"] <= 1 for r in log)
    assert log[-1]["agree"] > 0.5, log[-1]
