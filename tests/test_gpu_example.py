"""The example of routed microbatches: it learns, and a crash changes nothing."""
import importlib.util
import os

import pytest

from tests.gpu_util import have_gpu

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not have_gpu(), reason="no GPU")]

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "replay_after_crash.py")


def test_replay_after_crash():
    spec = importlib.util.spec_from_file_location("replay_after_crash", PATH)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    losses, moved, same = example.main(steps=8)
    assert same and moved >= 8
    assert losses[-1] < losses[0] - 0.5
