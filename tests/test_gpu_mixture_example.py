"""The example that trains a small mixture with the head's losses, the experts' dispatch and the optimizer step together."""
import importlib.util
import math
import os

import pytest

pytestmark = pytest.mark.gpu


def test_the_mixture_learns():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "mixture_step.py")
    spec = importlib.util.spec_from_file_location("mixture_step", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    history = example.train(60)
    # it starts near log(vocabulary) and has learnt most followers well before every token was seen often
    assert abs(history[0][1] - math.log(example.VOCAB)) < 1.0
    assert history[-1][1] < history[0][1] - 2.0 and history[-1][2] < history[0][2] - 1.0
