"""The path from scores to a better generator, as examples/learn_from_scores.py runs it."""
from __future__ import annotations

import importlib.util
import os

import pytest

from conftest import ROOT

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("loss", ["policy", "preference"])
def test_answers_score_higher_after_training(loss):
    spec = importlib.util.spec_from_file_location("learn_from_scores", os.path.join(ROOT, "examples", "learn_from_scores.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    history = example.train(steps=30, loss=loss)
    # a table of zeros samples tokens alike: the mean score starts near its own standard error and rises by
    # several standard deviations of one answer's score
    assert history[-1] > history[0] + 3.0, history
