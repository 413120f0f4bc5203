"""The operators together, as a program uses them: examples/train_packed_rows.py learns."""
import importlib.util
import os

import numpy as np
import pytest

from gpu_common import log

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "train_packed_rows.py")


def test_a_classifier_learns_from_packed_rows():
    spec = importlib.util.spec_from_file_location("train_packed_rows", PATH)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    losses, norms = example.train("tiny", steps=60)
    log(f"[example] first losses {losses[:3]}, last {losses[-3:]}")
    assert np.isfinite(losses).all() and np.isfinite(norms).all() and min(norms) > 0
    assert np.mean(losses[-5:]) < 0.7 * np.mean(losses[:5])           # the labels are decided by the rows: half of the loss is soon gone
    again, _ = example.train("tiny", steps=5)
    assert again == losses[:5]                                      # bit for bit
