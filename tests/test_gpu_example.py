"""The example trains: rollout tokens sampled, labels kept, the drafter distilled from them and its
table updated, all by the library's calls."""

import importlib.util
import os

import pytest
import torch

from paper_2609_38795_gb300 import build_lib

pytestmark = pytest.mark.gpu


def test_the_example_drafter_learns():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    build_lib.build()
    spec = importlib.util.spec_from_file_location(
        "distil_drafter", os.path.join(build_lib.ROOT, "examples", "distil_drafter.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    first, last = example.train(steps=150, rows=512, vocab=1024, dim=64, report=None)
    assert 0 < last < 0.5 * first
