"""The sequence example's own checks."""
from types import SimpleNamespace

import numpy as np
import pytest
import torch

from paper_2011_01383_amd import cortex as C
from paper_2011_01383_amd import sequence as Q
from tests.gpu_helpers import announce, need_gpu


def test_prompts_are_checked_before_the_device_sees_them():
    model = SimpleNamespace(vocab=10, rows=2, device="none")
    for prompts, what in (([[1], [2], [3]], "3 prompts, the model runs 2"), ([[1], []], "prompt 1 is empty"),
                          ([[1, 10]], "prompt 0 has a token outside"), ([[0], [-1]], "prompt 1 has a token outside")):
        with pytest.raises(ValueError, match=what):
            Q.write_trees(model, prompts)
    trees, logprob = Q.write_trees(model, [])
    assert trees == [] and logprob.shape == (0,)
