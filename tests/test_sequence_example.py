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


@pytest.mark.parametrize("left", [False, True])
def test_trees_deeper_than_the_interpreter_recurses(left):
    """A comb of 20,000 inner nodes, leaning either way."""
    n = 20000
    text = [0] * n + [5] * (n + 1) if left else [0, 5] * n + [7]
    children, words = Q.tree_arrays([text, [9]])
    assert words.tolist() == [-1 if t == 0 else t for t in text] + [9]
    children = children.reshape(-1, 2)
    if left:
        assert all(children[v].tolist() == [v + 1, 2 * n - v] for v in range(n))
    else:
        assert all(children[2 * v].tolist() == [2 * v + 1, 2 * v + 2] for v in range(n))
    assert (children[words >= 0] == -1).all()


def test_texts_that_are_no_tree():
    for text, what in (([0, 5], "a tree of 2 tokens lacks 1 subtrees"), ([], "a tree of 0 tokens lacks 1"), ([5, 0, 5], "2 tokens after the tree")):
        with pytest.raises(ValueError, match=what):
            Q.tree_arrays([text])


@pytest.mark.gpu
def test_a_call_that_failed_does_not_end_the_model():
    need_gpu()
    announce("sequence example, status of an earlier call")
    model = Q.SequenceModel(50, width=64, rows=3)
    prompts = [[3, 4], [5], [6, 7, 8]]
    trees, logprob = Q.write_trees(model, prompts, most=9, opening=3.0)
    # a step of a row that the pools do not have: the recurrences report it
    model.step(torch.tensor([1], dtype=torch.int32, device="cuda"), torch.tensor([7], dtype=torch.int32, device="cuda"))
    with pytest.raises(RuntimeError, match="device status %d" % C.CORTEX_ST_INPUT_RANGE):
        Q.write_trees(model, prompts, most=9, opening=3.0)
    again, logprob2 = Q.write_trees(model, prompts, most=9, opening=3.0)
    assert again == trees and np.array_equal(logprob, logprob2)
