"""The tree texts of the sequence example: grammar, arrays, and (GPU) the whole path."""
import numpy as np
import pytest
import torch

from oracle import cortex_oracle
from paper_2011_01383_amd import cortex as C
from paper_2011_01383_amd import sequence as Q
from tests.gpu_helpers import announce, need_gpu


def test_tree_arrays():
    children, words = Q.tree_arrays([[0, 5, 0, 7, 5], [9]])
    assert children.tolist() == [1, 2, -1, -1, 3, 4, -1, -1, -1, -1, -1, -1]
    assert words.tolist() == [-1, 5, -1, 7, 5, 9]
    with pytest.raises(ValueError, match="after the tree"):
        Q.tree_arrays([[5, 5]])


def test_masks():
    m = Q.tree_masks(70, device="cpu").numpy().view(np.uint8)
    bits = np.unpackbits(m, axis=1, bitorder="little")
    assert bits.shape == (3, 96) and not bits[:, 70:].any()
    assert bits[0, :70].all() and bits[1, 1:70].all() and not bits[1, 0] and not bits[2].any()


def model_state(model):
    return [t.clone() for l in model.layers for t in (l.conv_state, l.state)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_write_and_read_trees(dtype):
    need_gpu()
    announce("sequence example %s" % dtype)
    typ = torch.float32 if dtype == "f32" else torch.bfloat16
    model = Q.SequenceModel(200, width=128, rows=8, dtype=typ)
    rng = np.random.default_rng(3)
    prompts = [rng.integers(1, 200, n).tolist() for n in (3, 70, 1, 9, 33)]
    trees, logprob = Q.write_trees(model, prompts, most=25, repetition=1.2, frequency=0.2, presence=0.1, opening=6.0)
    again, logprob2 = Q.write_trees(model, prompts, most=25, repetition=1.2, frequency=0.2, presence=0.1, opening=6.0)
    assert trees == again and np.array_equal(logprob, logprob2)
    assert np.isfinite(logprob).all() and (logprob <= 0).all()
    assert max(len(t) for t in trees) <= 25 and any(len(t) > 1 for t in trees)
    H = 64
    g = torch.Generator().manual_seed(1)
    vectors = torch.randn(200, H, generator=g)
    U, b = 0.05 * (2 * torch.rand(2, 5, H, H, generator=g) - 1), 0.05 * (2 * torch.rand(5, H, generator=g) - 1)
    h, c, lin = Q.read_trees(trees, vectors.cuda(), U.cuda(), b.cuda())
    children, words = Q.tree_arrays(trees)
    ref = cortex_oracle.linearize(children, 2)
    assert lin.level_nodes.cpu().numpy().tolist() == ref["level_nodes"].tolist()
    # the roots' states, node by node in float64
    hh, cc = {}, {}
    w = U.double().numpy(), b.double().numpy()
    sig = lambda v: 1 / (1 + np.exp(-v))

    def node(v):
        l, r = children[2 * v], children[2 * v + 1]
        if l < 0:
            return vectors[words[v]].double().numpy(), np.zeros(H)
        (hl, cl), (hr, cr) = node(l), node(r)
        i, fl, fr, o, u = (w[0][0, k] @ hl + w[0][1, k] @ hr + w[1][k] for k in range(5))
        cn = sig(i) * np.tanh(u) + sig(fl) * cl + sig(fr) * cr
        return sig(o) * np.tanh(cn), cn

    rows = lin.node_row.cpu().numpy()
    at = 0
    for t in trees:
        want = node(at)[0]
        assert np.abs(h[rows[at]].cpu().double().numpy() - want).max() <= 1e-4
        at += len(t)


@pytest.mark.gpu
def test_tokens_continue_their_prompts():
    """Prompts and then tokens, one at a time, leave the states and logits of the whole texts
    read as prompts; a row that is not named keeps its own."""
    need_gpu()
    model = Q.SequenceModel(100, width=128, rows=4)
    rng = np.random.default_rng(5)
    texts = [rng.integers(0, 100, n) for n in (50, 40, 45)]
    cut = [40, 30, 35]
    ints = lambda v: torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")
    slots = ints([2, 0, 3])
    for l in model.layers:
        l.state[1] = 5.0
    whole = model.prompt(ints(np.concatenate(texts)), ints([0, 50, 90, 135]), slots)
    want = model_state(model)
    model.reset(slots)
    model.prompt(ints(np.concatenate([t[:c] for t, c in zip(texts, cut)])), ints([0] + np.cumsum(cut).tolist()), slots)
    for k in range(10):
        logits = model.step(ints([t[c + k] for t, c in zip(texts, cut)]), slots)
    torch.cuda.synchronize()
    assert int(model.status.item()) == 0
    # two layers of float32 sums in different orders, 50 tokens deep
    assert torch.allclose(logits, whole, rtol=0, atol=1e-4 * float(whole.abs().max()))
    for a, b in zip(model_state(model), want):
        assert torch.allclose(a, b, rtol=0, atol=1e-4 * max(1.0, float(b[[0, 2, 3]].abs().max())))
    assert all(bool((l.state[1] == 5.0).all()) for l in model.layers)
