"""The delta layer of the sequence model: its operators in a run, each against its definition on what the
one before it left, and the model that has such layers."""
import numpy as np
import pytest
import torch

from oracle import sequence_oracle as O
from paper_2011_01383_amd import cortex as C
from paper_2011_01383_amd import sequence as Q
from tests.delta_helpers import say
from tests.gpu_helpers import need_gpu
from tests.sequence_helpers import U, dev, host, offsets_of, type_step, within


def test_kinds_are_checked():
    with pytest.raises(ValueError, match="got 'other'"):
        Q.SequenceModel(10, device="cpu", kinds=("other",))


def linear(w, x, typ):
    q, s = O.quant_rows(x.astype(np.float32))
    y = (q.astype(np.int64) @ w.q.cpu().numpy().astype(np.int64).T) * s.astype(np.float64)[:, None] * host(w.scale)
    return y, (5 * U + type_step(typ)) * np.abs(y) + 1e-30


@pytest.mark.gpu
@pytest.mark.parametrize("typ", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("step", [False, True])
def test_operators_in_a_run(step, typ):
    need_gpu()
    say("delta layer", step, typ)
    g = torch.Generator().manual_seed(3)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    layer = Q._DeltaLayer(g, 96, 256, 6, typ, "cuda", status)
    layer.conv_state.copy_(torch.randn(layer.conv_state.shape, generator=g))
    layer.state.copy_(0.1 * torch.randn(layer.state.shape, generator=g))
    D, H, G, K, V = layer.D, layer.H, layer.G, 64, 64
    lens = [1] * 4 if step else [70, 3, 1, 129]
    T, off = sum(lens), offsets_of(lens)
    x = torch.randn(T, 96, generator=g).to("cuda", typ)
    index = np.array([2, 5, 0, 3], dtype=np.int32)
    conv0, state0 = host(layer.conv_state), host(layer.state)
    # the layer's own steps, one by one
    u = layer.w_in(x, status)
    within(host(u), *linear(layer.w_in, host(x), typ), "projection")
    z, c, b, dt = u.split([D, layer.conv_channels, H, H], 1)
    m = torch.empty_like(c, memory_format=torch.contiguous_format)
    pool = dict(state_index=dev(index, torch.int32), status=status)
    conv, state = layer.conv_state.clone(), layer.state.clone()
    offsets = dev(off, torch.int32)
    if step:
        C.check(C.cortex_conv_step(c, layer.conv_w, m, bias=layer.conv_b, state_in=conv, state_out=conv, **pool))
    else:
        C.check(C.cortex_conv_forward(c, layer.conv_w, offsets, m, bias=layer.conv_b, state_in=conv, state_out=conv, **pool))
    ref, mag, _ = O.conv(host(c), host(layer.conv_w), host(layer.conv_b), True, off, index, conv0)
    within(host(m), ref, 32 * U * mag * (1 + mag) + type_step(typ) * np.abs(ref) + 1e-30, "convolution")
    q, k, v = m[:, :G * K].unflatten(1, (G, K)), m[:, G * K:2 * G * K].unflatten(1, (G, K)), m[:, 2 * G * K:].unflatten(1, (H, V))
    before = host(q), host(k)
    C.check(C.cortex_qk_norm(q, q, k=k, k_out=k, norm=C.CORTEX_NORM_L2, status=status))
    for got, was, name in ((q, before[0], "queries"), (k, before[1], "keys")):
        ref, mag = O.qk_norm(was, "l2", float(np.float32(1e-6)))
        within(host(got), ref, (K / 2 + 32) * U * mag + type_step(typ) * np.abs(ref) + 1e-30, name)
    y = torch.empty(T, H, V, dtype=typ, device="cuda")
    kw = dict(dt=dt, A=layer.A, dt_bias=layer.dt_bias, scale=K ** -0.5, state_in=state, state_out=state, **pool)
    if step:
        C.check(C.cortex_delta_step(q, k, v, b, y, **kw))
    else:
        C.check(C.cortex_delta_forward(q, k, v, b, offsets, y, ws=C.workspace(C.cortex_delta_workspace_bytes(T, 4, H, K, V)), **kw))
    ref, mag, new = O.delta(host(q), host(k), host(v), host(b), off, host(dt), host(layer.A), host(layer.dt_bias), scale=K ** -0.5, index=index,
                            state=state0)
    # Keys rounded to 16 bits may have a norm above 1 by 2^-8: over these tokens, whose decays and updates
    # shrink a row far more, that is less than the bound's own factor.
    f32 = (2 * (K + 64) + 32) * U
    within(host(y), ref, f32 * mag + type_step(typ) * np.abs(ref) + 1e-30, "delta rule")
    for row, (h, hm) in new.items():
        within(host(state)[row], h, np.broadcast_to(f32 * hm + 1e-30, h.shape), "state")
    # the whole layer does the same, bit for bit
    C.check(C.cortex_qk_norm(y, y, norm=C.CORTEX_NORM_RMS, q_weight=layer.weight, status=status))
    gated = y.flatten(1) * torch.nn.functional.silu(z)
    out = x + layer.w_out(gated, status)
    got = layer(x, dev(index, torch.int32), status, None if step else offsets)
    assert torch.equal(got, out) and torch.equal(layer.state, state) and torch.equal(layer.conv_state, conv)
    assert int(status.item()) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_a_model_with_delta_layers_writes_trees(dtype):
    need_gpu()
    say("model with delta layers", dtype)
    model = Q.SequenceModel(50, width=64, layers=3, rows=4, dtype=dtype, kinds=("delta", "channel", "head"))
    prompts = [[3, 4], list(range(1, 49)) * 2, [5], [6, 7, 8]]
    trees, logprob = Q.write_trees(model, prompts, most=15, opening=3.0)
    children, words = Q.tree_arrays(trees)
    assert len(words) == sum(len(t) for t in trees) and np.isfinite(logprob).all()
    again, logprob2 = Q.write_trees(model, prompts, most=15, opening=3.0)
    assert again == trees and np.array_equal(logprob, logprob2)


@pytest.mark.gpu
def test_models_without_kinds_are_what_they_were():
    """The default's layers take their weights in the same order from the same generator."""
    need_gpu()
    say("default kinds")
    a, b = Q.SequenceModel(40, width=64), Q.SequenceModel(40, width=64, kinds=("channel", "head"))
    g = torch.Generator().manual_seed(0)
    assert torch.equal(a.embedding.cpu(), torch.randn(40, 64, generator=g))
    first = torch.randn(64, 256, generator=g) / 8
    assert torch.equal(a.layers[0].w_in.cpu(), first) and torch.equal(a.w_out, b.w_out)
