"""The causal convolution against its float64 definition: ragged prompts, single
tokens, states, strides, widths and types; broken batches."""
import numpy as np
import pytest
import torch

from oracle import sequence_oracle as O
from paper_2011_01383_amd import cortex as C
from tests.gpu_helpers import announce, need_gpu
from tests.sequence_helpers import DTYPES, U, columns, dev, host, offsets_of, type_step, within

pytestmark = pytest.mark.gpu

LENS = {"one": [1], "ragged": [5, 0, 33, 64, 31, 1, 100, 32, 2, 3], "empty": [0, 0, 0], "many": [k % 7 for k in range(150)],
        "long": [700]}


def make(seed, lens, ch, W, dtype, left=0):
    r = np.random.default_rng(seed)
    t = DTYPES[dtype]
    rnd = lambda a: torch.from_numpy(a).to(t).double().numpy()
    S, T = len(lens), sum(lens)
    index = r.permutation(S + 2)[:S].astype(np.int32)          # two rows of the pool that nobody names
    index[r.random(S) < 0.2] = -1
    f32 = lambda a: a.astype(np.float32).astype(np.float64)
    return dict(x=rnd(r.normal(size=(T, ch))), w=f32(r.normal(size=(ch, W))), b=f32(r.normal(size=ch)),
                state=rnd(r.normal(size=(S + 2, W - 1, ch))), index=index, offsets=offsets_of(lens), t=t, T=T, S=S, left=left)


def bound(p, y, mag, W):
    """W + 1 products and sums, each off by at most U of the magnitude, the silu's
    exponential by a few U of |v| <= mag, and the store's rounding."""
    return (4 * W + 16) * U * mag * (1 + mag) + type_step(p["t"]) * np.abs(y) + 1e-30


def run(p, step, act=True, bias=True, with_state=True, in_place=False, stream=None):
    x = columns(p["x"], p["t"], p["left"], p["left"])
    y = torch.full((p["T"], p["x"].shape[1] + p["left"]), float("nan"), dtype=p["t"], device="cuda")[:, :p["x"].shape[1]]
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    state = dev(p["state"], p["t"]) if with_state else None
    out = None if not with_state else state if in_place else torch.full_like(state, 7.0)
    kw = dict(bias=dev(p["b"]) if bias else None, silu=act, state_in=state, state_out=out,
              state_index=dev(p["index"], torch.int32) if with_state else None, status=status, stream=stream)
    if step:
        C.check(C.cortex_conv_step(x, dev(p["w"]), y, **kw))
    else:
        C.check(C.cortex_conv_forward(x, dev(p["w"]), dev(p["offsets"], torch.int32), y, **kw))
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    return y, out


def check(p, y, out, W, act=True, bias=True, with_state=True, in_place=False):
    ref, mag, new = O.conv(p["x"], p["w"], p["b"] if bias else None, act, p["offsets"], p["index"] if with_state else None,
                           p["state"] if with_state else None)
    within(host(y), ref, bound(p, ref, mag, W), "y")
    if with_state:
        got = host(out)
        for row in range(p["S"] + 2):
            want = new.get(row, p["state"][row] if in_place else np.full_like(p["state"][row], 7.0))
            np.testing.assert_array_equal(got[row], want, err_msg="state %d" % row)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("W", [2, 3, 4])
@pytest.mark.parametrize("lens", list(LENS))
def test_prompts(lens, W, dtype):
    need_gpu()
    for ch, left in ((64, 0), (37, 0), (520, 8), (40, 3)):
        announce("conv %s W %d %s channels %d left %d" % (lens, W, dtype, ch, left))
        p = make(W + ch, LENS[lens], ch, W, dtype, left)
        y, out = run(p, False)
        check(p, y, out, W)


@pytest.mark.parametrize("act,bias,with_state,in_place", [(False, False, False, False), (True, False, True, True),
                                                          (False, True, True, True)])
def test_options(act, bias, with_state, in_place):
    need_gpu()
    p = make(5, LENS["ragged"], 72, 4, "bf16")
    kw = dict(act=act, bias=bias, with_state=with_state, in_place=in_place)
    check(p, *run(p, False, **kw), 4, **kw)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("W", [2, 3, 4])
def test_single_tokens(W, dtype):
    need_gpu()
    for S, ch, left, in_place in ((1, 2304, 0, True), (7, 33, 0, False), (300, 64, 8, True), (5, 64, 1, True)):
        announce("conv step W %d %s rows %d channels %d" % (W, dtype, S, ch))
        p = make(S + W, [1] * S, ch, W, dtype, left)
        check(p, *run(p, True, in_place=in_place), W, in_place=in_place)


def test_prompt_then_tokens_is_the_whole_prompt():
    need_gpu()
    p = make(3, [40], 96, 4, "bf16")
    p["index"] = np.zeros(1, np.int32)
    whole, _ = run(p, False)
    x, w, b = dev(p["x"], p["t"]), dev(p["w"]), dev(p["b"])
    state, status = dev(p["state"], p["t"]), torch.zeros(1, dtype=torch.int32, device="cuda")
    y = torch.empty_like(x)
    off = torch.tensor([0, 25], dtype=torch.int32, device="cuda")
    C.check(C.cortex_conv_forward(x[:25], w, off, y[:25], bias=b, state_in=state, state_out=state, status=status))
    for t in range(25, 40):
        C.check(C.cortex_conv_step(x[t:t + 1], w, y[t:t + 1], bias=b, state_in=state, state_out=state, status=status))
    torch.cuda.synchronize()
    assert torch.equal(y, whole)


def test_broken_batches():
    need_gpu()
    x, w, y = torch.zeros(6, 64, device="cuda"), torch.zeros(64, 4, device="cuda"), torch.full((6, 64), 5.0, device="cuda")
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    state = torch.zeros(3, 3, 64, device="cuda")
    for off in ([0, 4, 3, 6], [0, 2, 4, 5], [1, 2, 4, 6], [0, 2, 4, 7], [0, -3, 4, 6]):
        status = ints([0])
        C.check(C.cortex_conv_forward(x, w, ints(off), y, state_in=state, state_out=state, status=status))
        torch.cuda.synchronize()
        assert int(status.item()) == C.CORTEX_ST_SEQ_OFFSETS, off
    for index in ([0, 3, 1], [0, -2, 1]):
        status = ints([0])
        C.check(C.cortex_conv_forward(x, w, ints([0, 2, 4, 6]), y, state_in=state, state_index=ints(index), status=status))
        C.check(C.cortex_conv_step(x[:3], w, y[:3], state_in=state, state_index=ints(index), status=(s2 := ints([0]))))
        torch.cuda.synchronize()
        assert int(status.item()) == C.CORTEX_ST_INPUT_RANGE and int(s2.item()) == C.CORTEX_ST_INPUT_RANGE
    # an earlier error leaves the outputs as they were
    status = ints([C.CORTEX_ST_CYCLE])
    y.fill_(5.0)
    C.check(C.cortex_conv_forward(x, w, ints([0, 2, 4, 6]), y, status=status))
    torch.cuda.synchronize()
    assert int(status.item()) == C.CORTEX_ST_CYCLE and bool((y == 5.0).all())
    # no sequence: nothing to do
    C.check(C.cortex_conv_forward(x[:0], w, ints([0]), y[:0], status=ints([0])))


def test_another_stream():
    need_gpu()
    p = make(9, LENS["ragged"], 64, 4, "f32")
    y, out = run(p, False)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    y2, out2 = run(p, False, stream=s)
    with torch.cuda.stream(s):
        y3, out3 = run(p, False)
    assert torch.equal(y, y2) and torch.equal(out, out2) and torch.equal(y, y3) and torch.equal(out, out3)


def test_long_batches():
    """Enough tokens for the longer chunks, aligned rows and others."""
    need_gpu()
    r = np.random.default_rng(1)
    for ch, left, lens in ((1040, 0, r.integers(0, 900, 24).tolist()), (300, 1, [5000, 0, 1, 15, 16, 17, 2100])):
        for W in (2, 4):
            announce("conv, %d tokens of %d channels W %d" % (sum(lens), ch, W))
            p = make(7, lens, ch, W, "bf16", left)
            y, out = run(p, False)
            check(p, y, out, W)
