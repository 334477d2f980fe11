"""The selective state space scan against its float64 definition, token by token:
both decay layouts, prompts and single tokens."""
import numpy as np
import pytest
import torch

from paper_2011_01383_amd import cortex as C
from tests.gpu_helpers import announce, need_gpu
from tests.sequence_helpers import Scan, U, dev, host, within

pytestmark = pytest.mark.gpu

LENS = {"one": [1], "ragged": [5, 0, 63, 64, 65, 1, 129, 2], "empty": [0, 0], "many": [k % 5 for k in range(90)],
        "long": [517], "chunks": [256, 255, 300, 0, 40]}
CHANNEL = [(64, 8, 1), (48, 16, 3), (37, 16, 1), (200, 32, 2), (64, 64, 1)]        # D, N, G
HEAD = [(64, 16, 1, 64), (96, 32, 1, 48), (128, 64, 2, 32), (128, 128, 1, 128), (256, 128, 2, 64), (32, 128, 1, 16),
        (256, 64, 1, 256)]                                                         # D, N, G, P


def run(p, label, step=False):
    """Prompt or tokens with a state in the pool, out of place: outputs and every row of the pool."""
    announce(label)
    d = p.upload()
    out = None if d["state"] is None else torch.full_like(d["state"], 7.0)
    C.check(p.call(step, state_out=out), label)
    torch.cuda.synchronize()
    assert int(d["status"].item()) == 0
    new = p.check(d["y"], out, label)
    if out is not None:
        for row in set(range(p.rows)) - set(new):
            assert bool((out[row] == 7.0).all()), "row %d of the pool belongs to nobody" % row
    return d["y"], out


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lens", list(LENS))
def test_channel_prompts(lens, dtype):
    need_gpu()
    for k, (D, N, G) in enumerate(CHANNEL):
        run(Scan(k, LENS[lens], D, N, G, dtype=dtype, left=8 * (k % 2)), "channel %s %s D %d N %d G %d" % (lens, dtype, D, N, G))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lens", list(LENS))
def test_head_prompts(lens, dtype):
    need_gpu()
    for k, (D, N, G, P) in enumerate(HEAD):
        run(Scan(k, LENS[lens], D, N, G, P, dtype=dtype, left=8 * (k % 2)),
            "head %s %s D %d N %d G %d P %d" % (lens, dtype, D, N, G, P))


OPTIONS = [dict(z=False), dict(skip=False), dict(bias=False, dt_scale=3.0), dict(soft=False), dict(state=False), dict(left=1),
           dict(left=3), dict(slow=True), dict(z=False, skip=False, bias=False, soft=False, state=False)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("k", range(len(OPTIONS)))
def test_options(k, dtype):
    need_gpu()
    lens = [70, 3, 0, 130]
    for P, D, N, G in ((0, 70, 16, 2), (32, 128, 64, 2)):
        run(Scan(k, lens, D, N, G, P, dtype=dtype, **OPTIONS[k]), "options %s %s P %d" % (OPTIONS[k], dtype, P))
        run(Scan(k, [1] * 5, D, N, G, P, dtype=dtype, **OPTIONS[k]), "options, step %s %s P %d" % (OPTIONS[k], dtype, P), True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("S", [1, 3, 130])
def test_single_tokens(S, dtype):
    need_gpu()
    for k, (D, N, G) in enumerate(CHANNEL):
        run(Scan(k, [1] * S, D, N, G, dtype=dtype, left=8 * (k % 2)), "channel step %s rows %d D %d N %d" % (dtype, S, D, N), True)
    for k, (D, N, G, P) in enumerate(HEAD):
        run(Scan(k, [1] * S, D, N, G, P, dtype=dtype, left=8 * (k % 2)), "head step %s rows %d D %d N %d" % (dtype, S, D, N), True)


@pytest.mark.parametrize("P", [0, 32])
@pytest.mark.parametrize("step", [False, True])
def test_pool_rows(P, step):
    """Sequences in any rows of a larger pool, some in none; in place and with no state written."""
    need_gpu()
    lens = [1] * 7 if step else [70, 3, 0, 130, 1, 64, 9]
    index = [9, -1, 3, 0, -1, 5, 1]
    p = Scan(1, lens, 64, 16, 1, P, index=index, rows=11)
    y, out = run(p, "pool P %d step %s" % (P, step), step)
    d = p.d
    old, y2 = d["state"].clone(), d["y"].clone()
    d["y"].fill_(float("nan"))
    C.check(p.call(step, state_out=d["state"]))               # in place
    torch.cuda.synchronize()
    assert torch.equal(d["y"], y2)
    named = [i for i in index if i >= 0]
    assert torch.equal(d["state"][named], out[named])
    rest = [i for i in range(11) if i not in named]
    assert torch.equal(d["state"][rest], old[rest])
    d["state"].copy_(old)
    d["y"].fill_(float("nan"))
    C.check(p.call(step, state_out=None))                      # read only
    torch.cuda.synchronize()
    assert torch.equal(d["y"], y2) and torch.equal(d["state"], old)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("P", [0, 64])
def test_prompt_then_tokens(P, dtype):
    """A prompt cut anywhere, its rest given token by token, ends in the state of the whole."""
    need_gpu()
    p = Scan(4, [300], 128, 64, 1, P, dtype=dtype)
    y, whole = run(p, "whole P %d" % P)
    d = p.d
    x, z, dt, B, Cm = d["x"], d["z"], d["dt"], d["B"], d["C"]
    state = d["state"].clone()
    y2 = torch.empty(300, 128, dtype=p.dtype, device="cuda")
    kw = dict(D=d["skip"], dt_bias=d["dt_bias"], status=d["status"], state_in=state, state_out=state)
    for a, b in ((0, 100), (100, 101), (101, 290)):
        off = torch.tensor([0, b - a], dtype=torch.int32, device="cuda")
        C.check(C.cortex_scan_forward(x[a:b], dt[a:b], d["A"], B[a:b], Cm[a:b], off, y2[a:b], z=z[a:b], ws=d["ws"], **kw))
    for t in range(290, 300):
        C.check(C.cortex_scan_step(x[t:t + 1], dt[t:t + 1], d["A"], B[t:t + 1], Cm[t:t + 1], y2[t:t + 1], z=z[t:t + 1], **kw))
    torch.cuda.synchronize()
    p.check(y2, state, "in parts P %d" % P)


@pytest.mark.parametrize("P", [0, 64])
def test_strong_and_absent_decay(P):
    """Step sizes from 0 to large: a state that is kept whole, and one that is forgotten at once."""
    need_gpu()
    for scale in (0.0, 40.0):
        p = Scan(6, [150, 20], 64, 16, 1, P, dtype="f32", soft=False)
        p.dt = np.full_like(p.dt, np.float32(0.02 * scale))
        p.dt_bias = None
        run(p, "dt %g P %d" % (0.02 * scale, P))


@pytest.mark.parametrize("P", [0, 64])
def test_masked_out_values_stay_in_their_sequence(P):
    """An infinity or NaN in one sequence, or in another sequence's row of the pool, reaches no other."""
    need_gpu()
    p = Scan(8, [40, 70, 33], 64, 16, 1, P, dtype="f32")
    y, out = run(p, "clean")
    y, out = y.clone(), out.clone()
    p.d["x"][45, 3] = float("nan")
    p.d["dt"][50] = float("inf")
    p.d["B"][60] = float("inf")
    p.d["state"][1, 5] = float("-inf")
    o2 = torch.full_like(out, 7.0)
    C.check(p.call(state_out=o2))
    torch.cuda.synchronize()
    assert torch.equal(p.d["y"][:40], y[:40]) and torch.equal(p.d["y"][110:], y[110:])
    assert torch.equal(o2[0], out[0]) and torch.equal(o2[2], out[2])
    assert not bool(torch.isfinite(p.d["y"][109]).all())


@pytest.mark.parametrize("P", [0, 32])
def test_broken_batches(P):
    need_gpu()
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    p = Scan(2, [2, 2, 2], 64, 16, 1, P)
    d = p.upload()
    for off in ([0, 4, 3, 6], [0, 2, 4, 5], [1, 2, 4, 6], [0, 2, 4, 7], [0, -3, 4, 6]):
        d["offsets"], d["status"] = ints(off), ints([0])
        C.check(p.call(state_out=None))
        torch.cuda.synchronize()
        assert int(d["status"].item()) == C.CORTEX_ST_SEQ_OFFSETS, off
    d["offsets"] = ints([0, 2, 4, 6])
    for index in ([0, 3, 1], [0, -2, 1]):
        d["index"], d["status"] = ints(index), ints([0])
        C.check(p.call(state_out=None))
        torch.cuda.synchronize()
        assert int(d["status"].item()) == C.CORTEX_ST_INPUT_RANGE
    d["index"], d["status"] = None, ints([C.CORTEX_ST_CYCLE])
    d["y"].fill_(5.0)
    out = torch.full_like(d["state"], 7.0)
    C.check(p.call(state_out=out))
    torch.cuda.synchronize()
    assert bool((d["y"] == 5.0).all()) and bool((out == 7.0).all()) and int(d["status"].item()) == C.CORTEX_ST_CYCLE


@pytest.mark.parametrize("P", [0, 64])
def test_graph_replays(P):
    """A captured prompt and step give the eager result at every replay."""
    need_gpu()
    announce("graph P %d" % P)
    p = Scan(3, [100, 70], 128, 32, 1, P)
    q = Scan(4, [1, 1, 1], 128, 32, 1, P)
    y, out = run(p, "eager")
    y1, out1 = run(q, "eager step", True)
    y, out, y1, out1 = y.clone(), out.clone(), y1.clone(), out1.clone()
    o, o1 = torch.zeros_like(out), torch.zeros_like(out1)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        C.check(p.call(state_out=o))
        C.check(q.call(True, state_out=o1))
    for k in range(4):
        p.d["y"].fill_(0), q.d["y"].fill_(0), o.fill_(0), o1.fill_(0)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(p.d["y"], y) and torch.equal(o, out) and torch.equal(q.d["y"], y1) and torch.equal(o1, out1), k


@pytest.mark.parametrize("P", [0, 64])
def test_deterministic_and_on_another_stream(P):
    need_gpu()
    p = Scan(5, [400, 37, 700], 128, 64, 1, P)
    y, out = run(p, "first")
    y, out = y.clone(), out.clone()
    s = torch.cuda.Stream()
    for k in range(3):
        o = torch.zeros_like(out)
        s.wait_stream(torch.cuda.current_stream())
        C.check(p.call(state_out=o, stream=s))
        torch.cuda.synchronize()
        assert torch.equal(p.d["y"], y) and torch.equal(o, out)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("P", [0, 64])
@pytest.mark.parametrize("what", ["x", "B", "dt", "C"])
def test_a_token_reaches_no_earlier_one(what, P, dtype):
    """An infinity or NaN at one token leaves the tokens before it as they were; in x it stays in its channel."""
    need_gpu()
    p = Scan(9, [150], 64, 16, 1, P, dtype=dtype)
    y, _ = run(p, "clean")
    y = y.clone()
    for at, v in ((100, float("inf")), (37, float("nan")), (0, float("-inf"))):
        p.upload()
        p.d[what][at, ..., 3 if what == "x" else slice(None)] = v
        C.check(p.call())
        torch.cuda.synchronize()
        assert torch.equal(p.d["y"][:at], y[:at]), at
        if what == "x":
            others = [c for c in range(64) if c != 3]
            assert torch.equal(p.d["y"][:, others], y[:, others]), at
            assert not bool(torch.isfinite(p.d["y"][at:, 3]).any()), at


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_many_sequences(dtype):
    """Enough sequences that each is walked whole, in one launch."""
    need_gpu()
    r = np.random.default_rng(0)
    run(Scan(1, r.integers(0, 6, 1100).tolist(), 64, 8, 1, dtype=dtype), "channel, 1100 sequences %s" % dtype)
    run(Scan(2, (r.integers(0, 40, 140) * 3).tolist(), 256, 32, 2, 64, dtype=dtype), "head, 140 sequences %s" % dtype)
    run(Scan(3, (r.integers(0, 40, 600)).tolist(), 128, 128, 1, 128, dtype=dtype), "head of 128, 600 sequences %s" % dtype)


def test_large_pools():
    """Batches that take two units a lane, and the loads past the caches: odd rows and channels."""
    need_gpu()
    run(Scan(1, [1] * 41, 2050, 64, 1, dtype="bf16"), "channel step, 41 x 2050 x 64", True)
    run(Scan(2, [1] * 17, 2064, 128, 1, 48), "head step, 17 x 2064 x 128", True)
    run(Scan(3, [1] * 35, 4112, 128, 1, 16, dtype="f32"), "head step, 35 x 4112 x 128", True)
    run(Scan(4, [1] * 135, 2049, 64, 3, dtype="f32"), "channel step, 135 x 2049 x 64", True)


@pytest.mark.parametrize("P", [0, 64])
def test_rows_far_apart(P):
    """Rows of a wide array: element offsets beyond 2^31."""
    need_gpu()
    T, D, N, ld = 80, 64, 16, 1 << 25
    p = Scan(6, [T], D, N, 1, P)
    d = p.upload()
    wide = torch.empty(T, ld, dtype=torch.bfloat16, device="cuda")
    at = 0
    for name in ("x", "z", "dt", "B", "C"):
        t = d[name]
        cols = t.flatten(1)
        v = wide[:, at:at + cols.shape[1]]
        v.copy_(cols)
        d[name] = v.unflatten(1, (1, N)) if t.dim() == 3 else v
        at += 64
    d["y"] = wide[:, at:at + D]
    out = torch.full_like(d["state"], 7.0)
    announce("rows %d elements apart P %d" % (ld, P))
    C.check(p.call(state_out=out))
    torch.cuda.synchronize()
    assert int(d["status"].item()) == 0
    p.check(d["y"], out, "far rows")
