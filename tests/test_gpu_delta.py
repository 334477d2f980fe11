"""The gated delta rule against its float64 definition: ragged prompts, single tokens, head layouts, states,
strides and types; what a NaN may touch; broken batches; streams and graphs."""
import numpy as np
import pytest
import torch

from paper_2011_01383_amd import cortex as C
from tests.delta_helpers import LENS, Delta, say
from tests.gpu_helpers import need_gpu
from tests.sequence_helpers import dev, host

pytestmark = pytest.mark.gpu


def run(p, step=False, in_place=False, with_state=True, stream=None):
    d = p.upload()
    out = None
    if with_state and p.state is not None:
        out = d["state"] if in_place else torch.full_like(d["state"], 7.0)
    C.check(p.call(step, state_in="state" if with_state else None, state_out=out, stream=stream))
    torch.cuda.synchronize()
    assert int(d["status"].item()) == 0
    return d["y"], out


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("K", [32, 64, 128])
@pytest.mark.parametrize("lens", sorted(LENS))
def test_prompts(lens, K, dtype):
    need_gpu()
    say("delta prompts", lens, K, dtype)
    p = Delta(1, LENS[lens], 2, 1, K, 32, dtype)
    y, out = run(p)
    p.check(y, out, "prompts")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,G,K,V", [(1, 1, 32, 16), (6, 3, 64, 48), (4, 4, 128, 128), (8, 1, 32, 80), (2, 1, 128, 256), (3, 3, 64, 112)])
def test_layouts(H, G, K, V, dtype):
    need_gpu()
    say("delta layouts", H, G, K, V, dtype)
    p = Delta(2, [70, 3, 0, 130], H, G, K, V, dtype)
    y, out = run(p)
    p.check(y, out, "layouts")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("left", [1, 2, 4, 8, 16])
def test_strides_and_alignments(left, dtype):
    need_gpu()
    say("delta strides", left, dtype)
    p = Delta(3, [66, 5], 3, 1, 64, 32, dtype, left=left)
    for step in (False, True):
        if step:
            p = Delta(3, [1] * 9, 3, 1, 64, 32, dtype, left=left)
        y, out = run(p, step)
        p.check(y, out, "strides")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kw", [dict(decay=False), dict(soft=False), dict(sig=False), dict(bias=False), dict(state=False), dict(lean=3.0),
                                dict(slow=0.01), dict(slow=30.0), dict(scale=-2.0)], ids=lambda k: "%s-%s" % list(k.items())[0])
def test_options(kw, dtype):
    need_gpu()
    say("delta options", kw, dtype)
    for step in (False, True):
        p = Delta(4, [1] * 5 if step else [100, 64, 7], 2, 2, 64, 32, dtype, **kw)
        y, out = run(p, step)
        p.check(y, out, "options")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("S,H,G,K,V", [(1, 1, 1, 32, 16), (5, 4, 2, 128, 128), (33, 3, 1, 64, 48), (300, 2, 2, 32, 32), (7, 2, 1, 128, 256)])
def test_tokens(S, H, G, K, V, dtype):
    need_gpu()
    say("delta tokens", S, H, G, K, V, dtype)
    p = Delta(5, [1] * S, H, G, K, V, dtype)
    y, out = run(p, True)
    p.check(y, out, "tokens")


@pytest.mark.parametrize("step", [False, True])
@pytest.mark.parametrize("in_place", [False, True])
def test_pool_rows(step, in_place):
    """Rows in any order, two without a row, rows that nobody names."""
    need_gpu()
    say("delta pool rows", step, in_place)
    lens = [1] * 6 if step else [65, 0, 3, 130, 64, 1]
    index = [4, 7, -1, 0, 2, -1]
    p = Delta(6, lens, 2, 1, 64, 32, index=index, rows=9)
    y, out = run(p, step, in_place)
    new = p.check(y, out, "pool")
    got = host(out)
    for row in set(range(9)) - set(new):
        assert np.array_equal(got[row], p.state[row] if in_place else np.full_like(p.state[row], 7.0)), row


def test_prompt_then_tokens_is_one_prompt():
    """The state that a prompt leaves is the one that its next tokens need."""
    need_gpu()
    say("delta prompt then tokens")
    whole = Delta(7, [70, 70, 70], 4, 2, 128, 64, "f32")
    y, end = run(whole)
    d = whole.d
    state = d["state"].clone()
    cut = [66, 69, 3]
    rows = np.concatenate([np.arange(70 * i, 70 * i + c) for i, c in enumerate(cut)])
    at = torch.from_numpy(rows).cuda()
    kw = dict(A=d["A"], dt_bias=d["dt_bias"], scale=whole.scale, state_in=state, state_out=state, status=d["status"])
    part = lambda name, i: d[name][i].contiguous()
    out = torch.empty_like(y)
    head = torch.empty(len(rows), 4, 64, device="cuda")
    C.check(C.cortex_delta_forward(part("q", at), part("k", at), part("v", at), part("b", at), dev(np.cumsum([0] + cut), torch.int32), head,
                                   dt=part("dt", at), ws=d["ws"], **kw))
    out[at] = head
    for j in range(70):
        live = [i for i in range(3) if cut[i] + j < 70]
        if not live:
            break
        at = torch.tensor([70 * i + cut[i] + j for i in live], device="cuda")
        one = torch.empty(len(live), 4, 64, device="cuda")
        C.check(C.cortex_delta_step(part("q", at), part("k", at), part("v", at), part("b", at), one, dt=part("dt", at),
                                    state_index=torch.tensor(live, dtype=torch.int32, device="cuda"), **kw))
        out[at] = one
    whole.check(out, state, "prompt then tokens")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("where", ["v", "k", "q", "b", "dt", "state"])
def test_what_is_not_finite_stays_behind_its_token(where, bad, dtype):
    """A value or a state entry reaches its row of the state, a key, share or step size its head, a query its own
    output; tokens before it and other sequences keep their results."""
    need_gpu()
    say("delta not finite", where, bad, dtype)
    p = Delta(8, [40, 150, 20], 4, 2, 64, 32, dtype)
    clean, end = (host(v) for v in run(p))
    t, head, row = 40 + 77, 3, 5                 # in the second sequence's second chunk; head 3 reads key head 1
    hit = np.zeros(clean.shape, dtype=bool)
    hit_end = np.zeros(end.shape, dtype=bool).reshape(3, 4, 32, 64)
    if where == "v":
        p.v[t, head, row] = bad
        hit[t:190, head, row] = hit_end[1, head, row] = True
    elif where == "k":
        p.k[t, 1, 9] = bad
        hit[t:190, 2:] = hit_end[1, 2:] = True
    elif where == "q":
        p.q[t, 1, 9] = bad
        hit[t, 2:] = True
    elif where == "b":
        p.b[t, head] = bad
        hit[t:190, head] = hit_end[1, head] = True
    elif where == "dt":
        p.dt[t, head] = bad
        hit[t:190, head] = hit_end[1, head] = True
    else:
        p.state[1, head * 32 + row, 3] = bad
        hit[40:190, head, row] = hit_end[1, head, row] = True
    got, got_end = (host(v) for v in run(p))
    hit_end = hit_end.reshape(end.shape)
    assert np.array_equal(got[~hit], clean[~hit]) and np.array_equal(got_end[~hit_end], end[~hit_end])
    # an infinite share is one or none, an infinite step forgets the state: finite either way
    if not (where in ("b", "dt") and np.isinf(bad)):
        assert not np.isfinite(got[hit]).any() and not np.isfinite(got_end[hit_end].reshape(-1, 64)).all(1).any()


@pytest.mark.parametrize("step", [False, True])
def test_broken_batches(step):
    need_gpu()
    say("delta broken batches", step)
    lens = [1, 1, 1] if step else [70, 3, 64]
    for index, offsets, want in (([0, 3, 1], None, C.CORTEX_ST_INPUT_RANGE), ([0, -2, 1], None, C.CORTEX_ST_INPUT_RANGE),
                                 (None, [0, 80, 73, 137], C.CORTEX_ST_SEQ_OFFSETS), (None, [1, 70, 73, 137], C.CORTEX_ST_SEQ_OFFSETS),
                                 (None, [0, 70, 73, 136], C.CORTEX_ST_SEQ_OFFSETS), (None, [0, -5, 73, 137], C.CORTEX_ST_SEQ_OFFSETS),
                                 (None, [0, 70, 73, 2 ** 31 - 1], C.CORTEX_ST_SEQ_OFFSETS)):
        if step and offsets is not None:
            continue
        p = Delta(9, lens, 2, 1, 32, 16, index=index)
        if offsets is not None:
            p.offsets = np.array(offsets)
        d = p.upload()
        out = torch.full_like(d["state"], 7.0)
        C.check(p.call(step, state_out=out))
        torch.cuda.synchronize()
        assert int(d["status"].item()) == want
        # the next call finds the status and writes nothing
        d["y"].fill_(5.0)
        out.fill_(7.0)
        C.check(p.call(step, state_out=out))
        torch.cuda.synchronize()
        assert (host(d["y"]) == 5.0).all() and (host(out) == 7.0).all()


def test_same_bits_on_another_stream_and_in_a_graph():
    need_gpu()
    say("delta streams and graphs")
    for step in (False, True):
        p = Delta(10, [1] * 9 if step else [70, 200, 3], 4, 2, 64, 32)
        y, out = run(p, step)
        y, out = y.clone(), out.clone()
        d = p.d
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        again = torch.empty_like(out)
        d["y"].zero_()
        torch.cuda.synchronize()
        C.check(p.call(step, state_out=again, stream=side))
        side.synchronize()
        assert torch.equal(d["y"], y) and torch.equal(again, out)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            C.check(p.call(step, state_out=again))
        for _ in range(3):
            d["y"].zero_()
            again.zero_()
            d["ws"].fill_(255)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(d["y"], y) and torch.equal(again, out)
        assert int(d["status"].item()) == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,G,K,V", [(8, 4, 64, 64), (4, 4, 128, 128), (40, 8, 32, 16), (12, 3, 64, 48)])
def test_many_prompts(H, G, K, V, dtype):
    """More heads of sequences than the GPU takes at once with few columns a workgroup."""
    need_gpu()
    say("delta many prompts", H, G, K, V, dtype)
    r = np.random.default_rng(11)
    S = 1200 // (H * V // 16) + 20
    p = Delta(11, [int(n) for n in r.integers(0, 100, S)], H, G, K, V, dtype, index=r.permutation(S).tolist())
    y, out = run(p)
    p.check(y, out, "many prompts")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,G,K,V,lens", [(1, 1, 32, 16, [1500]), (2, 1, 64, 48, [700, 0, 1, 900]), (1, 1, 128, 128, [1300]), (3, 3, 64, 64, [256, 257, 511]),
                                          (4, 2, 128, 32, [640, 0])])
def test_few_columns_and_long_prompts(H, G, K, V, lens, dtype):
    """Prompts cut into segments: their states come from the segments before, in the pool's rows or from zero."""
    need_gpu()
    say("delta long prompts", H, G, K, V, lens, dtype)
    S = len(lens)
    p = Delta(12, lens, H, G, K, V, dtype, index=[S - i for i in range(S)], rows=S + 1, slow=0.05)
    y, out = run(p)
    new = p.check(y, out, "long prompts")
    got = host(out)
    for row in set(range(S + 1)) - set(new):
        assert np.array_equal(got[row], np.full_like(got[row], 7.0))
    y, _ = run(Delta(12, lens, H, G, K, V, dtype, state=False, slow=0.05), with_state=False)
    Delta(12, lens, H, G, K, V, dtype, state=False, slow=0.05).check(y, None, "long prompts without states")


@pytest.mark.parametrize("where", ["v", "k", "state"])
def test_what_is_not_finite_in_a_long_prompt(where):
    need_gpu()
    say("delta long prompts, not finite", where)
    p = Delta(13, [1200, 90], 2, 1, 64, 32)
    clean, end = (host(v) for v in run(p))
    hit = np.zeros(clean.shape, dtype=bool)
    hit_end = np.zeros(end.shape, dtype=bool).reshape(2, 2, 32, 64)
    if where == "v":
        p.v[600, 1, 5] = np.nan
        hit[600:1200, 1, 5] = hit_end[0, 1, 5] = True
    elif where == "k":
        p.k[600, 0, 9] = np.inf
        hit[600:1200] = hit_end[0] = True
    else:
        p.state[0, 32 + 5, 3] = np.inf
        hit[:1200, 1, 5] = hit_end[0, 1, 5] = True
    got, got_end = (host(v) for v in run(p))
    hit_end = hit_end.reshape(end.shape)
    assert np.array_equal(got[~hit], clean[~hit]) and np.array_equal(got_end[~hit_end], end[~hit_end])
    assert not np.isfinite(got[hit]).any() and not np.isfinite(got_end[hit_end].reshape(-1, 64)).all(1).any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("left", [1, 2, 4, 8, 16])
def test_strides_and_alignments_of_many_prompts(left, dtype):
    need_gpu()
    say("delta strides of many prompts", left, dtype)
    p = Delta(14, [5, 70, 0, 1] * 32, 4, 1, 64, 48, dtype, left=left)
    y, out = run(p)
    p.check(y, out, "strides of many prompts")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("where", ["v", "k", "q", "b", "dt", "state"])
def test_what_is_not_finite_in_many_prompts(where, bad, dtype):
    """As in few: in every third of 66 prompts, at another token of each."""
    need_gpu()
    say("delta many prompts, not finite", where, bad, dtype)
    S, n, V, K = 66, 130, 64, 32
    p = Delta(15, [n] * S, 4, 2, K, V, dtype)
    clean, end = (host(v) for v in run(p))
    hit = np.zeros(clean.shape, dtype=bool)
    hit_end = np.zeros(end.shape, dtype=bool).reshape(S, 4, V, K)
    for s in range(0, S, 3):
        first, last, head, row = n * s, n * s + n, 2 + s % 2, s % V
        t = first + (s * 7) % n
        if where == "v":
            p.v[t, head, row] = bad
            hit[t:last, head, row] = hit_end[s, head, row] = True
        elif where == "k":
            p.k[t, 1, 9] = bad
            hit[t:last, 2:] = hit_end[s, 2:] = True
        elif where == "q":
            p.q[t, 1, 9] = bad
            hit[t, 2:] = True
        elif where == "state":
            p.state[s, head * V + row, 3] = bad
            hit[first:last, head, row] = hit_end[s, head, row] = True
        else:
            (p.b if where == "b" else p.dt)[t, head] = bad
            hit[t:last, head] = hit_end[s, head] = True
    got, got_end = (host(v) for v in run(p))
    hit_end = hit_end.reshape(end.shape)
    assert np.array_equal(got[~hit], clean[~hit]) and np.array_equal(got_end[~hit_end], end[~hit_end])
    # an infinite share is one or none, an infinite step forgets the state: finite either way
    if not (where in ("b", "dt") and np.isinf(bad)):
        assert not np.isfinite(got[hit]).any() and not np.isfinite(got_end[hit_end].reshape(-1, K)).all(1).any()


@pytest.mark.parametrize("many", [False, True])
def test_two_streams_at_once(many):
    """Two batches on two streams, each with its own workspace, over and over: what each gives alone."""
    need_gpu()
    say("delta two streams", many)
    ps = [Delta(16 + i, [30, 200, 65] * (24 if many else 1), 4, 2, 64, 64) for i in range(2)]
    alone = [tuple(t.clone() for t in run(p)) for p in ps]
    ends = [torch.empty_like(out) for _, out in alone]
    streams = [torch.cuda.Stream() for _ in ps]
    for p in ps:
        p.d["y"].zero_()
    torch.cuda.synchronize()
    for _ in range(5):
        for p, end, stream in zip(ps, ends, streams):
            C.check(p.call(False, state_out=end, stream=stream))
    torch.cuda.synchronize()
    for p, end, (y, out) in zip(ps, ends, alone):
        assert torch.equal(p.d["y"], y) and torch.equal(end, out) and int(p.d["status"].item()) == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,G,K,V,lens", [(8, 4, 128, 128, [1, 0, 1, 2, 0, 1, 1, 1]), (4, 4, 64, 64, [0, 1, 1, 0, 2, 0, 1, 1] * 5),
                                          (6, 2, 32, 32, [0, 0, 0, 3, 0]), (2, 1, 128, 16, [0, 0])])
def test_fewer_tokens_than_prompts(H, G, K, V, lens, dtype):
    need_gpu()
    say("delta fewer tokens than prompts", H, G, K, V, lens, dtype)
    S = len(lens)
    assert C.cortex_delta_segment_tokens(sum(lens), S, H, K, V) == 0
    p = Delta(17, lens, H, G, K, V, dtype, index=[S - 1 - i for i in range(S)])
    y, out = run(p)
    p.check(y, out, "fewer tokens than prompts")


def gates_at(p, name, value, places):
    """b or dt of every sequence's tokens at `places` (where it has them), another head each."""
    for s in range(p.S):
        for n, t in enumerate(places):
            if t < p.lens[s]:
                getattr(p, name)[p.offsets[s] + t, (s + n) % p.H] = value


FORMS = {"few": ([200, 64, 1, 65], 4, 2, 64, 32), "many": ([130, 0, 3, 64] * 17, 4, 2, 32, 64), "segments": ([1700, 1900], 3, 3, 64, 64),
         "tokens": ([1] * 9, 4, 2, 64, 32)}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("form", sorted(FORMS))
@pytest.mark.parametrize("name,value", [("b", np.inf), ("b", -np.inf), ("dt", np.inf), ("dt", -np.inf)])
def test_infinite_gates_are_none_or_whole(name, value, form, dtype):
    """A share of 0 or 1, a decay of 0 or 1: both forms give what the definition does."""
    need_gpu()
    say("delta infinite gates", name, value, form, dtype)
    lens, H, G, K, V = FORMS[form]
    assert (C.cortex_delta_segment_tokens(sum(lens), len(lens), H, K, V) > 0) == (form == "segments")
    p = Delta(18, lens, H, G, K, V, dtype, slow=0.2)
    gates_at(p, name, value, [0, 2, 17, 62, 63, 64, 128, 199, 700])
    y, out = run(p, form == "tokens")
    p.check(y, out, "infinite gates")


@pytest.mark.parametrize("form", sorted(FORMS))
@pytest.mark.parametrize("name,value,kw,A", [("b", np.inf, dict(sig=False), None), ("b", np.nan, dict(), None), ("dt", np.nan, dict(), None),
                                             ("dt", -np.inf, dict(soft=False), None), ("dt", np.inf, dict(), 0.0), ("dt", np.inf, dict(), 0.5)])
def test_gates_that_lose_a_head(name, value, kw, A, form):
    """A share or an exponent that is no finite number after the functions asked for."""
    need_gpu()
    say("delta gates that lose a head", name, value, kw, A, form)
    lens, H, G, K, V = FORMS[form]
    p = Delta(19, lens, H, G, K, V, "f32", slow=0.2, **kw)
    if A is not None:
        p.dt[:] = -8.0                           # a step of 3e-4, so that a growing state stays small
        p.dt_bias[:] = 0.0
        p.A[H - 1] = A
    clean, end = (host(v) for v in run(p, form == "tokens"))
    hit, hit_end = np.zeros(clean.shape, dtype=bool), np.zeros((p.S, H, V * K), dtype=bool)
    for s in range(0, p.S, 2):
        if lens[s]:
            t = p.offsets[s] + min(lens[s] - 1, 77)
            getattr(p, name)[t, H - 1] = value
            hit[t:p.offsets[s + 1], H - 1] = hit_end[s, H - 1] = True
    hit_end = hit_end.reshape(end.shape)
    got, got_end = (host(v) for v in run(p, form == "tokens"))
    assert np.array_equal(got[~hit], clean[~hit]) and np.array_equal(got_end[~hit_end], end[~hit_end])
    assert not np.isfinite(got[hit]).any() and not np.isfinite(got_end[hit_end]).any()


# Shapes that are cut into segments: of one and several heads, key groups, sequences, empty and short ones among them.
SEGMENTS = [(1, 1, 128, 128, [2100]), (3, 3, 64, 64, [1700, 1900]), (2, 2, 64, 32, [2900, 90]), (2, 1, 128, 48, [2600, 0, 2800]),
            (1, 1, 32, 256, [4200, 1]), (2, 1, 32, 16, [0, 6500, 64]), (1, 1, 64, 112, [256, 4000, 257])]


def in_segments(p):
    """The tokens of a segment of p's batch; some sequence has several."""
    Q = C.cortex_delta_segment_tokens(p.T, p.S, p.H, p.K, p.V)
    assert Q > 0 and max(p.lens) > Q, (Q, p.lens)
    return Q


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,G,K,V,lens", SEGMENTS)
def test_segments(H, G, K, V, lens, dtype):
    """States from the segments before, in the pool's rows, in place and not, without a row and without states."""
    need_gpu()
    say("delta segments", H, G, K, V, lens, dtype)
    S = len(lens)
    for n, in_place in enumerate((False, True)):
        index = [S + 1 - i for i in range(S)]
        if S > 1:
            index[n] = -1
        p = Delta(20, lens, H, G, K, V, dtype, index=index, rows=S + 2, slow=0.02)
        in_segments(p)
        y, out = run(p, in_place=in_place)
        new = p.check(y, out, "segments")
        got = host(out)
        for row in set(range(S + 2)) - set(new):
            assert np.array_equal(got[row], p.state[row] if in_place else np.full_like(got[row], 7.0))
    p = Delta(21, lens, H, G, K, V, dtype, state=False, decay=False, lean=2.0)
    y, _ = run(p, with_state=False)
    p.check(y, None, "segments without states")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("left", [1, 2, 4, 8, 16])
def test_segments_at_every_alignment(left, dtype):
    need_gpu()
    say("delta segments, alignments", left, dtype)
    for H, G, K, V, lens in ((2, 1, 64, 32, [2301, 3, 3030]), (1, 1, 128, 16, [2100])):
        p = Delta(22, lens, H, G, K, V, dtype, left=left, slow=0.05)
        in_segments(p)
        y, out = run(p)
        p.check(y, out, "segments, alignments")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("where", ["v", "k", "q", "state"])
def test_what_is_not_finite_in_segments(where, bad, dtype):
    """It passes from a segment to all that follow, of its row of the state or its head, and to nothing else."""
    need_gpu()
    say("delta segments, not finite", where, bad, dtype)
    H, G, K, V, lens = 4, 2, 64, 32, [2500, 0, 2900]
    p = Delta(23, lens, H, G, K, V, dtype, slow=0.05)
    Q = in_segments(p)
    clean, end = (host(v) for v in run(p))
    hit, hit_end = np.zeros(clean.shape, dtype=bool), np.zeros((3, H, V, K), dtype=bool)
    for s, t in ((0, Q + 77), (2, 3)):           # in a second segment and in a first one
        t, last, head, row = p.offsets[s] + t, p.offsets[s + 1], 2 + s // 2, 5 + s
        if where == "v":
            p.v[t, head, row] = bad
            hit[t:last, head, row] = hit_end[s, head, row] = True
        elif where == "k":
            p.k[t, 1, 9] = bad
            hit[t:last, 2:] = hit_end[s, 2:] = True
        elif where == "q":
            p.q[t, 1, 9] = bad
            hit[t, 2:] = True
        else:
            p.state[s, head * V + row, 3] = bad
            hit[p.offsets[s]:last, head, row] = hit_end[s, head, row] = True
    got, got_end = (host(v) for v in run(p))
    hit_end = hit_end.reshape(end.shape)
    assert np.array_equal(got[~hit], clean[~hit]) and np.array_equal(got_end[~hit_end], end[~hit_end])
    assert not np.isfinite(got[hit]).any() and not np.isfinite(got_end[hit_end].reshape(-1, K)).all(1).any()


def test_segments_of_broken_batches():
    need_gpu()
    say("delta segments, broken batches")
    for index, offsets, want in (([0, 3, 1], None, C.CORTEX_ST_INPUT_RANGE), ([0, -2, 1], None, C.CORTEX_ST_INPUT_RANGE),
                                 (None, [0, 2600, 2500, 5400], C.CORTEX_ST_SEQ_OFFSETS), (None, [1, 2500, 2700, 5400], C.CORTEX_ST_SEQ_OFFSETS),
                                 (None, [0, 2500, 2700, 5399], C.CORTEX_ST_SEQ_OFFSETS), (None, [0, -2500, 2700, 5400], C.CORTEX_ST_SEQ_OFFSETS),
                                 (None, [0, 2500, 2700, 2 ** 31 - 1], C.CORTEX_ST_SEQ_OFFSETS)):
        p = Delta(24, [2500, 200, 2700], 2, 1, 32, 16, index=index)
        in_segments(p)
        if offsets is not None:
            p.offsets = np.array(offsets)
        d = p.upload()
        out = torch.full_like(d["state"], 7.0)
        C.check(p.call(state_out=out))
        torch.cuda.synchronize()
        assert int(d["status"].item()) == want
        d["y"].fill_(5.0)
        out.fill_(7.0)
        C.check(p.call(state_out=out))
        torch.cuda.synchronize()
        assert (host(d["y"]) == 5.0).all() and (host(out) == 7.0).all()


def test_segments_on_two_streams_and_in_a_graph():
    """The same bits from two batches at once, each with its own workspace, and from every replay."""
    need_gpu()
    say("delta segments, streams and graph")
    ps = [Delta(25 + i, [1700, 1900], 3, 3, 64, 64, slow=0.05) for i in range(2)]
    for p in ps:
        in_segments(p)
    alone = [tuple(t.clone() for t in run(p)) for p in ps]
    ends = [torch.empty_like(out) for _, out in alone]
    streams = [torch.cuda.Stream() for _ in ps]
    for p in ps:
        p.d["y"].zero_()
    torch.cuda.synchronize()
    for _ in range(5):
        for p, end, stream in zip(ps, ends, streams):
            C.check(p.call(state_out=end, stream=stream))
    torch.cuda.synchronize()
    for p, end, (y, out) in zip(ps, ends, alone):
        assert torch.equal(p.d["y"], y) and torch.equal(end, out)
    p, end, (y, out) = ps[0], ends[0], alone[0]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        C.check(p.call(state_out=end))
    for _ in range(3):
        p.d["y"].zero_()
        end.zero_()
        p.d["ws"].fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(p.d["y"], y) and torch.equal(end, out)
    assert all(int(p.d["status"].item()) == 0 for p in ps)


def test_a_prompt_in_segments_then_tokens_is_one_prompt():
    need_gpu()
    say("delta segments then tokens")
    whole = Delta(27, [2120], 1, 1, 128, 64, "f32", slow=0.05)
    d = whole.upload()
    assert C.cortex_delta_segment_tokens(2100, 1, 1, 128, 64) > 0
    state, y, kw = d["state"].clone(), d["y"], dict(A=d["A"], dt_bias=d["dt_bias"], scale=whole.scale, status=d["status"])
    kw.update(state_in=state, state_out=state)
    part = lambda name, i, j: d[name][i:j]
    C.check(C.cortex_delta_forward(*(part(n, 0, 2100) for n in ("q", "k", "v", "b")), dev([0, 2100], torch.int32), y[:2100],
                                   dt=part("dt", 0, 2100), ws=d["ws"], **kw))
    for t in range(2100, 2120):
        C.check(C.cortex_delta_step(*(part(n, t, t + 1) for n in ("q", "k", "v", "b")), y[t:t + 1], dt=part("dt", t, t + 1), **kw))
    torch.cuda.synchronize()
    assert int(d["status"].item()) == 0
    whole.check(y, state, "segments then tokens")
