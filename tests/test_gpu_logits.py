"""The processing of logits against its definition.  The values are float32
operations rounded one by one, so they, and the tokens, are equal bit for bit;
the normaliser is compared with float64."""
import numpy as np
import pytest
import torch

from oracle import sequence_oracle as O
from paper_2011_01383_amd import cortex as C
from tests.gpu_helpers import announce, need_gpu
from tests.sequence_helpers import DTYPES, U, columns

pytestmark = pytest.mark.gpu


def ints(v):
    return torch.tensor(np.asarray(v, dtype=np.int32), device="cuda")


def floats(v):
    return torch.tensor(np.asarray(v, dtype=np.float32), device="cuda")


def pack(allowed):
    """[rows, V] booleans as rows of 32-bit words; the bits past V are set, and mean nothing."""
    rows, V = allowed.shape
    wide = np.ones((rows, (V + 31) // 32 * 32), dtype=bool)
    wide[:, :V] = allowed
    return np.packbits(wide, axis=1, bitorder="little").view(np.int32)


class Case:
    def __init__(self, seed, R, V, dtype="f32", history=True, cap=None, penalties=True, biases=True, mask=True, left=0):
        r = np.random.default_rng(seed)
        self.R, self.V, self.t, self.left = R, V, DTYPES[dtype], left
        self.v = torch.from_numpy(r.normal(size=(R, V)) * 2.5).to(self.t).float().numpy()
        self.hist = self.lens = self.prompt = self.rep = self.freq = self.pres = self.bias = self.allowed = self.index = None
        if history:
            cap = 40 if cap is None else cap
            self.hist = np.minimum((V ** r.random((R, cap))).astype(np.int32) - 1, V - 1).clip(0)
            self.lens = r.integers(0, cap + 1, R)
            self.prompt = (self.lens * r.random(R)).astype(np.int64)
            if penalties:
                f = lambda a: a.astype(np.float32)
                self.rep, self.freq, self.pres = f(1 + 0.5 * r.random(R)), f(r.random(R)), f(r.random(R))
        if biases:
            self.bias = [[(int(t), float(np.float32(b))) for t, b in zip(r.integers(0, V, n), 3 * r.normal(size=n))]
                         for n in r.integers(0, 12, R)]
        if mask:
            self.allowed = r.random((5, V)) < np.array([0.5, 1.0, 0.05, 0.9, 0.0])[:, None]
            self.index = r.integers(-1, 5, R)

    def call(self, out="new", token=True, lse=True, ws=None, stream=None):
        src = columns(self.v, self.t, self.left, self.left)
        dst = src if out == "same" else columns(self.v * 0 + 7, self.t, self.left) if out == "new" else None
        tok = torch.full((self.R,), 99, dtype=torch.int32, device="cuda") if token else None
        nrm = torch.full((self.R,), 99.0, device="cuda") if lse else None
        self.status = ints([0])
        kw = {}
        if self.hist is not None:
            kw.update(history=ints(self.hist), history_len=ints(self.lens), prompt_len=ints(self.prompt))
            if self.rep is not None:
                kw.update(repetition=floats(self.rep), frequency=floats(self.freq), presence=floats(self.pres))
        if self.bias is not None:
            flat = [p for row in self.bias for p in row]
            kw.update(bias_offsets=ints(np.cumsum([0] + [len(row) for row in self.bias])), bias_tokens=ints([t for t, _ in flat]),
                      bias_values=floats([b for _, b in flat]))
        if self.allowed is not None:
            kw.update(mask=ints(pack(self.allowed)), mask_index=ints(self.index))
        ws = C.workspace(C.cortex_logits_workspace_bytes(self.R, self.V)) if ws is None else ws
        C.check(C.cortex_logits_process(src, out=dst, token=tok, lse=nrm, status=self.status, ws=ws, stream=stream, **kw))
        torch.cuda.synchronize()
        return dst, tok, nrm

    def check(self, dst, tok, nrm):
        assert int(self.status.item()) == 0
        for i in range(self.R):
            at = lambda a: None if a is None else a[i]
            m = None if self.allowed is None or self.index[i] < 0 else self.allowed[self.index[i]]
            v, token, lse = O.logits(self.v[i], at(self.hist), at(self.lens), at(self.prompt), at(self.rep), at(self.freq),
                                     at(self.pres), at(self.bias), m)
            if dst is not None:
                want = torch.from_numpy(v).to(self.t).float().numpy()
                np.testing.assert_array_equal(dst[i].float().cpu().numpy(), want, err_msg="row %d" % i)
            if tok is not None:
                assert int(tok[i]) == token, i
            if nrm is not None:
                got = float(nrm[i])
                if np.isfinite(lse):
                    # exp and its argument's rounding: 4 U of |v - top| up to 90 for terms that still count; sums of
                    # partial sums, at most 64 deep; then the logarithm and the last addition
                    n = 64 + 4 * 90
                    assert abs(got - lse) <= n * U + 4 * U * abs(lse), (i, got, lse)
                else:
                    assert np.isnan(got) == np.isnan(lse) and (np.isnan(lse) or got == lse), (i, got, lse)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [1, 7, 31, 32, 33, 1000, 4096, 4097, 10007, 70000])
def test_sizes(V, dtype):
    need_gpu()
    announce("logits V %d %s" % (V, dtype))
    for left, out in ((0, "new"), (8, "same"), (3, "new"), (0, None)):
        c = Case(V + left, 5, V, dtype, left=left)
        c.check(*c.call(out))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kw", [dict(history=False), dict(penalties=False), dict(biases=False), dict(mask=False),
                                dict(history=False, biases=False, mask=False), dict(cap=0), dict(cap=6000)],
                         ids=lambda kw: "-".join(kw))
def test_parts(kw, dtype):
    need_gpu()
    for R, V in ((1, 9000), (37, 600)):
        c = Case(3, R, V, dtype, **kw)
        c.check(*c.call())


def test_outputs_alone():
    need_gpu()
    c = Case(1, 4, 9001)
    for kw in (dict(token=False, lse=False), dict(out=None, lse=False), dict(out=None, token=False)):
        c.check(*c.call(**kw))


def test_many_rows():
    need_gpu()
    c = Case(2, 3000, 129, "bf16")
    c.check(*c.call())


def test_one_workspace_for_calls_of_different_sizes():
    need_gpu()
    ws = C.workspace(C.cortex_logits_workspace_bytes(64, 70000))
    for k, (R, V) in enumerate([(64, 70000), (3, 9000), (64, 100), (1, 70000), (20, 5000), (64, 70000)]):
        c = Case(k, R, V)
        c.check(*c.call(ws=ws))


def test_ties_go_to_the_lowest_index():
    need_gpu()
    c = Case(1, 3, 20000, history=False, biases=False, mask=False)
    c.v[:] = -1.0
    c.v[0, [17000, 9000, 4095]] = 2.0
    c.v[1, [19999, 19998]] = 2.0
    _, tok, _ = out = c.call()
    c.check(*out)
    assert tok.tolist() == [4095, 19998, 0]


def test_rows_that_a_mask_leaves_empty():
    need_gpu()
    c = Case(1, 4, 9000)
    c.index[:] = [4, 1, 4, 0]
    c.v[0] = np.nan
    dst, tok, nrm = out = c.call()
    c.check(*out)
    assert tok.tolist()[0] == -1 and float(nrm[2]) == -np.inf and bool((dst[0] == -np.inf).all())


@pytest.mark.parametrize("value", [np.inf, -np.inf, np.nan, 3.4028235e38, -3.4028235e38])
def test_values_at_the_types_ends(value):
    """In masked places they are never used; in open ones they count as what they are."""
    need_gpu()
    for mask in (True, False):
        c = Case(4, 6, 9000, mask=mask)
        c.v[:, ::3] = value
        if mask:
            c.allowed[:, ::3] = False
        c.check(*c.call())
        c.v[0, :] = value
        c.check(*c.call())


def test_large_logits_do_not_overflow_the_normaliser():
    need_gpu()
    c = Case(5, 3, 5000, biases=False, history=False, mask=False)
    c.v[0] *= 1e30
    c.v[1] += 500
    c.v[2] -= 500
    c.check(*c.call())


def test_broken_rows():
    need_gpu()

    def status_of(**change):
        c = Case(1, 3, 5000)
        c.bias = [[(1, 1.0)], [], [(2, 2.0), (3, 1.0)]]
        c.lens[:] = [40, 3, 40]
        c.prompt[:] = [1, 1, 1]
        c.index[:] = [0, 1, -1]
        for name, (at, v) in change.items():
            getattr(c, name)[at] = v
        c.call()
        return int(c.status.item())

    assert status_of() == 0
    for change in (dict(hist=((0, 5), -1)), dict(hist=((2, 39), 5000)), dict(lens=(1, -1)), dict(lens=(1, 41)),
                   dict(prompt=(1, 4)), dict(prompt=(1, -1)), dict(index=(0, 5)), dict(index=(0, -2)),
                   dict(bias=(0, [(5000, 1.0)])), dict(bias=(2, [(-1, 1.0)]))):
        assert status_of(**change) == C.CORTEX_ST_INPUT_RANGE, change
    # a token past the row's length is not read
    assert status_of(hist=((1, 3), 70000)) == 0


def test_broken_bias_offsets():
    need_gpu()
    c = Case(1, 3, 5000, history=False, mask=False)
    src = columns(c.v, c.t)
    ws = C.workspace(C.cortex_logits_workspace_bytes(3, 5000))
    for off in ([0, 2, 1, 3], [1, 2, 2, 3], [0, 1, 2, 2], [0, 1, 2, 9], [0, -1, 2, 3]):
        status = ints([0])
        C.check(C.cortex_logits_process(src, token=ints([0, 0, 0]), bias_offsets=ints(off), bias_tokens=ints([1, 2, 3]),
                                        bias_values=floats([1, 1, 1]), status=status, ws=ws))
        torch.cuda.synchronize()
        assert int(status.item()) == C.CORTEX_ST_INPUT_RANGE, off
        ws.zero_()


def test_an_earlier_error_leaves_the_outputs():
    need_gpu()
    logits = torch.randn(2, 9000, device="cuda")
    out, token, status = torch.full_like(logits, 5.0), ints([7, 7]), ints([C.CORTEX_ST_CYCLE])
    ws = C.workspace(C.cortex_logits_workspace_bytes(2, 9000))
    C.check(C.cortex_logits_process(logits, out=out, token=token, status=status, ws=ws))
    torch.cuda.synchronize()
    assert bool((out == 5.0).all()) and token.tolist() == [7, 7] and int(status.item()) == C.CORTEX_ST_CYCLE


def test_graph_replays():
    need_gpu()
    announce("logits graph")
    c = Case(8, 4, 20000, "bf16")
    src, status = columns(c.v, c.t), ints([0])
    ws = C.workspace(C.cortex_logits_workspace_bytes(4, 20000))
    out, token, lse = torch.empty_like(src), ints([0] * 4), floats([0] * 4)
    kw = dict(history=ints(c.hist), history_len=ints(c.lens), prompt_len=ints(c.prompt), repetition=floats(c.rep),
              mask=ints(pack(c.allowed)), mask_index=ints(c.index), status=status, ws=ws)
    call = lambda: C.check(C.cortex_logits_process(src, out=out, token=token, lse=lse, **kw))
    call()
    torch.cuda.synchronize()
    want = out.clone(), token.clone(), lse.clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for k in range(4):
        out.zero_(), token.zero_(), lse.zero_()
        torch.cuda.synchronize()
        g.replay()
        call() if k == 2 else None
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((out, token, lse), want)), k


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_many_rows_of_several_tiles(dtype):
    need_gpu()
    for left in (0, 1):
        c = Case(11, 130, 33001, dtype, cap=200, left=left)
        c.check(*c.call("same"))


def test_long_history():
    """Histories that are counted in 32 bits, one token often."""
    need_gpu()
    for R, V in ((2, 5000), (140, 17000)):
        c = Case(12, R, V, cap=40000)
        c.hist[0, :] = 3
        c.lens[0], c.prompt[0] = 40000, 1000
        c.check(*c.call())
    c = Case(13, 2, 5000, cap=32767)                     # the longest in 16 bits
    c.hist[:] = 4999
    c.lens[:], c.prompt[:] = 32767, [0, 5]
    c.check(*c.call())


def test_biases_of_one_token():
    """Every entry names the same token or its neighbour: the last of each counts."""
    need_gpu()
    c = Case(14, 2, 5000, history=False, mask=False)
    c.bias = [[(10 + (k % 2), float(k)) for k in range(1500)], [(4999, 1.0), (4999, -2.0), (0, 4.0)]]
    c.check(*c.call())


def test_too_many_biases():
    need_gpu()
    for n, want in ((65535, 0), (65536, C.CORTEX_ST_INPUT_RANGE)):
        c = Case(15, 1, 70000, history=False, mask=False)
        c.bias = [[(k, 1.0) for k in range(n)]]
        c.call()
        assert int(c.status.item()) == want, n
