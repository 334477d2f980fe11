"""Inputs of the delta rule for its tests, and the bounds on what it must give."""
import numpy as np
import torch

from oracle import sequence_oracle as O
from paper_2011_01383_amd import cortex as C
from tests.gpu_helpers import announce
from tests.sequence_helpers import DTYPES, U, dev, host, offsets_of, type_step, within

LENS = {"one": [1], "two": [2], "chunk": [64], "less": [63], "more": [65], "ragged": [5, 0, 33, 64, 31, 1, 100, 32, 129, 3],
        "empty": [0, 0, 0], "many": [k % 7 for k in range(90)], "long": [400]}


def heads(a, dtype, left=0, right=0):
    """a [T, H, P] on the GPU as columns of a wider array of NaN."""
    T, H, P = a.shape
    wide = torch.full((T, left + H * P + right), float("nan"), dtype=dtype, device="cuda")
    wide[:, left:left + H * P] = torch.from_numpy(np.ascontiguousarray(a.reshape(T, H * P))).to("cuda", dtype)
    return wide[:, left:left + H * P].unflatten(1, (H, P))


class Delta:
    """Inputs of one call, rounded to the operator's types.  Keys have a norm just below 1 (their entries are
    rounded after a factor of 0.99), which the bounds rely on; ``lean`` gives the keys of a text a common direction."""

    def __init__(self, seed, lens, H, G, K, V, dtype="bf16", decay=True, bias=True, soft=True, sig=True, state=True, index=None,
                 rows=None, left=0, lean=0.5, scale=None, slow=1.0):
        r = np.random.default_rng(seed)
        self.dtype, self.left = DTYPES[dtype], left
        self.lens, self.H, self.G, self.K, self.V = list(lens), H, G, K, V
        T, S = int(sum(lens)), len(lens)
        self.T, self.S = T, S
        rnd = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(self.dtype).double().numpy()
        f32 = lambda a: a.astype(np.float32).astype(np.float64)
        unit = lambda a: 0.99 * a / np.sqrt((a * a).sum(-1, keepdims=True))
        self.q, self.k = rnd(unit(r.normal(size=(T, G, K)))), rnd(unit(r.normal(size=(T, G, K)) + lean))
        self.v = rnd(r.normal(size=(T, H, V)))
        self.soft, self.sig = soft, sig
        self.b = rnd(r.normal(size=(T, H)) if sig else r.random((T, H)))
        self.dt = self.A = self.dt_bias = None
        if decay:
            self.dt = rnd(0.5 * r.normal(size=(T, H)) if soft else 0.05 * r.random((T, H)))
            size = 0.001 * 100.0 ** r.random(H)
            self.dt_bias = f32(np.log(np.expm1(size)) if soft else size) if bias else None
            self.A = f32(-slow * (1 + 15 * r.random(H)))
        self.scale = float(np.float32(K ** -0.5 if scale is None else scale))
        self.rows = S if rows is None else rows
        self.index = index
        self.state = f32(0.3 * r.normal(size=(max(self.rows, 1), H * V, K))) if state else None
        self.offsets = offsets_of(lens)

    def reference(self):
        return O.delta(self.q, self.k, self.v, self.b, self.offsets, self.dt, self.A, self.dt_bias, self.soft, self.sig, self.scale,
                       self.index, self.state)

    def upload(self):
        t, l = self.dtype, self.left
        opt = lambda a: None if a is None else dev(a)
        flat = lambda a, r: None if a is None else heads(a[:, :, None], t, l, r)[:, :, 0]
        self.d = dict(q=heads(self.q, t, l), k=heads(self.k, t, 0, l), v=heads(self.v, t, l, l), b=flat(self.b, 0), dt=flat(self.dt, l),
                      A=opt(self.A), dt_bias=opt(self.dt_bias), offsets=dev(self.offsets, torch.int32),
                      index=None if self.index is None else dev(np.array(self.index), torch.int32), state=opt(self.state),
                      status=torch.zeros(1, dtype=torch.int32, device="cuda"),
                      ws=C.workspace(C.cortex_delta_workspace_bytes(self.T, self.S, self.H, self.K, self.V)))
        self.d["y"] = torch.full((self.T, self.H * self.V + l), float("nan"), dtype=t,
                                 device="cuda")[:, :self.H * self.V].unflatten(1, (self.H, self.V))
        return self.d

    def call(self, step=False, state_in="state", state_out=None, stream=None):
        d = self.d
        kw = dict(dt=d["dt"], A=d["A"], dt_bias=d["dt_bias"], softplus=self.soft, sigmoid=self.sig, scale=self.scale,
                  state_in=d["state"] if isinstance(state_in, str) else state_in, state_out=state_out, state_index=d["index"],
                  status=d["status"], stream=stream)
        if step:
            return C.cortex_delta_step(d["q"], d["k"], d["v"], d["b"], d["y"], **kw)
        return C.cortex_delta_forward(d["q"], d["k"], d["v"], d["b"], d["offsets"], d["y"], ws=d["ws"], **kw)

    def check(self, y, state, label):
        """Bounds: every float32 step of a token is a sum of at most K + 64 products, off by at most 2 U of the
        magnitudes added a term, and the exponentials and gates by a few U more; the oracle's magnitude passes
        these on through the tokens.  A decay's exponent is at most 6 where the decay leaves something, so
        its error is below 16 U.  Outputs are rounded once more."""
        ref, mag, new = self.reference()
        f32 = (2 * (self.K + 64) + 32) * U
        within(host(y), ref, f32 * mag + type_step(self.dtype) * np.abs(ref) + 1e-30, label + " y")
        if state is not None:
            got = host(state)
            for row, (h, m) in new.items():
                within(got[row], h, np.broadcast_to(f32 * m + 1e-30, h.shape), label + " state %d" % row)
        return new


def say(*what):
    announce(" ".join(str(w) for w in what))
