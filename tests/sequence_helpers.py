"""Shared helpers of the sequence operators' tests."""
import numpy as np
import torch

from paper_2011_01383_amd import cortex as C
from oracle import sequence_oracle as O

U = 2.0 ** -24            # half a unit in the last place of float32, relative
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def offsets_of(lens):
    return np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)


def dev(a, dtype=torch.float32):
    return torch.from_numpy(np.ascontiguousarray(a)).to(dtype).cuda()


def host(t):
    return t.detach().cpu().double().numpy()


def columns(a, dtype, left=0, right=0):
    """a [T, C] on the GPU as columns of a wider array."""
    T, cols = a.shape
    wide = torch.full((T, left + cols + right), float("nan"), dtype=dtype, device="cuda")
    wide[:, left:left + cols] = torch.from_numpy(np.ascontiguousarray(a)).to("cuda", dtype)
    return wide[:, left:left + cols]


def type_step(dtype):
    """Largest relative rounding of a store."""
    return 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24


def within(got, ref, tol, what):
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    assert np.isfinite(got).all(), "%s has non-finite values" % what
    d = np.abs(got - ref)
    bad = d > tol
    assert not bad.any(), "%s: %d of %d off, worst %.3g at %s (allowed %.3g)" % (
        what, bad.sum(), bad.size, d[bad].max(), np.argwhere(bad)[0], np.broadcast_to(tol, d.shape)[bad].min())


class Scan:
    """Inputs of one scan, rounded to the operator's types, and what it must give."""

    def __init__(self, seed, lens, D, N, G=1, P=0, dtype="bf16", z=True, skip=True, bias=True, soft=True, state=True,
                 index=None, rows=None, left=0, dt_scale=0.5, slow=False):
        r = np.random.default_rng(seed)
        self.dtype = DTYPES[dtype]
        self.lens, self.D, self.N, self.G, self.P = lens, D, N, G, P
        T, S = int(sum(lens)), len(lens)
        self.T, self.S, self.left = T, S, left
        H = D // P if P else D
        rnd = lambda a: torch.from_numpy(a).to(self.dtype).double().numpy()
        f32 = lambda a: a.astype(np.float32).astype(np.float64)
        self.x, self.B, self.C = rnd(r.normal(size=(T, D))), rnd(r.normal(size=(T, G, N))), rnd(r.normal(size=(T, G, N)))
        self.z = rnd(r.normal(size=(T, D))) if z else None
        self.soft = soft
        self.dt = rnd(r.normal(size=(T, H)) * dt_scale) if soft else rnd(np.abs(r.normal(size=(T, H))) * 0.05)
        size = 0.001 * 100.0 ** r.random(H)
        # without the softplus the bias is a part of the step size itself, which is not negative
        self.dt_bias = f32(np.log(np.expm1(size)) if soft else size) if bias else None
        a = 0.02 if slow else 1.0
        self.A = f32(-a * (1 + 15 * r.random(H))) if P else f32(-a * np.arange(1, N + 1) * (0.9 + 0.2 * r.random((D, N))))
        self.skip = f32(1 + 0.1 * r.normal(size=H)) if skip else None
        self.rows = S if rows is None else rows
        self.index = index
        self.state = f32(0.3 * r.normal(size=(max(self.rows, 1), D, N))) if state else None
        self.offsets = offsets_of(lens)

    def reference(self):
        return O.scan(self.x, self.dt, self.A, self.B, self.C, self.offsets, self.skip, self.z, self.dt_bias, self.soft,
                      self.index, self.state)

    def upload(self):
        opt = lambda a: None if a is None else dev(a)
        t, l = self.dtype, self.left
        flat = lambda a: a.reshape(self.T, self.G * self.N)
        self.d = dict(x=columns(self.x, t, l, l), dt=columns(self.dt, t, l), z=None if self.z is None else columns(self.z, t, 0, l),
                      B=columns(flat(self.B), t, l).unflatten(1, (self.G, self.N)),
                      C=columns(flat(self.C), t, l, l).unflatten(1, (self.G, self.N)), A=dev(self.A), skip=opt(self.skip),
                      dt_bias=opt(self.dt_bias), offsets=dev(self.offsets, torch.int32),
                      index=None if self.index is None else dev(np.array(self.index), torch.int32),
                      status=torch.zeros(1, dtype=torch.int32, device="cuda"))
        self.d["y"] = torch.full((self.T, self.D + l), float("nan"), dtype=t, device="cuda")[:, :self.D]
        self.d["state"] = None if self.state is None else dev(self.state)
        self.d["ws"] = C.workspace(C.cortex_scan_workspace_bytes(self.T, self.S, self.D, self.N, self.P))
        return self.d

    def call(self, step=False, state_in="state", state_out=None, stream=None):
        d = self.d
        kw = dict(D=d["skip"], z=d["z"], dt_bias=d["dt_bias"], softplus=self.soft,
                  state_in=d["state"] if state_in == "state" else state_in,
                  state_out=state_out, state_index=d["index"], status=d["status"], stream=stream)
        if step:
            return C.cortex_scan_step(d["x"], d["dt"], d["A"], d["B"], d["C"], d["y"], **kw)
        return C.cortex_scan_forward(d["x"], d["dt"], d["A"], d["B"], d["C"], d["offsets"], d["y"], ws=d["ws"], **kw)

    def check(self, y, state, label):
        """Bounds.  A state is a sum of terms, each multiplied by at most L decays.  A decay
        exp(dt A) carries the error of its exponent, a few U of |dt A| (below 6 here, a decay that
        large in the exponent leaves nothing to be wrong about) and of the step size, and one
        rounding: 8 U a token and term covers it.  N terms are added for y.  Outputs of 16 bits are
        rounded once more, after products whose operands may be held to 16 bits."""
        ref, mag, new = self.reference()
        L = max([1] + list(self.lens))
        f32 = 8 * (L + self.N + 8) * U
        tol = f32 * mag + type_step(self.dtype) * np.abs(ref) + (2.0 ** -14 * mag if self.dtype == torch.bfloat16 else 0)
        within(host(y), ref, tol + 1e-30, label + " y")
        if state is not None:
            got = host(state)
            for row, (h, m) in new.items():
                within(got[row], h, f32 * m + 1e-30, label + " state %d" % row)
        return new
