"""The per-head scan's products over sub-chunks of 32 tokens, emulated on the CPU in float32
with the library's splits into bf16 planes, so that a test's bound can be held against a form
that keeps too few of them.  Test infrastructure: nothing of the library calls it."""
import numpy as np

SUB = 32
f32 = np.float32


def upper(v):
    """The upper 16 bits of each float: a bf16 plane."""
    return (np.ascontiguousarray(v, f32).view(np.uint32) & np.uint32(0xffff0000)).view(f32)


def held(v, planes):
    """v as `planes` bf16 planes together hold it."""
    left, sum_ = np.array(v, f32), np.zeros_like(v, dtype=f32)
    for _ in range(planes):
        p = upper(left)
        sum_, left = (sum_ + p).astype(f32), (left - p).astype(f32)
    return sum_


def below(v, s):
    """v of the lane that the shift by s names, 0 where it leaves one out: 1, 2, 4 and 8 stay in a
    row of 16 lanes, 16 is lane 15 to the upper row."""
    b = np.zeros_like(v)
    if s == 16:
        b[16:] = v[15]
    else:
        b[s:16], b[16 + s:] = v[:16 - s], v[16:-s]
    return b


def prefix(e, low=None):
    """Inclusive sums over 32 tokens in the order of the lanes' shifts; `low`, if given, collects what
    their roundings left."""
    hi, lo = np.array(e, f32), np.zeros(SUB, f32)
    for s in (1, 2, 4, 8, 16):
        b, b_lo = below(hi, s), below(lo, s)
        total = (hi + b).astype(f32)
        t = (total - hi).astype(f32)
        lo = ((lo + b_lo) + ((hi - (total - t)) + (b - t))).astype(f32)
        hi = total
    if low is not None:
        low[:] = lo
    return hi


def head_scan(x, dt, A, B, C, h0, planes_score=3, planes_read=3, planes_add=3, exact_sums=True):
    """One head, one sequence of whole sub-chunks: x [T, P], dt [T], B and C [T, N], h0 [P, N].
    Returns y and the last state."""
    A2 = f32(f32(A) * f32(1.44269504088896340736))
    h, y = h0.astype(f32), np.zeros(x.shape, f32)
    lower = np.tril(np.ones((SUB, SUB), bool))
    for t0 in range(0, len(x), SUB):
        s = slice(t0, t0 + SUB)
        xs, Bs, Cs, d = x[s].astype(f32), B[s].astype(f32), C[s].astype(f32), dt[s].astype(f32)
        e = (d * A2).astype(f32)
        low = np.zeros(SUB, f32)
        cum = prefix(e, low)
        low *= exact_sums
        after = np.concatenate([prefix(e[::-1])[:-1][::-1], [f32(0)]])
        decay = np.exp2(prefix(e[::-1])[-1])
        with np.errstate(over="ignore", invalid="ignore"):
            between = (cum[:, None] - cum[None]) + (low[:, None] - low[None])
            score = ((Cs @ Bs.T) * (np.exp2(between) * d)).astype(f32)
        score = held(np.where(lower, score, f32(0)), planes_score)
        y[s] = (Cs @ held(h, planes_read).T) * np.exp2(cum)[:, None] + score @ xs
        weighted = held((xs * (np.exp2(after) * d)[:, None]).astype(f32), planes_add)
        h = (h * decay + weighted.T @ Bs).astype(f32)
    return y, h
