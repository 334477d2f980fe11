"""Plain float64 definitions of the sequence operators (test infrastructure).

Token by token over numpy arrays, no code shared with the GPU path.  Every
function also returns the magnitudes that an error bound is taken from: the same
sums with every term's absolute value.
"""
from __future__ import annotations

import numpy as np


def silu(v):
    return v / (1.0 + np.exp(-v))


def softplus(v):
    return np.logaddexp(v, 0.0)


def rows_of(offsets, index):
    """(sequence, first row, end row, pool row or -1)."""
    for i in range(len(offsets) - 1):
        yield i, int(offsets[i]), int(offsets[i + 1]), i if index is None else int(index[i])


def conv(x, weight, bias, act, offsets, index=None, state=None, rows=0):
    """y [T, C], magnitude [T, C], {pool row: new state [W-1, C]}."""
    T, C = x.shape
    W = weight.shape[1]
    y, mag, new = np.zeros((T, C)), np.zeros((T, C)), {}
    for _, a, b, row in rows_of(offsets, index):
        old = np.zeros((W - 1, C)) if row < 0 or state is None else state[row]
        text = np.concatenate([old, x[a:b]])
        for t in range(b - a):
            win = text[t:t + W].T
            y[a + t] = (win * weight).sum(1) + (0 if bias is None else bias)
            mag[a + t] = np.abs(win * weight).sum(1) + (0 if bias is None else np.abs(bias))
        if row >= 0:
            new[row] = text[b - a:]
    return (silu(y) if act else y), mag, new


def scan(x, dt, A, B, C, offsets, skip=None, z=None, dt_bias=None, soft=True, index=None, state=None):
    """y [T, D], its magnitude, {pool row: (new state [D, N], its magnitude)}."""
    T, D = x.shape
    G, N = B.shape[1:]
    H = A.shape[0]
    P = D // H
    per = lambda v: np.repeat(v, P, axis=-1)
    raw = dt + (0 if dt_bias is None else dt_bias)
    step = softplus(raw) if soft else raw
    AA = A if A.ndim == 2 else np.repeat(A[:, None], P, 0)          # [D, N] or [D, 1]
    y, mag, new = np.zeros((T, D)), np.zeros((T, D)), {}
    for _, a, b, row in rows_of(offsets, index):
        h = np.zeros((D, N)) if row < 0 or state is None else state[row].copy()
        m = np.abs(h)
        for t in range(a, b):
            d = per(step[t])[:, None] if A.ndim == 1 else step[t][:, None]
            Bt, Ct = np.repeat(B[t], D // G, 0), np.repeat(C[t], D // G, 0)
            decay, add = np.exp(d * AA), d * x[t][:, None] * Bt
            h, m = decay * h + add, decay * m + np.abs(add)
            y[t], mag[t] = (h * Ct).sum(1), (m * np.abs(Ct)).sum(1)
            if skip is not None:
                s = per(skip) if A.ndim == 1 else skip
                y[t] += s * x[t]
                mag[t] += np.abs(s * x[t])
        if row >= 0:
            new[row] = (h, m)
    if z is not None:
        y, mag = y * silu(z), mag * np.abs(silu(z))
    return y, mag, new


def logits(v, history=None, history_len=None, prompt_len=None, repetition=None, frequency=None, presence=None,
           biases=None, allowed=None):
    """One row, each operation in float32 (the operator states its roundings); the
    normaliser in float64.  biases: [(token, value)]; allowed: [V] booleans."""
    f = np.float32
    v = v.astype(f).copy()
    V = len(v)
    if history is not None:
        text = history[:history_len]
        n = np.bincount(text[prompt_len:], minlength=V)
        seen = np.bincount(text, minlength=V) > 0
        r = f(1 if repetition is None else repetition)
        with np.errstate(invalid="ignore", over="ignore"):
            v = np.where(seen, np.where(v > 0, v / r, v * r), v).astype(f)
            if frequency is not None:
                v = np.where(n > 0, v - f(frequency) * n.astype(f), v).astype(f)
            if presence is not None:
                v = np.where(n > 0, v - f(presence), v).astype(f)
    if biases:
        last = dict(biases)
        for t, b in last.items():
            v[t] = v[t] + f(b)
    if allowed is not None:
        v = np.where(allowed, v, f(-np.inf))
    if np.isnan(v).any():
        return v, int(np.argmax(np.isnan(v))), float("nan")
    top = v.max()
    if top == -np.inf:
        return v, -1, -np.inf
    token = int(np.argmax(v))
    if top == np.inf:
        return v, token, np.inf
    w = v.astype(np.float64)
    return v, token, float(top + np.log(np.exp(w - top).sum()))


def delta(q, k, v, b, offsets, dt=None, A=None, dt_bias=None, soft=True, sig=True, scale=1.0, index=None, state=None):
    """The gated delta rule: y [T, H, V], its magnitude, {pool row: (new state [H V, K], its magnitude [H V, 1])}.

    With |k| <= 1 and beta in [0, 1] a token's map of a state row shrinks (2-norm), so a row's error is at
    most a times what it was, plus what the token's own roundings add: those are parts of a |S| and of
    beta (|v| + a |S|).  The magnitude is that sum."""
    T, H, V = v.shape
    G, K = k.shape[1:]
    of = np.arange(H) // (H // G)
    raw = None if A is None else dt + (0 if dt_bias is None else dt_bias)
    a = np.ones((T, H)) if A is None else np.exp((softplus(raw) if soft else raw) * A)
    beta = 1.0 / (1.0 + np.exp(-b)) if sig else b
    y, mag, new = np.zeros((T, H, V)), np.zeros((T, H, V)), {}
    for _, i, j, row in rows_of(offsets, index):
        S = np.zeros((H, V, K)) if row < 0 or state is None else state[row].reshape(H, V, K).copy()
        m = np.sqrt((S * S).sum(-1))
        for t in range(i, j):
            kt, qt = k[t][of], q[t][of]
            S = S * a[t][:, None, None]
            old = np.sqrt((S * S).sum(-1))
            u = beta[t][:, None] * (v[t] - (S * kt[:, None]).sum(-1))
            S = S + u[..., None] * kt[:, None]
            m = a[t][:, None] * m + old + np.abs(beta[t])[:, None] * (np.abs(v[t]) + old)
            y[t] = scale * (S * qt[:, None]).sum(-1)
            mag[t] = abs(scale) * m * np.sqrt((qt * qt).sum(-1))[:, None]
        if row >= 0:
            new[row] = (S.reshape(H * V, K), m.reshape(H * V, 1))
    return y, mag, new


def qk_norm(x, norm, eps, weight=None, positions=None, freqs=None, interleaved=False):
    """x [T, H, P] normed per head, weighted and rotated; and the sum of the magnitudes behind every output."""
    P = x.shape[-1]
    size = 1.0 if norm == "none" else np.sqrt((x * x).sum(-1, keepdims=True) / (P if norm == "rms" else 1) + eps)
    v = x / size * (1.0 if weight is None else weight)
    mag = np.abs(v)
    if freqs is None or len(freqs) == 0:
        return v, mag
    R = 2 * len(freqs)
    f = positions.astype(np.float64)[:, None, None] * freqs
    i = np.arange(R // 2) * 2 if interleaved else np.arange(R // 2)
    j = i + 1 if interleaved else i + R // 2
    out, m = v.copy(), mag.copy()
    out[..., i] = v[..., i] * np.cos(f) - v[..., j] * np.sin(f)
    out[..., j] = v[..., j] * np.cos(f) + v[..., i] * np.sin(f)
    m[..., i] = m[..., j] = mag[..., i] + mag[..., j]
    return out, m


def quant_rows(x):
    """8-bit rows and their scales, by the float32 roundings that define them (x float32)."""
    x = x.astype(np.float32)
    bad = ~np.isfinite(x).all(1)
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        scale = np.abs(x).max(1) / np.float32(127)
        q = np.clip(np.rint(x / scale[:, None]), -127, 127)
    q[(scale == 0) | bad] = 0
    scale[bad] = np.nan
    return q.astype(np.int8), scale
