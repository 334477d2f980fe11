"""The chunks of the delta rule's prompts in float64, with operands held to fewer bits where asked: what a lost
plane of a product's operands would do."""
import numpy as np

from oracle import sequence_oracle as O

CHUNK = 64


def cut(a, bits):
    """a in `bits` bits, rounded to nearest."""
    if bits is None:
        return a
    m, e = np.frexp(a)
    return np.ldexp(np.rint(np.ldexp(m, bits)), e - bits)


def prompt(p, **bits):
    """y and {pool row: state} of p's prompts; bits of S (where keys and queries multiply it), T, P, R, U or W (the
    updates as the next state takes them), or of the state itself (`held`) at every chunk's end."""
    of = np.arange(p.H) // (p.H // p.G)
    keep = lambda name, a: cut(a, bits.get(name))
    raw = 0.0 if p.A is None else p.dt + (0 if p.dt_bias is None else p.dt_bias)
    e = np.zeros((p.T, p.H)) if p.A is None else (O.softplus(raw) if p.soft else raw) * p.A
    beta = 1 / (1 + np.exp(-p.b)) if p.sig else p.b
    y, new = np.zeros((p.T, p.H, p.V)), {}
    for _, i, j, row in O.rows_of(p.offsets, p.index):
        S = np.zeros((p.H, p.V, p.K)) if row < 0 or p.state is None else p.state[row].reshape(p.H, p.V, p.K).copy()
        for t in range(i, j, CHUNK):
            at = slice(t, min(t + CHUNK, j))
            n = at.stop - t
            k, q = p.k[at][:, of].transpose(1, 0, 2), p.q[at][:, of].transpose(1, 0, 2)         # [H, n, K]
            v, b, c = p.v[at].transpose(1, 0, 2), beta[at].T[..., None], np.cumsum(e[at], 0).T  # [H, n, V], [H, n, 1], [H, n]
            between = np.tril(np.exp(np.minimum(c[:, :, None] - c[:, None, :], 0.0)))
            L = np.tril(b * between * (k @ k.transpose(0, 2, 1)), -1)
            T = np.linalg.inv(np.eye(n) + L)
            P = p.scale * between * (q @ k.transpose(0, 2, 1))
            St, grow = keep("S", S).transpose(0, 2, 1), np.exp(c)[..., None]
            U = keep("T", T) @ keep("R", b * (v - grow * (k @ St)))
            y[at] = (p.scale * grow * (q @ St) + keep("P", P) @ keep("U", U)).transpose(1, 0, 2)
            S = np.exp(c[:, -1])[:, None, None] * S + keep("W", np.exp(c[:, -1:] - c)[..., None] * U).transpose(0, 2, 1) @ k
            S = keep("held", S)
        if row >= 0:
            new[row] = S.reshape(p.H * p.V, p.K)
    return y, new


def distance(got, ref):
    """||got - ref|| / ||ref||, 2-norms over all entries."""
    return float(np.sqrt(((got - ref) ** 2).sum() / (ref ** 2).sum()))
