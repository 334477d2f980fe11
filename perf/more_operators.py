"""Cases by which the operators of a layer with the gated delta rule are measured: the rule itself,
the norms and rotation of its queries and keys, and the 8-bit projections around it.

``kind`` of a case and what it stands for in a program that serves such a model:

* ``delta``        the gated delta rule over a batch of prompts of different lengths
* ``delta_step``   one new token of every running sequence, the states in a pool
* ``norm``         queries and keys of every head normed, weighted and rotated by their positions
* ``linear``       a projection with weights in 8 bits: tokens to 8 bits, the product, scales and bias

Inputs are what such a program has in hand: activations as the columns of packed projections, offsets
of the sequences on the GPU, states in a pool addressed by slot, weights quantised when they were loaded.
"""
import math
import random

import numpy as np
import torch

own = False
DEVICE = "cuda"
CHUNK = 64


def listed():
    return [
        # an ordinary batch of prompts, two heads of values for each of queries and keys
        {"name": "delta-prompts", "kind": "delta", "dtype": "bf16", "tokens": 8192, "seqs": 16, "heads": 32, "key_heads": 16, "key_dim": 128, "value_dim": 128},
        # the prompts of a small 32-bit model
        {"name": "delta-prompts-f32", "kind": "delta", "dtype": "f32", "tokens": 4099, "seqs": 5, "heads": 8, "key_heads": 8, "key_dim": 64, "value_dim": 64},
        # the largest: one long document
        {"name": "delta-long", "kind": "delta", "dtype": "bf16", "tokens": 32768, "seqs": 1, "heads": 32, "key_heads": 16, "key_dim": 128, "value_dim": 128},
        # a batch generating: the states' bytes
        {"name": "delta-tokens", "kind": "delta_step", "dtype": "bf16", "seqs": 64, "heads": 32, "key_heads": 16, "key_dim": 128, "value_dim": 128},
        # one interactive row: latency counts
        {"name": "delta-one-token", "kind": "delta_step", "dtype": "bf16", "seqs": 1, "heads": 32, "key_heads": 16, "key_dim": 128, "value_dim": 128},
        # a batch of prompts, fewer heads of keys than of queries
        {"name": "norm-prompts", "kind": "norm", "dtype": "bf16", "tokens": 8192, "heads": 32, "key_heads": 8, "head_dim": 128, "rotary": 128, "pairs": "halves", "norm": "rms"},
        # a few tokens, a quarter of each head rotated
        {"name": "norm-few-tokens", "kind": "norm", "dtype": "bf16", "tokens": 7, "heads": 16, "key_heads": 16, "head_dim": 128, "rotary": 32, "pairs": "halves", "norm": "l2"},
        # a 32-bit model's prompts, neighbouring elements rotated
        {"name": "norm-prompts-f32", "kind": "norm", "dtype": "f32", "tokens": 1021, "heads": 8, "key_heads": 8, "head_dim": 64, "rotary": 64, "pairs": "neighbours", "norm": "rms"},
        # one interactive row: the weights' bytes
        {"name": "linear-one-token", "kind": "linear", "dtype": "bf16", "tokens": 1, "inputs": 4096, "outputs": 8192, "bias": False},
        # a batch generating
        {"name": "linear-tokens", "kind": "linear", "dtype": "bf16", "tokens": 64, "inputs": 2048, "outputs": 8192, "bias": True},
        # a batch of prompts: the matrix units
        {"name": "linear-prompts", "kind": "linear", "dtype": "bf16", "tokens": 8192, "inputs": 4096, "outputs": 8192, "bias": False},
        # a short prompt of a 32-bit model, odd sizes
        {"name": "linear-odd-f32", "kind": "linear", "dtype": "f32", "tokens": 333, "inputs": 1001, "outputs": 2003, "bias": True},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the ranges above, odd sizes among them."""
    kind = rng.choice(["delta", "delta", "delta", "delta_step", "norm", "norm", "linear", "linear", "linear"])
    case = {"kind": kind, "dtype": rng.choice(["bf16", "bf16", "f32"])}
    if kind == "norm":
        case["tokens"] = _log_int(rng, 1, 8192)
        case["head_dim"] = rng.choice([32, 64, 80, 96, 128, 128, 256])
        case["key_heads"] = _log_int(rng, 1, 16)
        case["heads"] = case["key_heads"] * rng.choice([1, 1, 2, 4])
        case["rotary"] = 2 * int(case["head_dim"] // 2 * rng.choice([0, 0.25, 0.5, 1, 1]))
        case["pairs"] = rng.choice(["halves", "halves", "neighbours"])
        case["norm"] = rng.choice(["rms", "rms", "l2"])
        return case
    if kind == "linear":
        case["inputs"], case["outputs"] = _log_int(rng, 64, 8192), _log_int(rng, 64, 16384)
        most = 8192 * 4096 * 8192 // (case["inputs"] * case["outputs"])
        case["tokens"] = _log_int(rng, 1, min(8192, most))
        case["bias"] = rng.random() < 0.5
        return case
    case["key_heads"] = _log_int(rng, 1, 16)
    case["heads"] = case["key_heads"] * rng.choice([1, 1, 2, 4])
    case["key_dim"], case["value_dim"] = rng.choice([32, 64, 128, 128]), rng.choice([16, 32, 64, 128, 128, 256])
    state = case["heads"] * case["key_dim"] * case["value_dim"]
    if kind == "delta_step":
        case["seqs"] = _log_int(rng, 1, min(256, max(1, 33_000_000 // state)))
    else:
        case["tokens"] = _log_int(rng, 1, max(64, min(24576, 8_000_000_000 // state)))
        case["seqs"] = _log_int(rng, 1, min(64, max(1, 33_000_000 // state)))
    return case


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _lengths(case, seed):
    """Lengths of the sequences: a ramp that sums to ``tokens``, in the seed's order; where there are
    more sequences than tokens some have none."""
    T, S = case["tokens"], case["seqs"]
    ends = [T * i * (i + 1) // (S * (S + 1)) for i in range(S + 1)]
    lens = [b - a for a, b in zip(ends, ends[1:])]
    random.Random(seed).shuffle(lens)
    return lens


def prepare(case, seed):
    from types import SimpleNamespace
    kind = case["kind"]
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    typ = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=DEVICE, dtype=torch.float32)

    def unit(*shape):
        return torch.rand(*shape, generator=g, device=DEVICE, dtype=torch.float32)

    def ints(v):
        return torch.tensor(v, dtype=torch.int32, device=DEVICE)

    s = SimpleNamespace(case=case, kind=kind, status=ints([0]), workspace=None)
    if kind == "norm":
        T, H, Hk, P, R = case["tokens"], case["heads"], case["key_heads"], case["head_dim"], case["rotary"]
        s.norm, s.interleaved, s.eps = case["norm"], case["pairs"] == "neighbours", 1e-6
        packed = normal(T, (H + 2 * Hk) * P).to(typ)          # the projection's output: queries, keys and values
        s.q, s.k = packed[:, :H * P].unflatten(1, (H, P)), packed[:, H * P:(H + Hk) * P].unflatten(1, (Hk, P))
        s.q_weight, s.k_weight = 1.0 + 0.1 * normal(P), 1.0 + 0.1 * normal(P)
        # places in texts that have been running for up to 200,000 tokens
        begin = torch.randint(0, 200000, (8,), generator=g, device=DEVICE)
        at = torch.arange(T, device=DEVICE)
        s.positions = (begin[at * 8 // max(T, 1)] + at).to(torch.int32)
        s.freqs = (10000.0 ** (-torch.arange(0, R, 2, device=DEVICE, dtype=torch.float64) / max(R, 1))).float()
        s.q_out, s.k_out = torch.empty(T, H, P, dtype=typ, device=DEVICE), torch.empty(T, Hk, P, dtype=typ, device=DEVICE)
        return s
    if kind == "linear":
        T, K, N = case["tokens"], case["inputs"], case["outputs"]
        s.x = (normal(T, K) * torch.exp(0.5 * normal(T, 1))).to(typ)
        w = normal(N, K) / math.sqrt(K)
        s.w_scale = w.abs().amax(1) / 127.0
        s.w = torch.zeros(N, (K + 15) // 16 * 16, dtype=torch.int8, device=DEVICE)[:, :K]    # rows begin at 16 bytes
        s.w.copy_(torch.round(w / s.w_scale[:, None]).clamp(-127, 127))
        s.bias = 0.1 * normal(N) if case["bias"] else None
        s.y = torch.empty(T, N, dtype=typ, device=DEVICE)
        if own:                                  # the plain form needs none
            from paper_2011_01383_amd import cortex
            s.workspace = cortex.workspace(cortex.cortex_linear_i8_workspace_bytes(T, N, K), DEVICE)
        return s
    S, H, Hk, K, V = case["seqs"], case["heads"], case["key_heads"], case["key_dim"], case["value_dim"]
    step = kind == "delta_step"
    T = S if step else case["tokens"]
    lens = [1] * S if step else _lengths(case, seed)
    s.T, s.longest, s.scale = T, max(lens), K ** -0.5
    s.offsets = ints([0] + np.cumsum(lens).tolist())
    s.slots = torch.randperm(S, generator=g, device=DEVICE).to(torch.int32)
    # the convolution's output through its activation: keys of one text lean to one side; norms of one
    q, k = (_silu(normal(T, Hk, K)) for _ in range(2))
    s.q, s.k = ((v * torch.rsqrt((v * v).sum(-1, keepdim=True) + 1e-6)).to(typ) for v in (q, k))
    s.v = _silu(normal(T, 2 * Hk * K + H * V)).to(typ)[:, 2 * Hk * K:].unflatten(1, (H, V))
    ba = normal(T, 2 * H).to(typ)                # gates of the update and raw step sizes side by side
    s.b, s.dt = ba[:, :H], (0.5 * ba)[:, H:]
    # step sizes around 0.001 to 0.1 after the softplus, decays as such layers are initialised
    s.dt_bias = torch.log(torch.expm1(torch.exp(unit(H) * math.log(100.0)) * 0.001))
    s.A = -(1.0 + 15.0 * unit(H))
    s.state = 0.1 * normal(S, H * V, K)
    s.y, s.state_out = torch.empty(T, H, V, dtype=typ, device=DEVICE), torch.empty_like(s.state)
    if own and not step:
        from paper_2011_01383_amd import cortex
        s.workspace = cortex.workspace(cortex.cortex_delta_workspace_bytes(T, S, H, K, V), DEVICE)
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(state):
    return _own(state) if own else _PLAIN[state.kind](state)


def _own(s):
    from paper_2011_01383_amd import cortex
    if s.kind == "norm":
        norm = cortex.CORTEX_NORM_RMS if s.norm == "rms" else cortex.CORTEX_NORM_L2
        rotation = dict(positions=s.positions, freqs=s.freqs, interleaved=s.interleaved) if s.freqs.numel() else {}
        rc = cortex.cortex_qk_norm(s.q, s.q_out, k=s.k, k_out=s.k_out, norm=norm, eps=s.eps, q_weight=s.q_weight,
                                   k_weight=s.k_weight, status=s.status, **rotation)
        cortex.check(rc, "norm")
        return {"q": s.q_out, "k": s.k_out}
    if s.kind == "linear":
        rc = cortex.cortex_linear_i8(s.x, s.w, s.w_scale, s.y, bias=s.bias, status=s.status, ws=s.workspace)
        cortex.check(rc, "linear")
        return {"y": s.y}
    kw = dict(dt=s.dt, A=s.A, dt_bias=s.dt_bias, softplus=True, sigmoid=True, scale=s.scale, state_in=s.state,
              state_out=s.state_out, state_index=s.slots, status=s.status)
    if s.kind == "delta":
        rc = cortex.cortex_delta_forward(s.q, s.k, s.v, s.b, s.offsets, s.y, ws=s.workspace, **kw)
    else:
        rc = cortex.cortex_delta_step(s.q, s.k, s.v, s.b, s.y, **kw)
    cortex.check(rc, s.kind)
    return {"y": s.y, "state": s.state_out}


def _silu(v):
    return v / (1.0 + torch.exp(-v))


def _softplus(v):
    return torch.clamp(v, min=0) + torch.log1p(torch.exp(-torch.abs(v)))


def _plain_norm(s):
    R = 2 * s.freqs.numel()
    # far positions: angles in 64 bits
    angle = s.positions.double()[:, None, None] * s.freqs.double()
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()

    def one(x, weight):
        v = x.float()
        square = v * v
        v = v * torch.rsqrt((square.mean(-1, keepdim=True) if s.norm == "rms" else square.sum(-1, keepdim=True)) + s.eps) * weight
        turned = v[..., :R]
        if s.interleaved:
            a, b = turned[..., 0::2], turned[..., 1::2]
            turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
        else:
            a, b = turned[..., :R // 2], turned[..., R // 2:]
            turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
        return torch.cat([turned, v[..., R:]], -1).to(x.dtype)

    return {"q": one(s.q, s.q_weight), "k": one(s.k, s.k_weight)}


def _to_8_bits(x):
    """Whole numbers as floats, and the scale of every row; a row of zeros has a scale of 0."""
    v = x.float()
    scale = v.abs().amax(1) / 127.0
    return torch.where(scale[:, None] > 0, torch.round(v / scale[:, None]), 0.0), scale


def _plain_linear(s):
    # products and partial sums are whole numbers: the float32 product is at most a rounding off
    q, scale = _to_8_bits(s.x)
    y = torch.matmul(q, s.w.float().t().contiguous()) * scale[:, None] * s.w_scale
    return {"y": (y if s.bias is None else y + s.bias).to(s.x.dtype)}


def _per_head(v, heads, dim):
    return v.float().repeat_interleave(heads // v.shape[dim], dim)


def _steps(s):
    """log of the decay, and the update's share, per token and head."""
    return _softplus(s.dt.float() + s.dt_bias) * s.A, 1.0 / (1.0 + torch.exp(-s.b.float()))


def _plain_delta_step(s):
    H, V = s.v.shape[1:]
    g, beta = _steps(s)
    q, k = _per_head(s.q, H, 1), _per_head(s.k, H, 1)
    h = s.state[s.slots.long()].unflatten(1, (H, V)) * torch.exp(g)[:, :, None, None]
    u = beta[:, :, None] * (s.v.float() - (h * k[:, :, None]).sum(-1))
    h = h + u[..., None] * k[:, :, None]
    out = torch.empty_like(s.state)
    out[s.slots.long()] = h.flatten(1, 2)
    return {"y": (s.scale * (h * q[:, :, None]).sum(-1)).to(s.v.dtype), "state": out}


def _unit_lower_inverse(A):
    """(I + A)^-1 of strictly lower A [.., n, n], n a power of two: inverses of the diagonal's blocks, doubled."""
    n, size = A.shape[-1], 1
    X = torch.ones(A.shape[:-2] + (n, 1, 1), device=A.device, dtype=A.dtype)
    while size < n:
        blocks = A.unflatten(-1, (-1, 2 * size)).unflatten(-3, (-1, 2 * size)).diagonal(0, -4, -2).movedim(-1, -3)
        low = blocks[..., size:, :size].contiguous()
        X = X.unflatten(-3, (-1, 2))
        first, second = X[..., 0, :, :].contiguous(), X[..., 1, :, :].contiguous()
        corner = -torch.matmul(second, torch.matmul(low, first))
        X = torch.cat([torch.cat([first, torch.zeros_like(first)], -1), torch.cat([corner, second], -1)], -2)
        size *= 2
    return X.squeeze(-3)


def _plain_delta(s):
    """By chunks of CHUNK tokens of one sequence, as matrix products; a chunk maps the state that enters it to
    M state + N, and the maps are joined by doubling."""
    T, H, V = s.v.shape
    S, K, Q = s.slots.numel(), s.k.shape[2], CHUNK
    off = s.offsets.long()
    first, lens = off[:-1], off[1:] - off[:-1]
    seq = torch.repeat_interleave(torch.arange(S, device=DEVICE), lens, output_size=T)
    chunks = T // Q + S                          # at least as many as there are
    at = first // Q + torch.arange(S, device=DEVICE)   # first chunk of each sequence
    of = torch.searchsorted(at, torch.arange(chunks, device=DEVICE), right=True) - 1
    begin = (torch.arange(chunks, device=DEVICE) - at[of]) * Q
    tok = begin[:, None] + torch.arange(Q, device=DEVICE)
    live = tok < lens[of][:, None]
    tok = (first[of][:, None] + tok).clamp(max=T - 1)
    g, beta = (torch.where(live[:, :, None], v[tok], 0.0).permute(0, 2, 1) for v in _steps(s))      # [c, H, Q]
    k, q = (_per_head(v[tok], H, 2).permute(0, 2, 1, 3).contiguous() for v in (s.k, s.q))            # [c, H, Q, K]
    v = s.v.float()[tok].permute(0, 2, 1, 3)
    kt = k.transpose(2, 3).contiguous()
    cum = torch.cumsum(g, 2)
    strict = torch.ones(Q, Q, dtype=torch.bool, device=DEVICE).tril(-1)
    lower = torch.ones(Q, Q, dtype=torch.bool, device=DEVICE).tril()
    L = torch.exp(torch.where(lower, cum[..., :, None] - cum[..., None, :], -math.inf))
    inverse = _unit_lower_inverse(torch.where(strict, beta[..., None] * L * torch.matmul(k, kt), 0.0))
    W = torch.matmul(inverse, (beta * torch.exp(cum))[..., None] * k)
    U = torch.matmul(inverse, beta[..., None] * v)
    last = cum[..., -1:]
    kw = (kt * torch.exp(last - cum)[:, :, None]).contiguous()                                      # [c, H, K, Q]
    M = torch.exp(last)[..., None] * torch.eye(K, device=DEVICE) - torch.matmul(kw, W)
    N = torch.matmul(kw, U)
    enter = s.state[s.slots.long()].unflatten(1, (H, V)).transpose(2, 3).contiguous()               # [S, H, K, V]
    head = (begin == 0)[:, None, None, None]
    N = N + torch.where(head, torch.matmul(M, enter[of]), 0.0)
    M = torch.where(head, 0.0, M)
    d = 1
    while d < s.longest // Q + 2:
        N = torch.cat([N[:d], N[d:] + torch.matmul(M[d:], N[:-d])])
        M = torch.cat([M[:d], torch.matmul(M[d:], M[:-d])])
        d *= 2
    into = torch.where(head, enter[of], torch.cat([N[:1], N[:-1]]))
    U = U - torch.matmul(W, into)
    y = torch.exp(cum)[..., None] * torch.matmul(q, into) + torch.matmul(torch.matmul(q, kt) * L, U)
    y = s.scale * y.permute(0, 2, 1, 3).reshape(chunks * Q, H, V)
    t = torch.arange(T, device=DEVICE) - first[seq]
    end = N[at + (lens - 1).clamp(min=0) // Q].transpose(2, 3).reshape(S, H * V, K)
    out = torch.empty_like(s.state)
    out[s.slots.long()] = torch.where((lens > 0)[:, None, None], end, s.state[s.slots.long()])
    return {"y": y[at[seq] * Q + t].to(s.v.dtype), "state": out}


_PLAIN = {"delta": _plain_delta, "delta_step": _plain_delta_step, "norm": _plain_norm, "linear": _plain_linear}


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------

def work(case):
    """Every input read once, every output written once.  Of the delta rule a state entry and token: the decay, its
    parts of the two products with key and query, and the update (7 operations)."""
    kind, es = case["kind"], 2 if case["dtype"] == "bf16" else 4
    if kind == "norm":
        n = case["tokens"] * (case["heads"] + case["key_heads"]) * case["head_dim"]
        return {"bytes": float(2 * n * es + 4 * case["tokens"] + 8 * case["head_dim"] + 2 * case["rotary"]), "flops": float(8 * n)}
    if kind == "linear":
        T, K, N = case["tokens"], case["inputs"], case["outputs"]
        return {"bytes": float(T * K * es + N * K + T * N * es + 4 * N * (2 if case["bias"] else 1)), "flops": float(2 * T * K * N)}
    S, H, Hk, K, V = case["seqs"], case["heads"], case["key_heads"], case["key_dim"], case["value_dim"]
    T = case.get("tokens", S)
    rows = T * es * (2 * Hk * K + 2 * H * V + 2 * H)
    return {"bytes": float(rows + 8 * S * H * K * V + 8 * H + 8 * S), "flops": float(7 * T * H * K * V)}


# ---------------------------------------------------------------------------
# the definition in 64 bits
# ---------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    if s.kind == "norm":
        return {"q": _exact_norm(s, s.q, s.q_weight), "k": _exact_norm(s, s.k, s.k_weight)}
    if s.kind == "linear":
        q, scale = _exact_rows(s.x)
        y = (q @ s.w.double().t()) * scale[:, None] * s.w_scale.double()
        return {"y": y if s.bias is None else y + s.bias.double()}
    return _exact_delta(s)


def _exact_rows(x):
    """The 8-bit values are defined by float32 roundings: of the scale, and of the quotient before it is rounded to a
    whole number (a quotient next to a half may go either way in 64 bits)."""
    top = x.abs().amax(1).float()
    scale = top / 127.0
    safe = torch.where(scale > 0, scale, 1.0)
    return torch.round(x.float() / safe[:, None]).double(), scale.double()


def _exact_norm(s, x, weight):
    """Pairs as complex numbers times exp(i angle)."""
    v = x.double()
    size = v.square().sum(-1, keepdim=True) / (v.shape[-1] if s.norm == "rms" else 1) + s.eps
    v = v / size.sqrt() * weight.double()
    R = 2 * s.freqs.numel()
    if R == 0:
        return v
    turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEVICE), s.positions.double()[:, None, None] * s.freqs.double())
    pairs = v[..., :R].unflatten(-1, (R // 2, 2)) if s.interleaved else v[..., :R].unflatten(-1, (2, R // 2)).transpose(-1, -2)
    pairs = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
    return torch.cat([(pairs if s.interleaved else pairs.transpose(-1, -2)).flatten(-2), v[..., R:]], -1)


def _exact_delta(s):
    """Token by token, all sequences abreast."""
    T, H, V = s.v.shape
    K, each = s.k.shape[2], H // s.k.shape[1]
    off = s.offsets.long()
    lens, slots = off[1:] - off[:-1], s.slots.long()
    zero = torch.zeros((), dtype=torch.float64, device=DEVICE)
    decay = torch.exp(torch.logaddexp(s.dt.double() + s.dt_bias.double(), zero) * s.A.double())
    beta = torch.sigmoid(s.b.double())
    k, q, v = s.k.double(), s.q.double() * s.scale, s.v.double()
    order = torch.argsort(lens, descending=True, stable=True)        # the sequences still running come first
    left = sorted(lens.tolist(), reverse=True)
    h = s.state[slots[order]].double().reshape(len(left), H // each, each, V, K)
    y = torch.empty(T, H // each, each, V, dtype=torch.float64, device=DEVICE)
    firsts, n = off[:-1][order], len(left)
    for j in range(left[0] if left else 0):
        while left[n - 1] <= j:
            n -= 1
        t = firsts[:n] + j
        kt = k[t][:, :, None, :, None]
        live = h[:n]
        live.mul_(decay[t].reshape(n, H // each, each, 1, 1))
        u = (v[t].reshape(n, H // each, each, V, 1) - torch.matmul(live, kt)) * beta[t].reshape(n, H // each, each, 1, 1)
        live.add_(u * kt.transpose(-1, -2))
        y[t] = torch.matmul(live, q[t][:, :, None, :, None])[..., 0]
    out = torch.empty(s.state.shape, dtype=torch.float64, device=DEVICE)
    out[slots[order]] = h.reshape(len(left), H * V, K)
    return {"y": y.reshape(T, H, V), "state": out}
