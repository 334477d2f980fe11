"""Cases by which the sequence operators are measured: the causal convolution, the selective
state space scan and the processing of logits.

``kind`` of a case and what it stands for in a program that serves a recurrent language model:

* ``conv``        the short convolution over a batch of prompts of different lengths
* ``conv_step``   the same for one new token of every running sequence
* ``channel``     the scan with a decay per channel and state entry, over prompts
* ``head``        the scan with one decay per head of channels, over prompts
* ``channel_step``, ``head_step``  one new token of every running sequence, the states in a pool
* ``logits``      penalties for repeated tokens, biases and the grammar's mask on the last layer's
                  output, with the greedy token and the normaliser

Inputs are what such a program has in hand: activations, step sizes and B / C rows as the columns of
packed projections, offsets of the sequences on the GPU, states in a pool addressed by slot.
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
        # a batch of prompts: 24 of 1 to 700 tokens
        {"name": "conv-prompts", "kind": "conv", "dtype": "bf16", "tokens": 8192, "seqs": 24, "channels": 2304, "width": 4},
        # an interactive call: a few running sequences, latency counts
        {"name": "conv-few-tokens", "kind": "conv_step", "dtype": "bf16", "seqs": 7, "channels": 2304, "width": 4},
        # one short prompt of a small 32-bit model (the tree cells' hidden size 256, twice expanded): the smallest scan
        {"name": "channel-short-f32", "kind": "channel", "dtype": "f32", "tokens": 257, "seqs": 1, "channels": 512, "state": 16, "groups": 1},
        # an ordinary batch of prompts
        {"name": "channel-prompts", "kind": "channel", "dtype": "bf16", "tokens": 8192, "seqs": 16, "channels": 2048, "state": 16, "groups": 1},
        # one long document: the work is split over its length
        {"name": "channel-long", "kind": "channel", "dtype": "bf16", "tokens": 32768, "seqs": 1, "channels": 2048, "state": 16, "groups": 1},
        # a full batch generating: the state's bytes
        {"name": "channel-tokens", "kind": "channel_step", "dtype": "bf16", "seqs": 256, "channels": 2048, "state": 16, "groups": 1},
        # heads of 64 channels with a large state: an ordinary batch of prompts
        {"name": "head-prompts", "kind": "head", "dtype": "bf16", "tokens": 8192, "seqs": 16, "channels": 2048, "state": 128, "head": 64, "groups": 1},
        # the 32-bit model's prompts, two groups of heads
        {"name": "head-prompts-f32", "kind": "head", "dtype": "f32", "tokens": 4099, "seqs": 5, "channels": 1024, "state": 64, "head": 64, "groups": 2},
        # the largest: one long document through a wide layer
        {"name": "head-long", "kind": "head", "dtype": "bf16", "tokens": 32768, "seqs": 1, "channels": 4096, "state": 128, "head": 64, "groups": 1},
        # a batch generating
        {"name": "head-tokens", "kind": "head_step", "dtype": "bf16", "seqs": 64, "channels": 4096, "state": 128, "head": 64, "groups": 1},
        # one interactive row
        {"name": "logits-one", "kind": "logits", "dtype": "f32", "seqs": 1, "vocab": 32000, "history": 300},
        # a full batch with a large vocabulary
        {"name": "logits-batch", "kind": "logits", "dtype": "bf16", "seqs": 256, "vocab": 131072, "history": 2048},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the ranges above, odd sizes among them."""
    kind = rng.choice(["conv", "conv_step", "channel", "channel", "channel_step", "head", "head", "head_step", "logits", "logits"])
    case = {"kind": kind, "dtype": rng.choice(["bf16", "bf16", "f32"])}
    if kind == "logits":
        case["vocab"] = _log_int(rng, 1000, 160000)
        case["seqs"] = _log_int(rng, 1, min(256, 32_000_000 // case["vocab"]))
        case["history"] = _log_int(rng, 1, 8192)
        return case
    case["seqs"] = _log_int(rng, 1, 64)
    if kind in ("conv", "conv_step"):
        case["channels"] = _log_int(rng, 64, 6000)
        case["width"] = rng.choice([2, 3, 4, 4])
        if kind == "conv":
            case["tokens"] = _log_int(rng, 1, 16384)
        else:
            case["seqs"] = _log_int(rng, 1, 512)
        return case
    case["groups"] = rng.choice([1, 1, 2, 4])
    if kind in ("channel", "channel_step"):
        case["channels"] = case["groups"] * _log_int(rng, 64, 2048 // case["groups"])
        case["state"] = rng.choice([8, 16, 16, 32, 64])
    else:
        case["head"] = rng.choice([32, 64, 64, 128])
        case["channels"] = case["groups"] * case["head"] * _log_int(rng, 1, 4096 // (case["groups"] * case["head"]))
        case["state"] = rng.choice([16, 32, 64, 128, 128])
    if kind in ("channel", "head"):
        most = 400_000_000 if kind == "channel" else 2_000_000_000
        case["tokens"] = _log_int(rng, 1, max(64, min(24576, most // (case["channels"] * case["state"]))))
    else:
        case["seqs"] = _log_int(rng, 1, min(256, max(1, 60_000_000 // (case["channels"] * case["state"]))))
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


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def prepare(case, seed):
    from types import SimpleNamespace
    kind, S = case["kind"], case["seqs"]
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    typ = _dtype(case)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=DEVICE, dtype=torch.float32)

    def unit(*shape):
        return torch.rand(*shape, generator=g, device=DEVICE, dtype=torch.float32)

    def ints(v):
        return torch.tensor(v, dtype=torch.int32, device=DEVICE)

    s = SimpleNamespace(case=case, kind=kind, status=ints([0]))
    if kind == "logits":
        V, cap = case["vocab"], case["history"]
        r = np.random.default_rng(seed)
        s.logits = (normal(S, V) * 2.5).to(typ)
        s.out, s.token, s.lse = torch.empty_like(s.logits), ints([0] * S), torch.empty(S, device=DEVICE)
        # the text so far: frequent tokens have low ids, as in a sorted vocabulary
        s.history = torch.clamp((V ** unit(S, cap)).to(torch.int32) - 1, 0, V - 1)
        lens = r.integers(cap // 2, cap + 1, S)
        s.history_len, s.prompt_len = ints(lens.tolist()), ints((lens * r.random(S)).astype(int).tolist())
        s.repetition, s.frequency, s.presence = 1.0 + 0.3 * unit(S), 0.5 * unit(S), 0.5 * unit(S)
        # a few biases for some rows, no token twice in one
        count = np.where(r.random(S) < 0.5, r.integers(1, 65, S), 0)
        s.bias_offsets = ints([0] + np.cumsum(count).tolist())
        pick = random.Random(seed)
        s.bias_tokens = ints([t for n in count.tolist() for t in pick.sample(range(V), n)])
        s.bias_values = 2.0 * normal(int(count.sum()))
        # states of a grammar: few tokens, half of them, none; -1 is a row without a grammar
        words = (V + 31) // 32
        m = torch.randint(-2 ** 31, 2 ** 31, (8, words), generator=g, device=DEVICE, dtype=torch.int64)
        m[1] &= m[2] & m[3] & m[4] & m[5]
        m[7] = 0
        s.mask = m.to(torch.int32)
        s.mask_index = ints([int(i) for i in np.where(np.arange(S) % 64 == 63, 7, r.integers(-1, 7, S))])
        s.workspace = None
        if own:                                  # the plain form needs none
            from paper_2011_01383_amd import cortex
            s.workspace = cortex.workspace(cortex.cortex_logits_workspace_bytes(S, V), DEVICE)
        return s
    D, step = case["channels"], kind.endswith("_step")
    T = S if step else case["tokens"]
    lens = [1] * S if step else _lengths(case, seed)
    s.T, s.longest = T, max(lens)
    s.offsets = ints([0] + np.cumsum(lens).tolist())
    s.slots = torch.randperm(S, generator=g, device=DEVICE).to(torch.int32)
    if kind.startswith("conv"):
        W = case["width"]
        wide = normal(T, 2 * D).to(typ)        # the projection's output: gate and input side by side
        s.x = wide[:, D:]
        s.weight, s.bias = normal(D, W) / math.sqrt(W), 0.1 * normal(D)
        s.state = normal(S, W - 1, D).to(typ)
        s.y, s.state_out = torch.empty(T, D, dtype=typ, device=DEVICE), torch.empty_like(s.state)
        return s
    N, G = case["state"], case["groups"]
    H = D if "head" not in case else D // case["head"]
    xbc = normal(T, D + 2 * G * N).to(typ)      # the convolution's output: x, B and C side by side
    s.x = xbc[:, :D]
    s.B, s.C = xbc[:, D:D + G * N].unflatten(1, (G, N)), xbc[:, D + G * N:].unflatten(1, (G, N))
    s.z = normal(T, D).to(typ)
    s.dt = (0.5 * normal(T, H)).to(typ)
    # step sizes around 0.001 to 0.1 after the softplus, decays as such layers are initialised
    size = torch.exp(unit(H) * math.log(100.0)) * 0.001
    s.dt_bias = torch.log(torch.expm1(size))
    if "head" in case:
        s.A = -(1.0 + 15.0 * unit(H))
    else:
        s.A = -torch.arange(1, N + 1, device=DEVICE, dtype=torch.float32) * (0.9 + 0.2 * unit(D, N))
    s.skip = 1.0 + 0.1 * normal(H)
    s.state = 0.3 * normal(S, D, N)
    s.y, s.state_out = torch.empty(T, D, dtype=typ, device=DEVICE), torch.empty_like(s.state)
    s.workspace = None
    if own and not step:
        from paper_2011_01383_amd import cortex
        s.workspace = cortex.workspace(cortex.cortex_scan_workspace_bytes(T, S, D, N, case.get("head", 0)), DEVICE)
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(state):
    return _own(state) if own else _plain(state)


def _own(s):
    from paper_2011_01383_amd import cortex
    if s.kind == "logits":
        rc = cortex.cortex_logits_process(
            s.logits, out=s.out, token=s.token, lse=s.lse, history=s.history, history_len=s.history_len,
            prompt_len=s.prompt_len, repetition=s.repetition, frequency=s.frequency, presence=s.presence,
            bias_offsets=s.bias_offsets, bias_tokens=s.bias_tokens, bias_values=s.bias_values, mask=s.mask,
            mask_index=s.mask_index, status=s.status, ws=s.workspace)
        cortex.check(rc, "logits")
        return {"out": s.out, "token": s.token, "lse": s.lse}
    if s.kind == "conv":
        rc = cortex.cortex_conv_forward(s.x, s.weight, s.offsets, s.y, bias=s.bias, silu=True, state_in=s.state,
                                        state_out=s.state_out, state_index=s.slots, status=s.status)
    elif s.kind == "conv_step":
        rc = cortex.cortex_conv_step(s.x, s.weight, s.y, bias=s.bias, silu=True, state_in=s.state,
                                     state_out=s.state_out, state_index=s.slots, status=s.status)
    elif s.kind in ("channel", "head"):
        rc = cortex.cortex_scan_forward(s.x, s.dt, s.A, s.B, s.C, s.offsets, s.y, D=s.skip, z=s.z, dt_bias=s.dt_bias,
                                        softplus=True, state_in=s.state, state_out=s.state_out, state_index=s.slots,
                                        status=s.status, ws=s.workspace)
    else:
        rc = cortex.cortex_scan_step(s.x, s.dt, s.A, s.B, s.C, s.y, D=s.skip, z=s.z, dt_bias=s.dt_bias, softplus=True,
                                     state_in=s.state, state_out=s.state_out, state_index=s.slots, status=s.status)
    cortex.check(rc, s.kind)
    return {"y": s.y, "state": s.state_out}


def _plain(s):
    return _PLAIN[s.kind](s)


def _silu(v):
    return v / (1.0 + torch.exp(-v))


def _softplus(v):
    return torch.clamp(v, min=0) + torch.log1p(torch.exp(-torch.abs(v)))


def _ragged(s):
    """Sequence of every token, and the sequences' first tokens and lengths."""
    off = s.offsets.long()
    lens = off[1:] - off[:-1]
    return torch.repeat_interleave(torch.arange(len(lens), device=DEVICE), lens, output_size=s.T), off[:-1], lens


def _conv_act(s, taps):
    """taps [T, W, D]: the inputs under the window of each token."""
    return _silu((taps * s.weight.t()).sum(1) + s.bias).to(s.x.dtype)


def _plain_conv(s):
    W, S = s.weight.shape[1], s.slots.numel()
    seq, first, lens = _ragged(s)
    k = torch.arange(W, device=DEVICE)
    old = s.state[s.slots.long()].reshape(S * (W - 1), -1)
    rows = torch.cat([old, s.x])                 # row of sequence i's token j: S (W - 1) + first[i] + j; j < 0: its state

    def at(i, j):
        return torch.where(j < 0, i * (W - 1) + (W - 1) + j, S * (W - 1) + first[i] + j)

    t = torch.arange(s.T, device=DEVICE)
    y = _conv_act(s, rows[at(seq[:, None], (t - first[seq])[:, None] + k - (W - 1))].float())
    last = rows[at(torch.arange(S, device=DEVICE)[:, None], lens[:, None] + k[:W - 1] - (W - 1))]
    out = torch.empty_like(s.state)
    out[s.slots.long()] = last
    return {"y": y, "state": out}


def _plain_conv_step(s):
    taps = torch.cat([s.state[s.slots.long()], s.x[:, None]], 1)
    out = torch.empty_like(s.state)
    out[s.slots.long()] = taps[:, 1:]
    return {"y": _conv_act(s, taps.float()), "state": out}


def _per_channel(s, v):
    """A row of groups [.., G, N] as [.., D, N]: every channel its group's."""
    return v.float().repeat_interleave(s.x.shape[1] // v.shape[1], 1)


def _finish(s, y):
    """Skip connection and gate."""
    skip = s.skip.repeat_interleave(s.x.shape[1] // s.skip.numel())
    return ((y + skip * s.x.float()) * _silu(s.z.float())).to(s.x.dtype)


def _prefix(a, b, longest):
    """h[t] = a[t] h[t-1] + b[t] along the first axis, by doubling; a is 0 where a sequence begins."""
    d = 1
    while d < longest:
        b = torch.cat([b[:d], torch.addcmul(b[d:], a[d:], b[:-d])])
        a = torch.cat([a[:d], a[d:] * a[:-d]])
        d *= 2
    return b


def _store(s, last, lens):
    """The pool with the sequences' last states; one without tokens keeps its own."""
    out = torch.empty_like(s.state)
    out[s.slots.long()] = torch.where((lens > 0)[:, None, None], last, s.state[s.slots.long()])
    return out


def _plain_channel(s):
    seq, first, lens = _ragged(s)
    dt = _softplus(s.dt.float() + s.dt_bias)
    a = torch.exp(dt[:, :, None] * s.A)
    b = (dt * s.x.float())[:, :, None] * _per_channel(s, s.B)
    begins = first.clamp(max=s.T - 1)
    some = lens > 0
    # the entering state joins the first token's input; an empty sequence shares its place with a later one's
    # first token, or the last token, and adds nothing there
    b.index_put_((begins,), torch.where(some[:, None, None], a[begins] * s.state[s.slots.long()], 0.0), accumulate=True)
    keep = torch.ones(s.T, device=DEVICE)
    keep.index_put_((begins,), torch.where(some, -1.0, 0.0), accumulate=True)
    h = _prefix(a * keep[:, None, None], b, s.longest)
    y = (h * _per_channel(s, s.C)).sum(2)
    return {"y": _finish(s, y), "state": _store(s, h[(first + lens - 1).clamp(min=0)], lens)}


def _plain_channel_step(s):
    dt = _softplus(s.dt.float() + s.dt_bias)
    h = torch.exp(dt[:, :, None] * s.A) * s.state[s.slots.long()] + (dt * s.x.float())[:, :, None] * _per_channel(s, s.B)
    out = torch.empty_like(s.state)
    out[s.slots.long()] = h
    return {"y": _finish(s, (h * _per_channel(s, s.C)).sum(2)), "state": out}


def _plain_head(s):
    """By chunks of CHUNK tokens of one sequence, as matrix products."""
    T, D = s.x.shape
    S, G, N, H, Q = s.slots.numel(), s.B.shape[1], s.B.shape[2], s.A.numel(), CHUNK
    P = D // H
    seq, first, lens = _ragged(s)
    chunks = T // Q + S                          # at least as many as there are
    at = first // Q + torch.arange(S, device=DEVICE)   # first chunk of each sequence
    of = torch.searchsorted(at, torch.arange(chunks, device=DEVICE), right=True) - 1
    begin = (torch.arange(chunks, device=DEVICE) - at[of]) * Q
    tok = begin[:, None] + torch.arange(Q, device=DEVICE)
    live = tok < lens[of][:, None]
    tok = (first[of][:, None] + tok).clamp(max=T - 1)
    dt = torch.where(live[:, :, None], _softplus(s.dt.float() + s.dt_bias)[tok], 0.0)      # [c, Q, H]
    x = (s.x.float()[tok].unflatten(2, (H, P)) * dt[..., None]).permute(0, 2, 1, 3)         # [c, H, Q, P]
    B = s.B.float()[tok].permute(0, 2, 1, 3)                                                # [c, G, Q, N]
    C = s.C.float()[tok].permute(0, 2, 1, 3)
    cum = torch.cumsum(dt * s.A, 1).permute(0, 2, 1)                                        # [c, H, Q]
    lower = torch.ones(Q, Q, dtype=torch.bool, device=DEVICE).tril()
    L = torch.exp(torch.where(lower, cum[..., :, None] - cum[..., None, :], -math.inf))     # [c, H, Q, Q]
    each = H // G
    CB = torch.matmul(C, B.transpose(2, 3).contiguous()).repeat_interleave(each, 1)
    y = torch.matmul(CB * L, x)
    # the state that each chunk adds, then the one that enters it
    tail = torch.exp(cum[..., -1:] - cum)
    xw = (x * tail[..., None]).transpose(2, 3).contiguous()
    add = torch.matmul(xw, B.repeat_interleave(each, 1))                                    # [c, H, P, N]
    a = torch.exp(cum[..., -1])[..., None, None]
    enter = s.state[s.slots.long()].unflatten(1, (H, P))
    head = (begin == 0)[:, None, None, None]
    h = _prefix(torch.where(head, 0.0, a), add + torch.where(head, a * enter[of], 0.0), s.longest // Q + 2)
    into = torch.where(head, enter[of], torch.cat([h[:1], h[:-1]]))
    into = into.transpose(2, 3).contiguous()
    y = y + torch.exp(cum)[..., None] * torch.matmul(C.repeat_interleave(each, 1), into)
    y = y.permute(0, 2, 1, 3).reshape(chunks * Q, D)
    t = torch.arange(T, device=DEVICE) - first[seq]
    y = y[at[seq] * Q + t]
    last = h[(at + (lens - 1).clamp(min=0) // Q)].reshape(S, D, N)
    return {"y": _finish(s, y), "state": _store(s, last, lens)}


def _plain_head_step(s):
    T, D = s.x.shape
    P = D // s.A.numel()
    dt = _softplus(s.dt.float() + s.dt_bias)
    a = torch.exp(dt * s.A).repeat_interleave(P, 1)[:, :, None]
    u = (dt.repeat_interleave(P, 1) * s.x.float())[:, :, None]
    h = a * s.state[s.slots.long()] + u * _per_channel(s, s.B)
    out = torch.empty_like(s.state)
    out[s.slots.long()] = h
    return {"y": _finish(s, (h * _per_channel(s, s.C)).sum(2)), "state": out}


def _plain_logits(s):
    rows, V = s.logits.shape
    cap = s.history.shape[1]
    j = torch.arange(cap, device=DEVICE)
    live = j < s.history_len[:, None]
    said = live & (j >= s.prompt_len[:, None])
    tok = s.history.long()
    seen = torch.zeros(rows, V, device=DEVICE).scatter_add_(1, tok, live.float()) > 0
    n = torch.zeros(rows, V, device=DEVICE).scatter_add_(1, tok, said.float())
    v = s.logits.float()
    r = s.repetition[:, None]
    v = torch.where(seen, torch.where(v > 0, v / r, v * r), v)
    v = v - s.frequency[:, None] * n
    v = v - s.presence[:, None] * (n > 0)
    count = (s.bias_offsets[1:] - s.bias_offsets[:-1]).long()
    row = torch.repeat_interleave(torch.arange(rows, device=DEVICE), count, output_size=s.bias_tokens.numel())
    v.index_put_((row, s.bias_tokens.long()), s.bias_values, accumulate=True)
    words = s.mask[s.mask_index.clamp(min=0).long()]
    bit = torch.arange(32, device=DEVICE, dtype=torch.int32)
    allowed = ((words[:, :, None] >> bit) & 1).reshape(rows, -1)[:, :V] != 0
    v = torch.where(allowed | (s.mask_index < 0)[:, None], v, -math.inf)
    top = v.amax(1)
    # the first of the largest; -1 where the mask leaves nothing
    first = torch.where(v == top[:, None], torch.arange(V, device=DEVICE), V).amin(1)
    token = torch.where(top > -math.inf, first, -1).to(torch.int32)
    base = torch.where(top > -math.inf, top, 0.0)
    lse = base + torch.log(torch.exp(v - base[:, None]).sum(1))
    return {"out": v.to(s.logits.dtype), "token": token, "lse": lse}


_PLAIN = {"conv": _plain_conv, "conv_step": _plain_conv_step, "channel": _plain_channel, "channel_step": _plain_channel_step,
          "head": _plain_head, "head_step": _plain_head_step, "logits": _plain_logits}


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------

def work(case):
    """Every input read once, every output written once; a state entry's update and its part of the output
    are five operations, with a decay of its own an exponential more."""
    kind, S = case["kind"], case["seqs"]
    es = 2 if case["dtype"] == "bf16" else 4
    if kind == "logits":
        V = case["vocab"]
        return {"bytes": float(S * (2 * V * es + (V + 31) // 32 * 4 + 3 * case["history"] + 40)), "flops": float(S * V * 6)}
    D, T = case["channels"], case.get("tokens", S)
    if kind.startswith("conv"):
        W = case["width"]
        return {"bytes": float(es * (2 * T * D + 2 * S * (W - 1) * D) + 4 * D * (W + 1) + 8 * S), "flops": float(T * D * (2 * W + 4))}
    N, G = case["state"], case["groups"]
    H = D // case["head"] if "head" in case else D
    rows = T * es * (3 * D + H + 2 * G * N)
    fixed = 4 * (2 * H + (H if "head" in case else D * N)) + 8 * S
    return {"bytes": float(rows + 8 * S * D * N + fixed), "flops": float(T * D * (N * (5 if "head" in case else 6) + 10))}


# ---------------------------------------------------------------------------
# the definition in 64 bits
# ---------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return _exact_logits(s) if s.kind == "logits" else _exact_conv(s) if s.kind.startswith("conv") else _exact_scan(s)


def _exact_conv(s):
    """Sequence by sequence: the state's inputs, then its own, under a sliding window."""
    x, w, W = s.x.double(), s.weight.double(), s.weight.shape[1]
    off, slots = s.offsets.tolist(), s.slots.tolist()
    y, out = torch.empty_like(x), torch.empty(s.state.shape, dtype=torch.float64, device=DEVICE)
    for i, slot in enumerate(slots):
        text = torch.cat([s.state[slot].double(), x[off[i]:off[i + 1]]])
        v = (text.unfold(0, W, 1) * w).sum(-1) + s.bias.double() if off[i + 1] > off[i] else text[:0]
        y[off[i]:off[i + 1]] = v * torch.sigmoid(v)
        out[slot] = text[text.shape[0] - (W - 1):]
    return {"y": y, "state": out}


def _exact_scan(s):
    """Token by token, all sequences abreast."""
    x, z, B, C = s.x.double(), s.z.double(), s.B.double(), s.C.double()
    T, D = x.shape
    H, N, G = s.dt.shape[1], B.shape[2], B.shape[1]
    off = s.offsets.long()
    lens, slots = off[1:] - off[:-1], s.slots.long()
    dt = torch.logaddexp(s.dt.double() + s.dt_bias.double(), torch.zeros((), dtype=torch.float64, device=DEVICE))
    A = s.A.double().reshape(G, H // G, 1, -1)                       # [G, heads, channels of one, N or 1]
    order = torch.argsort(lens, descending=True, stable=True)        # the sequences still running come first
    left = sorted(lens.tolist(), reverse=True)
    h = s.state[slots[order]].double().reshape(len(left), G, H // G, D // H, N)
    y = torch.empty(T, D, dtype=torch.float64, device=DEVICE)
    firsts, n = off[:-1][order], len(left)
    for j in range(left[0] if left else 0):
        while left[n - 1] <= j:
            n -= 1
        t = firsts[:n] + j
        d = dt[t].reshape(n, G, H // G, 1, 1)
        u = x[t].reshape(n, G, H // G, D // H, 1)
        live = h[:n]
        live.mul_(torch.exp(d * A)).add_(d * u * B[t][:, :, None, None, :])
        y[t] = (live * C[t][:, :, None, None, :]).sum(-1).reshape(n, D)
    skip = s.skip.double()[:, None].expand(H, D // H).reshape(D)
    y = (y + skip * x) * z * torch.sigmoid(z)
    out = torch.empty(s.state.shape, dtype=torch.float64, device=DEVICE)
    out[slots[order]] = h.reshape(len(left), D, N)
    return {"y": y, "state": out}


def _exact_logits(s):
    out, lse = [], []
    bits = np.unpackbits(s.mask.cpu().numpy().view(np.uint8), axis=1, bitorder="little")
    off = s.bias_offsets.tolist()
    for i in range(s.logits.shape[0]):
        v = s.logits[i].double()
        text = s.history[i, :int(s.history_len[i])].long()
        seen = torch.unique(text)
        r = s.repetition[i].double()
        v[seen] = torch.where(v[seen] > 0, v[seen] / r, v[seen] * r)
        said, n = torch.unique(text[int(s.prompt_len[i]):], return_counts=True)
        v[said] -= s.frequency[i].double() * n + s.presence[i].double()
        v[s.bias_tokens[off[i]:off[i + 1]].long()] += s.bias_values[off[i]:off[i + 1]].double()
        m = int(s.mask_index[i])
        if m >= 0:
            v[torch.from_numpy(bits[m, :v.numel()] == 0).to(DEVICE)] = -math.inf
        out.append(v)
        lse.append(torch.logsumexp(v, 0))
    return {"out": torch.stack(out), "token": None, "lse": torch.stack(lse)}
