"""A recurrent sequence model that writes trees, and the tree cell that reads them.

The third structure kind beside trees and DAGs (Sec. 3 of the paper) as a program
uses it: ``SequenceModel`` reads a batch of prompts of different lengths, then
writes one token a step for every sequence.  Its tokens are words and one mark
that opens an inner node, so a text in prefix order is a binary tree; a grammar
mask keeps every text one.  The finished trees go to a tree cell in one call.

    python -m paper_2011_01383_amd.sequence

runs it with random weights.  The recurrences, convolutions and the choice of the
next token are the library's kernels (``cortex_conv_*``, ``cortex_scan_*``,
``cortex_logits_process``, ``cortex_tree_infer``); the projections between them are
plain matrix products of the framework that also supplies the memory.
"""
from __future__ import annotations

import numpy as np
import torch

from . import cortex as C


class _Layer:
    """Projection, convolution, scan, gate and projection back.  ``heads`` = 0: a
    decay per channel and state entry, step sizes of low rank; else one decay per
    head, and x, B and C convolved together."""

    def __init__(self, g, width: int, channels: int, N: int, heads: int, rows: int, dtype, device, W: int = 4):
        def normal(a, b):
            return (torch.randn(a, b, generator=g) / a ** 0.5).to(device, dtype)

        self.D, self.N, self.heads, self.rank = channels, N, heads, max(1, width // 16)
        D = channels
        rates = heads or D
        self.conv_channels = D + 2 * N if heads else D
        self.w_in = normal(width, D + self.conv_channels + heads)
        if not heads:
            self.w_x, self.w_dt = normal(D, self.rank + 2 * N), normal(self.rank, D)
        self.w_out = normal(D, width)
        self.conv_w = (torch.randn(self.conv_channels, W, generator=g) / W ** 0.5).to(device)
        self.conv_b = torch.zeros(self.conv_channels, device=device)
        size = 0.001 * 100.0 ** torch.rand(rates, generator=g)
        self.dt_bias = torch.log(torch.expm1(size)).to(device)
        self.A = (-(1 + 15 * torch.rand(heads, generator=g)) if heads else -torch.arange(1.0, N + 1).repeat(D, 1)).to(device)
        self.skip = torch.ones(rates, device=device)
        self.conv_state = torch.zeros(rows, W - 1, self.conv_channels, dtype=dtype, device=device)
        self.state = torch.zeros(rows, D, N, device=device)

    def __call__(self, x, slots, status, offsets=None):
        """x [T, width]: prompts with their offsets, or one token of every sequence."""
        D, N, T = self.D, self.N, x.shape[0]
        u = x @ self.w_in
        z, v = u[:, :D], u[:, D:D + self.conv_channels]
        c = torch.empty_like(v, memory_format=torch.contiguous_format)
        states = dict(state_in=self.conv_state, state_out=self.conv_state, state_index=slots, status=status)
        if offsets is None:
            C.check(C.cortex_conv_step(v, self.conv_w, c, bias=self.conv_b, **states), "cortex_conv_step")
        else:
            C.check(C.cortex_conv_forward(v, self.conv_w, offsets, c, bias=self.conv_b, **states), "cortex_conv_forward")
        xs = c[:, :D]
        if self.heads:
            dt, bc = u[:, D + self.conv_channels:], c[:, D:]
        else:
            p = c @ self.w_x
            dt, bc = p[:, :self.rank] @ self.w_dt, p[:, self.rank:]
        B, Cm = bc[:, :N].unflatten(1, (1, N)), bc[:, N:].unflatten(1, (1, N))
        y = torch.empty(T, D, dtype=x.dtype, device=x.device)
        kw = dict(D=self.skip, z=z, dt_bias=self.dt_bias, state_in=self.state, state_out=self.state, state_index=slots,
                  status=status)
        if offsets is None:
            C.check(C.cortex_scan_step(xs, dt, self.A, B, Cm, y, **kw), "cortex_scan_step")
        else:
            head_dim = D // self.heads if self.heads else 0
            ws = C.workspace(C.cortex_scan_workspace_bytes(T, offsets.numel() - 1, D, N, head_dim), x.device)
            C.check(C.cortex_scan_forward(xs, dt, self.A, B, Cm, offsets, y, ws=ws, **kw), "cortex_scan_forward")
        return x + y @ self.w_out


class SequenceModel:
    """Embedding, layers (decays per channel and per head in turn), output weights.

    ``rows`` sequences can run at once; each has a row of every state pool."""

    def __init__(self, vocab: int, width: int = 256, layers: int = 2, rows: int = 64, dtype=torch.float32, device="cuda",
                 seed: int = 0):
        C.load()
        g = torch.Generator().manual_seed(seed)
        self.vocab, self.device, self.rows = vocab, device, rows
        self.embedding = torch.randn(vocab, width, generator=g).to(device, dtype)
        self.layers = [_Layer(g, width, 2 * width, 64 if k % 2 else 16, 2 * width // 64 if k % 2 else 0, rows, dtype, device)
                       for k in range(layers)]
        self.w_out = (torch.randn(width, vocab, generator=g) / width ** 0.5).to(device, dtype)
        self.status = torch.zeros(1, dtype=torch.int32, device=device)

    def _run(self, tokens, slots, offsets=None):
        x = self.embedding[tokens.long()]
        for layer in self.layers:
            x = layer(x, slots, self.status, offsets)
        x = x.float()
        return (x * torch.rsqrt((x * x).mean(1, keepdim=True) + 1e-6)).to(self.w_out.dtype)

    def reset(self, slots) -> None:
        """Rows start from zero."""
        for layer in self.layers:
            layer.conv_state[slots.long()] = 0
            layer.state[slots.long()] = 0

    def check(self) -> None:
        """Raises what the calls since the last check reported, and clears it: a status left in
        place would make every later call a no-op."""
        code = int(self.status.item())
        if code != 0:
            self.status.zero_()
            raise RuntimeError("device status %d" % code)

    def prompt(self, tokens, offsets, slots):
        """Logits after the last token of each prompt (none may be empty)."""
        x = self._run(tokens, slots, offsets)
        return x[offsets[1:].long() - 1] @ self.w_out

    def step(self, tokens, slots):
        """Logits after one more token of each sequence."""
        return self._run(tokens, slots) @ self.w_out


NODE = 0        # opens an inner node: two subtrees follow.  Other tokens are words, the leaves.


def tree_masks(vocab: int, device="cuda") -> torch.Tensor:
    """Rows of allowed tokens: 0 a word or an inner node, 1 words only, 2 nothing."""
    allowed = np.ones((3, (vocab + 31) // 32 * 32), dtype=bool)
    allowed[:, vocab:] = False
    allowed[1, NODE] = False
    allowed[2] = False
    words = np.packbits(allowed, axis=1, bitorder="little").view(np.int32)
    return torch.from_numpy(words.copy()).to(device)


def write_trees(model: SequenceModel, prompts, most: int = 40, repetition: float = 1.0, frequency: float = 0.0,
                presence: float = 0.0, opening: float = 0.0):
    """Continues every prompt (lists of tokens) with one tree in prefix order of at most ``most``
    tokens, greedily under the grammar.  ``opening`` is a bias for another inner node.
    Returns the trees' tokens and their log-probabilities under the masked, penalised logits."""
    # on the device a token or row out of range would end the process, and an empty prompt
    # would continue its neighbour's
    if len(prompts) > model.rows:
        raise ValueError("%d prompts, the model runs %d at once" % (len(prompts), model.rows))
    for i, p in enumerate(prompts):
        if len(p) == 0:
            raise ValueError("prompt %d is empty" % i)
        if min(p) < 0 or max(p) >= model.vocab:
            raise ValueError("prompt %d has a token outside [0, %d)" % (i, model.vocab))
    if not prompts:
        return [], np.zeros(0, dtype=np.float32)
    S, dev = len(prompts), model.device
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=dev)
    full = lambda v: torch.full((S,), float(v), device=dev)
    lens = [len(p) for p in prompts]
    slots = torch.arange(S, dtype=torch.int32, device=dev)
    model.reset(slots)
    # the text so far, filled in place as it grows
    history = torch.zeros(S, max(lens) + most, dtype=torch.int32, device=dev)
    for i, p in enumerate(prompts):
        history[i, :len(p)] = ints(p)
    prompt_len = ints(lens)
    at = prompt_len.clone()
    masks = tree_masks(model.vocab, dev)
    token, lse = ints([0] * S), torch.zeros(S, device=dev)
    ws = C.workspace(C.cortex_logits_workspace_bytes(S, model.vocab), dev)
    penalties = dict(repetition=full(repetition), frequency=full(frequency), presence=full(presence))
    biases = dict(bias_offsets=ints(list(range(S + 1))), bias_tokens=ints([NODE] * S), bias_values=full(opening))
    missing = torch.ones(S, dtype=torch.int32, device=dev)       # subtrees still to be written
    logprob = torch.zeros(S, device=dev)
    rows = torch.arange(S, device=dev)
    logits = model.prompt(ints([t for p in prompts for t in p]), ints([0] + np.cumsum(lens).tolist()), slots).contiguous()
    for left in range(most, 0, -1):
        # another node needs room for two more subtrees; a finished tree is left alone
        done = missing == 0
        index = torch.where(done, 2, torch.where(missing + 2 <= left, 0, 1)).to(torch.int32)
        C.check(C.cortex_logits_process(logits, out=logits, token=token, lse=lse, history=history, history_len=at,
                                        prompt_len=prompt_len, mask=masks, mask_index=index, status=model.status, ws=ws,
                                        **penalties, **biases), "cortex_logits_process")
        chosen = torch.where(done, 1, token)
        logprob += torch.where(done, torch.zeros_like(lse), logits[rows, chosen.long()].float() - lse)
        history[rows, torch.where(done, at - 1, at).long()] = torch.where(done, history[rows, (at - 1).long()], chosen)
        at += (~done).to(torch.int32)
        missing += torch.where(done, 0, torch.where(chosen == NODE, 1, -1)).to(torch.int32)
        if left > 1:
            # a finished sequence keeps its states: its row of the pools is not named
            logits = model.step(chosen, torch.where(done, -1, slots).to(torch.int32)).contiguous()
    text, ends = history.cpu().numpy(), at.cpu().numpy()
    model.check()
    return [text[i, lens[i]:ends[i]].tolist() for i in range(S)], logprob.cpu().numpy()


def tree_arrays(trees):
    """Prefix texts as the arrays of a batch: children [N * 2] and the word of every node, -1 inside."""
    children, words = [], []
    for text in trees:
        open_slots = [None]                     # (node, slot) that the coming subtrees fill, the next one last
        for pos, t in enumerate(text):
            if not open_slots:
                raise ValueError("%d tokens after the tree" % (len(text) - pos))
            v, slot = len(words), open_slots.pop()
            if slot is not None:
                children[slot[0]][slot[1]] = v
            words.append(-1 if t == NODE else t)
            children.append([-1, -1])
            if t == NODE:
                open_slots += [(v, 1), (v, 0)]
        if open_slots:
            raise ValueError("a tree of %d tokens lacks %d subtrees" % (len(text), len(open_slots)))
    return np.array(children, dtype=np.int32).reshape(-1), np.array(words, dtype=np.int32)


def read_trees(trees, vectors: torch.Tensor, U: torch.Tensor, b: torch.Tensor):
    """The binary N-ary TreeLSTM's states of every node of the texts, in row order, and the linearization."""
    children, words = tree_arrays(trees)
    N, H, dev = len(words), vectors.shape[1], vectors.device
    lin = C.Linearization.alloc(N, 2, dev)
    h, c = torch.empty(N, H, device=dev), torch.empty(N, H, device=dev)
    status = torch.zeros(1, dtype=torch.int32, device=dev)
    ws = C.workspace(C.cortex_tree_infer_workspace_bytes(C.CORTEX_NARY_TREELSTM, N, 2, H), dev)
    up = lambda a: torch.from_numpy(a).to(dev)
    C.check(C.cortex_tree_infer(C.CORTEX_NARY_TREELSTM, H, up(children), lin, vectors, vectors.shape[0], up(words), None,
                                W=None, U=U, b=b, W_M=None, h=h, c_or_P=c, status=status, ws=ws), "cortex_tree_infer")
    if int(status.item()) != 0:
        raise RuntimeError("device status %d" % int(status.item()))
    return h, c, lin


def main() -> None:
    vocab, H = 1000, 64
    model = SequenceModel(vocab, dtype=torch.bfloat16)
    rng = np.random.default_rng(0)
    prompts = [rng.integers(1, vocab, n).tolist() for n in (3, 17, 1, 64, 130, 9, 33, 5)]
    trees, logprob = write_trees(model, prompts, most=31, repetition=1.1, frequency=0.5, opening=6.0)
    for i, (t, p) in enumerate(zip(trees, logprob)):
        print("prompt of %3d tokens: %2d tokens, log-probability %8.3f: %s" % (len(prompts[i]), len(t), p, t))
    g = torch.Generator().manual_seed(1)
    vectors = torch.randn(vocab, H, generator=g).cuda()
    U, b = 0.05 * (2 * torch.rand(2, 5, H, H, generator=g) - 1), 0.05 * (2 * torch.rand(5, H, generator=g) - 1)
    h, _, lin = read_trees(trees, vectors, U.cuda(), b.cuda())
    print("tree cell: %d nodes, %d levels, |h| %.4f" % (lin.N, int(lin.num_levels.item()), float(h.norm())))


if __name__ == "__main__":
    main()
