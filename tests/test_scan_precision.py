"""What the per-head scan keeps of its operands, by inputs that show it: outputs that are small
differences of large terms, and states as a whole.  The bounds are held against an emulation of
the products that keeps less (CPU), and the library against the bounds (GPU)."""
import numpy as np
import pytest
import torch

from paper_2011_01383_amd import cortex as C
from oracle import sequence_oracle as O
from tests import scan_planes as E
from tests.gpu_helpers import announce, need_gpu
from tests.sequence_helpers import Scan, U, host, offsets_of, type_step

T = 96


def bf16(a):
    return torch.from_numpy(np.asarray(a, np.float64)).to(torch.bfloat16).double().numpy()


def close_states(N, H, P, seed=0, T=T):
    """y is the difference of two entries of the state that are the same to 15 bits: no inputs, no decay."""
    r = np.random.default_rng(seed)
    D = H * P
    p = Scan(seed, [T], D, N, 1, P, dtype="bf16", z=False, skip=False, bias=False, soft=False)
    p.x[:], p.dt[:], p.B[:], p.C[:], p.state[:] = 0, 0, 0, 0, 0
    a, b = 1, N - 2
    c = bf16(r.normal(size=T))
    p.C[:, 0, a], p.C[:, 0, b] = c, -c
    h = r.normal(size=D).astype(np.float32)
    p.state[0, :, a], p.state[0, :, b] = h, (h * np.float32(1 - 2.0 ** -15)).astype(np.float32)
    return p


def close_scores(N, H, P, seed=0, T=T):
    """Two neighbouring tokens of every 32 have opposite inputs, and their decays differ in the 14th bit."""
    r = np.random.default_rng(seed)
    D = H * P
    p = Scan(seed, [T], D, N, 1, P, dtype="bf16", z=False, skip=False, state=False)
    p.x[:], p.dt[:], p.B[:], p.C[:] = 0, 0, 0, 0
    size = 0.02 + 0.02 * r.random(H)
    p.dt_bias = np.log(np.expm1(size)).astype(np.float32).astype(np.float64)
    p.A = (-2.0 ** -9 * (1 + r.random(H))).astype(np.float32).astype(np.float64)
    n = N // 2 + 3
    p.C[:, 0, n] = bf16(r.normal(size=T))
    for t in range(0, T, 32):
        v = bf16(r.normal(size=D))
        p.x[t + 3], p.x[t + 4] = v, -v
        p.B[t + 3, 0, n] = p.B[t + 4, 0, n] = bf16(r.normal())
    return p


def bound(p, ref, mag):
    """Few terms: for each the step size's softplus (the same for both, it cancels), an exponential (2 U), two
    products (2 U), and the additions of at most six parts (6 U); twice that, and the store's rounding."""
    return 20 * U * mag + type_step(p.dtype) * np.abs(ref) + 1e-30


def emulated(p, **planes):
    ref, mag, _ = p.reference()
    H, P = len(p.A), p.P
    raw = p.dt + (0 if p.dt_bias is None else p.dt_bias)
    dt = (O.softplus(raw) if p.soft else raw).astype(np.float32)
    state = np.zeros((p.D, p.N)) if p.state is None else p.state[0]
    y = np.zeros((p.T, p.D))
    for k in range(H):
        c = slice(k * P, k * P + P)
        y[:, c] = E.head_scan(p.x[:, c], dt[:, k], p.A[k], p.B[:, 0], p.C[:, 0], state[c], **planes)[0]
    return np.abs(bf16(y) - ref) / bound(p, ref, mag)


@pytest.mark.parametrize("N", [16, 64, 128])
def test_bounds_tell_two_planes_from_three(N):
    assert emulated(close_states(N, 2, 32)).max() <= 1
    assert emulated(close_states(N, 2, 32), planes_read=2).max() > 2
    assert emulated(close_scores(N, 8, 32)).max() <= 1
    assert emulated(close_scores(N, 8, 32), planes_score=2).max() > 2


@pytest.mark.gpu
@pytest.mark.parametrize("N", [16, 32, 64, 128])
@pytest.mark.parametrize("make", [close_states, close_scores])
@pytest.mark.parametrize("sequences", [1, 600])
def test_small_differences_of_large_terms(make, N, sequences):
    """bf16 prompts in segments (one sequence) and walked whole (many)."""
    need_gpu()
    announce("%s N %d, %d sequences" % (make.__name__, N, sequences))
    p = make(N, 4, 32)
    if sequences > 1:                            # the same one, every time
        p.lens, p.S, p.rows, p.T = [T] * sequences, sequences, sequences, T * sequences
        p.offsets = offsets_of(p.lens)
        tiled = lambda a: None if a is None else np.concatenate([a] * sequences)
        one = p.x, p.dt, p.B, p.C, p.state
        p.x, p.dt, p.B, p.C, p.state = map(tiled, one)
    d = p.upload()
    C.check(p.call())
    torch.cuda.synchronize()
    assert int(d["status"].item()) == 0
    got = host(d["y"])
    if sequences > 1:
        assert np.array_equal(got.reshape(sequences, T, -1), np.broadcast_to(got[:T], (sequences, T, p.D)))
        p.lens, p.S, p.T, p.offsets = [T], 1, T, offsets_of([T])
        p.x, p.dt, p.B, p.C, p.state = one
    ref, mag, _ = p.reference()
    worst = np.abs(got[:T] - ref) / bound(p, ref, mag)
    assert worst.max() <= 1, (float(worst.max()), np.argwhere(worst > 1)[0])


def slow(dtype, N, P, seed=3):
    """A hundred tokens and more stay in the state; step sizes as a model has them."""
    return Scan(seed, [320, 96], 2 * P, N, 1, P, dtype=dtype, slow=True, z=False, skip=False)


# Relative error over a whole output.  A state is summed over ten sub-chunks: each multiplies by a decay (an exponential
# and its argument, below 1 here: 3 U) and adds float32 products of its 32 tokens (their weights 4 U each, independent);
# the square root of ten times some 5 U, and as much again.
WHOLE = 1e-6


def norm_error(got, ref):
    return float(np.linalg.norm(got - ref) / np.linalg.norm(ref))


@pytest.mark.parametrize("N", [16, 64, 128])
def test_the_norm_tells_a_state_of_two_planes(N):
    p = slow("bf16", N, 32)
    new = p.reference()[2]
    dt = O.softplus(p.dt + p.dt_bias).astype(np.float32)

    def error(**planes):
        got, want = [], []
        for i in range(2):
            a, b = p.offsets[i], p.offsets[i + 1]
            for k in range(2):
                c = slice(k * 32, k * 32 + 32)
                got.append(E.head_scan(p.x[a:b, c], dt[a:b, k], p.A[k], p.B[a:b, 0], p.C[a:b, 0], p.state[i][c], **planes)[1])
                want.append(new[i][0][c])
        return norm_error(np.array(got, np.float64), np.array(want))

    assert error() <= WHOLE / 2
    assert error(planes_add=2) > 2 * WHOLE


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N", [16, 32, 64, 128])
def test_whole_outputs(N, dtype):
    """States of both types, and float32 outputs, to a few U over the whole of them."""
    need_gpu()
    for P in (32, 64, 128):
        announce("whole outputs %s N %d P %d" % (dtype, N, P))
        p = slow(dtype, N, P)
        d = p.upload()
        out = torch.zeros_like(d["state"])
        C.check(p.call(state_out=out))
        torch.cuda.synchronize()
        ref, _, new = p.reference()
        states = np.array([new[i][0] for i in range(2)])
        assert norm_error(host(out), states) <= WHOLE
        if dtype == "f32":
            assert norm_error(host(d["y"]), ref) <= WHOLE


# ---- ordinary tokens after a large step ----

def large_step(dtype, size, N=64, P=32, A=16.0):
    """Token 40 has a step of `size`, so nothing of the tokens before it is left; the others' are small."""
    p = Scan(11, [T], 2 * P, N, 1, P, dtype=dtype, z=False, skip=False, bias=False, soft=False, state=False)
    p.A[:] = -A
    p.dt[:] = bf16(0.002 + 0.006 * np.random.default_rng(1).random(p.dt.shape))
    p.dt[40] = bf16(size)
    p.x[40] = 0                                  # its own input would hide the others'
    return p


@pytest.mark.parametrize("size,wrong", [(20.0, 1.5e-6), (100.0, 1e-5), (1000.0, 1e-4), (20000.0, 2e-3)])
def test_the_norm_tells_sums_that_lose_small_steps(size, wrong):
    p = large_step("f32", size)
    ref = p.reference()[0][:, :32]

    def error(**kw):
        y, _ = E.head_scan(p.x[:, :32], p.dt[:, 0].astype(np.float32), p.A[0], p.B[:, 0], p.C[:, 0], np.zeros((32, 64)), **kw)
        return norm_error(y[41:].astype(np.float64), ref[41:])

    assert error() <= WHOLE / 2
    assert error(exact_sums=False) > wrong


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [20.0, 100.0, 1000.0, 20000.0])
def test_tokens_after_a_large_step(size, dtype):
    """As exact as without it.  A bf16 output is off by its store's rounding, 2^-9 at most.  Its float32
    value is off by some 3e-7, which takes it to the other side of a rounding's tie in 2 * 3e-7 / 2^-8 of
    the outputs, a few times more where the terms cancel."""
    need_gpu()
    for N in (16, 64, 128):
        announce("a step of %g, %s N %d" % (size, dtype, N))
        p = large_step(dtype, size, N)
        d = p.upload()
        C.check(p.call())
        torch.cuda.synchronize()
        assert int(d["status"].item()) == 0
        ref = p.reference()[0][41:]
        got = host(d["y"])[41:]
        assert norm_error(got, ref) <= (WHOLE if dtype == "f32" else 2.0 ** -9)
        if dtype == "bf16":
            # the rounded reference itself: few outputs fall on the other side of a tie
            assert np.mean(got != bf16(ref)) <= 0.002


# ---- 16-bit outputs are the rounded float32 ones ----

@pytest.mark.gpu
@pytest.mark.parametrize("form", ["channel", "head"])
@pytest.mark.parametrize("step", [False, True])
def test_outputs_are_rounded_once(form, step):
    """Float32 sums are off by half a U of their terms' magnitudes on average, and those are some sqrt(N) <= 11 of the
    sum: some 5e-7 of an output, 1e-6 with the smaller ones among them.  That is on the other side of a rounding's tie in
    2 * 1e-6 / 2^-8 = 0.05 percent of them.  Operands held to 16 bits put 0.1 to 0.25 percent there."""
    need_gpu()
    shapes = [(130, 16, 1, 0), (128, 64, 2, 0)] if form == "channel" else [(128, 16, 1, 32), (256, 64, 2, 64), (256, 128, 1, 128)]
    for D, N, G, P in shapes:
        for lens in ([[1] * 400] if step else [[70, 3, 0, 330], [5] * 1100]):
            announce("rounded once: %s step %s D %d N %d, %d sequences" % (form, step, D, N, len(lens)))
            p = Scan(7, lens, D, N, G, P, dtype="bf16")
            d = p.upload()
            C.check(p.call(step))
            torch.cuda.synchronize()
            assert int(d["status"].item()) == 0
            assert np.mean(host(d["y"]) != bf16(p.reference()[0])) <= 0.0005
