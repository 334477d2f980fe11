"""What the delta rule keeps of its operands: outputs and states as a whole against the definition, and inputs whose
outputs are small differences of large terms, which a 16-bit store shows too.  The bounds are held against an
emulation of the chunks that keeps two planes of three (CPU), and the library against the bounds (GPU)."""
import numpy as np
import pytest
import torch

from paper_2011_01383_amd import cortex as C
from tests import delta_planes as E
from tests.delta_helpers import Delta, say
from tests.gpu_helpers import need_gpu
from tests.sequence_helpers import U, host, type_step

# 2-norm of the errors over the 2-norm of the results.  Roundings are taken as independent, so that squares add.  On its
# way through a chunk a value is rounded in at most 40 sums and products of float32 (K / 32 or two
# steps of three parts in each of the four products, the solution's substitution and joins), each by at most U, U / sqrt 3 in the
# mean square: 3.7 U.  Its gates (an exponent's product, the exponential, the reciprocal in beta) are off by at most 3 U each, 5.2 U
# together, and the parts of products left out are 3 U: 7 U a chunk in all.  What later chunks keep of a chunk's errors they
# keep of its values as well; with four chunks' errors on top of each other that is 14 U.
NORM = 16 * U
# The largest 16-bit rounding is 2^-8; spread evenly over a step and over the logarithm, its mean square is 0.43 of that.
NORM_16 = 0.6 * 2.0 ** -8

# Sequences, heads, key heads, V; all for K of 32 to 128.
FORMS = {"few": ([200, 64, 1, 130], 2, 1, 32), "many": ([100, 3, 0, 130] * 20, 4, 2, 64), "segments": ([2900, 90], 1, 1, 32),
         "tokens": ([1] * 70, 4, 2, 64)}


def whole(form, K, dtype, seed=31):
    lens, H, G, V = FORMS[form]
    return Delta(seed, lens, H, G, K, V, dtype, slow=0.05, lean=1.0)


def norms(p, y, states, ref, new):
    """The distances of y and of each state, in parts of what is allowed."""
    allowed = NORM + (NORM_16 if p.dtype == torch.bfloat16 else 0.0)
    return E.distance(y, ref) / allowed, [E.distance(states[row], h) / NORM for row, (h, _) in new.items()]


@pytest.mark.parametrize("K", [32, 64, 128])
@pytest.mark.parametrize("form", ["few", "many"])
def test_two_planes_of_three_do_not_pass(form, K):
    """Emulated: with all bits nothing is off; two planes of any operand of a product are seen in float32 outputs, those of T, of R, of
    the state's updates and of the state itself in states too."""
    p = whole(form, K, "f32")
    ref, _, new = p.reference()
    y, states = norms(p, *E.prompt(p), ref, new)
    assert y < 1e-3 and max(states) < 1e-3
    for name in ("S", "T", "P", "R", "U", "W", "held"):
        y, states = norms(p, *E.prompt(p, **{name: 16}), ref, new)
        assert y > 1.25, (name, y)
        if name in ("T", "R", "W", "held"):
            assert max(states) > 1.25, (name, states)


def pair(form, K, dtype, decay, **kw):
    """No inputs but two tokens one behind the other in each sequence, with orthogonal keys and the same value; queries are the
    difference of the two keys.  (a, n): the keys' entries."""
    lens, H, G, V = FORMS[form]
    p = Delta(32, lens, H, G, K, V, dtype, decay=decay, bias=False, **kw)
    r = np.random.default_rng(K)
    rnd = lambda a: torch.from_numpy(np.asarray(a, np.float64)).to(torch.bfloat16).double().numpy()
    a, n = 1, K - 2
    c = rnd(0.5 + 0.4 * r.random((p.T, G)))
    p.q[:], p.k[:], p.v[:] = 0, 0, 0
    p.q[:, :, a], p.q[:, :, n] = c, -c
    at = [p.offsets[s] + (37 * s + 3) % (l - 1) for s, l in enumerate(lens) if l > 1]
    for t in at:
        p.k[t, :, a], p.k[t + 1, :, n] = 1, 1
        p.v[t] = p.v[t + 1] = rnd(r.normal(size=(H, V)))
    return p, c, at, (a, n)


def close_states(form, K, dtype):
    """y is the difference of two entries of the state that are the same to 15 bits: no inputs, no decay."""
    p, c, at, (a, n) = pair(form, K, dtype, False)
    p.k[:], p.v[:], p.state[:] = 0, 0, 0
    h = np.random.default_rng(K).normal(size=p.state.shape[:2]).astype(np.float32)
    p.state[:, :, a], p.state[:, :, n] = h, (h * np.float32(1 - 2.0 ** -15)).astype(np.float32)
    size = np.concatenate([np.broadcast_to(np.abs(h[s]).reshape(1, p.H, p.V), (l, p.H, p.V)) for s, l in enumerate(p.lens)])
    return p, 2 * abs(p.scale) * size * c.repeat(p.H // p.G, 1)[..., None]


def close_scores(form, K, dtype):
    """The two tokens' decays differ in the 12th bit, their shares are 1."""
    p, c, at, _ = pair(form, K, dtype, True, soft=False, sig=False, state=False)
    p.dt[:], p.b[:] = 2.0 ** -4, 1.0
    p.A = (-2.0 ** -8 * (1 + np.random.default_rng(K).random(p.H))).astype(np.float32).astype(np.float64)
    return p, magnitude(p, c, at, 1.0)


def close_updates(form, K, dtype):
    """The two tokens' shares differ in the 14th bit, no decay."""
    p, c, at, _ = pair(form, K, dtype, False, state=False)
    r = np.random.default_rng(K)
    p.b[:] = 0
    for t in at:
        p.b[t] = torch.from_numpy(2.0 ** -14 * (1 + r.random(p.H))).to(torch.bfloat16).double().numpy()
        p.b[t + 1] = -p.b[t]
    return p, magnitude(p, c, at, 0.5)


def magnitude(p, c, at, share):
    """Of the two terms whose difference y is (the decays after them, which shrink both, left out)."""
    size = np.zeros((p.T, p.H, p.V))
    for t in at:
        end = p.offsets[np.searchsorted(p.offsets, t, side="right")]
        size[t:end] = 2 * share * np.abs(p.v[t])
    return abs(p.scale) * size * c.repeat(p.H // p.G, 1)[..., None]


def close(p, mag, y, ref):
    """The worst error in parts of what is allowed.  Each term is rounded by at most: the gates 8 U (two exponentials, the sigmoid's
    reciprocal and sum), the products that form R, P, W and the outputs 6 U, the sums of parts 6 U, and by the state's sum and decay
    in chunks that follow, 2 U each; what a decay of several chunks is off by is the same for both and not seen.  24 U of the
    magnitude in all, and the store."""
    return float((np.abs(y - ref) / (24 * U * mag + type_step(p.dtype) * np.abs(ref) + 1e-30)).max())


CLOSE = {"states": close_states, "scores": close_scores, "updates": close_updates}


@pytest.mark.parametrize("K", [32, 64, 128])
@pytest.mark.parametrize("form", ["few", "many"])
@pytest.mark.parametrize("what,names", [("states", "S"), ("scores", "PWS"), ("updates", "RUW")])
def test_two_planes_do_not_pass_in_16_bits(what, names, form, K):
    p, mag = CLOSE[what](form, K, "bf16")
    ref, _, _ = p.reference()
    assert close(p, mag, E.prompt(p)[0], ref) < 1e-3
    for name in names:
        assert close(p, mag, E.prompt(p, **{name: 16})[0], ref) > 1.25, name


def run(p, form):
    if form != "tokens":
        assert (C.cortex_delta_segment_tokens(p.T, p.S, p.H, p.K, p.V) > 0) == (form == "segments")
    d = p.upload()
    out = None if p.state is None else torch.full_like(d["state"], 7.0)
    C.check(p.call(form == "tokens", state_out=out))
    torch.cuda.synchronize()
    assert int(d["status"].item()) == 0
    return host(d["y"]), None if out is None else host(out)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("K", [32, 64, 128])
@pytest.mark.parametrize("form", sorted(FORMS))
def test_outputs_and_states_as_a_whole(form, K, dtype):
    need_gpu()
    say("delta precision", form, K, dtype)
    p = whole(form, K, dtype)
    ref, _, new = p.reference()
    y, states = norms(p, *run(p, form), ref, new)
    say("y %.3f of the bound, states %.3f" % (y, max(states)))
    assert y <= 1 and max(states) <= 1


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("K", [32, 64, 128])
@pytest.mark.parametrize("form", ["few", "many", "segments"])
@pytest.mark.parametrize("what", sorted(CLOSE))
def test_small_differences(what, form, K, dtype):
    need_gpu()
    say("delta precision, close", what, form, K, dtype)
    p, mag = CLOSE[what](form, K, dtype)
    ref, _, _ = p.reference()
    worst = close(p, mag, run(p, form)[0], ref)
    say("%.3f of the bound" % worst)
    assert worst <= 1
