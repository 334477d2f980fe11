"""Norms of queries and keys with their rotation, against the float64 definition."""
import numpy as np
import pytest
import torch

from oracle import sequence_oracle as O
from paper_2011_01383_amd import cortex as C
from tests.delta_helpers import heads, say
from tests.gpu_helpers import need_gpu
from tests.sequence_helpers import DTYPES, U, dev, host, type_step, within

pytestmark = pytest.mark.gpu
NORMS = {"none": C.CORTEX_NORM_NONE, "rms": C.CORTEX_NORM_RMS, "l2": C.CORTEX_NORM_L2}


def make(seed, T, H, G, P, R, dtype, far=300000):
    r = np.random.default_rng(seed)
    t = DTYPES[dtype]
    rnd = lambda a: torch.from_numpy(a).to(t).double().numpy()
    f32 = lambda a: a.astype(np.float32).astype(np.float64)
    return dict(q=rnd(r.normal(size=(T, H, P))), k=rnd(r.normal(size=(T, G, P))) if G else None, qw=f32(1 + 0.1 * r.normal(size=P)),
                kw=f32(1 + 0.1 * r.normal(size=P)), at=r.integers(-far, far, T).astype(np.int32),
                freqs=f32(10000.0 ** (-np.arange(R // 2) / max(R // 2, 1))), t=t, T=T, H=H, G=G, P=P, R=R)


def bound(p, ref, mag):
    """The norm is a sum of P squares (P U), a quotient and a root, the weight and the rotation six roundings of
    the magnitude; a cosine is off by at most 2 U, plus the angle's 2^-22 of a turn at 2^31 positions, here below U."""
    return (p["P"] / 2 + 32) * U * mag + type_step(p["t"]) * np.abs(ref) + 1e-30


def run(p, norm, interleaved, eps=1e-6, weights=True, left=0, in_place=False, graph=False, stream=None):
    q, k = heads(p["q"], p["t"], left, left), None if p["k"] is None else heads(p["k"], p["t"], 0, left)
    qo = q if in_place else heads(np.full_like(p["q"], 5.0), p["t"], 0, left)
    ko = k if in_place or k is None else heads(np.full_like(p["k"], 5.0), p["t"], left)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    kw = dict(k=k, k_out=ko, norm=NORMS[norm], eps=eps, interleaved=interleaved, status=status, stream=stream)
    if weights:
        kw.update(q_weight=dev(p["qw"]), k_weight=dev(p["kw"]) if k is not None else None)
    if p["R"]:
        kw.update(positions=dev(p["at"], torch.int32), freqs=dev(p["freqs"]))
    torch.cuda.synchronize()
    C.check(C.cortex_qk_norm(q, qo, **kw))
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    for x, w, out, name in ((p["q"], p["qw"], qo, "q"), (p["k"], p["kw"], ko, "k")):
        if x is None:
            continue
        ref, mag = O.qk_norm(x, norm, float(np.float32(eps)), w if weights else None, p["at"], p["freqs"], interleaved)
        within(host(out), ref, bound(p, ref, mag), name)
    return qo, ko


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("norm", sorted(NORMS))
@pytest.mark.parametrize("P,R", [(128, 128), (128, 32), (64, 64), (64, 0), (32, 32), (256, 128), (80, 40), (96, 96), (512, 512), (2, 2),
                                 (66, 10), (16, 16), (512, 16), (256, 6)])
def test_heads(P, R, norm, interleaved, dtype):
    need_gpu()
    say("norm heads", P, R, norm, interleaved, dtype)
    run(make(1, 5, 3, 2, P, R, dtype), norm, interleaved)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,H,G", [(1, 1, 0), (1, 40, 8), (700, 1, 1), (33, 17, 5), (2000, 9, 3), (5000, 4, 0)])
def test_sizes(T, H, G, dtype):
    need_gpu()
    say("norm sizes", T, H, G, dtype)
    run(make(2, T, H, G, 64, 64, dtype), "rms", False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("left", [1, 2, 3, 8])
def test_strides_and_alignments(left, dtype):
    need_gpu()
    say("norm strides", left, dtype)
    for interleaved in (False, True):
        run(make(3, 9, 3, 2, 64, 32, dtype), "l2", interleaved, left=left)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("norm", sorted(NORMS))
@pytest.mark.parametrize("P,R", [(128, 64), (66, 66)])
def test_in_place(P, R, norm, dtype):
    need_gpu()
    say("norm in place", P, R, norm, dtype)
    for interleaved in (False, True):
        run(make(4, 50, 5, 3, P, R, dtype), norm, interleaved, in_place=True, left=8)


def test_rows_beside_stay_as_they_are():
    need_gpu()
    say("norm rows beside")
    q = torch.randn(7, 2, 64, device="cuda")
    wide = torch.full((9, 300), 3.0, device="cuda")
    out = wide[1:8, 100:228].unflatten(1, (2, 64))
    C.check(C.cortex_qk_norm(q, out, status=torch.zeros(1, dtype=torch.int32, device="cuda")))
    torch.cuda.synchronize()
    mask = torch.zeros(9, 300, dtype=torch.bool)
    mask[1:8, 100:228] = True
    assert (wide.cpu()[~mask] == 3.0).all() and (wide.cpu()[mask] != 3.0).all()


@pytest.mark.parametrize("P", [64, 66])
def test_zeros_and_what_is_not_finite(P):
    """A row of zeros stays zeros (with eps), an infinity or NaN stays in its head."""
    need_gpu()
    say("norm zeros", P)
    p = make(5, 6, 2, 1, P, 2 * (P // 4), "f32")
    q = dev(p["q"].reshape(6, -1)).reshape(6, 2, P)
    q[1] = 0.0
    q[2, 0, 5], q[3, 1, 7] = float("nan"), float("inf")
    out, status = torch.empty_like(q), torch.zeros(1, dtype=torch.int32, device="cuda")
    C.check(C.cortex_qk_norm(q, out, norm=C.CORTEX_NORM_L2, positions=dev(p["at"], torch.int32), freqs=dev(p["freqs"]), status=status))
    torch.cuda.synchronize()
    assert (out[1] == 0).all() and torch.isnan(out[2, 0]).all()
    assert torch.isnan(out[3, 1]).any() and torch.isfinite(out[[0, 1, 4, 5]]).all() and torch.isfinite(out[2, 1]).all()
    assert torch.isfinite(out[3, 0]).all()


def test_far_positions():
    """Positions to the ends of their type: the angle's own rounding in 64 bits, 2^31 * 2^-53 turns, is below 2^-21 of one."""
    need_gpu()
    say("norm far positions")
    p = make(6, 64, 1, 0, 64, 64, "f32", far=2 ** 31 - 1)
    p["at"][:4] = [2 ** 31 - 1, -2 ** 31, 0, -1]
    run(p, "none", False, weights=False)


def test_same_bits_on_another_stream_and_in_a_graph():
    need_gpu()
    say("norm streams and graphs")
    p = make(7, 30, 4, 2, 64, 64, "bf16")
    qo, ko = (t.clone() for t in run(p, "rms", False))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    q2, k2 = run(p, "rms", False, stream=side)
    assert torch.equal(q2, qo) and torch.equal(k2, ko)
    q, k, status = heads(p["q"], p["t"]), heads(p["k"], p["t"]), torch.zeros(1, dtype=torch.int32, device="cuda")
    kw = dict(q_weight=dev(p["qw"]), k_weight=dev(p["kw"]), positions=dev(p["at"], torch.int32), freqs=dev(p["freqs"]), status=status)
    graph, q3, k3 = torch.cuda.CUDAGraph(), torch.empty_like(q), torch.empty_like(k)
    with torch.cuda.graph(graph):
        C.check(C.cortex_qk_norm(q, q3, k=k, k_out=k3, **kw))
    for _ in range(3):
        q3.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(q3, qo) and torch.equal(k3, ko)


def test_an_earlier_error_leaves_outputs():
    need_gpu()
    say("norm earlier error")
    q = torch.randn(5, 2, 64, device="cuda")
    for P in (64, 62):
        out = torch.full((5, 2, P), 5.0, device="cuda")
        status = torch.full((1,), C.CORTEX_ST_CYCLE, dtype=torch.int32, device="cuda")
        C.check(C.cortex_qk_norm(q[:, :, :P].contiguous(), out, status=status))
        torch.cuda.synchronize()
        assert (out == 5.0).all() and int(status.item()) == C.CORTEX_ST_CYCLE


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("norm", sorted(NORMS))
@pytest.mark.parametrize("P,R", [(128, 128), (128, 32), (64, 64), (64, 0), (32, 32), (256, 128), (80, 48), (96, 96), (512, 512), (16, 16),
                                 (512, 16), (256, 6), (66, 10)])
def test_heads_of_many_rows(P, R, norm, interleaved, dtype):
    """More rows than have a wave each."""
    need_gpu()
    say("norm many rows", P, R, norm, interleaved, dtype)
    run(make(8, 823, 3, 2, P, R, dtype), norm, interleaved)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,H,G", [(64, 65, 0), (101, 40, 8), (513, 9, 1), (1025, 17, 5), (4099, 1, 0), (4500, 4, 4)])
def test_sizes_of_many_rows(T, H, G, dtype):
    need_gpu()
    say("norm sizes of many rows", T, H, G, dtype)
    run(make(9, T, H, G, 64, 64, dtype), "rms", False)
    run(make(9, T, H, G, 32, 16, dtype), "l2", True, left=8, in_place=True)


def test_special_values_in_many_rows():
    """As in few: zeros, NaN, infinities, positions to the ends of their type, an earlier error, a graph."""
    need_gpu()
    say("norm special values in many rows")
    p = make(10, 4200, 1, 1, 64, 64, "f32", far=2 ** 31 - 1)
    p["at"][:4] = [2 ** 31 - 1, -2 ** 31, 0, -1]
    run(p, "none", True, weights=False)
    q = dev(p["q"].reshape(4200, -1)).reshape(4200, 1, 64)
    q[1] = 0.0
    q[2, 0, 5], q[3, 0, 7] = float("nan"), float("inf")
    out, status = torch.full_like(q, 5.0), torch.full((1,), C.CORTEX_ST_CYCLE, dtype=torch.int32, device="cuda")
    kw = dict(norm=C.CORTEX_NORM_L2, positions=dev(p["at"], torch.int32), freqs=dev(p["freqs"]), status=status)
    C.check(C.cortex_qk_norm(q, out, **kw))
    torch.cuda.synchronize()
    assert (out == 5.0).all() and int(status.item()) == C.CORTEX_ST_CYCLE
    status.zero_()
    C.check(C.cortex_qk_norm(q, out, **kw))
    torch.cuda.synchronize()
    assert (out[1] == 0).all() and torch.isnan(out[2]).all() and torch.isnan(out[3]).any()
    assert torch.isfinite(out[0]).all() and torch.isfinite(out[4:]).all()
    graph, again = torch.cuda.CUDAGraph(), torch.empty_like(q)
    with torch.cuda.graph(graph):
        C.check(C.cortex_qk_norm(q, again, **kw))
    for _ in range(3):
        again.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(again[4:], out[4:]) and torch.equal(again[:2], out[:2])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("P,R", [(64, 0), (64, 16), (128, 96), (32, 32), (66, 10), (80, 40)])
def test_what_is_not_finite_without_a_norm_stays_with_its_element(P, R, bad, interleaved, dtype):
    """An element outside the rotation reaches its own output, one inside that of its pair too, in few rows and in many."""
    need_gpu()
    say("norm none, not finite", P, R, bad, interleaved, dtype)
    for T in (6, 1400):
        p = make(11, T, 2, 1, P, R, dtype)
        kw = dict(norm=C.CORTEX_NORM_NONE, interleaved=interleaved, q_weight=dev(p["qw"]), status=torch.zeros(1, dtype=torch.int32, device="cuda"))
        if R:
            kw.update(positions=dev(p["at"], torch.int32), freqs=dev(p["freqs"]))
        k = heads(p["k"], p["t"])
        q, hit = heads(p["q"], p["t"]), np.zeros((T, 2, P), dtype=bool)
        clean, k_clean = torch.empty_like(q, memory_format=torch.contiguous_format), torch.empty_like(k, memory_format=torch.contiguous_format)
        C.check(C.cortex_qk_norm(q, clean, k=k, k_out=k_clean, **kw))
        for t in range(min(T, P)):               # every place of a head, in another token each
            q[t, t % 2, t] = bad
            hit[t, t % 2, t] = True
            if t < R:
                hit[t, t % 2, t ^ 1 if interleaved else (t + R // 2) % R] = True
        got, k_got = torch.empty_like(clean), torch.empty_like(k_clean)
        C.check(C.cortex_qk_norm(q, got, k=k, k_out=k_got, **kw))
        torch.cuda.synchronize()
        assert torch.equal(k_got, k_clean)
        assert np.array_equal(host(got)[~hit], host(clean)[~hit]) and not np.isfinite(host(got)[hit]).any()
        for t in range(R, min(T, P)):
            assert np.array_equal(host(got)[t, t % 2, t], bad, equal_nan=True)


@pytest.mark.parametrize("norm", ["rms", "l2"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("P,R", [(64, 0), (128, 32), (66, 10)])
def test_an_infinity_in_a_norm_leaves_zeros_beside_it(P, R, interleaved, norm):
    """x / infinity is 0 but for the infinite element itself, which has no value."""
    need_gpu()
    say("norm of an infinity", P, R, interleaved, norm)
    for T in (6, 4200):
        p = make(12, T, 1, 0, P, R, "f32")
        q = heads(p["q"], p["t"])
        q[:6, 0, P - 3] = float("inf")
        kw = dict(positions=dev(p["at"], torch.int32), freqs=dev(p["freqs"])) if R else {}
        out = torch.empty_like(q)
        C.check(C.cortex_qk_norm(q, out, norm=NORMS[norm], interleaved=interleaved, status=torch.zeros(1, dtype=torch.int32, device="cuda"), **kw))
        torch.cuda.synchronize()
        rest = [i for i in range(P) if i != P - 3]
        assert torch.isnan(out[:6, 0, P - 3]).all() and (out[:6, 0, rest] == 0).all() and torch.isfinite(out[6:]).all()


@pytest.mark.parametrize("T", [5, 4200])
def test_sums_of_squares_past_the_float_range(T):
    need_gpu()
    say("norm past the float range", T)
    q, status = torch.randn(T, 1, 64, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    q[1], q[3] = 1e20, 1e-30
    for norm in ("rms", "l2"):
        out = torch.empty_like(q)
        C.check(C.cortex_qk_norm(q, out, norm=NORMS[norm], eps=0.0, status=status))
        torch.cuda.synchronize()
        assert (out[1] == 0).all() and not torch.isfinite(out[3]).any() and torch.isfinite(out[[0, 2, 4]]).all()
