"""Rows to 8 bits and the projection over them: whole numbers are exact, the rest is a few float32 roundings."""
import numpy as np
import pytest
import torch

from oracle import sequence_oracle as O
from paper_2011_01383_amd import cortex as C
from tests.delta_helpers import say
from tests.gpu_helpers import need_gpu
from tests.sequence_helpers import DTYPES, U, columns, dev, host, type_step, within

pytestmark = pytest.mark.gpu


def status_word():
    return torch.zeros(1, dtype=torch.int32, device="cuda")


def rows8(a, left=0):
    """An int8 array on the GPU in rows of whole 16-byte pieces; what lies between them is no zero."""
    rows, cols = a.shape
    wide = torch.full((rows, left + (cols + 15) // 16 * 16), 77, dtype=torch.int8, device="cuda")
    wide[:, left:left + cols] = torch.from_numpy(a).cuda()
    return wide[:, left:left + cols]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("left", [0, 1, 8])
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 7), (5, 8), (2, 16), (70, 100), (9, 2048), (4, 4099), (2, 131071), (1000, 64)])
def test_quant(rows, cols, left, dtype):
    need_gpu()
    say("quant", rows, cols, left, dtype)
    r = np.random.default_rng(rows + cols)
    x = columns(r.normal(size=(rows, cols)) * np.exp(3 * r.normal(size=(rows, 1))), DTYPES[dtype], left, left)
    q = torch.full((rows, cols + left), 77, dtype=torch.int8, device="cuda")[:, :cols]
    scale, status = torch.full((rows,), 5.0, device="cuda"), status_word()
    C.check(C.cortex_quant_i8(x, q, scale, status=status))
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    want, s = O.quant_rows(x.float().cpu().numpy())
    assert np.array_equal(scale.cpu().numpy(), s) and np.array_equal(q.cpu().numpy(), want)
    assert (q._base.cpu()[:, cols:] == 77).all()


def test_quant_of_special_rows():
    need_gpu()
    say("quant special rows")
    x = np.random.default_rng(0).normal(size=(9, 40)).astype(np.float32)
    x[0] = 0.0
    x[1, 3], x[2, 4], x[3, 5] = np.nan, np.inf, -np.inf
    x[4] *= np.float32(2.0 ** -148)               # denormals: the scale is none or a few of the smallest
    x[5] *= np.float32(2.0 ** -140)
    x[6] = 3.0e38
    x[7] = np.arange(40) - 20 + 0.5               # halves, where the scale is 1
    x[7, 0] = 127.0
    x[8] = -0.0
    q, scale, status = torch.empty(9, 40, dtype=torch.int8, device="cuda"), torch.empty(9, device="cuda"), status_word()
    C.check(C.cortex_quant_i8(dev(x), q, scale, status=status))
    torch.cuda.synchronize()
    want, s = O.quant_rows(x)
    assert np.array_equal(scale.cpu().numpy(), s, equal_nan=True) and np.array_equal(q.cpu().numpy(), want)


def reference(q, scale, w, w_scale, bias):
    """Sums in whole numbers, then float64; the magnitude of what is added."""
    acc = q.astype(np.int64) @ w.astype(np.int64).T
    y = acc.astype(np.float64) * scale.astype(np.float64)[:, None] * w_scale.astype(np.float64)
    mag = np.abs(y) + (0 if bias is None else np.abs(bias))
    return (y if bias is None else y + bias), mag


def product(T, K, N, dtype, given=False, bias=True, left=0, seed=0, stream=None, full=False):
    r = np.random.default_rng(seed + T + K + N)
    t = DTYPES[dtype]
    w = r.integers(-128 if full else -127, 128, (N, K)).astype(np.int8)
    w_scale = (0.01 * (0.5 + r.random(N))).astype(np.float32)
    b = r.normal(size=N).astype(np.float32) if bias else None
    status = status_word()
    ws = torch.full((C.cortex_linear_i8_workspace_bytes(T, N, K),), 255, dtype=torch.uint8, device="cuda")
    y = torch.full((T, N + left), float("nan"), dtype=t, device="cuda")[:, :N]
    kw = dict(bias=None if b is None else dev(b), status=status, ws=ws, stream=stream)
    if given:
        q = r.integers(-128, 128, (T, K)).astype(np.int8)
        scale = (0.01 * (0.5 + r.random(T))).astype(np.float32)
        x = rows8(q, left)
        kw["x_scale"] = dev(scale)
    else:
        x = columns(r.normal(size=(T, K)), t, left, left)
        q, scale = O.quant_rows(x.float().cpu().numpy())
    wd, sd = rows8(w), dev(w_scale)
    torch.cuda.synchronize()
    C.check(C.cortex_linear_i8(x, wd, sd, y, **kw))
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    ref, mag = reference(q, scale, w, w_scale, b)
    # the sum to float32, two products and a sum: four roundings of the magnitude, and the store's
    within(host(y), ref, 5 * U * mag + type_step(t) * np.abs(ref) + 1e-30, "y")
    if left:
        assert torch.isnan(y._base[:, N:]).all()
    return y


SIZES = [(1, 64, 16), (1, 1, 1), (1, 4096, 1000), (2, 100, 33), (3, 128, 128), (5, 777, 130), (16, 2048, 512), (17, 40, 300), (33, 1001, 257),
         (64, 512, 1024), (65, 130, 129), (127, 256, 200), (128, 128, 128), (129, 1000, 515), (300, 640, 700), (1000, 144, 1030),
         (2100, 512, 1024), (1500, 1040, 2200)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("given", [False, True])
@pytest.mark.parametrize("T,K,N", SIZES)
def test_products(T, K, N, given, dtype):
    need_gpu()
    say("linear", T, K, N, given, dtype)
    product(T, K, N, dtype, given)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("given", [False, True])
@pytest.mark.parametrize("left", [1, 2, 3, 4, 16])
@pytest.mark.parametrize("T", [3, 70, 600])
def test_strides_and_alignments(T, left, given, dtype):
    need_gpu()
    say("linear strides", T, left, given, dtype)
    product(T, 208, 140, dtype, given, bias=False, left=left)


@pytest.mark.parametrize("T", [2, 300])
def test_largest_sums(T):
    """-128 times -128 over the most inputs: the sum is 2^31 - 2^14."""
    need_gpu()
    say("linear largest sums", T)
    K, N = 131071, 48
    x, w = torch.full((T, 131072), -128, dtype=torch.int8, device="cuda")[:, :K], torch.full((N, 131072), -128, dtype=torch.int8, device="cuda")[:, :K]
    y, status = torch.empty(T, N, device="cuda"), status_word()
    ws = C.workspace(C.cortex_linear_i8_workspace_bytes(T, N, K))
    one = torch.ones(max(T, N), device="cuda")
    C.check(C.cortex_linear_i8(x, w, one[:N].contiguous(), y, x_scale=one[:T].contiguous(), status=status, ws=ws))
    torch.cuda.synchronize()
    assert (host(y) == float(np.float32(K * 16384))).all()


@pytest.mark.parametrize("T", [1, 40, 500])
def test_a_row_that_is_not_finite_stays_alone(T):
    need_gpu()
    say("linear not finite", T)
    r = np.random.default_rng(1)
    x = dev(r.normal(size=(T, 96)))
    x[T // 2, 5] = float("inf")
    w, one = rows8(r.integers(-127, 128, (50, 96)).astype(np.int8)), torch.ones(50, device="cuda")
    y, status, ws = torch.empty(T, 50, device="cuda"), status_word(), C.workspace(C.cortex_linear_i8_workspace_bytes(T, 50, 96))
    C.check(C.cortex_linear_i8(x, w, one, y, status=status, ws=ws))
    torch.cuda.synchronize()
    odd = torch.isnan(y).all(1).cpu().numpy()
    assert odd[T // 2] and odd.sum() == 1 and torch.isfinite(y).all(1).sum().item() == T - 1


@pytest.mark.parametrize("T", [1, 40, 500])
def test_same_bits_on_another_stream_and_in_a_graph(T):
    need_gpu()
    say("linear streams and graphs", T)
    y = product(T, 512, 300, "bf16").clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    assert torch.equal(product(T, 512, 300, "bf16", stream=side), y)
    r = np.random.default_rng(2)
    x, w, s = dev(r.normal(size=(T, 512)), torch.bfloat16), rows8(r.integers(-127, 128, (300, 512)).astype(np.int8)), torch.ones(300, device="cuda")
    y, again, status = torch.empty(T, 300, dtype=torch.bfloat16, device="cuda"), torch.empty(T, 300, dtype=torch.bfloat16, device="cuda"), status_word()
    ws = C.workspace(C.cortex_linear_i8_workspace_bytes(T, 300, 512))
    C.check(C.cortex_linear_i8(x, w, s, y, status=status, ws=ws))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        C.check(C.cortex_linear_i8(x, w, s, again, status=status, ws=ws))
    for _ in range(3):
        again.zero_()
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(again, y)


@pytest.mark.parametrize("T", [1, 40, 500])
def test_an_earlier_error_leaves_outputs(T):
    need_gpu()
    say("linear earlier error", T)
    x, w = torch.randn(T, 64, device="cuda"), torch.ones(32, 64, dtype=torch.int8, device="cuda")
    y, status = torch.full((T, 32), 5.0, device="cuda"), torch.full((1,), C.CORTEX_ST_CYCLE, dtype=torch.int32, device="cuda")
    q, scale = torch.full((T, 64), 3, dtype=torch.int8, device="cuda"), torch.full((T,), 5.0, device="cuda")
    ws = C.workspace(C.cortex_linear_i8_workspace_bytes(T, 32, 64))
    C.check(C.cortex_linear_i8(x, w, torch.ones(32, device="cuda"), y, status=status, ws=ws))
    C.check(C.cortex_quant_i8(x, q, scale, status=status))
    torch.cuda.synchronize()
    assert (y == 5.0).all() and (q == 3).all() and (scale == 5.0).all() and int(status.item()) == C.CORTEX_ST_CYCLE


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("given", [False, True])
@pytest.mark.parametrize("T,K,N", [(1, 16384, 40), (1, 16385, 40), (2, 16385, 17), (4, 8200, 50), (9, 100, 8203), (24, 100, 8203),
                                   (32, 1000, 8177), (50, 200, 8190), (64, 70, 8176)])
def test_few_tokens_of_many_channels_and_inputs(T, K, N, given, dtype):
    need_gpu()
    say("linear few tokens", T, K, N, given, dtype)
    product(T, K, N, dtype, given)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("left", [0, 1, 2, 3, 4, 16])
def test_one_token(left, dtype):
    need_gpu()
    say("linear one token", left, dtype)
    for K in (15, 16, 208, 2048, 2050, 4100):
        product(1, K, 139, dtype, left=left)


def test_one_token_of_special_values():
    """A NaN or an infinity makes the outputs NaN, a row of zeros leaves the bias, an earlier error everything."""
    need_gpu()
    say("linear one token of special values")
    w, ws = torch.ones(20, 48, dtype=torch.int8, device="cuda")[:, :40], C.workspace(C.cortex_linear_i8_workspace_bytes(1, 20, 40))
    one, bias, status = torch.ones(20, device="cuda"), torch.arange(20.0, device="cuda"), status_word()
    for bad in (float("nan"), float("inf"), 0.0):
        x, y = torch.zeros(1, 40, device="cuda"), torch.full((1, 20), 5.0, device="cuda")
        x[0, 3] = bad
        C.check(C.cortex_linear_i8(x, w, one, y, bias=bias, status=status, ws=ws))
        torch.cuda.synchronize()
        assert torch.equal(y[0], bias) if bad == 0.0 else torch.isnan(y).all()
    status.fill_(C.CORTEX_ST_CYCLE)
    y = torch.full((1, 20), 5.0, device="cuda")
    C.check(C.cortex_linear_i8(torch.zeros(1, 40, device="cuda"), w, one, y, bias=bias, status=status, ws=ws))
    torch.cuda.synchronize()
    assert (y == 5.0).all() and int(status.item()) == C.CORTEX_ST_CYCLE


@pytest.mark.parametrize("cols", [1000, 2048, 5000])
def test_quant_near_halves(cols):
    """Quotients within a few steps of n + 1/2, where a quotient off by one step would be another whole number; scales
    over the whole range of the type."""
    need_gpu()
    say("quant near halves", cols)
    r = np.random.default_rng(cols)
    tops = (2.0 ** r.uniform(-145, 127, 400) * (1 + r.random(400))).astype(np.float32)
    scale = tops / np.float32(127)
    x = (r.integers(-127, 127, (400, cols)) + 0.5).astype(np.float32) * scale[:, None]
    x = (x.view(np.int32) + r.integers(-2, 3, x.shape).astype(np.int32)).view(np.float32)
    x = np.where(np.abs(x) <= tops[:, None], x, np.float32(0))
    x[:, 7] = tops
    q, s, status = torch.empty(400, cols, dtype=torch.int8, device="cuda"), torch.empty(400, device="cuda"), status_word()
    C.check(C.cortex_quant_i8(dev(x), q, s, status=status))
    torch.cuda.synchronize()
    want, ws = O.quant_rows(x)
    assert np.array_equal(s.cpu().numpy(), ws) and np.array_equal(q.cpu().numpy(), want)


@pytest.mark.parametrize("T,N", [(5, 50), (20, 50), (60, 50), (20, 8200), (60, 8200)])
def test_few_tokens_of_every_number_of_shares(T, N):
    """Inputs of one, two and more 64-byte shares for each of eight waves, and of fewer than waves."""
    need_gpu()
    say("linear shares", T, N)
    for K in (64, 65, 512, 513, 1024, 1025, 2048, 2100):
        product(T, K, N, "bf16", given=K % 2 == 1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("left", [0, 1, 8])
@pytest.mark.parametrize("rows,cols", [(7, 1024), (3, 1025), (7, 2049), (5, 4096), (3, 4097), (5, 8192), (3, 8193), (3, 16384), (2, 16385),
                                       (300, 6098)])
def test_quant_of_every_number_of_waves(rows, cols, left, dtype):
    test_quant(rows, cols, left, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N", [1, 50, 1000])
def test_one_token_of_every_number_of_shares(N, dtype):
    need_gpu()
    say("linear one token, shares", N, dtype)
    for K in (1, 63, 64, 512, 513, 1024, 1025, 4032, 4033, 4096, 4100, 8192, 8193, 16384):
        product(1, K, N, dtype)
