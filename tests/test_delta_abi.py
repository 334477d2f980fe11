"""Refusals of the delta rule, the norms of queries and keys and the 8-bit projection that need no GPU."""
import ctypes
import os

import pytest
import torch

from paper_2011_01383_amd import cortex as C

P8 = 256                       # a pointer that is never followed: the checks come first


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(C.LIB_PATH):
        from paper_2011_01383_amd import build
        build.build()
    return C.load()


def delta_args(**kw):
    a = dict(dtype=1, num_seqs=2, num_tokens=2, heads=4, key_heads=2, key_dim=64, value_dim=32, softplus=1, sigmoid=1,
             state_rows=2, scale=1.0, seq_offsets=P8, state_index=None, q=P8, k=P8, v=P8, b=P8, dt=P8, q_ld=128, k_ld=128,
             v_ld=128, b_ld=4, dt_ld=4, A=P8, dt_bias=None, state_in=P8, state_out=P8, y=P8, y_ld=128)
    a.update(kw)
    return C.cortex_delta_t(**a)


@pytest.mark.parametrize("bad", [
    dict(dtype=2), dict(num_seqs=-1), dict(num_tokens=-1), dict(heads=0), dict(key_heads=0), dict(key_heads=3), dict(key_dim=16),
    dict(key_dim=48), dict(key_dim=256, q_ld=512, k_ld=512), dict(value_dim=8), dict(value_dim=24),
    dict(value_dim=272, v_ld=1088, y_ld=1088), dict(heads=2048, value_dim=256, v_ld=1 << 19, y_ld=1 << 19, b_ld=2048, dt_ld=2048),
    dict(state_rows=1), dict(state_rows=-1), dict(q=None), dict(k=None), dict(v=None), dict(b=None), dict(dt=None), dict(y=None),
    dict(q_ld=127), dict(k_ld=127), dict(v_ld=127), dict(y_ld=127), dict(b_ld=3), dict(dt_ld=3), dict(q_ld=(1 << 25) + 1),
    dict(state_in=P8 + 4), dict(state_out=P8 + 8), dict(num_seqs=0), dict(num_tokens=2 ** 31 - 1)])
def test_delta_refuses(lib, bad):
    args = ctypes.byref(delta_args(**bad))
    assert lib.cortex_delta_forward(args, P8, P8, 1 << 50, None) == C.CORTEX_E_INVAL
    assert lib.cortex_delta_step(args, P8, None) == C.CORTEX_E_INVAL


def test_delta_refuses_by_form(lib):
    ok = delta_args()
    assert lib.cortex_delta_forward(ctypes.byref(delta_args(seq_offsets=None)), P8, P8, 1 << 50, None) == C.CORTEX_E_INVAL
    assert lib.cortex_delta_forward(None, P8, P8, 1 << 50, None) == C.CORTEX_E_INVAL
    assert lib.cortex_delta_forward(ctypes.byref(ok), None, P8, 1 << 50, None) == C.CORTEX_E_INVAL
    assert lib.cortex_delta_forward(ctypes.byref(ok), P8, None, 1 << 50, None) == C.CORTEX_E_INVAL
    assert lib.cortex_delta_step(ctypes.byref(delta_args(num_tokens=1)), P8, None) == C.CORTEX_E_INVAL
    assert lib.cortex_delta_step(ctypes.byref(delta_args(num_tokens=3)), P8, None) == C.CORTEX_E_INVAL
    for off in (1, 2, 4, 8):
        assert lib.cortex_delta_forward(ctypes.byref(ok), P8, P8 + off, 1 << 50, None) == C.CORTEX_E_INVAL
    need = lib.cortex_delta_workspace_bytes(2, 2, 4, 64, 32)
    assert need > 0
    assert lib.cortex_delta_forward(ctypes.byref(ok), P8, P8, need - 1, None) == C.CORTEX_E_WORKSPACE


@pytest.mark.parametrize("size", [(-1, 1, 4, 64, 32), (1, -1, 4, 64, 32), (1, 1, 0, 64, 32), (1, 1, 4, 100, 32), (1, 1, 4, 64, 20)])
def test_delta_workspace_of_invalid_sizes(lib, size):
    assert lib.cortex_delta_workspace_bytes(*size) == 0


def test_delta_workspace_serves_smaller_batches(lib):
    need = lib.cortex_delta_workspace_bytes
    for T, S in ((1, 1), (64, 1), (1000, 7), (5000, 300), (0, 9)):
        assert need(T + 1, S, 8, 128, 64) >= need(T, S, 8, 128, 64)
        assert need(T, S + 1, 8, 128, 64) >= need(T, S, 8, 128, 64)


def test_delta_of_nothing(lib):
    for T in (0,):
        a = ctypes.byref(delta_args(num_seqs=0, num_tokens=T, state_rows=0, q=None, k=None, v=None, b=None, dt=None, y=None))
        assert lib.cortex_delta_forward(a, P8, P8, 1 << 50, None) == C.CORTEX_OK
        assert lib.cortex_delta_step(a, P8, None) == C.CORTEX_OK


def test_delta_of_more_than_a_grid_holds(lib):
    a = delta_args(num_seqs=1 << 25, num_tokens=1 << 25, heads=1, key_heads=1, value_dim=16, state_rows=1 << 25)
    assert lib.cortex_delta_step(ctypes.byref(a), P8, None) == C.CORTEX_E_INVAL
    assert lib.cortex_delta_forward(ctypes.byref(a), P8, P8, 1 << 62, None) == C.CORTEX_E_INVAL


def test_delta_of_more_chunks_than_a_grid_holds(lib):
    for T, S, heads in ((1 << 29, 1, 1), (64, 1 << 23, 1), ((1 << 29) // 32, 1, 32)):
        a = delta_args(num_seqs=S, num_tokens=T, heads=heads, key_heads=1, value_dim=16, state_rows=S, q_ld=1 << 12, k_ld=1 << 12,
                       v_ld=1 << 12, y_ld=1 << 12, b_ld=1 << 12, dt_ld=1 << 12)
        assert lib.cortex_delta_forward(ctypes.byref(a), P8, P8, 1 << 62, None) == C.CORTEX_E_INVAL


def norm_args(**kw):
    a = dict(dtype=0, num_tokens=2, heads=4, key_heads=2, head_dim=64, rotary_dim=32, interleaved=0, norm=1, eps=1e-6, q=P8, k=P8,
             q_ld=256, k_ld=128, q_weight=None, k_weight=None, positions=P8, freqs=P8, q_out=P8, k_out=P8, q_out_ld=256,
             k_out_ld=128)
    a.update(kw)
    return C.cortex_qk_norm_t(**a)


@pytest.mark.parametrize("bad", [
    dict(dtype=2), dict(num_tokens=-1), dict(heads=0), dict(key_heads=-1), dict(head_dim=0), dict(head_dim=63), dict(head_dim=514),
    dict(rotary_dim=-2), dict(rotary_dim=31), dict(rotary_dim=66), dict(norm=-1), dict(norm=3), dict(eps=-1.0),
    dict(eps=float("nan")), dict(q=None), dict(k=None), dict(q_out=None), dict(k_out=None), dict(positions=None),
    dict(freqs=None), dict(q_ld=255), dict(k_ld=127), dict(q_out_ld=255), dict(k_out_ld=127), dict(num_tokens=1 << 24)])
def test_norm_refuses(lib, bad):
    assert lib.cortex_qk_norm(ctypes.byref(norm_args(**bad)), P8, None) == C.CORTEX_E_INVAL


def test_norm_of_nothing(lib):
    assert lib.cortex_qk_norm(ctypes.byref(norm_args(num_tokens=0, q=None, k=None)), P8, None) == C.CORTEX_OK
    assert lib.cortex_qk_norm(None, P8, None) == C.CORTEX_E_INVAL
    assert lib.cortex_qk_norm(ctypes.byref(norm_args()), None, None) == C.CORTEX_E_INVAL


def quant_args(**kw):
    a = dict(dtype=0, rows=2, columns=8, x=P8, x_ld=8, q=P8, q_ld=8, scale=P8)
    a.update(kw)
    return C.cortex_quant_i8_t(**a)


@pytest.mark.parametrize("bad", [dict(dtype=2), dict(rows=-1), dict(rows=1 << 24), dict(rows=1 << 22), dict(columns=0),
                                 dict(columns=131072, x_ld=131072, q_ld=131072), dict(x=None), dict(q=None), dict(scale=None),
                                 dict(x_ld=7), dict(q_ld=7)])
def test_quant_refuses(lib, bad):
    assert lib.cortex_quant_i8(ctypes.byref(quant_args(**bad)), P8, None) == C.CORTEX_E_INVAL


def linear_args(**kw):
    a = dict(dtype=1, tokens=2, inputs=40, outputs=8, x=P8, x_ld=40, x_scale=None, w=P8, w_ld=48, w_scale=P8, bias=None, y=P8, y_ld=8)
    a.update(kw)
    return C.cortex_linear_i8_t(**a)


@pytest.mark.parametrize("bad", [
    dict(dtype=2), dict(tokens=-1), dict(inputs=0), dict(inputs=131072, x_ld=131072, w_ld=131072), dict(outputs=0), dict(x=None),
    dict(w=None), dict(w_scale=None), dict(y=None), dict(x_ld=39), dict(w_ld=40), dict(w_ld=56), dict(w_ld=32), dict(y_ld=7),
    dict(w=P8 + 8), dict(w_ld=(1 << 24) + 16), dict(tokens=1 << 24), dict(tokens=1 << 22)])
def test_linear_refuses(lib, bad):
    assert lib.cortex_linear_i8(ctypes.byref(linear_args(**bad)), P8, P8, 1 << 50, None) == C.CORTEX_E_INVAL


@pytest.mark.parametrize("size", [(1, (1 << 26) + 16), (1 << 12, (1 << 25) + 16), ((1 << 24) - 1, 1 << 14)])
def test_linear_of_more_than_a_grid_holds(lib, size):
    tokens, outputs = size
    a = linear_args(tokens=tokens, outputs=outputs, y_ld=outputs)
    assert lib.cortex_linear_i8(ctypes.byref(a), P8, P8, 1 << 62, None) == C.CORTEX_E_INVAL
    assert lib.cortex_linear_i8_workspace_bytes(tokens, outputs, 40) == 0


def test_linear_workspace(lib):
    a = ctypes.byref(linear_args())
    need = lib.cortex_linear_i8_workspace_bytes
    assert need(-1, 8, 40) == need(2, 0, 40) == need(2, 8, 0) == need(2, 8, 131072) == 0
    assert lib.cortex_linear_i8(a, P8, None, 1 << 50, None) == C.CORTEX_E_INVAL
    assert lib.cortex_linear_i8(a, P8, P8 + 8, 1 << 50, None) == C.CORTEX_E_INVAL
    assert lib.cortex_linear_i8(a, P8, P8, 0, None) == C.CORTEX_E_WORKSPACE
    for T, N, K in ((1, 8, 40), (17, 5000, 4096), (300, 64, 100), (5000, 1000, 1000)):
        assert 0 < need(T, N, K) <= need(T + 1, N, K)


def test_linear_and_quant_of_nothing(lib):
    assert lib.cortex_linear_i8(ctypes.byref(linear_args(tokens=0, x=None, y=None)), P8, None, 0, None) == C.CORTEX_OK
    assert lib.cortex_quant_i8(ctypes.byref(quant_args(rows=0, x=None)), P8, None) == C.CORTEX_OK


Z, I32, I8 = torch.zeros, torch.int32, torch.int8
STATUS = Z(1, dtype=I32)
WS = Z(256, dtype=torch.uint8)


def test_binding_refuses_delta():
    good = dict(q=Z(3, 2, 32), k=Z(3, 2, 32), v=Z(3, 4, 16), b=Z(3, 4), offsets=Z(2, dtype=I32), y=Z(3, 4, 16), status=STATUS, ws=WS)
    for kw, what in ((dict(), "in device memory"), (dict(v=Z(3, 64)), "v must be a"), (dict(v=Z(3, 4, 16).half()), "v must be a"),
                     (dict(k=Z(3, 2, 64)), r"k must be \[3, 2, 32\]"), (dict(k=Z(3, 4, 32)), r"k must be \[3, 2, 32\]"),
                     (dict(q=Z(2, 2, 32)), "q must have 3 rows"), (dict(q=Z(3, 2, 32).bfloat16()), "q must be torch.float32"),
                     (dict(y=Z(3, 4, 32)), "y must be"), (dict(b=Z(3, 3)), "b must be"), (dict(dt=Z(3, 4)), "A is required"),
                     (dict(A=Z(4)), "dt is required"), (dict(A=Z(3), dt=Z(3, 4)), "A holds 3 elements"),
                     (dict(offsets=None), "offsets must be"), (dict(ws=None), "ws is required"), (dict(status=None), "status is required"),
                     (dict(scale="1"), "scale must be a number"), (dict(scale=Z(1)), "scale must be a number"),
                     (dict(state_in=Z(1, 64, 16)), r"must be \[rows, 64, 32\]"), (dict(state_in=Z(0, 64, 32)), "have 0 rows"),
                     (dict(q=Z(3, 32, 2).transpose(1, 2)), "contiguous rows")):
        with pytest.raises(ValueError, match=what):
            C.cortex_delta_forward(**{**good, **kw})


def test_binding_refuses_norm():
    good = dict(q=Z(3, 4, 32), q_out=Z(3, 4, 32), status=STATUS)
    for kw, what in ((dict(), "in device memory"), (dict(q=Z(3, 128)), "q must be a"), (dict(q_out=Z(3, 4, 16)), "q_out must be"),
                     (dict(k=Z(3, 2, 16), k_out=Z(3, 2, 16)), "k must be"), (dict(k=Z(3, 2, 32)), "k_out must be a"),
                     (dict(k_out=Z(3, 2, 32)), "k is required"), (dict(positions=Z(3, dtype=I32)), "freqs is required"),
                     (dict(freqs=Z(8)), "positions is required"), (dict(freqs=Z(8), positions=Z(2, dtype=I32)), "positions holds 2"),
                     (dict(freqs=Z(8), positions=Z(3)), "positions must be torch.int32"), (dict(q_weight=Z(31)), "q_weight holds 31"),
                     (dict(freqs=[1.0], positions=Z(3, dtype=I32)), "freqs must be a torch.Tensor"), (dict(norm="rms"), "norm must be one of"),
                     (dict(status=None), "status is required")):
        with pytest.raises(ValueError, match=what):
            C.cortex_qk_norm(**{**good, **kw})


def test_binding_refuses_linear():
    good = dict(x=Z(3, 40), w=Z(8, 48, dtype=I8)[:, :40], w_scale=Z(8), y=Z(3, 8), status=STATUS, ws=WS)
    for kw, what in ((dict(), "in device memory"), (dict(x=Z(3, 48)), "x must be"), (dict(x=Z(3, 40, dtype=I8)), "x must be torch.float32"),
                     (dict(x_scale=Z(3)), "x must be torch.int8"), (dict(w=Z(8, 40, dtype=I8)), "16-byte boundaries"),
                     (dict(w=Z(8, 40)), "w must be torch.int8"), (dict(w=Z(8 * 48 + 8, dtype=I8)[8:].view(8, 48)[:, :40]), "16-byte boundaries"),
                     (dict(w=Z(7 * 48 + 40, dtype=I8).as_strided((8, 40), (48, 1))), "its last row too"),
                     (dict(w_scale=Z(7)), "w_scale holds 7"), (dict(bias=Z(7)), "bias holds 7"), (dict(y=Z(3, 9)), "w must be"),
                     (dict(ws=None), "ws is required")):
        with pytest.raises(ValueError, match=what):
            C.cortex_linear_i8(**{**good, **kw})
    for kw, what in ((dict(), "in device memory"), (dict(q=Z(3, 40)), "q must be torch.int8"), (dict(scale=Z(2)), "scale holds 2"),
                     (dict(q=Z(3, 41, dtype=I8)), "q must be")):
        with pytest.raises(ValueError, match=what):
            C.cortex_quant_i8(**{**dict(x=Z(3, 40), q=Z(3, 40, dtype=I8), scale=Z(3), status=STATUS), **kw})


@pytest.mark.parametrize("T,S,H,K,V", [(0, 1, 1, 128, 128), (0, 9, 8, 128, 128), (1, 2, 1, 32, 16), (7, 8, 8, 128, 128), (30, 40, 4, 64, 64),
                                       (3, 10, 6, 128, 128), (1, 15, 10, 64, 32), (63, 64, 1, 32, 16), (64, 64, 1, 32, 16), (1, 1, 1, 128, 128)])
def test_delta_takes_short_prompts_whole(lib, T, S, H, K, V):
    """Two launches, also where sequences have less than a token each."""
    assert lib.cortex_delta_segment_tokens(T, S, H, K, V) == 0


@pytest.mark.parametrize("T,S,H,K,V", [(24576, 1, 1, 128, 128), (8192, 1, 2, 128, 128), (8192, 1, 8, 128, 128), (2048, 1, 4, 64, 64)])
def test_delta_cuts_long_prompts_of_few_columns(lib, T, S, H, K, V):
    Q = lib.cortex_delta_segment_tokens(T, S, H, K, V)
    assert 0 < Q < T and Q % 64 == 0


@pytest.mark.parametrize("size", [(-1, 1, 4, 64, 32), (9999, 0, 4, 64, 32), (9999, 1, 0, 64, 32), (9999, 1, 4, 100, 32), (9999, 1, 4, 64, 20),
                                  (1 << 20, 128, 64, 64, 64)])
def test_delta_cuts_nothing_of_sizes_that_it_refuses_or_of_many_columns(lib, size):
    assert lib.cortex_delta_segment_tokens(*size) == 0


def test_delta_limits_of_the_header(lib):
    """Sequences times heads times V / 16 and the strides, on either side: what is admitted asks for its workspace."""
    size = dict(heads=2, key_heads=1, key_dim=32, q_ld=32, k_ld=32, b_ld=2, dt_ld=2)
    for V, S in ((256, 1 << 20), (128, 1 << 21)):
        for n, want in ((S - 1, C.CORTEX_E_WORKSPACE), (S, C.CORTEX_E_INVAL)):
            a = delta_args(value_dim=V, v_ld=2 * V, y_ld=2 * V, num_seqs=n, num_tokens=n, state_rows=n, **size)
            assert lib.cortex_delta_forward(ctypes.byref(a), P8, P8, 1 << 20, None) == want
        assert lib.cortex_delta_step(ctypes.byref(a), P8, None) == C.CORTEX_E_INVAL
    for name in ("q_ld", "k_ld", "v_ld", "y_ld", "b_ld", "dt_ld"):
        for ld, want in ((1 << 25, C.CORTEX_E_WORKSPACE), ((1 << 25) + 1, C.CORTEX_E_INVAL)):
            assert lib.cortex_delta_forward(ctypes.byref(delta_args(**{name: ld})), P8, P8, 0, None) == want


@pytest.mark.parametrize("bad", [dict(heads=65537, q_ld=65537 * 64, q_out_ld=65537 * 64), dict(key_heads=65537, k_ld=65537 * 64, k_out_ld=65537 * 64),
                                 dict(num_tokens=(1 << 25) // 8, key_heads=4, k_ld=256, k_out_ld=256),
                                 dict(num_tokens=512, heads=32768, key_heads=32768, q_ld=1 << 21, k_ld=1 << 21, q_out_ld=1 << 21, k_out_ld=1 << 21)])
def test_norm_limits_of_the_header(lib, bad):
    assert lib.cortex_qk_norm(ctypes.byref(norm_args(**bad)), P8, None) == C.CORTEX_E_INVAL
