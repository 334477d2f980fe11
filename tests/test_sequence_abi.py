"""Refusals of the sequence operators that need no GPU: the library's host checks
and the binding's."""
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


def conv_args(**kw):
    a = dict(dtype=0, num_seqs=2, num_tokens=2, channels=8, width=4, silu=1, state_rows=2, seq_offsets=P8, state_index=None,
             x=P8, x_ld=8, weight=P8, bias=None, state_in=P8, state_out=P8, y=P8, y_ld=8)
    a.update(kw)
    return C.cortex_conv_t(**a)


@pytest.mark.parametrize("bad", [
    dict(dtype=2), dict(num_seqs=-1), dict(num_tokens=-1), dict(channels=0), dict(width=1), dict(width=5), dict(state_rows=1),
    dict(state_rows=-1), dict(x=None), dict(y=None), dict(weight=None), dict(x_ld=7), dict(y_ld=7),
    dict(num_seqs=0), dict(num_tokens=2 ** 31 - 1)])
def test_conv_refuses(lib, bad):
    for call in (lib.cortex_conv_forward, lib.cortex_conv_step):
        assert call(ctypes.byref(conv_args(**bad)), P8, None) == C.CORTEX_E_INVAL


def test_conv_refuses_by_form(lib):
    assert lib.cortex_conv_forward(ctypes.byref(conv_args(seq_offsets=None)), P8, None) == C.CORTEX_E_INVAL
    assert lib.cortex_conv_step(ctypes.byref(conv_args(num_tokens=3)), P8, None) == C.CORTEX_E_INVAL
    assert lib.cortex_conv_forward(None, P8, None) == C.CORTEX_E_INVAL
    assert lib.cortex_conv_forward(ctypes.byref(conv_args()), None, None) == C.CORTEX_E_INVAL


def scan_args(**kw):
    a = dict(dtype=1, num_seqs=2, num_tokens=2, channels=128, head_dim=64, groups=2, state_size=64, softplus=1, state_rows=2,
             seq_offsets=P8, state_index=None, x=P8, z=None, dt=P8, B=P8, C=P8, x_ld=128, z_ld=0, dt_ld=2, B_ld=128, C_ld=128,
             A=P8, skip=None, dt_bias=None, state_in=P8, state_out=P8, y=P8, y_ld=128)
    a.update(kw)
    return C.cortex_scan_t(**a)


@pytest.mark.parametrize("bad", [
    dict(dtype=3), dict(num_seqs=-1), dict(channels=0), dict(groups=0), dict(groups=3), dict(head_dim=-16), dict(head_dim=24),
    dict(head_dim=272, channels=544, x_ld=544, y_ld=544), dict(head_dim=128), dict(state_size=8), dict(state_size=256),
    dict(state_size=48), dict(head_dim=0, state_size=128, dt_ld=128, B_ld=256, C_ld=256), dict(state_rows=1), dict(x=None),
    dict(dt=None), dict(B=None), dict(C=None), dict(A=None), dict(y=None), dict(x_ld=127), dict(dt_ld=1), dict(B_ld=127),
    dict(C_ld=127), dict(y_ld=127), dict(z=P8, z_ld=127), dict(state_in=P8 + 4), dict(state_out=P8 + 8), dict(num_seqs=0)])
def test_scan_refuses(lib, bad):
    args = ctypes.byref(scan_args(**bad))
    assert lib.cortex_scan_forward(args, P8, P8, 1 << 40, None) == C.CORTEX_E_INVAL
    assert lib.cortex_scan_step(args, P8, None) == C.CORTEX_E_INVAL


def test_scan_refuses_by_form(lib):
    assert lib.cortex_scan_forward(ctypes.byref(scan_args(seq_offsets=None)), P8, P8, 1 << 40, None) == C.CORTEX_E_INVAL
    assert lib.cortex_scan_forward(ctypes.byref(scan_args()), P8, None, 1 << 40, None) == C.CORTEX_E_INVAL
    need = C.cortex_scan_workspace_bytes(2, 2, 128, 64, 64)
    assert need > 0
    assert lib.cortex_scan_forward(ctypes.byref(scan_args()), P8, P8, need - 1, None) == C.CORTEX_E_WORKSPACE
    assert lib.cortex_scan_step(ctypes.byref(scan_args(num_tokens=1)), P8, None) == C.CORTEX_E_INVAL
    for bad in ((-1, 1, 128, 64, 64), (1, -1, 128, 64, 64), (1, 1, 0, 64, 64), (1, 1, 128, 5, 0), (1, 1, 128, 64, 24)):
        assert C.cortex_scan_workspace_bytes(*bad) == 0


def logits_args(**kw):
    a = dict(dtype=0, rows=2, vocab=100, history_cap=10, num_biases=1, mask_rows=2, logits=P8, logits_ld=100, history=P8,
             history_ld=10, history_len=P8, prompt_len=None, repetition=P8, frequency=None, presence=None, bias_offsets=P8,
             bias_tokens=P8, bias_values=P8, mask=P8, mask_ld=4, mask_index=None, out=P8, out_ld=100, token=P8, lse=P8)
    a.update(kw)
    return C.cortex_logits_t(**a)


@pytest.mark.parametrize("bad", [
    dict(dtype=7), dict(rows=-1), dict(rows=65536), dict(vocab=0), dict(logits=None), dict(logits_ld=99), dict(out_ld=99),
    dict(history_len=None), dict(history_cap=-1), dict(history_ld=9), dict(history=None), dict(num_biases=-1),
    dict(bias_tokens=None), dict(bias_values=None), dict(mask_ld=3), dict(mask_rows=1), dict(out=None, token=None, lse=None)])
def test_logits_refuses(lib, bad):
    args = ctypes.byref(logits_args(**bad))
    assert lib.cortex_logits_process(args, P8, P8, 1 << 40, None) == C.CORTEX_E_INVAL


def test_logits_refuses_a_small_workspace(lib):
    need = C.cortex_logits_workspace_bytes(2, 100)
    args = ctypes.byref(logits_args())
    assert lib.cortex_logits_process(args, P8, P8, need - 1, None) == C.CORTEX_E_WORKSPACE
    assert lib.cortex_logits_process(args, P8, None, need, None) == C.CORTEX_E_INVAL
    assert lib.cortex_logits_process(args, None, P8, need, None) == C.CORTEX_E_INVAL
    assert C.cortex_logits_workspace_bytes(-1, 100) == 0 and C.cortex_logits_workspace_bytes(1, 0) == 0


def z(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype)


def test_binding_refuses_conv():
    x, w, off = z(3, 8), z(8, 4), z(2, dtype=torch.int32)
    call = lambda **kw: C.cortex_conv_forward(**{**dict(x=x, weight=w, offsets=off, y=z(3, 8), status=z(1, dtype=torch.int32)), **kw})
    for kw, what in ((dict(x=z(3, 8, dtype=torch.float16)), "x must be torch.float32 or torch.bfloat16"),
                     (dict(x=z(24)), "x must be a 2-dimensional"), (dict(weight=z(7, 4)), "weight must be"),
                     (dict(weight=z(8, 4, dtype=torch.bfloat16)), "weight must be torch.float32"),
                     (dict(offsets=off.long()), "offsets must be torch.int32"), (dict(offsets=None), "offsets must be"),
                     (dict(state_in=z(1, 2, 8)), "state_in and state_out must be"),
                     (dict(state_in=z(0, 3, 8)), "the states have 0 rows"),
                     (dict(bias=z(7)), "bias holds 7"), (dict(status=None), "status is required"),
                     (dict(), "must be in device memory")):
        with pytest.raises(ValueError, match=what):
            call(**kw)


def test_binding_refuses_scan():
    i32 = torch.int32
    base = dict(x=z(3, 64), dt=z(3, 64), A=z(64, 16), B=z(3, 1, 16), C=z(3, 1, 16), offsets=z(2, dtype=i32), y=z(3, 64),
                status=z(1, dtype=i32), ws=z(256, dtype=torch.uint8))
    for kw, what in ((dict(A=z(63, 16)), "A must be"), (dict(A=z(64, 8)), "A must be"), (dict(A=z(5)), "A must hold a divisor"),
                     (dict(B=z(2, 1, 16)), "B must have 3 rows"), (dict(B=z(3, 16)), r"B must be a \[T, G, N\]"),
                     (dict(C=z(3, 1, 32)), "B and C must have"), (dict(B=z(3, 1, 16, dtype=torch.bfloat16)), "B must be"),
                     (dict(state_in=z(1, 64, 8)), "state_in and state_out"), (dict(ws=None), "ws is required"),
                     (dict(D=z(3)), "D holds 3"), (dict(), "must be in device memory")):
        with pytest.raises(ValueError, match=what):
            C.cortex_scan_forward(**{**base, **kw})


def test_binding_refuses_logits():
    i32 = torch.int32
    base = dict(logits=z(2, 100), token=z(2, dtype=i32), status=z(1, dtype=i32), ws=z(256, dtype=torch.uint8))
    for kw, what in ((dict(token=None), "out, token or lse"), (dict(token=z(2)), "token must be torch.int32"),
                     (dict(repetition=z(2)), "history is required"), (dict(bias_tokens=z(1, dtype=i32)), "bias_offsets is required"),
                     (dict(mask_index=z(2, dtype=i32)), "mask is required"), (dict(logits=z(100)), "2-dimensional"),
                     (dict(mask=z(1, 4, dtype=i32)), "mask has 1 rows, 2 rows"),
                     (dict(mask=z(2, 4, dtype=i32)), "must be in device memory"), (dict(), "must be in device memory")):
        with pytest.raises(ValueError, match=what):
            C.cortex_logits_process(**{**base, **kw})
