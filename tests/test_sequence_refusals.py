"""More refusals of the sequence operators that need no GPU."""
import ctypes
import os

import pytest
import torch

from paper_2011_01383_amd import cortex as C
from tests.test_sequence_abi import P8, logits_args, scan_args


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(C.LIB_PATH):
        from paper_2011_01383_amd import build
        build.build()
    return C.load()


@pytest.mark.parametrize("off", [1, 2, 4, 8])
def test_workspaces_start_at_16_bytes(lib, off):
    """The scan stores 16 bytes at once, the logits count arrivals with atomics."""
    assert lib.cortex_scan_forward(ctypes.byref(scan_args()), P8, P8 + off, 1 << 40, None) == C.CORTEX_E_INVAL
    assert lib.cortex_logits_process(ctypes.byref(logits_args()), P8, P8 + off, 1 << 40, None) == C.CORTEX_E_INVAL


@pytest.mark.parametrize("S,P", [(1 << 25, 64), (1 << 23, 64), (1 << 22, 256), (3 << 28, 16)])
def test_prompts_of_more_heads_than_a_grid_holds(lib, S, P):
    """Their number was cut to 32 bits: 2^32 and more of them ran too few workgroups, or none."""
    D = 2 * P if P < 256 else P
    a = scan_args(num_seqs=S, num_tokens=64, channels=D, head_dim=P, groups=1, state_rows=S, x_ld=D, y_ld=D, dt_ld=D // P)
    assert lib.cortex_scan_forward(ctypes.byref(a), P8, P8, 1 << 50, None) == C.CORTEX_E_INVAL


def test_binding_refuses_biases_that_are_no_tensors():
    z, i32 = torch.zeros, torch.int32
    for kw, what in ((dict(bias_tokens=[1]), "bias_tokens must be a torch.Tensor, got list"),
                     (dict(bias_tokens=z(1, dtype=i32), bias_values=[1.0]), "bias_values must be a torch.Tensor"),
                     (dict(bias_tokens=None, bias_values=z(1)), "bias_tokens is required"),
                     (dict(bias_offsets=[0, 0, 0], bias_tokens=z(1, dtype=i32), bias_values=z(1)), "bias_offsets must be a torch.Tensor")):
        with pytest.raises(ValueError, match=what):
            C.cortex_logits_process(z(2, 100), **{**dict(token=z(2, dtype=i32), status=z(1, dtype=i32), ws=z(256, dtype=torch.uint8),
                                                         bias_offsets=z(3, dtype=i32)), **kw})
