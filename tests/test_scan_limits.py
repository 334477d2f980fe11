"""The scan at the ends of its types' ranges and of its arguments'."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2011_01383_amd import cortex as C
from tests.gpu_helpers import announce, need_gpu
from tests.sequence_helpers import Scan, host

LOWEST = -3.4028234663852886e38


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("P", [0, 32])
@pytest.mark.parametrize("A,size", [(LOWEST, 0.05), (LOWEST, 8.0), (-1e30, 1e10), (-1e30, 1e-30)])
def test_decays_that_leave_the_float_range(A, size, P, dtype):
    """A step forgets the state at once, a step of 0 keeps it: prompts of whole and broken sub-chunks, and tokens."""
    need_gpu()
    for lens, step in (([70, 3, 0, 96], False), ([1] * 6, True), ([5] * 1100, False)):
        announce("A %g steps of %g %s P %d, %d sequences" % (A, size, dtype, P, len(lens)))
        p = Scan(1, lens, 64, 16, 1, P, dtype=dtype, z=False, skip=False, bias=False, soft=False)
        p.A[:] = A
        taken = np.random.default_rng(2).random(p.dt.shape) < 0.3
        p.dt = torch.from_numpy(np.where(taken, size, 0.0)).to(p.dtype).double().numpy()
        d = p.upload()
        out = torch.full_like(d["state"], 7.0)
        C.check(p.call(step, state_out=out))
        torch.cuda.synchronize()
        assert int(d["status"].item()) == 0
        p.check(d["y"], out, "A %g" % A)


@pytest.mark.gpu
@pytest.mark.parametrize("z_ld", [-1, 0, 1 << 40])
def test_no_gate_has_no_stride(z_ld):
    """z NULL: its stride is not looked at."""
    need_gpu()
    announce("no gate, z_ld %d" % z_ld)
    p = Scan(3, [1, 1, 1], 64, 16, 1, 32, dtype="f32", z=False)
    d = p.upload()
    for step in (False, True):
        C.check(p.call(step))
        torch.cuda.synchronize()
        want = d["y"].clone()
        d["y"].fill_(float("nan"))
        at = lambda t: None if t is None else t.data_ptr()
        a = C.cortex_scan_t(dtype=C.CORTEX_F32, num_seqs=3, num_tokens=3, channels=64, head_dim=32, groups=1, state_size=16,
                            softplus=1, state_rows=3, seq_offsets=at(d["offsets"]), x=at(d["x"]), dt=at(d["dt"]), B=at(d["B"]),
                            C=at(d["C"]), x_ld=d["x"].stride(0), z_ld=z_ld, dt_ld=d["dt"].stride(0), B_ld=d["B"].stride(0),
                            C_ld=d["C"].stride(0), A=at(d["A"]), skip=at(d["skip"]), dt_bias=at(d["dt_bias"]),
                            state_in=at(d["state"]), y=at(d["y"]), y_ld=d["y"].stride(0))
        lib, status = C.load(), at(d["status"])
        if step:
            C.check(lib.cortex_scan_step(ctypes.byref(a), status, None))
        else:
            C.check(lib.cortex_scan_forward(ctypes.byref(a), status, at(d["ws"]), d["ws"].numel(), None))
        torch.cuda.synchronize()
        assert int(d["status"].item()) == 0 and torch.equal(d["y"], want)
