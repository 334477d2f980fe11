"""The scan at the ends of its types' ranges and of its arguments'."""
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
