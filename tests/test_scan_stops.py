"""A batch in which one sequence is broken: what the scan has written of the others when it stops is
their result, and the rest is as it was."""
import numpy as np
import pytest
import torch

from paper_2011_01383_amd import cortex as C
from tests.gpu_helpers import announce, need_gpu
from tests.sequence_helpers import Scan


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("P", [0, 32, 128])
@pytest.mark.parametrize("S", [5, 900])
def test_other_sequences_are_whole_or_left_alone(S, P, dtype):
    """S = 5 is split over the length, 900 are walked whole."""
    need_gpu()
    lens = (np.random.default_rng(0).integers(1, 40 if S > 5 else 400, S)).tolist()
    p = Scan(2, lens, 256, 32, 1, P, dtype=dtype, index=list(range(S)), rows=S)
    announce("one broken index of %d, %s P %d" % (S, dtype, P))
    d = p.upload()
    old = d["state"].clone()
    new = torch.zeros_like(old)
    C.check(p.call(state_out=new))
    torch.cuda.synchronize()
    y = d["y"].clone()
    for at in (0, S // 2, S - 1):
        d["index"].copy_(torch.arange(S, dtype=torch.int32))
        d["index"][at] = S
        d["state"].copy_(old)
        d["y"].fill_(float("nan"))
        d["status"].zero_()
        C.check(p.call(state_out=d["state"]))
        torch.cuda.synchronize()
        assert int(d["status"].item()) == C.CORTEX_ST_INPUT_RANGE
        assert bool(((d["state"] == old) | (d["state"] == new)).all())
        assert torch.equal(d["state"][at], old[at])
        assert bool(((d["y"] == y) | d["y"].isnan()).all())
