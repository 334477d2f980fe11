"""When the scan splits prompts over their length: the workspace tells (CPU), and the results do not (GPU)."""
import numpy as np
import pytest
import torch

from paper_2011_01383_amd import cortex as C
from tests import test_scan_precision as precision
from tests.gpu_helpers import announce, need_gpu
from tests.sequence_helpers import Scan, host

WHOLE_SEQUENCES = 256          # bytes of workspace of a call that does not split


@pytest.mark.parametrize("T,S,D,N,P", [
    (5000, 1, 12800, 128, 32),              # 400 heads: the GPU holds one segment of each
    (100000, 1, 385 * 16, 128, 16),         # 385
    (300, 1, 399 * 64, 64, 64),
    (96, 1, 2048, 128, 64), (160, 1, 64, 64, 64), (128, 64, 256, 64, 64),
    (32, 1, 512, 16, 0), (36, 4, 64, 64, 0)])
def test_one_launch(T, S, D, N, P):
    """A prompt that one segment would hold is not split, nor is one that ends sooner than three launches."""
    assert C.cortex_scan_workspace_bytes(T, S, D, N, P) == WHOLE_SEQUENCES


@pytest.mark.parametrize("T,S,D,N,P", [
    (32768, 1, 4096, 128, 64), (4099, 5, 1024, 64, 64), (8192, 8, 2048, 128, 64), (8192, 16, 2048, 16, 0), (257, 1, 512, 16, 0)])
def test_segments(T, S, D, N, P):
    assert C.cortex_scan_workspace_bytes(T, S, D, N, P) > 2 * D * N * 4


@pytest.mark.gpu
@pytest.mark.parametrize("T,S,whole", [(8192, 15, True), (8192, 16, True), (8192, 12, False), (8192, 1, False), (224, 1, True),
                                       (225, 1, False)])
def test_one_launch_needs_no_workspace(T, S, whole):
    """32 heads of 64: a call that does not split takes 256 bytes, one that does refuses them."""
    need_gpu()
    D, N, H = 2048, 128, 32
    announce("%d tokens of %d prompts in 256 bytes" % (T, S))
    z = lambda *s: torch.zeros(*s, dtype=torch.bfloat16, device="cuda")
    off = torch.tensor([T * i // S for i in range(S + 1)], dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    rc = C.cortex_scan_forward(z(T, D), z(T, H), torch.zeros(H, device="cuda"), z(T, 1, N), z(T, 1, N), off, z(T, D),
                               status=status, ws=C.workspace(WHOLE_SEQUENCES))
    torch.cuda.synchronize()
    assert rc == (C.CORTEX_OK if whole else C.CORTEX_E_WORKSPACE) and int(status.item()) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,D,N,P", [(193, 64, 16, 64), (163, 64, 64, 64), (162, 64, 64, 64), (700, 3200, 128, 16),
                                     (36, 70, 16, 0), (37, 70, 16, 0)])
def test_either_side_of_the_rule(T, D, N, P, dtype):
    need_gpu()
    announce("%d tokens of %d channels N %d P %d %s" % (T, D, N, P, dtype))
    p = Scan(5, [T], D, N, 1, P, dtype=dtype)
    d = p.upload()
    out = torch.full_like(d["state"], 7.0)
    C.check(p.call(state_out=out))
    torch.cuda.synchronize()
    assert int(d["status"].item()) == 0
    p.check(d["y"], out, "%d tokens" % T)


@pytest.mark.gpu
@pytest.mark.parametrize("N", [16, 32, 64, 128])
@pytest.mark.parametrize("make", [precision.close_states, precision.close_scores])
def test_segments_keep_all_bits(make, N):
    """The small differences of large terms, over segments of a longer prompt."""
    need_gpu()
    announce("%s N %d in segments" % (make.__name__, N))
    p = make(N, 4, 32, T=384)
    assert C.cortex_scan_workspace_bytes(384, 1, 128, N, 32) > WHOLE_SEQUENCES
    d = p.upload()
    C.check(p.call())
    torch.cuda.synchronize()
    assert int(d["status"].item()) == 0
    ref, mag, _ = p.reference()
    worst = np.abs(host(d["y"]) - ref) / precision.bound(p, ref, mag)
    assert worst.max() <= 1, (float(worst.max()), np.argwhere(worst > 1)[0])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("P", [0, 32])
def test_segments_with_decays_that_leave_the_float_range(P, dtype):
    need_gpu()
    for A, size in ((-3.4028234663852886e38, 0.05), (-1e30, 1e10)):
        announce("A %g steps of %g %s P %d in segments" % (A, size, dtype, P))
        p = Scan(1, [300, 0, 9, 111], 64, 16, 1, P, dtype=dtype, z=False, skip=False, bias=False, soft=False)
        p.A[:] = A
        taken = np.random.default_rng(2).random(p.dt.shape) < 0.02
        p.dt = torch.from_numpy(np.where(taken, size, 0.0)).to(p.dtype).double().numpy()
        assert C.cortex_scan_workspace_bytes(p.T, p.S, 64, 16, P) > WHOLE_SEQUENCES
        d = p.upload()
        out = torch.full_like(d["state"], 7.0)
        C.check(p.call(state_out=out))
        torch.cuda.synchronize()
        assert int(d["status"].item()) == 0
        p.check(d["y"], out, "A %g" % A)
