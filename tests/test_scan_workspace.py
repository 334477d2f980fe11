"""One workspace of the scan, sized for the largest batch, serves every smaller one."""
import random

import pytest
import torch

from paper_2011_01383_amd import cortex as C
from tests.gpu_helpers import announce, need_gpu
from tests.sequence_helpers import Scan


@pytest.mark.parametrize("D,N,P", [(2048, 16, 0), (64, 64, 0), (70000, 8, 0), (1, 8, 0), (2048, 128, 64), (64, 16, 64), (12768, 128, 32),
                                   (512, 64, 256)])
def test_bytes_rise_with_tokens_and_sequences(D, N, P):
    r = random.Random(D)
    tokens = sorted({int(2 ** r.uniform(0, 24)) for _ in range(300)} | set(range(0, 2000, 7)))
    for S in (0, 1, 2, 5, 6, 7, 15, 16, 31, 32, 100, 1023, 1024, 5000):
        sizes = [C.cortex_scan_workspace_bytes(T, S, D, N, P) for T in tokens]
        assert sizes == sorted(sizes) and sizes[0] >= 256, S
    for T in tokens[::5]:
        sizes = [C.cortex_scan_workspace_bytes(T, S, D, N, P) for S in range(0, 1100, 3)]
        assert sizes == sorted(sizes), T


@pytest.mark.gpu
@pytest.mark.parametrize("D,N,P", [(130, 16, 0), (128, 32, 64)])
def test_one_workspace_for_batches_of_different_sizes(D, N, P):
    need_gpu()
    ws = C.workspace(C.cortex_scan_workspace_bytes(6000, 600, D, N, P))
    r = random.Random(1)
    for k, (T, S) in enumerate([(6000, 600), (6000, 1), (3000, 3), (700, 40), (40, 1), (33, 600), (5999, 12), (1200, 255), (2100, 2)]):
        announce("workspace of 6,000 tokens and 600 sequences, %d and %d, D %d" % (T, S, D))
        cuts = sorted(r.randint(0, T) for _ in range(S - 1))
        p = Scan(k, [b - a for a, b in zip([0] + cuts, cuts + [T])], D, N, 1, P, dtype="f32", z=False)
        d = p.upload()
        d["ws"] = ws
        out = torch.full_like(d["state"], 7.0)
        C.check(p.call(state_out=out))
        torch.cuda.synchronize()
        assert int(d["status"].item()) == 0
        p.check(d["y"], out, "%d tokens of %d sequences" % (T, S))
