"""The logits' mask turned off by its pointer alone, through the C ABI (the binding asks for a mask
with its indices)."""
import ctypes

import pytest
import torch

from paper_2011_01383_amd import cortex as C
from tests.gpu_helpers import announce, need_gpu


@pytest.mark.gpu
@pytest.mark.parametrize("mask_rows", [0, 3])
@pytest.mark.parametrize("V", [5000, 70000])
def test_indices_without_a_mask_are_not_read(V, mask_rows):
    need_gpu()
    announce("logits V %d, no mask, indices, %d rows" % (V, mask_rows))
    R = 4
    g = torch.Generator(device="cuda").manual_seed(1)
    logits = torch.randn(R, V, generator=g, device="cuda")
    ints = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")
    ws = C.workspace(C.cortex_logits_workspace_bytes(R, V))

    def call(mask_index, rows):
        out, token, lse, status = torch.zeros_like(logits), ints(*[7] * R), torch.zeros(R, device="cuda"), ints(0)
        a = C.cortex_logits_t(dtype=C.CORTEX_F32, rows=R, vocab=V, mask_rows=rows, logits=logits.data_ptr(), logits_ld=V,
                              mask_index=None if mask_index is None else mask_index.data_ptr(), out=out.data_ptr(), out_ld=V,
                              token=token.data_ptr(), lse=lse.data_ptr())
        C.check(C.load().cortex_logits_process(ctypes.byref(a), status.data_ptr(), ws.data_ptr(), ws.numel(), None))
        torch.cuda.synchronize()
        return out, token, lse, status

    plain, got = call(None, 0), call(ints(-1, 0, 2, 1), mask_rows)
    assert int(got[3].item()) == 0
    assert all(torch.equal(a, b) for a, b in zip(plain, got))
    assert torch.equal(got[0], logits) and torch.equal(got[1].long(), logits.argmax(1))
