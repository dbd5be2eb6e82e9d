"""Products with 4-bit weights where they can go wrong: waits that run out."""
import pytest
import torch

import paper_2607_07409_gb300 as dels

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16


# ---------------------------------------------------------------- waits that run out

@pytest.mark.parametrize("stall", [1, 2])
@pytest.mark.parametrize("form", [0, 1, 2, 3])
@pytest.mark.parametrize("B,V,K", [(1, 256, 1024), (2, 128, 32), (8, 80000, 256), (12, 4096, 700), (24, 3000, 512),
                                   (64, 256, 1024), (64, 40000, 256), (100, 512, 4096)])
def test_a_wait_that_runs_out_is_reported(B, V, K, form, stall):
    """Blocks that never come, products whose end is never reported: the kernel returns all the same, says so, and the
    context goes on."""
    nbytes = dels.dels_selftest_w4_timeout_bytes(B, V, K)
    ws = torch.zeros(nbytes, dtype=torch.uint8, device=DEV)
    assert dels.dels_selftest_w4_timeout(form, stall, B, V, K, ws, nbytes) == 0
    assert dels.dels_read_status(ws) == dels.DELS_STATUS_TIMEOUT
    codes = torch.full((300, 64), 9, dtype=torch.uint8, device=DEV)
    w = dels.pack_w4(codes, torch.ones(300, 2, dtype=BF16, device=DEV), group=32)
    x = torch.ones(B, 64, dtype=F32 if form == 1 else BF16, device=DEV)
    assert (w.project(x) == 64).all() and w.status() == 0
