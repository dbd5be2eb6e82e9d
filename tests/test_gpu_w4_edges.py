"""Products with 4-bit weights where they can go wrong: waits that run out, features of very different sizes in one request."""
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


# ---------------------------------------------------------------- what is held of a feature

@pytest.mark.parametrize("B", [1, 12, 30, 64])
@pytest.mark.parametrize("x,held", [(BF16, 2.0 ** -40), (F32, 2.0 ** -35)])
@pytest.mark.parametrize("lead", [1.0, 1.9921875, 2.0 ** -100, 1e35])
def test_small_features_beside_large_ones(lead, x, held, B):
    """A request's largest feature meets weights of 0: what is left are features from 2^-1 to 2^-38 of it, one to a group
    of 32 inputs, each held to `held` of the largest. The rest is rounding: a code's products with a feature's terms are exact, three
    of them, a scale of 1 and what takes the power of two back leave the sum of one feature with two roundings at most,
    2^-23 of it; 38 features' groups are added one after another, 2 38 2^-24 of the sum of magnitudes."""
    n, G = 38, 32
    K = (n + 1) * G
    g = torch.Generator().manual_seed(B)
    wide = torch.zeros(B, K, dtype=torch.float64)
    wide[:, 0] = lead
    wide[:, G * torch.arange(1, n + 1)] = (torch.rand(B, n, generator=g, dtype=torch.float64) + 1) / 2 * lead * \
        2.0 ** -torch.arange(1, n + 1, dtype=torch.float64)
    feats = wide.to(x)
    # outputs of one feature each, and of those from one size on
    codes = torch.full((2 * n, K), 8, dtype=torch.uint8)
    for v in range(n):
        codes[v, G * (v + 1)] = 8 + 1 + v % 7
        codes[n + v, G * torch.arange(v + 1, n + 1)] = 8 - 1 - v % 8
    w = dels.pack_w4(codes.to(DEV), torch.ones(2 * n, n + 1, dtype=BF16, device=DEV), group=G)
    got = w.project(feats.to(DEV)).cpu().double()
    wt = codes.double() - 8
    want, size = feats.double() @ wt.T, feats.double().abs() @ wt.abs().T
    tol = held * feats.double().abs().amax(-1, keepdim=True) * wt.abs().sum(-1)
    tol[:, :n] += 2.0 ** -23 * size[:, :n]
    tol[:, n:] += 2 * n * 2.0 ** -24 * size[:, n:]
    err = (got - want).abs()
    assert w.status() == 0 and (err <= tol + 2.0 ** -149).all(), (err / tol).max()
