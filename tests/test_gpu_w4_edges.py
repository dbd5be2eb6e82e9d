"""Products with 4-bit weights where they can go wrong: waits that run out, features of very different sizes in one
request; how exact they are."""
import math

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


# ---------------------------------------------------------------- how exact products are

@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("x", [BF16, F32])
@pytest.mark.parametrize("B,V,K,G", [(1, 4000, 256, 32), (8, 3000, 1024, 64), (12, 3000, 2560, 128), (30, 1000, 600, 32),
                                     (64, 1000, 1280, 64)])
def test_products_norm(B, V, K, G, x, zeros):
    """||y - W x|| / ||W x|| of float32 outputs. Of n groups one after another each addition is off by 0.3 steps of 2^-23 (rms)
    of the sum so far, which grows with its root: 0.3 2^-23 sqrt(n / 2). A group's own sum is cut, not rounded, after each 16
    inputs, by half a step of 2^-24 to 2^-23 on average, of what is two thirds of it on average, always towards 0, as the
    group's and so the whole's: 2^-25 G / 16. (Codes without an exponent were off by 8e-7.)"""
    g = torch.Generator().manual_seed(K + B)
    n = -(-K // G)
    codes = torch.randint(0, 16, (V, K), generator=g, dtype=torch.uint8)
    scales = (torch.rand(V, n, generator=g) * 0.02 + 1e-3).to(BF16)
    zero = torch.randint(6, 10, (V, n), generator=g, dtype=torch.uint8) if zeros else None
    feats = torch.randn(B, K, generator=g).to(x)
    of = torch.arange(K) // G
    wt = (codes.double() - (8.0 if zero is None else zero.double()[:, of])) * scales.double()[:, of]
    want = feats.double() @ wt.T
    w = dels.pack_w4(codes.to(DEV), scales.to(DEV), None if zero is None else zero.to(DEV), group=G)
    got = w.project(feats.to(DEV)).cpu().double()
    tol = 0.3 * 2.0 ** -23 * math.sqrt(n / 2) + 2.0 ** -25 * G / 16
    assert (got - want).norm() <= tol * want.norm(), ((got - want).norm() / want.norm(), tol)
