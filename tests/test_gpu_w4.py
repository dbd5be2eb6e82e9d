"""Products with 4-bit weights against float64.

Tolerance of an output: the products of a weight without its scale and a feature (a term of it) are exact in float32;
the tensor cores add 16 of them and the sum so far at a time, each off by at most 2^-24 of the
largest in truncating and rounding it, so 17 2^-24 of the sum of all magnitudes for each 16 inputs and term of a group;
the groups' sums take the scale's product and an addition each, and 8 more roundings may follow:
(17 terms G / 16 + groups + 10) 2^-24 sum_k |w_k x_k| in all; bf16 half a step, 2^-8. Features are held to 2^-40 of
their request's largest, m: 2^-40 m sum_k |w_k| more.
"""
import math

import pytest
import torch

import paper_2607_07409_gb300 as dels

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16
INF, NAN = math.inf, math.nan


class Case:
    def __init__(self, B, V, K, group, zeros, x=BF16, seed=0, scale=0.02):
        g = torch.Generator().manual_seed(seed + V * 3 + K + B)
        groups = -(-K // group)
        self.B, self.V, self.K, self.group = B, V, K, group
        self.codes = torch.randint(0, 16, (V, K), generator=g, dtype=torch.uint8)
        self.scales = (torch.rand(V, groups, generator=g) * scale + 1e-3).to(BF16)
        self.scales[::3] *= -1
        self.zeros = torch.randint(0, 16, (V, groups), generator=g, dtype=torch.uint8) if zeros else None
        self.x = torch.randn(B, K, generator=g).to(x)

    def pack(self):
        z = None if self.zeros is None else self.zeros.to(DEV)
        return dels.pack_w4(self.codes.to(DEV), self.scales.to(DEV), z, group=self.group)

    def weights(self):
        of = torch.arange(self.K) // self.group
        z = 8.0 if self.zeros is None else self.zeros.double()[:, of]
        return (self.codes.double() - z) * self.scales.double()[:, of]

    def want(self, out):
        w, x = self.weights(), self.x.double()
        y = x @ w.T
        terms = 3 if self.x.dtype is F32 else 1
        groups, G = -(-self.K // self.group), min(self.group, 32 * -(-self.K // 32))
        eps = (17 * terms * G / 16 + groups + 10) * 2.0 ** -24
        tol = eps * (x.abs() @ w.abs().T) + 2.0 ** -40 * x.abs().amax(-1, keepdim=True) * w.abs().sum(-1)
        return y, tol + (2.0 ** -8 * y.abs() if out is BF16 else 0.0) + 1e-37


def put(x, offset=0, pitch=None):
    rows, n = x.shape
    pitch = pitch or n
    buf = torch.full((offset + rows * pitch,), NAN, dtype=x.dtype, device=DEV)
    view = buf.as_strided((rows, n), (pitch, 1), offset)
    view.copy_(x)
    return view


def check(c, out=F32, w=None, offset=0, pitch=None):
    w = w or c.pack()
    got = w.project(put(c.x, offset, pitch), dtype=out)
    y, tol = c.want(out)
    err = (got.cpu().double() - y).abs()
    assert got.dtype is out and (err <= tol).all(), (err / tol).max()
    assert w.status() == 0


@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("B,V,K", [(1, 1, 1), (1, 1024, 128), (2, 31, 33), (3, 33, 127), (7, 100, 129), (8, 640, 160),
                                   (9, 1003, 1000), (1, 4099, 2560), (16, 2048, 256), (17, 999, 96), (33, 500, 320),
                                   (64, 3001, 256), (65, 70, 500), (130, 257, 192)])
def test_w4(B, V, K, group, zeros):
    c = Case(B, V, K, group, zeros)
    w = c.pack()
    check(c, F32, w)
    check(c, BF16, w)
    f = Case(B, V, K, group, zeros, x=F32)
    check(f, F32)


@pytest.mark.parametrize("B,V,K,group,zeros,x", [(1, 151936, 256, 64, False, BF16), (4, 50257, 1024, 128, True, BF16),
                                                 (64, 32003, 512, 32, True, F32), (5, 8000, 4096, 32, False, F32),
                                                 (64, 1500, 4096, 128, True, BF16), (1, 700, 65536, 64, True, BF16),
                                                 (3, 129, 20000, 32, True, F32), (64, 80000, 128, 32, True, BF16),
                                                 (40, 100000, 64, 64, False, BF16), (20, 79992, 96, 128, True, F32),
                                                 # tiles that several groups of warps share, one each and several
                                                 (2, 1264, 4096, 64, False, F32), (1, 50257, 4096, 32, True, BF16),
                                                 (10, 50257, 4096, 128, True, BF16), (16, 20000, 1100, 64, False, F32),
                                                 (20, 3000, 700, 32, True, F32), (64, 1500, 1024, 64, False, BF16),
                                                 (64, 45000, 1024, 128, True, BF16)])
def test_w4_larger(B, V, K, group, zeros, x):
    c = Case(B, V, K, group, zeros, x)
    check(c, F32)
    check(c, BF16)


def test_every_code_and_zero_point():
    """The weights themselves, one at a time: x is a row of the identity, its products exact."""
    V, K, G = 48, 96, 32
    codes = (torch.arange(V * K) % 16).view(V, K).to(torch.uint8)
    zeros = (torch.arange(V * 3) // 3 % 16).view(V, 3).to(torch.uint8)
    scales = (torch.arange(V * 3).view(V, 3) % 7 + 1).to(BF16)
    w = dels.pack_w4(codes.to(DEV), scales.to(DEV), zeros.to(DEV), group=G)
    of = torch.arange(K) // G
    want = (codes.float() - zeros.float()[:, of]) * scales.float()[:, of]
    for x in (BF16, F32):
        assert torch.equal(w.project(torch.eye(K, dtype=x, device=DEV)).cpu(), want.T)


@pytest.mark.parametrize("x,offset,pitch", [(BF16, 1, 0), (BF16, 0, 1), (BF16, 8, 8), (BF16, 3, 5), (F32, 1, 0),
                                            (F32, 0, 1), (F32, 4, 4), (F32, 3, 2)])
@pytest.mark.parametrize("K", [128, 333])
def test_features_anywhere(K, x, offset, pitch):
    check(Case(6, 777, K, 64, True, x), F32, offset=offset, pitch=K + pitch)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V,offset,pitch", [(1000, 0, 1003), (1001, 1, 1001), (96, 3, 103), (1024, 8, 1032)])
def test_outputs_anywhere(V, offset, pitch, dtype):
    """Rows of any alignment; what lies between them stays."""
    B = 11
    c = Case(B, V, 160, 32, False)
    big = torch.full((offset + B * pitch,), -7.0, dtype=dtype, device=DEV)
    out = big.as_strided((B, V), (pitch, 1), offset)
    got = c.pack().project(put(c.x), out=out)
    assert got is out
    y, tol = c.want(dtype)
    assert ((out.cpu().double() - y).abs() <= tol).all()
    big = big.cpu()
    assert (big[:offset] == -7).all()
    for b in range(B):
        assert (big[offset + b * pitch + V:offset + (b + 1) * pitch] == -7).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("B,V,pitch,offset", [(17, 8, 8, 0), (32, 1000, 1000, 0), (33, 1004, 1008, 8), (40, 129, 136, 0),
                                              (64, 4096, 4096, 16), (64, 4096, 4100, 0), (65, 1003, 1003, 1),
                                              (100, 260, 264, 0)])
def test_outputs_of_many_requests(B, V, pitch, offset, dtype):
    """Rows that start on 16 bytes and others; what lies between and behind them stays."""
    c = Case(B, V, 200, 32, True)
    big = torch.full((offset + (B + 1) * pitch,), -7.0, dtype=dtype, device=DEV)
    out = big.as_strided((B, V), (pitch, 1), offset)
    c.pack().project(put(c.x), out=out)
    y, tol = c.want(dtype)
    assert ((out.cpu().double() - y).abs() <= tol).all()
    out.fill_(-7)
    assert (big == -7).all()


def test_float32_features_to_their_last_bit():
    """Features of 24 significant bits, from the smallest to the largest, each alone against a weight of 1."""
    K = 64
    g = torch.Generator().manual_seed(1)
    m = torch.randint(1 << 23, 1 << 24, (K,), generator=g).double()
    e = torch.linspace(-120, 100, K).round()
    x = (m * 2.0 ** e).float()
    x[0], x[1] = torch.finfo(F32).max, -torch.finfo(F32).max
    codes = torch.full((40, K), 9, dtype=torch.uint8)
    w = dels.pack_w4(codes.to(DEV), torch.ones(40, 1, dtype=BF16, device=DEV), group=64)
    got = w.project(torch.diag(x).to(DEV)).cpu()
    assert torch.equal(got, x[:, None].expand(K, 40))


def test_non_finite_features_and_scales():
    """A request with an infinity or NaN has NaN throughout, the others their products; scales likewise by rows."""
    for x in (BF16, F32):
        c = Case(11, 100, 200, 32, False, x)
        c.x[1, 7], c.x[2, 190], c.x[9, 0] = INF, NAN, -INF
        got = c.pack().project(put(c.x)).cpu()
        bad = [1, 2, 9]
        assert torch.isnan(got[bad]).all()
        c.x[bad] = 0
        y, tol = c.want(F32)
        keep = [i for i in range(11) if i not in bad]
        assert ((got.double() - y).abs() <= tol)[keep].all()
    c.scales[5, 2], c.scales[6, 0] = NAN, INF
    got = c.pack().project(put(c.x)).cpu()
    assert torch.isnan(got[0, 5]) and torch.isinf(got[0, 6]) and torch.isfinite(got[0, [4, 7]]).all()


def test_far_outputs_and_features():
    B, V, K, far = 3, 200, 100, (1 << 31) + 1
    c = Case(B, V, K, 32, True)
    buf = torch.empty(2 * far + V, dtype=BF16, device=DEV)
    out = buf.as_strided((B, V), (far, 1))
    x = torch.empty(2 * far + K, dtype=BF16, device=DEV).as_strided((B, K), (far, 1))
    x.copy_(c.x)
    c.pack().project(x, out=out)
    y, tol = c.want(BF16)
    assert ((out.cpu().double() - y).abs() <= tol).all()


def test_matrix_past_4_gb():
    """Packed rows past 2^32 bytes."""
    V, K, G = (1 << 20) + 77, 8200, 128
    codes = torch.randint(0, 16, (V, K), dtype=torch.uint8, device=DEV)
    scales = torch.rand(V, -(-K // G), device=DEV).to(BF16)
    w = dels.pack_w4(codes, scales, group=G)
    assert w.data.numel() > 1 << 32
    x = torch.randn(2, K, device=DEV).to(BF16)
    got = w.project(x)
    at = torch.cat([torch.arange(64), torch.arange(V - 200, V)]).to(DEV)
    of = torch.arange(K, device=DEV) // G
    wt = (codes[at].double() - 8) * scales[at].double()[:, of]
    want, size = x.double() @ wt.T, x.double().abs() @ wt.abs().T
    eps = (17 * 8 + 65 + 10) * 2.0 ** -24 + 2.0 ** -37
    assert ((got[:, at].double() - want).abs() <= eps * size).all()


def test_refusals():
    codes, scales = torch.zeros(64, 96, dtype=torch.uint8, device=DEV), torch.ones(64, 3, dtype=BF16, device=DEV)
    zeros = torch.zeros(64, 3, dtype=torch.uint8, device=DEV)
    for a, kw in [((codes.int(), scales), {}), ((codes, scales.float()), {}), ((codes, scales[:, :2]), {}),
                  ((codes, None), {}), ((codes, scales, zeros.int()), {}), ((codes, scales, zeros[:5]), {}),
                  ((codes[:, ::2], scales), {}), ((codes, scales.cpu()), {})]:
        with pytest.raises(ValueError):
            dels.pack_w4(*a, group=32, **kw)
    with pytest.raises(dels.DelsError):
        dels.pack_w4(codes, scales, group=16)
    for where in ("codes", "zeros"):
        c, z = codes.clone(), zeros.clone()
        (c if where == "codes" else z)[63, 2] = 16
        with pytest.raises(ValueError, match="0 .. 15"):
            dels.pack_w4(c, scales, z, group=32)
    w = dels.pack_w4(codes, scales, zeros, group=32)
    x = torch.zeros(2, 96, dtype=BF16, device=DEV)
    for a in [(x[:, :95],), (x.half(),), (x.cpu(),), (x[0],), (x.T.contiguous().T,),
              (x, torch.empty(2, 63, device=DEV)), (x, torch.empty(2, 64, dtype=torch.half, device=DEV)),
              (x, torch.empty(64, device=DEV).expand(2, 64))]:
        with pytest.raises(ValueError):
            w.project(*a)
    assert w.project(x[:0]).shape == (0, 64)
    with pytest.raises(ValueError):
        dels.W4Matrix(w.data[:-1], 64, 96, 32, True)


def test_streams_graphs_and_equal_bits():
    c = Case(20, 3001, 900, 64, True)
    w, x = c.pack(), c.x.to(DEV)
    one = w.project(x).clone()
    s, t = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    outs = []
    for k in range(6):                       # one matrix, two streams at a time
        with torch.cuda.stream(s if k % 2 else t):
            outs.append(w.project(x))
    torch.cuda.synchronize()
    assert all(torch.equal(one, o) for o in outs)
    graph, out = torch.cuda.CUDAGraph(), torch.empty_like(one)
    with torch.cuda.graph(graph):
        w.project(x, out=out)
    x2 = torch.randn(20, 900, device=DEV).to(BF16)
    x.copy_(x2)
    graph.replay()
    graph.replay()
    assert torch.equal(out, w.project(x2)) and not torch.equal(out, one)
    v = out._version
    w.project(x2, out=out)
    assert out._version > v


def test_behind_a_kernel_on_its_stream():
    """Features, and the matrix itself, that the kernel before has just written."""
    c = Case(4, 5000, 512, 128, False)
    x = c.x.to(DEV)
    codes, scales = c.codes.to(DEV), c.scales.to(DEV)
    y, tol = c.want(F32)
    nbytes = dels.dels_w4_bytes(5000, 512, 128, False)
    ws = torch.zeros(256, dtype=torch.uint8, device=DEV)
    data = torch.zeros(nbytes, dtype=torch.uint8, device=DEV)
    w = dels.W4Matrix(data, 5000, 512, 128, False)
    for _ in range(20):
        data.zero_()
        assert dels.dels_w4_pack(codes, scales, None, 5000, 512, 128, data, nbytes, ws, 256) == 0
        got = w.project(x)
        assert ((got.cpu().double() - y).abs() <= tol).all()
    for k in range(20):
        z = x * 2.0 ** (k % 3)
        got = w.project(z)
        z.zero_()
        assert ((got.cpu().double() - y * 2.0 ** (k % 3)).abs() <= tol * 4).all()


@pytest.mark.parametrize("handle", [False, True])
def test_another_stream_than_the_current_one(handle):
    """Memory that the current stream has still to write, given back and taken again, and codes that it has still to
    make: the outputs of a call on another stream are its own, and so is what is packed there."""
    c = Case(3, 9000, 300, 64, True)
    y, tol = c.want(F32)
    s = torch.cuda.Stream()
    on = s.cuda_stream if handle else s
    w, x = c.pack(), c.x.to(DEV)
    source = [t.to(DEV) for t in (c.codes, c.scales, c.zeros)]
    rows = torch.randn(16, 4000, device=DEV)
    probs = torch.softmax(rows.double(), -1)
    torch.cuda.synchronize()
    # torch's own memory of these sizes is free again, with the current stream's fills ahead of it
    busy = [torch.empty(3, 9000, device=DEV), torch.empty(16, 4000, device=DEV),
            torch.empty(w.data.numel(), dtype=torch.uint8, device=DEV)]
    torch.cuda._sleep(50_000_000)
    for t in busy:
        t.fill_(7)
    del t, busy
    got = w.project(x, stream=on)
    p = dels.RowProbs(16, 4000)(rows, stream=on)
    torch.cuda.synchronize()
    assert ((got.cpu().double() - y).abs() <= tol).all()
    # an exponent's difference and product, 13 at most, a rounding each; the exponential, the sum and the quotient
    assert torch.allclose(p.double(), probs, rtol=(2 * 13 + 14) * 2.0 ** -24, atol=0)
    torch.cuda._sleep(50_000_000)
    late = [t.clone() for t in source]
    packed = dels.pack_w4(*late, group=64, stream=on)
    check(c, F32, packed)
