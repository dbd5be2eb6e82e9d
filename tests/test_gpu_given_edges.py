"""The verification from given numbers where it can go wrong: empty columns beside a border, sums at
float32's end, rows far longer than a vocabulary, handles built behind unfinished work; how
exact probabilities are."""
import math
from fractions import Fraction

import pytest
import torch

import paper_2607_07409_gb300 as dels
from test_gpu_given import Block

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
NAN = math.nan
F32, BF16 = torch.float32, torch.bfloat16
NONFINITE = dels.DELS_STATUS_NONFINITE


def draw(p, u, h=None):
    """One draw a row of p [B, V] with uniforms u: (columns, status), from outputs that held -9 before."""
    B, V = p.shape
    h = h or dels.BlockVerifier(B, 0, V, device=DEV)
    h.accept_len.fill_(-9)
    h.bonus.fill_(-9)
    _, bonus = h(None, p.view(B, 1, V), torch.as_tensor(u, dtype=F32).expand(B).reshape(B, 1).contiguous().to(DEV))
    return bonus.tolist(), h.status()


# ---------------------------------------------------------------- borders beside what has no weight

# Three weights whose sums in float64 depend on their order: (x1 + x2) + x0 = 1 + 2^-52, x2 + (x1 + x0) = 1 + 2^-51.
X0, X1, X2 = 1.0, 2.0 ** -53 * (1 + 2.0 ** -23), 2.0 ** -53


@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("V,step,more,u", [
    (32768, 4096, {4 * 4096: 1.0}, 0.5),                       # a CTA's slice a step: the fourth has none
    (32768, 256, {5 * 4096: 1.0}, 0.5),                        # a warp's run a step
    (524288, 256, {5 * 256: 2.0 ** -50, 6 * 65536: 3.0}, 0.25),          # a part of a run a step
])
def test_the_border_lies_where_there_is_weight(V, step, more, u, offset):
    """u times the whole comes out between two sums up to the same column, taken in two orders: the column is one
    with weight all the same, and it is written. Sums here take 16 float64 additions at most, 2^-49 of the whole: of the
    columns with weight those whose sums enclose u times the whole to that."""
    weights = {0: X0, step: X1, 2 * step: X2, **more}
    p = torch.zeros(1, V + offset, dtype=F32)
    for v, w in weights.items():
        p[0, offset + v] = w
    bonus, status = draw(p.to(DEV)[:, offset:], u)
    total = sum(map(Fraction, weights.values()))
    at, near, right = Fraction(u) * total, total * Fraction(2) ** -49, []
    upto = Fraction(0)
    for v, w in sorted(weights.items()):
        if upto - near <= at <= upto + Fraction(w) + near:
            right.append(v)
        upto += Fraction(w)
    assert status == 0 and bonus[0] in right


# ---------------------------------------------------------------- sums at float32's end

@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("B,V", [(1, 32768), (1, 100), (40, 32768), (200, 9001)])
def test_sums_above_float32(B, V, offset):
    """A row whose entries are finite and whose sum is not within float32 is flagged wherever the entries lie, in any
    batch; one that sums to float32's largest number is not."""
    most = torch.finfo(F32).max
    rows = []
    for cols, values, ok in [([0, V - 1], [2e38, 2e38], False), ([5, 6], [2e38, 2e38], False),
                             ([5, V // 2], [2e38, 2e38], False), ([0, V // 3, V - 1], [1.2e38] * 3, False),
                             ([7], [most], True), ([7, V - 2], [most, 2.0 ** 80], False),
                             ([3, V - 1], [2.0 ** 127, most - 2.0 ** 127], True)]:
        rows.append((cols, values, ok))
    for cols, values, ok in rows:
        buf = torch.zeros(B * (V + offset), dtype=F32)
        p = buf.as_strided((B, V), (V + offset, 1), offset) if offset else buf.view(B, V)
        p[:, 1] = 1.0
        p[B // 2] = 0.0
        for c, x in zip(cols, values):
            p[B // 2, c] = x
        dev = buf.to(DEV)
        p = dev.as_strided((B, V), (V + offset, 1), offset) if offset else dev.view(B, V)
        bonus, status = draw(p, 0.25)
        assert (bonus[B // 2], status) == ((cols[0], 0) if ok else (-1, NONFINITE)), (cols, values)
        assert all(x == 1 for b, x in enumerate(bonus) if b != B // 2)


# ---------------------------------------------------------------- rows far longer than a vocabulary

@pytest.mark.parametrize("V,offset", [(1 << 28, 0), ((1 << 26) + 8, 1)])
def test_a_long_row(V, offset):
    """Weights of a = 1.1 (as float32) in the first half, of 1 behind them: the column is floor(u total - a V / 2) + V / 2 for
    the larger uniforms. No border of these lies within 0.05 of a weight, 2^-33 of the whole (a sum kept
    in float32 pairs throughout has lost 2^-24 of the first half, and comes out some columns off)."""
    a = torch.tensor(1.1, dtype=F32).item()
    p = torch.ones(1, V + offset, dtype=F32, device=DEV)[:, offset:]
    p[:, :V // 2] = a
    front, total = Fraction(a) * (V // 2), (Fraction(a) + 1) * (V // 2)
    h = dels.BlockVerifier(1, 0, V, device=DEV)
    u = 0.53 + 0.4 * torch.rand(40, generator=torch.Generator().manual_seed(5))
    n = 0
    for x in u.tolist():
        at = Fraction(x) * total - front
        if not 0.05 < at - math.floor(at) < 0.95:
            continue
        assert draw(p, x, h) == ([V // 2 + math.floor(at)], 0)
        n += 1
    assert n > 20


@pytest.mark.parametrize("p,q", [(F32, F32), (BF16, BF16), (BF16, F32), (F32, None), (BF16, None)])
@pytest.mark.parametrize("B,n,V,offset", [(2, 2, 2200008, 0), (1, 3, 2200001, 1), (160, 1, 262403, 0)])
def test_long_rows_of_blocks(B, n, V, offset, p, q):
    """Blocks whose rows are closed in parts: against the definition."""
    Block(B, n, V, B + n, p, q).check(offset=offset, pitch=V + offset)


# ---------------------------------------------------------------- handles built behind unfinished work

@pytest.mark.parametrize("handle", [False, True])
def test_a_handle_built_behind_unfinished_work(handle):
    """Built on a stream that still has to fill the memory that the handle is given, called on another one: what the
    call writes, and the status it raises, stay."""
    B, n, V = 64, 3, 5000
    g = torch.Generator().manual_seed(2)
    p = torch.softmax(torch.randn(B, n + 1, V, generator=g) * 3, -1).to(DEV)
    tokens = p[:, :n].argmax(-1).to(torch.int32)
    u = torch.rand(B, n + 1, generator=g).to(DEV)
    rows = torch.randn(16, V, generator=g)
    rows[5, 7] = NAN
    rows = rows.to(DEV)
    codes = torch.randint(0, 16, (500, 64), generator=g, dtype=torch.uint8).to(DEV)
    scales = torch.ones(500, 2, dtype=BF16, device=DEV)
    x = torch.randn(3, 64, generator=g).to(BF16).to(DEV)
    one = dels.BlockVerifier(B, n, V, device=DEV)
    want = [t.clone() for t in one(tokens, p, u)]
    assert one.status() == 0
    packed = dels.pack_w4(codes, scales, group=32)
    y = packed.project(x).clone()
    s = torch.cuda.Stream()
    on = s.cuda_stream if handle else s
    torch.cuda.synchronize()

    def behind(make):
        """make() with memory that the current stream has still to fill with other numbers."""
        busy = [torch.empty(m, dtype=torch.uint8, device=DEV) for m in (256, 512, 1024, 256, 512) for _ in range(8)]
        torch.cuda._sleep(100_000_000)
        for t in busy:
            t.fill_(1)
        del t, busy
        return make()

    h = behind(lambda: dels.BlockVerifier(B, n, V, device=DEV))
    acc, bonus = h(tokens, p, u, stream=on)
    s.synchronize()
    torch.cuda.synchronize()
    assert torch.equal(acc, want[0]) and torch.equal(bonus, want[1]) and h.status() == 0
    h = behind(lambda: dels.RowProbs(16, V, device=DEV))
    got = h(rows, stream=on)
    assert h.status(on) == NONFINITE
    torch.cuda.synchronize()
    assert torch.isnan(got[5]).all() and torch.isfinite(got[4]).all() and h.status() == 0
    m = behind(lambda: dels.W4Matrix(packed.data, 500, 64, 32, False))
    got = m.project(x, stream=on)
    assert m.status(on) == 0
    torch.cuda.synchronize()
    assert torch.equal(got, y) and m.status() == 0


def test_handles_in_a_capture():
    """Built before it and first called in it, on the capture's own stream; and built in it."""
    g = torch.Generator().manual_seed(3)
    x, u = torch.randn(4, 700, generator=g).to(DEV), torch.rand(4, 1, generator=g).to(DEV)
    probs, pick = dels.RowProbs(4, 700, device=DEV), dels.BlockVerifier(4, 0, 700, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _, one = pick(None, probs(x).view(4, 1, 700), u)
        p2, v2 = dels.RowProbs(4, 700, device=DEV), dels.BlockVerifier(4, 0, 700, device=DEV)
        _, two = v2(None, p2(x).view(4, 1, 700), u)
    for _ in range(2):
        x.mul_(0.7)
        graph.replay()
        p = torch.softmax(x.double(), -1).cumsum(-1)
        want = torch.searchsorted(p, u.double() * p[:, -1:], right=True).view(-1).tolist()
        assert one.tolist() == two.tolist() == want
    assert [h.status() for h in (probs, pick, p2, v2)] == [0] * 4


# ---------------------------------------------------------------- how exact probabilities are

def below(c):
    """The float32 number at or below c."""
    f = torch.tensor(c, dtype=F32)
    return (f if f.item() <= c else torch.nextafter(f, torch.tensor(0.0))).item()


def rough(lo, hi):
    """A temperature whose log2(e) / T lies nearly a whole step above a float32 number."""
    ts = torch.linspace(lo, hi, 4001, dtype=F32).tolist()
    return max(ts, key=lambda t: 1 - below(math.log2(math.e) / t) / (math.log2(math.e) / t))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V,T", [(1000, 1.0), (32003, 0.7), (151936, 1.0), (500009, 1.0)])
def test_probabilities_norm(V, T, dtype):
    """||p - softmax|| / ||softmax|| of float32 outputs. The norm is the likely entries', whose exponents are within 16 of the
    largest: the difference and its product are rounded by 0.3 steps of 2^-20 (rms), each 2e-7 of such an entry and 1e-7 over
    all; the exponential by 2^-23 or so, the row's own factor by three roundings, 2^-23 together: 3e-7 holds them all."""
    g = torch.Generator().manual_seed(V)
    x = (torch.randn(8, V, generator=g) * 3).to(dtype).to(DEV)
    h = dels.RowProbs(8, V, device=DEV)
    want = torch.softmax(x.double() / T, -1)
    got = h(x, temperature=T).double()
    assert h.status() == 0
    assert ((got - want).norm(dim=-1) <= 3e-7 * want.norm(dim=-1)).all(), ((got - want).norm(dim=-1) / want.norm(dim=-1)).max()


@pytest.mark.parametrize("V", [20011, 151936, 500009])
def test_the_scale_of_all_exponents(V):
    """A likely entry beside many that are far below and together have as much: roundings of their exponents differ and go
    both ways, so that the likely one's probability is off by those of the row's factor, 3 2^-24, and of a sum of
    exponentials of 2^-23, 3e-7 in all. (With log2(e) / T cut to float32 all exponents are off the same way by 12 2^-23,
    times the others' share: 4e-7 and more.)"""
    T = rough(0.95, 1.05)
    x = torch.randn(4, V, generator=torch.Generator().manual_seed(V)).to(DEV)
    x[:, 77] = math.log(V) + 0.5
    h = dels.RowProbs(4, V, device=DEV)
    got = h(x, temperature=T).double()[:, 77] / torch.softmax(x.double() / T, -1)[:, 77]
    assert h.status() == 0 and ((got - 1).abs() <= 3e-7).all(), got - 1
