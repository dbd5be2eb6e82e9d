"""Probabilities of rows, and verification from given probabilities and uniforms, against float64.

Tolerances of a probability, relative: an entry's exponent takes at most 8 float32 roundings of
its distance from the row's largest over T, and where terms are added up 8 of the size of its own and
of the largest entry's terms, a sum of V exponentials of hardware accuracy (2^-22) V / 256 additions in a row at most and 64 more to join them,
the product with its reciprocal 2; bf16 half a step, 2^-8. Below float32's normal numbers a
probability may be flushed to 0. What the verification returns are whole numbers and have to be equal:
its sums are exact to about 2^-45, and no border of these cases lies that near.
"""
import math

import pytest
import torch

import paper_2607_07409_gb300 as dels

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
INF, NAN = math.inf, math.nan
F32, BF16 = torch.float32, torch.bfloat16
NONFINITE, BAD_TOKEN, BAD_VALUE = dels.DELS_STATUS_NONFINITE, dels.DELS_STATUS_BAD_TOKEN, dels.DELS_STATUS_BAD_VALUE


def gen(seed):
    return torch.Generator().manual_seed(seed)


def put(x, offset=0, pitch=None):
    """x [..., V] on the device, `offset` elements into its buffer, rows `pitch` apart, NaN between them."""
    V, pitch = x.shape[-1], pitch or x.shape[-1]
    rows = x.numel() // V
    buf = torch.full((offset + rows * pitch,), NAN, dtype=x.dtype, device=DEV)
    strides, step = [1], pitch
    for n in reversed(x.shape[:-1]):
        strides.insert(0, step)
        step *= n
    view = buf.as_strided(x.shape, strides, offset)
    view.copy_(x)
    return view


# ---------------------------------------------------------------- probabilities

class Rows:
    def __init__(self, rows, V, dtype, seed, fused, n=1):
        g = gen(seed)
        self.rows, self.V, self.dtype = rows, V, dtype
        self.long = (torch.randn(rows, V, generator=g) * 3).to(dtype)
        self.short = torch.randn(rows, V, generator=g).to(dtype) if fused else None
        self.prior = torch.log_softmax(torch.randn(V, generator=g) * 2, 0) if fused else None
        self.alpha = torch.rand(n, generator=g) + 0.2 if fused else None
        self.beta = torch.rand(n, generator=g) + 0.1 if fused else None

    def terms(self):
        at = lambda w: w.double()[torch.arange(self.rows) % w.numel()][:, None]
        t = [self.long.double()]
        if self.short is not None:
            t += [at(self.alpha) * self.short.double()] if self.alpha is not None else [self.short.double()]
        if self.prior is not None:
            t += [-at(self.beta) * self.prior.double()] if self.beta is not None else [-self.prior.double().expand(self.rows, -1)]
        return t

    def want(self, T, out):
        terms = self.terms()
        x = sum(terms)
        p = torch.softmax(x / T, -1)
        m, at = x.max(-1, keepdim=True)
        size = (x - m).abs()
        if len(terms) > 1:
            size = size + sum(t.abs() + t.abs().gather(1, at) for t in terms)
        rel = torch.expm1(8 * 2.0 ** -24 * size / T) + (16 * math.ceil(self.V / 4096) + 66) * 2.0 ** -24 + 2.0 ** -20
        rel = rel + (2.0 ** -8 if out is BF16 else 0.0)
        return p, torch.where(p > 0, rel * p, 0.0) + 2.0 ** -126

    def run(self, T=1.0, out=F32, offset=0, pitch=None, into=None, **kw):
        dev = lambda t: None if t is None else t.to(DEV)
        h = dels.RowProbs(self.rows, self.V, out, device=DEV)
        y = h(put(self.long, offset, pitch), short=None if self.short is None else put(self.short, offset, pitch),
              log_prior=dev(self.prior), alpha=dev(self.alpha), beta=dev(self.beta), temperature=T, out=into, **kw)
        return y.cpu(), h.status()


def check(c, T=1.0, out=F32, **kw):
    got, status = c.run(T, out, **kw)
    p, tol = c.want(T, out)
    assert status == 0 and got.dtype is out
    err = (got.double() - p).abs()
    assert (err <= tol).all(), (err / tol).max()


@pytest.mark.parametrize("fused", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,V", [(1, 1), (3, 2), (2, 7), (5, 255), (4, 1024), (3, 4099), (7, 32003), (300, 2050),
                                    (2, 50257), (3, 151936), (2, 470001), (1, 1000003)])
def test_probs(rows, V, dtype, fused):
    for T, out in [(1.0, F32), (0.7, BF16)]:
        check(Rows(rows, V, dtype, rows + V, fused, n=min(rows, 3)), T, out)


@pytest.mark.parametrize("out", [F32, BF16])
@pytest.mark.parametrize("dtype,offset,pitch", [(F32, 1, 0), (F32, 0, 3), (BF16, 1, 0), (BF16, 3, 5), (BF16, 0, 9),
                                                (BF16, 8, 8)])
@pytest.mark.parametrize("V", [1000, 9000, 33001])
def test_probs_anywhere(V, dtype, offset, pitch, out):
    """Rows of any alignment and pitch, in and out; what lies between the outputs' rows stays."""
    c = Rows(5, V, dtype, 3, True, n=2)
    big = torch.full((3 + 5 * (V + 5),), -1.0, dtype=out, device=DEV)
    view = big.as_strided((5, V), (V + 5, 1), 3)
    check(c, 1.3, out, offset=offset, pitch=V + pitch if pitch else None, into=view)
    big = big.cpu()
    assert (big[:3] == -1).all()
    for r in range(5):
        assert (big[3 + r * (V + 5) + V:3 + (r + 1) * (V + 5)] == -1).all()


@pytest.mark.parametrize("what", ["long+short", "long+prior", "short+prior", "no weights"])
def test_probs_terms(what):
    c = Rows(6, 5001, BF16, 11, True, n=3)
    if what == "long+short":
        c.prior = c.beta = None
    elif what == "long+prior":
        c.short = c.alpha = None
    elif what == "no weights":
        c.alpha = c.beta = None
    if what == "short+prior":
        kept = [put(c.short)] + [t.to(DEV) for t in (c.prior, c.alpha, c.beta)]
        x = dels.rows_of(6, 5001, None, *kept)
        h = dels.RowProbs(6, 5001, device=DEV)
        out = torch.empty(6, 5001, device=DEV)
        assert dels.dels_row_probs(x, 6, 5001, out, 0, 0, h.workspace, h.ws_bytes) == 0
        torch.cuda.synchronize()
        c.long = torch.zeros_like(c.long)
        p, tol = c.want(1.0, F32)
        assert ((out.cpu().double() - p).abs() <= tol).all()
        return
    check(c)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_probs_masks(dtype):
    """Masked entries have probability 0; rows masked to one entry, by the lowest value, from the front."""
    low = torch.finfo(dtype).min
    c = Rows(8, 20011, dtype, 5, False)
    c.long[0, 1:] = -INF
    c.long[1, :-1] = -INF
    c.long[2, :15000] = -INF
    c.long[3, ::2] = low
    c.long[4] = low                       # equal values: uniform
    c.long[5] = 3e38 if dtype is F32 else low
    c.long[6, 1:] = -1e9
    c.long[7] = -INF
    c.long[7, 777] = low
    check(c)
    got, _ = c.run()
    assert got[0, 0] == 1 and got[1, -1] == 1 and got[7, 777] == 1 and got[7].sum() == 1
    assert (got[2, :15000] == 0).all()


@pytest.mark.parametrize("T", [1e-30, 1e-4, 1e30])
def test_probs_temperatures(T):
    c = Rows(3, 5000, F32, 9, False)
    got, status = c.run(T)
    p = torch.softmax(c.long.double() / T, -1)
    assert status == 0
    # of the largest entry the distance is exact; what is below it by more than 2^-20 T has no part at 1e-4
    tol = 2.0 ** -18 if T < 1 else 1e-5 * p.max()
    assert ((got.double() - p).abs() <= tol).all()


@pytest.mark.parametrize("V", [100, 40001])
@pytest.mark.parametrize("bad", [NAN, INF, "none"])
def test_probs_flags(V, bad):
    c = Rows(5, V, F32, 2, False)
    c.long[3] = -INF if bad == "none" else c.long[3]
    if bad != "none":
        c.long[3, V - 1] = bad
    got, status = c.run()
    assert status == NONFINITE and torch.isnan(got[3]).all()
    p, tol = c.want(1.0, F32)
    keep = [0, 1, 2, 4]
    assert ((got.double() - p).abs() <= tol)[keep].all()


def test_probs_no_rows_and_refusals():
    h = dels.RowProbs(0, 10, device=DEV)
    assert h(torch.empty(0, 10, device=DEV)).shape == (0, 10) and h.status() == 0
    with pytest.raises(dels.DelsError):
        dels.RowProbs(1, 0, device=DEV)
    h = dels.RowProbs(2, 10, device=DEV)
    x = torch.zeros(2, 10, device=DEV)
    with pytest.raises(ValueError):
        h(x.cpu())
    with pytest.raises(ValueError):
        h(x.half())
    with pytest.raises(ValueError):
        h(x, out=torch.empty(2, 10, dtype=BF16, device=DEV))
    with pytest.raises(ValueError, match="overlap"):
        h(x, out=torch.empty(10, device=DEV).expand(2, 10))
    with pytest.raises(dels.DelsError):
        h(x, temperature=0.0)


def test_probs_far_rows():
    """Rows past 2^32 elements of their buffer."""
    V, pitch = 1003, (1 << 31) + 1
    buf = torch.empty(2 * pitch + V, dtype=BF16, device=DEV)
    x = buf.as_strided((3, V), (pitch, 1))
    c = Rows(3, V, BF16, 4, False)
    x.copy_(c.long)
    h = dels.RowProbs(3, V, BF16, device=DEV)
    got = h(x).cpu()
    p, tol = c.want(1.0, BF16)
    assert h.status() == 0 and ((got.double() - p).abs() <= tol).all()


# ---------------------------------------------------------------- verification

def oracle(tokens, p, q, u, lengths):
    """From the definition in float64, a request at a time."""
    B, n = tokens.shape
    acc, bonus = [], []
    for b in range(B):
        a, end = 0, n if lengths is None else int(lengths[b])
        while a < end:
            t = int(tokens[b, a])
            if not float(u[b, a]) * (float(q[b, a, t]) if q is not None else 1.0) < float(p[b, a, t]):
                break
            a += 1
        w = p[b, a].double()
        if a < end:
            r = torch.relu(w - q[b, a].double()) if q is not None else w.clone()
            if q is None:
                r[int(tokens[b, a])] = 0
            if r.max() > 0:
                w = r
        c = torch.cumsum(w, 0)
        acc.append(a)
        bonus.append(int(torch.searchsorted(c, float(u[b, n]) * c[-1], right=True)))
    return acc, bonus


class Block:
    def __init__(self, B, n, V, seed, p=F32, q=F32, near=0.5):
        g = gen(seed)
        x = torch.randn(B, n + 1, V, generator=g) * 3
        self.p = torch.softmax(x + near * torch.randn(B, n + 1, V, generator=g), -1).to(p)
        self.q = torch.softmax(x[:, :n], -1).to(q) if q is not None else None
        flat = torch.softmax(x[:, :n], -1).reshape(-1, V)
        self.tokens = (torch.multinomial(flat, 1, generator=g) if n and q is not None else flat.argmax(-1)
                       ).reshape(B, n).to(torch.int32)
        self.u = torch.rand(B, n + 1, generator=g)
        self.lengths = None
        self.B, self.n, self.V = B, n, V

    def run(self, offset=0, pitch=None, h=None, **kw):
        dev = lambda t: None if t is None else t.to(DEV)
        h = h or dels.BlockVerifier(self.B, self.n, self.V, device=DEV)
        q = None if self.q is None else put(self.q, offset and offset + 1, pitch)
        acc, bonus = h(dev(self.tokens), put(self.p, offset, pitch), dev(self.u), draft=q, lengths=dev(self.lengths), **kw)
        return acc.tolist(), bonus.tolist(), h.status()

    def check(self, **kw):
        acc, bonus, status = self.run(**kw)
        assert (acc, bonus) == oracle(self.tokens, self.p, self.q, self.u, self.lengths) and status == 0


@pytest.mark.parametrize("p,q", [(F32, F32), (BF16, BF16), (F32, BF16), (BF16, F32), (F32, None), (BF16, None)])
@pytest.mark.parametrize("B,n,V", [(1, 0, 1), (1, 1, 1), (3, 2, 2), (2, 5, 33), (1, 8, 1000), (33, 4, 4099), (5, 7, 50257),
                                   (9, 16, 8191), (2, 3, 151936), (3, 0, 151936), (200, 1, 3000)])
def test_verify(B, n, V, p, q):
    Block(B, n, V, B + n + V, p, q).check()


@pytest.mark.parametrize("p,q", [(F32, F32), (BF16, BF16), (BF16, F32), (F32, None)])
@pytest.mark.parametrize("offset,pitch", [(1, 0), (0, 1), (3, 7), (8, 8)])
@pytest.mark.parametrize("V", [500, 20000])
def test_verify_anywhere(V, offset, pitch, p, q):
    b = Block(6, 4, V, 77, p, q)
    b.lengths = torch.tensor([0, 1, 2, 3, 4, 4], dtype=torch.int32)
    b.check(offset=offset, pitch=V + pitch)


def test_verify_many_lengths_and_tokens():
    b = Block(64, 9, 700, 5, near=0.2)
    b.lengths = torch.randint(0, 10, (64,), generator=gen(1), dtype=torch.int32)
    b.check()
    b.u[:, :9] = 0.0            # kept wherever p > 0
    b.check()
    b.u[:, :9] = 1 - 2.0 ** -24
    b.check()


@pytest.mark.parametrize("V", [64, 1024, 40960])
@pytest.mark.parametrize("q", [F32, None])
def test_verify_borders(V, q):
    """Dyadic probabilities: every sum is exact, and uniforms lie on the borders themselves."""
    g = gen(V)
    B = 80
    w = torch.randint(0, 4, (B, 2, V), generator=g).double() * (torch.rand(B, 2, V, generator=g) < 40.0 / V)
    w[:, :, -1] = 0
    w[:, :, V // 3] += 1
    w[..., 0] += 1024 - w.sum(-1)
    b = Block(B, 1, V, 3, F32, q)
    b.p = (w / 1024).float()
    if q is not None:
        b.q = torch.zeros(B, 1, V)
        b.q[:, 0, 0] = 1.0
    b.tokens = torch.zeros(B, 1, dtype=torch.int32)
    b.u[:, 0] = b.p[:, 0, 0]              # u q = p: not kept
    for k in range(3):
        # on a border of the weights that are drawn from
        r = b.p[:, 0].double().clone()
        r[:, 0] = 0
        total = r.sum(-1)
        # borders j / 1024 of a total t / 1024: u = j / t is dyadic only for some; whole ones are exact
        b.u[:, 1] = 0.0 if k == 0 else (0.5 if k == 1 else 0.25)
        assert (total > 0).all()
        b.check()
    b.lengths = torch.zeros(B, dtype=torch.int32)      # from the whole row, of total 1
    b.u[:, 1] = torch.randint(0, 1024, (B,), generator=g) / 1024
    b.check()


def test_verify_nothing_left():
    """p = q (or below q) leaves no weight at a rejection: the token is drawn from p."""
    b = Block(12, 3, 3001, 8)
    b.p[:, :3] = b.q * 0.5
    b.u[:, :3] = 0.75
    acc, bonus, status = b.run()
    assert acc == [0] * 12 and status == 0
    b.check()
    one = torch.zeros(4, 2, 9)
    one[:, :, 4] = 1.0                     # a single token has it all: rejected by u q = p, nothing else left
    c = Block(4, 1, 9, 1, F32, None)
    c.p, c.tokens = one * 0.5, torch.full((4, 1), 4, dtype=torch.int32)
    c.u[:, 0] = 0.5
    assert c.run() == ([0] * 4, [4] * 4, 0)


@pytest.mark.parametrize("V", [5, 9001])
def test_verify_extremes(V):
    """The smallest and largest uniforms, weights at the ends, tiny and subnormal weights, sums above 1."""
    b = Block(6, 0, V, 2, F32, None)
    b.p = torch.zeros(6, 1, V)
    b.p[0, 0, V - 1] = 1e-30
    b.p[1, 0, 0] = 1e-45
    b.p[2, 0, :] = 1e-40
    b.p[3, 0, 1:4] = 1e37
    b.p[4, 0, :] = 1.0
    b.p[5, 0, 2] = 1.0
    b.p[5, 0, 3] = 2.0 ** -60
    for u in (0.0, 0.5, 1 - 2.0 ** -24, 2.0 ** -149):
        b.u[:] = u
        b.check()
    assert b.run()[1][0] == V - 1 and b.run()[1][1] == 0


def test_verify_small_differences():
    """Residuals of one unit in the last place, beside large equal entries."""
    V = 4000
    b = Block(16, 1, V, 21)
    bits = b.q.clone()
    up = torch.rand(16, 1, V, generator=gen(3)) < 0.01
    near = torch.nextafter(bits, torch.ones(()))
    b.p[:, :1] = torch.where(up, near, bits)
    b.tokens[:, 0] = up[:, 0].float().argmin(-1).to(torch.int32)     # p = q there
    b.u[:, 0] = 1 - 2.0 ** -24
    # u q < p would be kept: make it a rejection
    b.p[torch.arange(16), 0, b.tokens[:, 0].long()] = 0.0
    b.check()


@pytest.mark.parametrize("V", [50, 30000])
def test_verify_flags(V):
    ok = Block(9, 2, V, 4)
    ok.u[:, :2] = 0.0
    ok.tokens[:] = 1
    ok.p[:] = 1.0 / V

    def run(change):
        b = Block(9, 2, V, 4)
        b.p, b.q, b.u, b.tokens = ok.p.clone(), ok.q.clone(), ok.u.clone(), ok.tokens.clone()
        b.lengths = torch.full((9,), 2, dtype=torch.int32)
        change(b)
        acc, bonus, status = b.run()
        for i in (0, 1, 2, 3, 5, 6, 7, 8):     # the others as ever
            assert acc[i] == 2 and 0 <= bonus[i] < V
        return acc[4], bonus[4], status

    def at(name, *where, value):
        return lambda b: getattr(b, name).__setitem__((4,) + where, value)

    assert run(at("tokens", 1, value=-1)) == (1, -1, BAD_TOKEN)
    assert run(at("tokens", 0, value=V)) == (0, -1, BAD_TOKEN)
    assert run(at("u", 1, value=1.0)) == (1, -1, BAD_VALUE)
    assert run(at("u", 0, value=NAN)) == (0, -1, BAD_VALUE)
    assert run(at("u", 2, value=-0.5)) == (0, -1, BAD_VALUE)
    assert run(at("lengths", value=3)) == (0, -1, BAD_VALUE)
    assert run(at("lengths", value=-1)) == (0, -1, BAD_VALUE)
    assert run(at("p", 1, 1, value=NAN)) == (1, -1, NONFINITE)
    assert run(at("p", 1, 1, value=INF)) == (1, -1, NONFINITE)
    assert run(at("q", 0, 1, value=-0.1)) == (0, -1, NONFINITE)
    for value in (NAN, INF, -INF, -1e-3):
        for v in (0, V - 1, V // 2):
            assert run(at("p", 2, v, value=value)) == (2, -1, NONFINITE)
    assert run(at("p", 2, value=0.0)) == (2, -1, NONFINITE)          # a row without any

    def rejected(b):
        b.u[4, 1] = 0.5
        b.p[4, 1, 1] = 0.0
        b.q[4, 1, V - 2] = NAN

    assert run(rejected) == (1, -1, NONFINITE)

    def behind(b):
        rejected(b)
        b.q[4, 1, V - 2] = 0.0
        b.p[4, 2], b.tokens[4, 1] = NAN, 1
    acc, bonus, status = run(behind)       # behind the token that decides nothing is looked at
    assert acc == 1 and 0 <= bonus < V and status == 0

    def minus_zero(b):
        b.p[4, 2], b.p[4, 2, 3] = -0.0, 1.0
    assert run(minus_zero) == (2, 3, 0)


def test_verify_shorter_than_drafted():
    """Tokens, draft rows and uniforms behind a length are not read."""
    b = Block(5, 6, 2000, 6)
    b.lengths = torch.tensor([0, 2, 3, 6, 1], dtype=torch.int32)
    want = oracle(b.tokens, b.p, b.q, b.u, b.lengths)
    for i, n in enumerate(b.lengths.tolist()):
        b.tokens[i, n:] = -7
        b.q[i, n:] = NAN
        b.p[i, n + 1:] = NAN
        b.u[i, n:6] = NAN
    acc, bonus, status = b.run()
    assert (acc, bonus) == want and status == 0


def test_verify_far_rows():
    V, far = 1001, (1 << 31) + 3
    buf = torch.empty(3 * far, dtype=BF16, device=DEV)
    b = Block(3, 2, V, 6, BF16, BF16)
    p = buf.as_strided((3, 3, V), (far, V + 1, 1))
    q = buf.as_strided((3, 2, V), (far, V + 1, 1), 1 << 20)
    p.copy_(b.p)
    q.copy_(b.q)
    h = dels.BlockVerifier(3, 2, V, device=DEV)
    acc, bonus = h(b.tokens.to(DEV), p, b.u.to(DEV), draft=q)
    assert (acc.tolist(), bonus.tolist()) == oracle(b.tokens, b.p, b.q, b.u, None) and h.status() == 0


def test_verify_draws_follow_the_target():
    """Kept and drawn tokens together follow p (a chi-square of 20 categories, 3 significant tokens drafted badly)."""
    V, B = 20, 20000
    g = gen(9)
    p, q = (torch.softmax(torch.randn(V, generator=g), -1) for _ in range(2))
    tokens = torch.multinomial(q, B, replacement=True, generator=g)
    b = Block(1, 1, V, 1)
    b.B, b.p, b.q = B, p.expand(B, 2, V).contiguous(), q.expand(B, 1, V).contiguous()
    b.tokens, b.u = tokens[:, None].to(torch.int32), torch.rand(B, 2, generator=g)
    acc, bonus, status = b.run()
    first = torch.where(torch.tensor(acc) > 0, tokens, torch.tensor(bonus))
    n = torch.bincount(first, minlength=V).double()
    chi = ((n - B * p.double()) ** 2 / (B * p.double())).sum()
    assert status == 0 and chi < 19 + 6 * math.sqrt(2 * 19)


def test_verify_refusals():
    h = dels.BlockVerifier(2, 3, 10, device=DEV)
    t, p, u = torch.zeros(2, 3, dtype=torch.int32, device=DEV), torch.rand(2, 4, 10, device=DEV), torch.rand(2, 4, device=DEV)
    for args, kw in [((t.long(), p, u), {}), ((None, p, u), {}), ((t, p[:, :3], u), {}), ((t, p.half(), u), {}),
                     ((t, p, u[:, :3]), {}), ((t, p, None), {}), ((t, p.cpu(), u), {}), ((t, p, u), dict(draft=p)),
                     ((t, p, u), dict(lengths=t[0])), ((t, p[:1].expand(2, 4, 10), u), {}),
                     ((t, p.transpose(1, 2).contiguous().transpose(1, 2), u), {})]:
        with pytest.raises(ValueError):
            h(*args, **kw)
    with pytest.raises(dels.DelsError):
        dels.BlockVerifier(2, 1025, 10, device=DEV)
    e = dels.BlockVerifier(0, 3, 10, device=DEV)
    acc, bonus = e(t[:0], p[:0], u[:0])
    assert acc.shape == bonus.shape == (0,)


# ---------------------------------------------------------------- as they are used

def test_drafted_rows_then_verified():
    """Probabilities of the drafter's fused rows, a token of each, probabilities of the target's, verification."""
    B, n, V = 4, 5, 3203
    c, t = Rows(B * n, V, F32, 1, True, n=n), Rows(B * (n + 1), V, F32, 2, False)
    t.long = (c.long.view(B, n, V)[:, torch.arange(n + 1).clamp(max=n - 1)] + 0.3 * t.long.view(B, n + 1, V)).reshape(-1, V)
    g = gen(4)
    u0, u = torch.rand(B * n, 1, generator=g), torch.rand(B, n + 1, generator=g)
    dev = lambda x: x.to(DEV)
    draft, target = dels.RowProbs(B * n, V, device=DEV), dels.RowProbs(B * (n + 1), V, device=DEV)
    pick, verify = dels.BlockVerifier(B * n, 0, V, device=DEV), dels.BlockVerifier(B, n, V, device=DEV)
    args = [dev(x) for x in (c.long, c.short, c.prior, c.alpha, c.beta, t.long, u0, u)]

    def step():
        q = draft(args[0], short=args[1], log_prior=args[2], alpha=args[3], beta=args[4])
        _, x = pick(None, q.view(B * n, 1, V), args[6])
        p = target(args[5])
        return q, x, p, verify(x.view(B, n), p.view(B, n + 1, V), args[7], draft=q.view(B, n, V))

    q, x, p, (acc, bonus) = step()
    qh, ph = q.cpu(), p.cpu()
    _, drawn = oracle(torch.zeros(B * n, 0, dtype=torch.int32), qh.view(B * n, 1, V), None, u0, None)
    assert x.tolist() == drawn
    want = oracle(x.cpu().view(B, n), ph.view(B, n + 1, V), qh.view(B, n, V), u, None)
    assert (acc.tolist(), bonus.tolist()) == want
    # captured on a stream of its own and replayed over new numbers
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    u0, u = torch.rand(B * n, 1, generator=g), torch.rand(B, n + 1, generator=g)
    args[6].copy_(u0)
    args[7].copy_(u)
    args[5].mul_(0.9)
    graph.replay()
    graph.replay()
    q, x, p, (acc, bonus) = out
    qh, ph = q.cpu(), p.cpu()
    assert x.tolist() == oracle(torch.zeros(B * n, 0, dtype=torch.int32), qh.view(B * n, 1, V), None, u0, None)[1]
    assert (acc.tolist(), bonus.tolist()) == oracle(x.cpu().view(B, n), ph.view(B, n + 1, V), qh.view(B, n, V), u, None)
    for h in (draft, target, pick, verify):
        assert h.status() == 0


def test_equal_calls_give_equal_bits_on_any_stream():
    c = Rows(40, 30011, BF16, 1, True, n=4)
    one, _ = c.run()
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        two, _ = c.run()
    three, _ = c.run(stream=s)
    assert torch.equal(one, two) and torch.equal(one, three)


def test_outputs_are_marked_as_written():
    h = dels.RowProbs(2, 10, device=DEV)
    x = torch.zeros(2, 10, device=DEV)
    y = h(x)
    v = y._version
    h(x)
    assert y._version > v
    b = dels.BlockVerifier(2, 0, 10, device=DEV)
    u = torch.rand(2, 1, device=DEV)
    acc, bonus = b(None, y.view(2, 1, 10), u)
    v = acc._version, bonus._version
    b(None, y.view(2, 1, 10), u)
    assert acc._version > v[0] and bonus._version > v[1]
