"""Scoring and distillation of vocabulary rows against their definitions in float64.

Tolerances, from the operations: a fused entry takes three float32 roundings, a
scaled one (x - m) / T two more (each 2^-24 of the values' size); a sum of V
exponentials of hardware accuracy (2^-22) is taken 8 V / 4096 terms in a row at
most (a slice may be a whole row), then through trees of at most 32 steps:

    eps_z(row) = 8 * 2^-24 * max(|terms|) / T,   eps_sum(V) = (8 ceil(V / 4096) + 32) 2^-24 + 2^-21

A log-probability is off by 2 eps_z + eps_sum at most, an entropy by that times
(1 + the largest ln q that has weight, taken as ln V + 2), a probability by the
same relatively; a gradient entry by that of its probabilities, and bf16 by half
a unit of its last place (8 significant bits: 2^-8 of the value at most).
"""
import math

import numpy as np
import pytest
import torch

import paper_2607_07409_gb300 as dels

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
INF = math.inf
LOW = {torch.float32: torch.finfo(torch.float32).min, torch.bfloat16: torch.finfo(torch.bfloat16).min}


def eps_sum(V):
    return (8 * math.ceil(V / 4096) + 32) * 2.0 ** -24 + 2.0 ** -21


def gen(seed):
    return torch.Generator().manual_seed(seed)


def put(x, offset=0, pitch=None):
    """x [rows, V] on the device, `offset` elements into its buffer, rows `pitch` apart."""
    rows, V = x.shape
    pitch = pitch or V
    buf = torch.full((offset + rows * pitch,), float("nan"), dtype=x.dtype, device=DEV)   # what lies between rows
    view = buf.as_strided((rows, V), (pitch, 1), offset)
    view.copy_(x)
    return view


class Case:
    """Rows on the host (as stored) and on the device."""

    def __init__(self, rows, V, dtype, seed, fused, n=1, offset=0, pitch=None, scale=3.0):
        g = gen(seed)
        self.rows, self.V, self.dtype, self.fused = rows, V, dtype, fused
        self.long = (torch.randn(rows, V, generator=g) * scale).to(dtype)
        self.short = torch.randn(rows, V, generator=g).to(dtype) if fused else None
        self.prior = torch.log_softmax(torch.randn(V, generator=g) * 2, 0).float() if fused else None
        self.alpha = (torch.rand(n, generator=g) + 0.2).float() if fused else None
        self.beta = (torch.rand(n, generator=g) + 0.1).float() if fused else None
        self.offset, self.pitch = offset, pitch

    def at(self, w):
        return w[torch.arange(self.rows) % w.numel()][:, None]

    def x32(self):
        """The fused rows as the library defines them: float32, rounded after every operation."""
        if not self.fused:
            return self.long.float()
        x = self.long.float() + self.at(self.alpha) * self.short.float()
        return x - self.at(self.beta) * self.prior

    def size(self):
        """Largest finite term of each row."""
        parts = [self.long.float()]
        if self.fused:
            parts += [self.at(self.alpha) * self.short.float(), (self.at(self.beta) * self.prior).expand(self.rows, -1)]
        return sum(torch.where(p.isfinite(), p.abs(), torch.zeros_like(p)).amax(-1).double() for p in parts)

    def dev(self, name):
        t = getattr(self, name)
        if t is None:
            return None
        return put(t, self.offset, self.pitch) if t.dim() == 2 else t.to(DEV)

    def kwargs(self):
        return {k: self.dev(k2) for k, k2 in (("log_prior", "prior"), ("alpha", "alpha"), ("beta", "beta"))}


def top_order(x, K):
    """Entries of each float32 row by (value descending, index ascending); -1 for what is missing."""
    order = np.argsort(-x.numpy(), axis=1, kind="stable")[:, :K].copy()
    val = np.take_along_axis(x.numpy(), order, 1)
    order[val == -INF] = -1
    out = np.full((x.shape[0], K), -1, dtype=np.int64)
    out[:, :order.shape[1]] = order
    return out


def check_score(c, K, T=1.0, tokens=None, rows_ok=None):
    x32, V = c.x32(), c.V
    tokens = torch.randint(0, V, (c.rows,), generator=gen(5)) if tokens is None else tokens
    sc = dels.TokenScorer(c.rows, V, K, device=DEV)
    lp, ent, ids, tlp = sc(c.dev("long"), tokens.to(torch.int32).to(DEV), short=c.dev("short"), temperature=T, **c.kwargs())
    status = sc.status()
    z = x32.double() / T
    lq = torch.log_softmax(z, -1)
    tol = 2 * 8 * 2.0 ** -24 * c.size() / T + eps_sum(V)
    ok = torch.ones(c.rows, dtype=torch.bool) if rows_ok is None else rows_ok
    ref = lq.gather(1, tokens.clamp(min=0)[:, None])[:, 0]
    got = lp.cpu().double()
    fin = ok & ref.isfinite()
    # a log-probability far below is rounded to its own last place too
    assert ((got - ref).abs()[fin] <= tol[fin] + ref.abs()[fin] * 2.0 ** -22).all()
    assert (got[ok & ~ref.isfinite()] == -INF).all()
    h = torch.special.entr(lq.exp()).sum(-1)
    assert ((ent.cpu().double() - h).abs()[ok] <= (tol * (math.log(V) + 3))[ok]).all()
    if K:
        want = torch.from_numpy(top_order(x32, K))
        assert torch.equal(ids.cpu().long()[ok], want[ok])
        ref_t = torch.where(want >= 0, lq.gather(1, want.clamp(min=0)), torch.full_like(want, -INF, dtype=torch.float64))
        t = tlp.cpu().double()
        f = ref_t.isfinite() & ok[:, None]
        assert ((t - ref_t).abs() <= tol[:, None] + ref_t.abs() * 2.0 ** -22)[f].all()
        assert (t[~ref_t.isfinite() & ok[:, None]] == -INF).all()
    return lp, ent, ids, tlp, status


SCORE_SIZES = [
    # rows, V, K, offset, pitch: one column and one vector, one past a vector, one item per thread and one past it
    (3, 1, 1, 0, None), (2, 2, 5, 0, None), (5, 7, 3, 0, None), (4, 8, 8, 0, None), (3, 9, 256, 0, None),
    (2, 31, 20, 0, None), (3, 1000, 1, 0, None), (2, 4096, 20, 0, None), (2, 4097, 33, 0, None),
    (1, 8191, 64, 0, None), (2, 20011, 128, 0, None), (1, 40000, 256, 0, None), (1, 151936, 20, 0, None),
    # rows that start off a 16-byte boundary, and padded ones
    (4, 1000, 7, 1, None), (3, 1000, 7, 0, 1003), (4, 1001, 7, 0, 1008), (3, 5000, 16, 8, 5008), (3, 4099, 5, 3, 4101),
    # many rows: one CTA a row
    (700, 1030, 4, 0, None), (640, 9001, 2, 0, None),
    # few entries a thread and many asked for: more candidates than are sorted at once
    (2, 1024, 128, 0, None), (2, 2048, 256, 0, None), (300, 3000, 200, 0, None),
]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("fused", [False, True], ids=["plain", "fused"])
@pytest.mark.parametrize("rows,V,K,offset,pitch", SCORE_SIZES)
def test_score_matches_float64(rows, V, K, offset, pitch, fused, dtype):
    c = Case(rows, V, dtype, rows * V + K, fused, n=3, offset=offset, pitch=pitch)
    assert check_score(c, K, T=1.0 if V % 2 else 0.7)[-1] == 0


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("V", [30000, 30001])
def test_score_rounds_fused_values_step_by_step(V, dtype):
    """Enough fused entries that neighbours in the order differ in their last bits:
    a contracted product would exchange some."""
    assert check_score(Case(48, V, dtype, 77, True, n=5), 256)[-1] == 0


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("V,offset", [(9000, 0), (9001, 0), (131072, 0), (131073, 0)])
def test_score_orders_ties_and_crowded_threads(V, offset, dtype):
    """Rows whose alternatives meet in few threads, more entries above the
    threshold than are kept at once, and ties by the thousand."""
    rows = []
    i = torch.arange(V)
    rows.append(torch.full((V,), 2.5))                                   # all equal
    rows.append((i % 7).float())                                         # seven values
    rows.append(i.float() / V)                                           # rising: every entry beats those before it
    rows.append(-(i.float()) / V)
    rows.append(torch.where(i % 4096 < 8, 50.0 + i / V, i / V))          # one thread of each CTA
    rows.append(torch.where(i % 4096 < 255 * 8, 100.0 + i / V, torch.where(i % 4096 == 3000, 1.0, -i / V)))
    rows.append(torch.where(i % 512 < 255, 100.0 + i / V, torch.where(i % 512 == 300, 1.0, -i / V)))
    rows.append(torch.where(i % 3 == 0, 0.0, -0.0))                      # zeros of both signs are equal
    for K in (1, 64, 256):
        c = Case(len(rows), V, dtype, 1, False, offset=offset)
        c.long = torch.stack(rows).to(dtype)
        assert check_score(c, K)[-1] == 0


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("V", [100, 4097, 12000])
def test_score_masks_and_bad_rows(V, dtype):
    c = Case(12, V, dtype, 9, False)
    x = c.long.float()
    low = LOW[dtype]
    x[0, 3:] = -INF                      # three entries left
    x[1] = -INF                          # nothing left
    x[2] = low                           # the type's lowest value alone: a uniform row
    x[3, 5:] = low
    x[4, V // 2] = float("nan")
    x[5, V // 2] = INF
    x[6] = -INF
    x[6, V - 1] = -7.0                   # one entry
    x[7] = -1e30
    x[7, 1] = -1.5e30
    x[8, :] = torch.where(torch.arange(V) % 2 == 0, -INF, 1.0)
    x[9] = 3e38
    x[10, 0] = 3e38
    c.long = x.to(dtype)
    ok = torch.ones(12, dtype=torch.bool)
    ok[[1, 4, 5]] = False
    # rows of huge values: their differences are exact or infinite, the rest has no mass
    c.size = lambda: torch.where(c.long.float().abs().nan_to_num(0, 0, 0).amax(-1) > 1e20, 1.0, 30.0).double()
    tok = torch.zeros(12, dtype=torch.int64)
    lp, ent, ids, tlp, status = check_score(c, 8, tokens=tok, rows_ok=ok)
    assert status == dels.DELS_STATUS_NONFINITE
    for t in (lp, ent, tlp):
        assert torch.isnan(t[[1, 4, 5]]).all()
    assert (ids[[1, 4, 5]] == -1).all()
    assert abs(float(ent[2]) - math.log(V)) < 1e-5 and abs(float(ent[6])) == 0.0


def test_score_left_out_rows_and_bad_tokens():
    c = Case(6, 3000, torch.float32, 2, True, n=2)
    sc = dels.TokenScorer(6, 3000, 4, device=DEV)
    tok = torch.tensor([5, -1, 2999, 3000, -2, 0], dtype=torch.int32, device=DEV)
    long = c.dev("long")
    long[1] = float("nan")               # a left-out row is not read
    lp, ent, ids, tlp = sc(long, tok, short=c.dev("short"), **c.kwargs())
    assert sc.status() == dels.DELS_STATUS_BAD_TOKEN
    assert lp[1] == 0 and ent[1] == 0 and (ids[1] == -1).all() and (tlp[1] == -INF).all()
    assert torch.isnan(lp[[3, 4]]).all() and torch.isfinite(lp[[0, 2, 5]]).all()
    assert torch.isfinite(ent[[0, 2, 3, 4, 5]]).all() and (ids[[0, 2, 3, 4, 5]] >= 0).all()
    # without tokens every row is read
    c.long[1] = 1.0
    lp, ent2, ids2, _ = sc(c.dev("long"), short=c.dev("short"), **c.kwargs())
    assert lp is None and sc.status() == 0 and (ids2[1] >= 0).all()
    assert torch.equal(ent2[[0, 2, 5]], ent[[0, 2, 5]])


def test_score_terms_may_be_absent():
    """A head's logits alone with a weight, a prior alone beside the drafter's."""
    c = Case(5, 2003, torch.bfloat16, 3, True, n=5)
    sc = dels.TokenScorer(5, 2003, 3, device=DEV)
    al, be, pr = c.alpha.to(DEV), c.beta.to(DEV), c.prior.to(DEV)
    got = sc(c.dev("long"), log_prior=pr, beta=be)[1].clone()
    ref = torch.log_softmax((c.long.float() - c.at(c.beta) * c.prior).double(), -1)
    assert ((got.cpu() - torch.special.entr(ref.exp()).sum(-1)).abs() < 1e-4).all()
    short = c.dev("short")
    x = dels.rows_of(5, 2003, None, short, None, al)
    ent = torch.empty(5, device=DEV)
    ws = torch.zeros(256, dtype=torch.uint8, device=DEV)
    assert dels.dels_score_rows(x, 5, 2003, None, 0, None, ent, None, None, ws, 256) == 0
    ref = torch.log_softmax((c.at(c.alpha) * c.short.float()).double(), -1)
    assert ((ent.cpu() - torch.special.entr(ref.exp()).sum(-1)).abs() < 1e-4).all()


def test_score_offsets_past_32_bits():
    """Rows beyond 2^31 elements; the last ones against the same rows alone."""
    V, rows = 151936, 14200
    x = torch.empty(rows, V, dtype=torch.bfloat16, device=DEV)
    x.fill_(-3.0)
    tail = torch.randn(4, V, generator=gen(8)).mul(3).to(torch.bfloat16).to(DEV)
    x[-4:] = tail
    assert x.numel() > 2 ** 31
    tok = torch.arange(rows, dtype=torch.int32, device=DEV)
    a = dels.TokenScorer(rows, V, 5, device=DEV)(x, tok)
    b = dels.TokenScorer(4, V, 5, device=DEV)(tail, tok[-4:])
    assert torch.equal(a[2][-4:], b[2])
    for k in (0, 1, 3):
        assert ((a[k][-4:] - b[k]).abs() < 2e-5).all()


def test_score_repeats_its_bits_on_any_stream():
    c = Case(9, 30011, torch.bfloat16, 4, True, n=3)
    long, short, kw = c.dev("long"), c.dev("short"), c.kwargs()
    tok = torch.arange(9, dtype=torch.int32, device=DEV)
    sc = dels.TokenScorer(9, 30011, 40, device=DEV)
    first = [t.clone() for t in sc(long, tok, short=short, **kw)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(3):
            again = sc(long, tok, short=short, **kw)
    torch.cuda.synchronize()
    for u, v in zip(first, again):
        assert torch.equal(u, v)


# --------------------------------------------------------------------------- distillation

def teacher(c, K, seed, tail, T, missing=True):
    """Entries of a row near the student's own, as a teacher that differs from it."""
    g = gen(seed)
    z = (c.x32().nan_to_num(0.0, 0.0, -1e4) + torch.randn(c.rows, c.V, generator=g) * 2).double() / T
    k = min(K, c.V)
    v, i = torch.log_softmax(z, -1).topk(k, -1)
    ids = torch.full((c.rows, K), -1, dtype=torch.int32)
    lp = torch.full((c.rows, K), -INF)
    ids[:, :k], lp[:, :k] = i.to(torch.int32), v.float()
    if missing and k > 2:
        ids[::2, 1] = -1
        lp[1::3, 2] = -INF
    return ids, lp


def reference(c, ids, t, tail, T, weight, up):
    """Losses and gradients in float64 from the definition, by PyTorch's engine."""
    x = c.long.double() if not c.fused else None
    s = (c.short if c.fused else c.long).double().requires_grad_()
    al = c.alpha.double().requires_grad_() if c.fused else None
    be = c.beta.double().requires_grad_() if c.fused else None
    at = torch.arange(c.rows)
    x = c.long.double() + al[at % al.numel(), None] * s - be[at % be.numel(), None] * c.prior.double() if c.fused else s
    lq = torch.log_softmax(x / T, -1)
    losses = []
    for r in range(c.rows):
        keep = [(int(i), float(v)) for i, v in zip(ids[r], t[r]) if i >= 0 and i < c.V and v > -INF]
        if not keep or weight[r] == 0:
            losses.append((lq[r] * 0).nan_to_num(0).sum() * 0)
            continue
        lv = torch.tensor([v for _, v in keep], dtype=torch.float64)
        lp = lv if tail else torch.log_softmax(lv / T, -1)
        p = lp.exp()
        loss = sum(p[k] * (lp[k] - lq[r, i]) for k, (i, _) in enumerate(keep) if p[k] > 0)
        if tail:
            others = torch.ones(c.V, dtype=torch.bool)
            others[[i for i, _ in keep]] = False
            rest = max(0.0, 1.0 - float(p.sum()))
            if rest > 0 and bool(others.any()) and bool((lq[r, others] > -INF).any()):
                loss = loss + rest * (math.log(rest) - torch.logsumexp(lq[r, others], -1))
        losses.append(weight[r] * loss)
    losses = torch.stack(losses)
    (losses * up).sum().backward()
    return losses.detach(), s.grad.nan_to_num(0.0), al.grad if c.fused else None, be.grad if c.fused else None, lq.detach()


def check_distill(c, K, tail, T=1.0, seed=7, weight=None, via="step", ids_t=None, in_place=False, rest_tol=None):
    ids, t = ids_t or teacher(c, K, seed, tail, T)
    weight = torch.rand(c.rows, generator=gen(3)) + 0.5 if weight is None else weight
    up = torch.rand(c.rows, generator=gen(4)) + 0.5 if via != "step" else torch.ones(c.rows)
    ref = reference(c, ids, t, tail, T, weight.double(), up.double())
    short = c.dev("short") if c.fused else c.dev("long")
    long = c.dev("long") if c.fused else None
    args = dict(long=long, row_weight=weight.float().to(DEV), **c.kwargs())
    n = c.alpha.numel() if c.fused else 1
    if via == "step":
        d = dels.Distiller(c.rows, c.V, K, c.dtype, n_weights=n, tail=tail, temperature=T, device=DEV)
        loss, g, ga, gb = d.step(short, ids.to(DEV), t.to(DEV), out=short if in_place else None, **args)
        status = d.status()
    else:
        leaves = [short.requires_grad_()]
        if c.fused:
            leaves += [args["alpha"].requires_grad_(), args["beta"].requires_grad_()]
        loss = dels.distill_loss(short, ids.to(DEV), t.to(DEV), tail=tail, temperature=T, **args)
        g, *rest = torch.autograd.grad(loss, leaves, up.to(DEV))
        ga, gb = rest if c.fused else (None, None)
        status = 0
    V, w = c.V, (weight * up).double()
    lq = ref[4]
    # a log-probability's error, which is the relative one of a probability
    e = 2 * 8 * 2.0 ** -24 * c.size() / T + eps_sum(V)
    live = t[t > -INF]
    e_t = 2.0 ** -23 * (float(live.abs().max()) if live.numel() else 0.0) / T + 2.0 ** -20
    e_row = (e + e_t)[:, None]
    # the loss: terms p (ln p - ln q) of both errors, |ln p| + |ln q| of relative size
    big = 2 + math.log(max(V, 3)) + float(ref[4][ref[4] > -INF].abs().max()) * 2.0 ** -10
    assert ((loss.detach().cpu().double() - ref[0]).abs() <= weight.double() * e_row[:, 0] * big).all()
    # a tail's gradient is q (M - p_t / q_t): the teacher's rest is known to 2^-22 of 1
    q = lq.exp()
    p = torch.zeros_like(q)
    r_t = torch.zeros(c.rows, 1, dtype=torch.float64)
    for r in range(c.rows):
        lv = torch.tensor([v if 0 <= i < V else -INF for i, v in zip(ids[r].tolist(), t[r].tolist())]).double()
        if (lv > -INF).any():
            pr = lv.exp() if tail else torch.softmax(lv / T, -1)
            p[r].index_add_(0, ids[r].clamp(0, V - 1).long(), pr.nan_to_num(0.0))
            if tail:
                qt = q[r][p[r] == 0].sum()
                r_t[r] = 2.0 ** -21 / max(float(qt), 1e-30) + float(max(0.0, 1 - pr.sum()) / max(float(qt), 1e-30)) * 2 * float(e_row[r])
    a_row = (c.at(c.alpha).double() if c.fused else torch.ones(c.rows, 1, dtype=torch.float64)).abs()
    bound = (w[:, None] / T) * a_row * (2 * e_row * (q + p) + q * r_t)
    half = 2.0 ** -8 if c.dtype == torch.bfloat16 else 2.0 ** -24
    err = (g.cpu().double() - ref[1]).abs()
    assert (err <= bound + half * ref[1].abs() + 1e-37).all(), float((err - bound).max())
    if c.fused:
        at = torch.arange(c.rows) % n
        # the sums' own rounding beside the entries'
        for got, want, val in ((ga, ref[2], c.short.double().nan_to_num(0.0, 0.0, 0.0).abs()),
                               (gb, ref[3], c.prior.double().abs().expand(c.rows, -1))):
            per = ((bound / a_row + 2.0 ** -20 * (w[:, None] / T) * (q + p)) * val).sum(-1)
            lim = torch.zeros(n, dtype=torch.float64).index_add_(0, at, per)
            assert ((got.cpu().double() - want).abs() <= lim + 1e-12).all()
    return loss, g, ga, gb, status


DISTILL_SIZES = [
    # rows, V, K, offset, pitch
    (3, 1, 1, 0, None), (3, 2, 1, 0, None), (4, 5, 5, 0, None), (4, 8, 3, 0, None), (3, 9, 20, 0, None),
    (5, 1000, 16, 0, None), (2, 4096, 64, 0, None), (3, 4097, 33, 0, None), (2, 20011, 256, 0, None),
    (1, 151936, 64, 0, None), (4, 1001, 7, 1, None), (3, 1000, 7, 0, 1003), (4, 1001, 7, 0, 1008),
    (3, 5000, 16, 8, 5008), (640, 1100, 4, 0, None),
]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("tail", [False, True], ids=["renormalised", "tail"])
@pytest.mark.parametrize("fused", [False, True], ids=["plain", "fused"])
@pytest.mark.parametrize("rows,V,K,offset,pitch", DISTILL_SIZES)
def test_distill_matches_float64(rows, V, K, offset, pitch, fused, tail, dtype):
    c = Case(rows, V, dtype, rows * V + K, fused, n=3, offset=offset, pitch=pitch)
    T = 1.0 if K % 2 else 2.0
    assert check_distill(c, K, tail, T)[-1] == 0


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("tail", [False, True], ids=["renormalised", "tail"])
@pytest.mark.parametrize("fused", [False, True], ids=["plain", "fused"])
def test_distill_through_autograd(fused, tail, dtype):
    c = Case(6, 3001, dtype, 11, fused, n=2)
    check_distill(c, 9, tail, 1.5, via="autograd")
    c = Case(7, 12000, dtype, 12, fused, n=7)
    check_distill(c, 40, tail, 1.0, via="autograd")


@pytest.mark.parametrize("tail", [False, True], ids=["renormalised", "tail"])
def test_distill_gradient_against_differences(tail):
    """Central differences of the losses themselves in the weights and in single logits: the
    loss is known to about 1e-6, a step of 2^-5 leaves 1e-4 of that and 3e-4 of third-order terms."""
    c = Case(4, 40, torch.float32, 13, True, n=4, scale=1.0)
    ids, t = teacher(c, 6, 1, tail, 1.0)
    long, short, kw = c.dev("long"), c.dev("short"), c.kwargs()
    d = dels.Distiller(4, 40, 6, torch.float32, n_weights=4, tail=tail, device=DEV)
    ids, t = ids.to(DEV), t.to(DEV)
    loss, g, ga, gb = [v.clone() for v in d.step(short, ids, t, long=long, **kw)]
    h = 2.0 ** -5
    for name, grad in (("alpha", ga), ("beta", gb)):
        for j in range(4):
            moved = []
            for sign in (1, -1):
                k2 = dict(kw, **{name: kw[name].clone()})
                k2[name][j] += sign * h
                moved.append(float(d.loss(short, ids, t, long=long, **k2).double().sum()))
            assert abs((moved[0] - moved[1]) / (2 * h) - float(grad[j])) < 2e-3 * (1 + abs(float(grad[j])) * 5)
    for r, v in ((0, int(ids[0, 0])), (1, int(ids[1, 3])), (2, 17), (3, 0)):
        moved = []
        for sign in (1, -1):
            s2 = short.clone()
            s2[r, v] += sign * h
            moved.append(float(d.loss(s2, ids, t, long=long, **kw).double().sum()))
        assert abs((moved[0] - moved[1]) / (2 * h) - float(g[r, v])) < 2e-3


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("V", [2000, 2001, 33000])
def test_distill_in_place_and_strided_gradient(V, dtype):
    c = Case(5, V, dtype, 21, True, n=5)
    a = [x.clone() for x in check_distill(c, 12, True)[:4]]
    b = check_distill(c, 12, True, in_place=True)
    for u, v in zip(a, b):
        assert torch.equal(u, v)
    ids, t = teacher(c, 12, 7, True, 1.0)
    weight = (torch.rand(5, generator=gen(3)) + 0.5).float().to(DEV)
    d = dels.Distiller(5, V, 12, dtype, n_weights=5, tail=True, device=DEV)
    wide = torch.full((5, V + 13), 7.0, dtype=dtype, device=DEV)
    out = d.step(c.dev("short"), ids.to(DEV), t.to(DEV), long=c.dev("long"), row_weight=weight, out=wide[:, :V], **c.kwargs())
    assert torch.equal(out[1], a[1]) and (wide[:, V:] == 7.0).all()      # nothing past the rows is written


@pytest.mark.parametrize("tail", [False, True], ids=["renormalised", "tail"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_distill_listed_twice_and_whole_vocabulary(dtype, tail):
    c = Case(4, 4100, dtype, 31, True, n=2)
    ids, t = teacher(c, 8, 2, tail, 1.0, missing=False)
    ids[0, 3] = ids[0, 0]
    ids[1, 5] = ids[1, 4]
    ids[1, 6] = ids[1, 4]
    t = t - 1.0                                  # sums below 1 whatever is listed twice
    check_distill(c, 8, tail, ids_t=(ids, t))
    c = Case(3, 12, dtype, 32, True, n=1)        # every id listed: no tail is left
    ids, t = teacher(c, 12, 2, tail, 1.0, missing=False)
    check_distill(c, 12, tail, ids_t=(ids, t))


@pytest.mark.parametrize("tail", [False, True], ids=["renormalised", "tail"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("V", [300, 4500])
def test_distill_left_out_masked_and_bad_rows(V, dtype, tail):
    rows = 10
    c = Case(rows, V, dtype, 41, True, n=rows)
    ids, t = teacher(c, 6, 3, tail, 1.0, missing=False)
    ids[1] = -1                                  # no entries
    t[2] = -INF
    weight = torch.ones(rows)
    weight[3] = 0.0
    c.long[3, 0] = float("nan")                  # not read
    c.long[4, :] = torch.where(torch.arange(V) % 3 == 0, c.long[4].float(), -INF).to(dtype)   # a mask
    c.long[4, ids[4].long()] = 1.0
    c.long[5, V // 2:] = LOW[dtype]              # a mask of the type's lowest value
    c.long[5, ids[5].long()] = 0.5
    ids[6, 2] = V + 3                            # not a column: left out
    c.size = lambda: torch.full((rows,), 40.0).double()
    good = Case.__new__(Case)
    good.__dict__.update(c.__dict__)
    good.long = c.long.clone()
    good.long[3] = 0.0
    # the reference has no NaN row to skip
    loss, g, ga, gb, status = check_distill(good, 6, tail, weight=weight, ids_t=(ids, t))
    assert status == dels.DELS_STATUS_BAD_TOKEN
    d = dels.Distiller(rows, V, 6, dtype, n_weights=rows, tail=tail, device=DEV)
    c.short[7, 1] = float("nan")
    c.long[8, 2] = INF
    t[9, 0] = float("nan")
    args = dict(long=c.dev("long"), row_weight=weight.to(DEV), **c.kwargs())
    out = d.step(c.dev("short"), ids.to(DEV), t.to(DEV), **args)
    assert d.status() == dels.DELS_STATUS_BAD_TOKEN | dels.DELS_STATUS_NONFINITE
    assert torch.isnan(out[0][7:]).all() and torch.isnan(out[1][7:].float()).all()
    assert torch.isnan(out[2][7:]).all() and torch.isnan(out[3][7:]).all()
    for r in (1, 2, 3):
        assert out[0][r] == 0 and (out[1][r] == 0).all() and out[2][r] == 0 and out[3][r] == 0
    assert torch.equal(out[0][:7], loss[:7]) and torch.equal(out[1][:7], g[:7])
    c.short[:], c.long[:] = 0.0, -INF            # nothing left in any row
    out = d.step(c.dev("short"), ids.to(DEV), t.to(DEV), long=c.dev("long"), row_weight=weight.to(DEV), **c.kwargs())
    assert torch.isnan(out[0][[0, 4, 5, 6, 7, 8, 9]]).all() and d.status() & dels.DELS_STATUS_NONFINITE


def test_distill_peaked_rows_keep_their_digits():
    """A student and a teacher that are both nearly certain: losses of 1e-4 and less, tails of 1e-5. The loss and the
    tail's gradient hold to 1e-3 of themselves (a sum next to 1 would keep 6e-8 of 1: 6e-3 of a tail of 1e-5)."""
    V, rows = 6000, 4
    c = Case(rows, V, torch.float32, 51, False, scale=1.0)
    c.long[:, 77] = torch.tensor([19.0, 20.0, 20.5, 21.0])
    z = c.long.double().clone()
    z[:, 77] += 0.5
    lp, i = torch.log_softmax(z, -1).topk(4, -1)
    ids, t = i.to(torch.int32), lp.float()
    ref = reference(c, ids, t, True, 1.0, torch.ones(rows).double(), torch.ones(rows).double())
    d = dels.Distiller(rows, V, 4, torch.float32, tail=True, device=DEV)
    loss, g, _, _ = d.step(c.dev("long"), ids.to(DEV), t.to(DEV))
    assert ((loss.cpu().double() - ref[0]).abs() <= 1e-3 * ref[0].abs()).all()
    assert ((g.cpu().double() - ref[1]).norm(dim=-1) <= 1e-3 * ref[1].norm(dim=-1)).all()


def test_distill_learns_from_what_scoring_writes():
    """The teacher's table is the scorer's output; at the teacher's own logits the loss and its gradient vanish."""
    rows, V, K = 9, 7000, 32
    x = (torch.randn(rows, V, generator=gen(61)) * 3).to(DEV)
    x[4, 20:] = -INF                               # fewer entries than K
    ids, lp = dels.TokenScorer(rows, V, K, device=DEV)(x)[2:]
    for tail in (False, True):
        d = dels.Distiller(rows, V, K, torch.float32, tail=tail, device=DEV)
        loss, g, ga, gb = d.step(x, ids, lp)
        assert d.status() == 0 and ga is None and gb is None
        if tail:
            assert (loss.abs() < 1e-5).all() and (g.abs() < 1e-5).all()
        else:
            assert (loss >= -1e-6).all()


def test_distill_rows_of_many_weights_and_none():
    """More weights than rows: those without rows get 0."""
    c = Case(3, 500, torch.float32, 71, True, n=8)
    ids, t = teacher(c, 4, 1, False, 1.0)
    d = dels.Distiller(3, 500, 4, torch.float32, n_weights=8, device=DEV)
    _, _, ga, gb = d.step(c.dev("short"), ids.to(DEV), t.to(DEV), long=c.dev("long"), **c.kwargs())
    assert (ga[3:] == 0).all() and (gb[3:] == 0).all() and (ga[:3] != 0).all()
    d = dels.Distiller(3, 500, 4, torch.float32, device=DEV)
    _, _, ga, gb = d.step(c.dev("short"), ids.to(DEV), t.to(DEV), long=c.dev("long"))
    assert ga is None and gb is None


def test_distill_repeats_its_bits():
    c = Case(20, 40001, torch.bfloat16, 81, True, n=4)
    ids, t = teacher(c, 50, 1, True, 1.0)
    d = dels.Distiller(20, 40001, 50, torch.bfloat16, n_weights=4, tail=True, device=DEV)
    args = (c.dev("short"), ids.to(DEV), t.to(DEV))
    kw = dict(long=c.dev("long"), **c.kwargs())
    first = [v.clone() for v in d.step(*args, **kw)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(3):
            again = d.step(*args, **kw)
    torch.cuda.synchronize()
    for u, v in zip(first, again):
        assert torch.equal(u, v)


def test_distill_refusals():
    c = Case(3, 64, torch.float32, 91, True, n=3)
    ids, t = teacher(c, 4, 1, False, 1.0)
    d = dels.Distiller(3, 64, 4, torch.float32, n_weights=3, device=DEV)
    short, long, kw = c.dev("short"), c.dev("long"), c.kwargs()
    ids, t = ids.to(DEV), t.to(DEV)
    with pytest.raises(ValueError):
        d.step(short, ids[:, :3].contiguous(), t[:, :3].contiguous(), long=long, **kw)      # another k
    with pytest.raises(ValueError):
        d.step(short.bfloat16(), ids, t, long=long, **kw)                                   # another type
    with pytest.raises(ValueError):
        d.step(short, ids.long(), t, long=long, **kw)
    with pytest.raises(ValueError):
        d.step(short, ids, t.cpu(), long=long, **kw)
    with pytest.raises(ValueError):
        d.step(short, ids, t, long=long.bfloat16(), **kw)
    with pytest.raises(ValueError):
        d.step(short, ids, t, long=long, **dict(kw, alpha=kw["alpha"][:2].contiguous()))
    with pytest.raises(ValueError):
        d.step(short.t().contiguous().t(), ids, t, long=long, **kw)                         # columns are not dense
    with pytest.raises(ValueError):
        d.step(short, ids, t, long=long, out=short[:1].expand(3, 64), **kw)                 # rows overlap
    with pytest.raises(ValueError):
        d.step(short[:1].expand(3, 64), ids, t, long=long, **kw)
    with pytest.raises(dels.DelsError):
        dels.Distiller(3, (1 << 22) + 1, 4, torch.float32, device=DEV)
    with pytest.raises(ValueError):
        dels.TokenScorer(3, 64, 4, device=DEV)(long.cpu())
    with pytest.raises(dels.DelsError):
        dels.TokenScorer(3, 64, 257, device=DEV)(long)
    with pytest.raises(dels.DelsError):
        dels.TokenScorer(3, 64, 2, device=DEV)(long, temperature=0.0)


def test_row_ops_with_no_rows():
    z = torch.empty(0, 50, device=DEV)
    assert dels.TokenScorer(0, 50, 3, device=DEV)(z, torch.empty(0, dtype=torch.int32, device=DEV))[0].numel() == 0
    d = dels.Distiller(0, 50, 2, torch.float32, n_weights=2, device=DEV)
    w = torch.ones(2, device=DEV)
    out = d.step(z, torch.empty(0, 2, dtype=torch.int32, device=DEV), torch.empty(0, 2, device=DEV), alpha=w)
    assert out[0].numel() == 0 and (out[2] == 0).all()


def test_row_ops_under_a_graph():
    """Both operators captured in one CUDA graph and replayed on new inputs."""
    rows, V, K = 16, 5000, 8
    x, s = torch.empty(rows, V, device=DEV), torch.empty(rows, V, device=DEV)
    sc, d = dels.TokenScorer(rows, V, K, device=DEV), dels.Distiller(rows, V, K, torch.float32, tail=True, device=DEV)

    def both():
        _, ent, ids, lp = sc(x)
        return (ent, ids, lp) + d.step(s, ids, lp)[:2]

    x.normal_()
    s.normal_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = both()
    for seed in (1, 2):
        torch.manual_seed(seed)
        x.normal_()
        s.normal_()
        g.replay()
        torch.cuda.synchronize()
        got = [v.clone() for v in out]
        for u, v in zip(got, both()):
            assert torch.equal(u, v)
