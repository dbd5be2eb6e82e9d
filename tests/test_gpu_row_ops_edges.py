"""Scoring and distillation of vocabulary rows where the kernels change their way of
working: entries far above a row's first ones, masks in the local head's logits, terms
that are absent or lie differently against 16-byte boundaries, slices that leave room
for one CTA on an SM or none, the largest vocabularies. Bounds as in test_gpu_row_ops."""
import math

import pytest
import torch

import paper_2607_07409_gb300 as dels
from test_gpu_row_ops import DEV, INF, LOW, Case, check_distill, check_score, eps_sum, gen, put, teacher

pytestmark = pytest.mark.gpu

DTYPES = pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
TAIL = pytest.mark.parametrize("tail", [False, True], ids=["renormalised", "tail"])
VIA = pytest.mark.parametrize("via", ["step", "autograd"])


class Placed(Case):
    """A Case whose tensors on the device differ from the ones it computes with: `absent` ones are not passed
    (they are zero on the host), `offsets` of their own, `masked` columns of the local head at -inf (on the host
    the drafter's are, and the local head's are 0 there: the same rows, and sums without 0 * inf)."""

    def __init__(self, *args, absent=(), offsets=None, **kw):
        super().__init__(*args, **kw)
        self.absent, self.offsets, self.masked = absent, offsets or {}, None
        for name in absent:
            getattr(self, name).zero_()

    def mask(self, columns):
        self.masked = columns
        self.long[:, columns] = -INF
        self.short[:, columns] = 0.0
        self.plain_long = torch.zeros_like(self.long)

    def dev(self, name):
        if name in self.absent:
            return None
        t = getattr(self, name)
        if self.masked is not None and name in ("long", "short"):
            t = t.clone()
            t[:, self.masked] = -INF if name == "short" else 1.0
        if name == "prior":
            t = put(t[None], self.offsets.get(name, 0))[0]
            return t
        return put(t, self.offsets.get(name, self.offset), self.pitch) if t.dim() == 2 else t.to(DEV)


@DTYPES
@TAIL
@VIA
@pytest.mark.parametrize("fused", [False, True], ids=["plain", "fused"])
def test_distill_entries_far_above_the_first(fused, via, tail, dtype):
    """Unlisted entries up to e^10000 times as likely as those that a row begins with, and rows that begin with such."""
    V, rows = 20000, 8
    c = Case(rows, V, dtype, 101, fused, n=3)
    ids, t = teacher(c, 9, 3, tail, 1.0, missing=False)
    free = [v for v in range(V - 1, 0, -1) if not (ids == v).any()]
    for r, far in enumerate((75.0, 90.0, 200.0, 1e4)):
        c.long[r, free[r]] = far
    c.long[4, free[4]] = c.long[4, free[5]] = 150.0
    first = [v for v in reversed(free) if v < 2000][:20]
    c.long[5, first] = 500.0                       # the rest has nothing beside these
    c.long[6, :16000] = torch.where(torch.arange(16000) % 2 == 0, -INF, c.long[6, :16000].float()).to(dtype)
    c.long[6, ids[6].long()] = 1.0
    c.long[7, :17000] = -INF                       # nothing in the first items of any lane
    c.long[7, ids[7].long()] = 2.0
    check_distill(c, 9, tail, ids_t=(ids, t), via=via)


@DTYPES
@VIA
@pytest.mark.parametrize("fused", [False, True], ids=["plain", "fused"])
def test_distill_entries_that_pass_the_range_together(fused, via, dtype):
    """Sums of warps that are finite each, and not together: 2^126.96 sixty-four times, and other sizes near it."""
    V, rows = 20000, 6
    c = Case(rows, V, dtype, 109, fused, n=2, scale=0.0)
    if fused:
        c.short *= 0.01
        c.prior *= 0.01
    ids = torch.tensor([[3, 9, 12345]] * rows, dtype=torch.int32)
    t = torch.log_softmax(torch.tensor([1.0, 0.5, 0.25, 0.0]), 0)[:3].expand(rows, 3).clone()
    for r, far in enumerate((88.0, 87.0, 86.0, 84.0, 70.0, 60.0)):
        c.long[r, 4000::250] = far
    check_distill(c, 3, True, ids_t=(ids, t), via=via)


@DTYPES
@pytest.mark.parametrize("V", [3001, 20000])
def test_row_ops_that_begin_with_the_lowest_value(V, dtype):
    """Rows whose first part is masked by the type's lowest value, in one term and in all that have it."""
    for fused in (False, True):
        c = Case(5, V, dtype, 110, fused, n=5)
        ids, t = teacher(c, 8, 3, True, 1.0, missing=False)
        for r in range(4):
            c.long[r, :V * (r + 1) // 5] = LOW[dtype]
            c.long[r, ids[r].long()] = 1.0
        c.size = lambda: torch.full((5,), 40.0).double()
        check_distill(c, 8, True, ids_t=(ids, t))
        check_distill(c, 8, False, ids_t=(ids, t), via="autograd")
        assert check_score(c, 64)[-1] == 0


@DTYPES
@TAIL
@VIA
def test_distill_masks_in_the_local_head(via, tail, dtype):
    """-inf among the local head's logits, listed ones too: no weight, no gradient, no NaN in the weights' gradients."""
    c = Placed(6, 9000, dtype, 102, fused=True, n=2)
    ids, t = teacher(c, 7, 3, tail, 1.0, missing=False)
    listed = set(ids.flatten().tolist())
    c.mask([v for v in range(0, 9000, 3) if v not in listed] + [8999 - v for v in range(40) if 8999 - v not in listed])
    _, g, ga, gb, _ = check_distill(c, 7, tail, ids_t=(ids, t), via=via)
    assert (g[:, c.masked] == 0).all() and torch.isfinite(ga).all() and torch.isfinite(gb).all()


@DTYPES
@VIA
@pytest.mark.parametrize("absent", [("long",), ("prior",), ("long", "prior")], ids="-".join)
@pytest.mark.parametrize("V", [777, 12000])
def test_distill_terms_may_be_absent(V, absent, via, dtype):
    """The prior's weight has no gradient without a prior."""
    c = Placed(5, V, dtype, 103, fused=True, n=3, absent=absent)
    ids, t = teacher(c, 6, 3, True, 1.0)
    kw = dict(long=c.dev("long"), log_prior=c.dev("prior"), alpha=c.dev("alpha"))
    if "prior" not in absent:
        check_distill(c, 6, True, ids_t=(ids, t), via=via)
        return
    # (the reference with a prior of zeros; its beta's gradient is zero)
    c2 = Case(5, V, dtype, 103, True, n=3)
    c2.long, c2.prior = c.long, c.prior
    loss, g, ga, _, _ = check_distill(c2, 6, True, ids_t=(ids, t), via=via)
    weight = (torch.rand(5, generator=gen(3)) + 0.5).to(DEV)
    short = c.dev("short")
    if via == "step":
        d = dels.Distiller(5, V, 6, dtype, n_weights=3, tail=True, device=DEV)
        loss1, g1, ga1, gb1 = d.step(short, ids.to(DEV), t.to(DEV), row_weight=weight, **kw)
        assert gb1 is None
    else:
        up = torch.rand(5, generator=gen(4)) + 0.5
        short, al = short.requires_grad_(), kw.pop("alpha").requires_grad_()
        loss1 = dels.distill_loss(short, ids.to(DEV), t.to(DEV), alpha=al, row_weight=weight, tail=True, **kw)
        g1, ga1 = torch.autograd.grad(loss1, (short, al), up.to(DEV))
    # the same numbers but for the order of their sums: twice the bounds that c2 holds
    e = 2 * (16 * 2.0 ** -24 * c2.size() + eps_sum(V) + 2.0 ** -18).to(DEV)
    assert ((loss1 - loss).abs().double() <= e * (2 + loss.abs().double() + math.log(V) + 20)).all()
    unit = 2.0 ** -7 if dtype is torch.bfloat16 else 2.0 ** -18
    assert ((g1 - g).double().norm(dim=-1) <= (unit + 8 * e) * g.double().norm(dim=-1)).all()
    assert ((ga1 - ga).abs().double() <= 8 * float(e.max()) * 5 * float(c2.short.abs().max())).all()


@DTYPES
@TAIL
@pytest.mark.parametrize("V", [1000, 5003, 30000])
@pytest.mark.parametrize("offsets", [dict(long=1), dict(short=3), dict(prior=1), dict(long=5, short=2, prior=3)],
                         ids=["long", "short", "prior", "all"])
def test_row_ops_terms_that_lie_differently(offsets, V, tail, dtype):
    """Terms whose rows begin at different places against 16-byte boundaries."""
    c = Placed(4, V, dtype, 104, fused=True, n=4, offsets=offsets)
    check_distill(c, 11, tail)
    if tail:
        assert check_score(c, 20)[-1] == 0
    else:
        check_distill(c, 11, tail, via="autograd")


@DTYPES
@pytest.mark.parametrize("fused", [False, True], ids=["plain", "fused"])
@pytest.mark.parametrize("rows,V,K", [(20, 151936, 16), (1000, 300, 4), (1, 420001, 9), (2, 1 << 22, 12)])
def test_distill_step_by_one_launch_or_two(rows, V, K, fused, dtype):
    """Sizes on both sides of the step's choice; in place, as the second launch reads what it overwrites."""
    c = Case(rows, V, dtype, 105, fused, n=4)
    a = [None if x is None else x.clone() for x in check_distill(c, K, True)[:4]]
    b = check_distill(c, K, True, in_place=True)
    for u, v in zip(a, b):
        assert u is None or torch.equal(u, v)


@DTYPES
def test_rows_past_the_last_whole_round(dtype):
    """More rows than the device takes at once, in two launches side by side: the rows of the second against the
    same rows alone, among them ones that are left out, and what the next call on the stream reads and overwrites."""
    V, rows, n = 151936, 152 * 4 + 40, 3
    g = torch.Generator(DEV).manual_seed(111)
    long = torch.empty(rows, V, dtype=dtype, device=DEV).normal_(0, 3, generator=g)
    short = torch.empty(rows, V, dtype=dtype, device=DEV).normal_(generator=g)
    prior = torch.log_softmax(torch.randn(V, device=DEV, generator=g), 0)
    alpha, beta = torch.tensor([0.5, 0.7, 0.2], device=DEV), torch.tensor([0.3, 0.1, 0.2], device=DEV)
    kw = dict(log_prior=prior, alpha=alpha, beta=beta)
    token = torch.randint(0, V, (rows,), device=DEV, generator=g, dtype=torch.int32)
    weight = torch.rand(rows, device=DEV, generator=g)
    token[-3], weight[-3] = -1, 0.0
    sc = dels.TokenScorer(rows, V, 8, device=DEV)
    d = dels.Distiller(rows, V, 8, dtype, n_weights=n, tail=True, device=DEV)
    for _ in range(2):
        score = sc(long, token, short=short, **kw)
        _, _, ids, lp = score
        target = lp - 0.1
        out = d.step(short, ids, target, long=long, row_weight=weight, **kw)
        copy = [x.clone() for x in score + out]                    # right behind them on the stream
    assert sc.status() == 0 and d.status() == 0
    for a, b in zip(copy, score + out):
        assert torch.equal(a, b)
    loss = dels.distill_loss(short, ids, target, long=long, row_weight=weight, tail=True, **kw)
    assert torch.equal(loss, out[0]) or (loss - out[0]).abs().max() <= 1e-4
    some = list(range(0, rows, 97)) + list(range(rows - 41, rows))
    first = torch.tensor([r for r in some if r % n == 0], device=DEV)
    kw1 = dict(log_prior=prior, alpha=alpha[:1], beta=beta[:1])
    alone = dels.TokenScorer(len(first), V, 8, device=DEV)(long[first], token[first], short=short[first], **kw1)
    assert torch.equal(alone[2], ids[first])
    for k in (0, 1, 3):
        assert torch.allclose(alone[k], score[k][first], rtol=0, atol=1e-4)
    d1 = dels.Distiller(len(first), V, 8, dtype, tail=True, device=DEV)
    alone = d1.step(short[first], ids[first], target[first], long=long[first], row_weight=weight[first], **kw1)
    assert torch.allclose(alone[0], out[0][first], rtol=0, atol=1e-4)
    # the order of sums differs: 2^-12 of a row's largest, and bf16's last place
    close = 2.0 ** -12 + (2.0 ** -7 if dtype is torch.bfloat16 else 0.0)
    a, b = alone[1].float(), out[1][first].float()
    assert ((a - b).abs() <= close * b.abs() + 2.0 ** -16 * b.abs().amax(-1, keepdim=True)).all()
    # the weights' gradients are the rows': each alone
    ga = torch.zeros(n, device=DEV, dtype=torch.float64)
    dl = dels.Distiller(rows, V, 8, dtype, n_weights=rows, tail=True, device=DEV)
    each = dl.step(short, ids, target, long=long, row_weight=weight, log_prior=prior, alpha=alpha.repeat(rows)[:rows],
                   beta=beta.repeat(rows)[:rows])
    ga.index_add_(0, torch.arange(rows, device=DEV) % n, each[2].double())
    assert ((ga - out[2]).abs() <= 1e-5 * each[2].double().abs().sum()).all()


def test_distill_is_differentiable_once():
    c = Case(3, 200, torch.float32, 106, False)
    ids, t = teacher(c, 4, 1, False, 1.0)
    short = c.dev("long").requires_grad_()
    loss = dels.distill_loss(short, ids.to(DEV), t.to(DEV)).sum()
    with pytest.raises(RuntimeError):
        torch.autograd.grad(loss, short, create_graph=True)
    loss = dels.distill_loss(short, ids.to(DEV), t.to(DEV)).sum()
    with torch.no_grad():
        short.add_(1.0)                            # what the gradient reads has changed
    with pytest.raises(RuntimeError):
        loss.backward()


@pytest.mark.parametrize("V", [150_000_001, 40_000_000])
def test_score_very_long_rows(V):
    """Alternatives and the token among hundreds of millions of columns, the first and the last of them too."""
    x = torch.empty(1, V, dtype=torch.bfloat16, device=DEV)
    x.normal_(generator=torch.Generator(DEV).manual_seed(107))
    at = torch.randperm(V // 1000, generator=gen(108))[:64] * 1000
    at[0], at[1] = 0, V - 1
    top = torch.arange(64, 0, -1).float() + 16.0
    x[0, at.to(DEV)] = top.to(torch.bfloat16).to(DEV)
    token = torch.tensor([V - 1], dtype=torch.int32, device=DEV)
    sc = dels.TokenScorer(1, V, 64, device=DEV)
    lp, ent, ids, tlp = sc(x, token)
    assert sc.status() == 0
    assert torch.equal(ids[0].cpu().long(), at)
    m, total, weighted = float(top[0]), 0.0, 0.0
    for part in x[0].split(1 << 24):
        z = part.double() - m
        total += float(z.exp().sum())
        weighted += float((z.exp() * z).sum())
    ln = math.log(total)
    tol = 2 * 8 * 2.0 ** -24 * m + eps_sum(V)
    assert ((tlp[0].cpu().double() - (top.double() - m - ln)).abs() <= tol).all()
    assert abs(float(lp[0]) - (float(top[1]) - m - ln)) <= tol
    assert abs(float(ent[0]) - (ln - weighted / total)) <= tol * (math.log(V) + 3)


def test_rows_past_the_last_whole_round_under_a_graph():
    """The two launches side by side captured, between calls of their own kind, and replayed on new inputs."""
    V, rows = 151936, 152 * 3 + 50
    long, short = (torch.empty(rows, V, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    alpha, prior = torch.ones(1, device=DEV), torch.full((V,), -math.log(V), device=DEV)
    sc = dels.TokenScorer(rows, V, 4, device=DEV)
    d = dels.Distiller(rows, V, 4, torch.bfloat16, tail=True, device=DEV)

    def calls():
        first = [x.clone() for x in sc(long, short=short, log_prior=prior, alpha=alpha)[1:]]
        return first + list(d.step(short, first[1], first[2] - 0.5, long=long, log_prior=prior, alpha=alpha)[:3])

    long.normal_(0, 2)
    short.normal_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls()
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = calls()
    for seed in (1, 2, 3):
        torch.manual_seed(seed)
        long.normal_(0, 2)
        short.normal_()
        g.replay()
        got = [x.clone() for x in out]
        for a, b in zip(got, calls()):
            assert torch.equal(a, b)
