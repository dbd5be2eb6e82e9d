"""Distillation of rows whose first columns say nothing of their largest: the references that the sums
are relative to then lie far below them. Bounds as in test_gpu_row_ops."""
import pytest
import torch

import paper_2607_07409_gb300 as dels
from test_gpu_row_ops import DEV, INF, Case, check_distill, eps_sum, gen, reference, teacher

pytestmark = pytest.mark.gpu

DTYPES = pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
VIA = pytest.mark.parametrize("via", ["step", "autograd"])
V = 20000
# columns that are in the first items of no warp, with one CTA a row and with two (a slice of 10240 columns)
LATE = [v for v in range(V) if v % 10240 >= 6000]


def low_first(rows, dtype, fused, seed, low, others, listed):
    """Rows of about `low`, but for 3 listed late columns and every 100th late one that is not listed."""
    c = Case(rows, V, dtype, seed, fused, n=2, scale=0.25)
    if fused:
        c.short *= 0.05
        c.prior *= 0.05
    c.long += low
    ids = torch.tensor([[LATE[11], LATE[1017], LATE[-30]]] * rows, dtype=torch.int32)
    for r in range(rows):
        c.long[r, LATE[50::100]] = others[r] + 0.25 * torch.randn(len(LATE[50::100]), generator=gen(seed + r)).to(dtype)
        c.long[r, ids[r].long()] = torch.tensor(listed).to(dtype)
    t = torch.log_softmax(torch.tensor([1.0, 0.5, 0.25, 0.5]), 0)[:3].expand(rows, 3).clone()
    return c, ids, t


@DTYPES
@VIA
@pytest.mark.parametrize("fused", [False, True], ids=["plain", "fused"])
@pytest.mark.parametrize("low,T", [(-42.5, 1.0), (-50.0, 1.0), (-60.0, 1.0), (-25.0, 0.5), (-6.0, 0.125)])
def test_tail_next_to_listed_ids_far_above_the_first_columns(low, T, fused, via, dtype):
    """Listed entries and others of the same size, 42 to 60 (times T) above the first columns."""
    c, ids, t = low_first(6, dtype, fused, 301, low, [-2.0 * T, 0.0, 5.0 * T, -8.0 * T, 2.0 * T, -20.0 * T],
                          [0.1 * T, 0.0, -0.2 * T])
    for tail in (True, False):
        check_distill(c, 3, tail, T, ids_t=(ids, t), via=via)


@DTYPES
@VIA
@pytest.mark.parametrize("fused", [False, True], ids=["plain", "fused"])
def test_entries_that_are_not_listed_beside_listed_ones_past_the_range(fused, via, dtype):
    """Listed entries 2^120 to 2^140 times as likely as the first columns, others 2^20 to 2^40 times less than they:
    their gradients, of 1e-12 to 1e-6, hold to their own digits."""
    c, ids, t = low_first(5, dtype, fused, 302, -84.0, [-14.0, -18.0, -20.0, -25.0, -28.0], [4.0, 1.0, 0.0])
    for r, up in enumerate((0.0, 3.0, 4.0, 6.0, 9.0)):
        c.long[r, ids[r].long()] += up
    check_distill(c, 3, False, ids_t=(ids, t), via=via)
    check_distill(c, 3, True, ids_t=(ids, t), via=via)


def weight_grads_of(c, ids, t, via, w):
    """The weights' gradients by the step or by the engine."""
    kw = dict(long=c.dev("long"), row_weight=w.to(DEV), **c.kwargs())
    short, ids, t = c.dev("short"), ids.to(DEV), t.to(DEV)
    if via == "step":
        d = dels.Distiller(c.rows, c.V, ids.shape[1], c.dtype, n_weights=c.alpha.numel(), tail=True, device=DEV)
        return [g.cpu().double() for g in d.step(short, ids, t, **kw)[2:]]
    leaves = [kw["alpha"].requires_grad_(), kw["beta"].requires_grad_()]
    loss = dels.distill_loss(short, ids, t, tail=True, **kw)
    return [g.cpu().double() for g in torch.autograd.grad(loss.sum(), leaves)]


def centred_bound(c, ids, t, w, lq, terms, around):
    """The bound of a sum over the columns of gradient entries times what `terms` have beside `around`, one of them:
    the entries' own bounds (as in check_distill, the fused value's size being that of its last operations, since a
    product is not rounded before it is added), and 2^-20 of the sum of the products."""
    size = (c.long.double() + c.at(c.alpha).double() * c.short.double()).abs().amax(-1) \
        + (c.at(c.beta).double() * c.prior.double()).abs().amax(-1)
    e = (2 * 8 * 2.0 ** -24 * size + eps_sum(c.V) + 2.0 ** -23 * float(t[t > -INF].abs().max()) + 2.0 ** -20)[:, None]
    q, p = lq.exp(), torch.zeros_like(lq)
    p.scatter_add_(1, ids.long(), t.double().exp())
    rest = (1 - p.sum(-1, keepdim=True)).clamp(min=0.0)
    q_t = q.masked_fill(p > 0, 0.0).sum(-1, keepdim=True)
    per = 2 * e * (q + p) + q * (2.0 ** -21 + 2 * e * rest) / q_t + 2.0 ** -20 * (q + p * (1 + rest / q_t))
    far = (terms.double() - around).abs()
    far = far + torch.where(far < 1e3, far, torch.zeros_like(far)).amax(-1, keepdim=True)   # (the reference is one of them)
    return (w.double()[:, None] * per * far).sum(-1)


@VIA
@pytest.mark.parametrize("V", [3001, 20000])
def test_the_gradient_of_alpha_where_the_heads_logits_share_an_offset(V, via):
    """A row's gradient sums to zero: an offset of 2^14 in l_S, which l_L takes away again, changes no gradient. (The
    sums of products with the logits themselves would be off by some 2^-22 of it.)"""
    c = Case(6, V, torch.float32, 303, True, n=6)
    ids, t = teacher(c, 7, 3, True, 1.0, missing=False)
    c.short = c.short + 16384.0
    c.long = (c.long.double() - c.at(c.alpha).double() * 16384.0).float()
    w = torch.rand(6, generator=gen(3)) + 0.5
    ref = reference(c, ids, t, True, 1.0, w.double(), torch.ones(6).double())
    got = weight_grads_of(c, ids, t, via, w)
    bound = centred_bound(c, ids, t, w, ref[4], c.short, 16384.0)
    assert ((got[0] - ref[2]).abs() <= bound).all(), ((got[0] - ref[2]).abs() / bound).max()


@VIA
@pytest.mark.parametrize("V", [3001, 20000])
@pytest.mark.parametrize("far", [-1e6, -1e9])
def test_the_gradient_of_beta_where_the_prior_has_values_far_below(far, V, via):
    """Some of the prior's values far below the others (columns that l_L masks, the middle one and every 7th): they
    have no part in a gradient, and take no digits from it."""
    c = Case(6, V, torch.float32, 304, True, n=6)
    ids, t = teacher(c, 7, 3, True, 1.0, missing=False)
    listed = set(ids.flatten().tolist())
    gone = [v for v in sorted({V // 2, *range(0, V, 7)} - {V // 4, V - 1 - V // 4}) if v not in listed]
    c.long[:, gone] = -INF
    c.prior[gone] = 0.0                                       # (the reference's rows: the same columns without weight)
    w = torch.rand(6, generator=gen(3)) + 0.5
    ref = reference(c, ids, t, True, 1.0, w.double(), torch.ones(6).double())
    # (the others' largest sets the bound: columns of no weight take no part in it)
    c.long[:, gone] = 0.0
    bound = centred_bound(c, ids, t, w, ref[4], c.prior, float(c.prior[c.prior != 0].median()))
    c.long[:, gone] = -INF
    c.prior[gone] = far
    got = weight_grads_of(c, ids, t, via, w)
    assert ((got[1] - ref[3]).abs() <= bound).all(), ((got[1] - ref[3]).abs() / bound).max()
    assert ((got[0] - ref[2]).abs() <= 16 * bound).all()
