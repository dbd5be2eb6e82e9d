"""distill_loss where PyTorch gives backward() other tensors than forward() had: rows made again under
checkpointing, tensors kept on the host, and what a call writes over."""
import pytest
import torch
from torch.utils.checkpoint import checkpoint

import paper_2607_07409_gb300 as dels
from test_gpu_row_ops import DEV, Case, teacher

pytestmark = pytest.mark.gpu

DTYPES = pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])


class Head:
    """A head's product before the loss, as a training loop has it."""

    def __init__(self, dtype, V, seed, rows=6, n=3, K=9):
        c = Case(rows, V, dtype, seed, True, n=n)
        g = torch.Generator().manual_seed(seed)
        ids, t = teacher(c, K, 3, True, 1.0)
        self.h = torch.randn(rows, 16, generator=g).to(DEV)
        self.w = (torch.randn(V, 16, generator=g) * 0.25).to(DEV).requires_grad_()
        self.alpha, self.beta = c.alpha.to(DEV).requires_grad_(), c.beta.to(DEV).requires_grad_()
        self.dtype, self.ids, self.t = dtype, ids.to(DEV), t.to(DEV)
        self.kw = dict(long=c.dev("long"), log_prior=c.prior.to(DEV), tail=True)
        self.up = (torch.rand(rows, generator=g) + 0.5).to(DEV)

    def loss(self, h):
        short = (h @ self.w.T).to(self.dtype)
        return dels.distill_loss(short, self.ids, self.t, alpha=self.alpha, beta=self.beta, **self.kw)

    def grads(self, loss):
        return torch.autograd.grad(loss, (self.w, self.alpha, self.beta), self.up)


@DTYPES
@pytest.mark.parametrize("V", [1001, 30000])
def test_gradients_under_checkpointing(V, dtype):
    """The first rows are freed after forward, others are written to their place before backward."""
    m = Head(dtype, V, 201)
    plain = m.grads(m.loss(m.h))
    loss = checkpoint(m.loss, m.h, use_reentrant=False)
    fill = [torch.full((6, V), 9.0, dtype=dtype, device=DEV) for _ in range(8)]
    again = m.grads(loss)
    for a, b in zip(plain, again):
        assert torch.equal(a, b)
    del fill


@DTYPES
def test_gradients_with_the_saved_tensors_on_the_host(dtype):
    m = Head(dtype, 5003, 202)
    plain = m.grads(m.loss(m.h))
    for pin in (False, True):
        with torch.autograd.graph.save_on_cpu(pin_memory=pin):
            loss = m.loss(m.h)
        for a, b in zip(plain, m.grads(loss)):
            assert torch.equal(a, b)


def test_gradients_of_rows_that_come_back_with_another_pitch():
    """Padded rows whose copies from the host are dense."""
    m = Head(torch.float32, 777, 203)
    wide = torch.zeros(6, 800, device=DEV)
    wide[:, :777] = (m.h @ m.w.T).detach()
    short = wide[:, :777].requires_grad_()

    def grads():
        loss = dels.distill_loss(short, m.ids, m.t, alpha=m.alpha, beta=m.beta, **m.kw)
        return lambda: torch.autograd.grad(loss, (short, m.alpha, m.beta), m.up)

    plain = grads()()
    with torch.autograd.graph.save_on_cpu():
        later = grads()
    for a, b in zip(plain, later()):
        assert torch.allclose(a, b, rtol=1e-5, atol=1e-7)      # (other alignments: the same sums in another order)


def two_batches(rows=6, V=3001):
    g = torch.Generator(DEV).manual_seed(204)
    return [torch.randn(rows, V, generator=g, device=DEV) * 3 for _ in range(2)]


def test_a_table_that_was_scored_over_is_refused():
    """The scorer's own table of one batch in a loss, and the next batch scored before the first one's backward."""
    first, second = two_batches()
    rows, V = first.shape
    sc = dels.TokenScorer(rows, V, 8, device=DEV)
    short = torch.randn(rows, V, device=DEV).requires_grad_()
    _, _, ids, lp = sc(first)
    loss = dels.distill_loss(short, ids, lp, tail=True)
    want = torch.autograd.grad(dels.distill_loss(short, ids.clone(), lp.clone(), tail=True).sum(), short)[0]
    assert torch.equal(torch.autograd.grad(loss.sum(), short, retain_graph=True)[0], want)
    kept = dels.distill_loss(short, ids.clone(), lp.clone(), tail=True)
    sc(second)
    with pytest.raises(RuntimeError):
        loss.sum().backward()
    assert torch.equal(torch.autograd.grad(kept.sum(), short)[0], want)      # a copy of the table outlasts it


def test_logits_that_a_step_wrote_over_are_refused():
    first, second = two_batches()
    rows, V = first.shape
    ids = torch.arange(rows * 4, dtype=torch.int32, device=DEV).view(rows, 4)
    lp = torch.full((rows, 4), -2.0, device=DEV)
    short = first.clone().requires_grad_()
    loss = dels.distill_loss(short, ids, lp)
    d = dels.Distiller(rows, V, 4, torch.float32, device=DEV)
    d.step(short, ids, lp)
    loss.sum().backward(retain_graph=True)                                   # another place: nothing has changed
    d.step(short, ids, lp, out=short)
    with pytest.raises(RuntimeError):
        loss.sum().backward()


def test_what_the_library_writes_is_marked_as_written():
    first, _ = two_batches()
    rows, V = first.shape
    ids = torch.arange(rows * 4, dtype=torch.int32, device=DEV).view(rows, 4)
    lp = torch.full((rows, 4), -2.0, device=DEV)
    w, prior = torch.ones(2, device=DEV), torch.zeros(V, device=DEV)
    tok = torch.zeros(rows, dtype=torch.int32, device=DEV)

    def moved(call, *written):
        before = [t._version for t in written]
        call()
        return all(t._version > b for t, b in zip(written, before))

    sc = dels.TokenScorer(rows, V, 4, device=DEV)
    assert moved(lambda: sc(first, tok), sc.logprob, sc.entropy, sc.top_ids, sc.top_logprob)
    d = dels.Distiller(rows, V, 4, torch.float32, n_weights=2, device=DEV)
    loss = d.loss(first, ids, lp)
    assert moved(lambda: d.loss(first, ids, lp), loss)
    kw = dict(long=first, log_prior=prior, alpha=w, beta=w)
    out = d.step(first, ids, lp, **kw)
    assert moved(lambda: d.step(first, ids, lp, **kw), *out)
    read = [first, ids, lp, w, prior]
    before = [t._version for t in read]
    d.step(first, ids, lp, **kw)
    assert [t._version for t in read] == before
    # the calls by their C names, tensors or addresses
    x, t = dels.rows_of(rows, V, first, first, prior, w, w), dels.teacher_of(rows, ids, lp)
    ws = torch.zeros(dels.dels_distill_workspace_bytes(rows, V), dtype=torch.uint8, device=DEV)
    state = torch.zeros(dels.dels_distill_state_bytes(rows), dtype=torch.uint8, device=DEV)
    los, g, ga, gb = torch.empty(rows, device=DEV), torch.empty_like(first), torch.empty_like(w), torch.empty_like(w)
    assert moved(lambda: dels.dels_distill_loss(x, rows, V, t, los, state, state.numel(), ws, ws.numel()), los, state)
    assert moved(lambda: dels.dels_distill_grad(x, rows, V, t, None, state, state.numel(), g, V, ga, gb), g, ga, gb)
    assert moved(lambda: dels.dels_distill_step(x, rows, V, t, los, g, V, ga, gb, ws, ws.numel()), los, g, ga, gb)
    ent, top, tlp = torch.empty(rows, device=DEV), torch.empty_like(ids), torch.empty_like(lp)
    assert moved(lambda: dels.dels_score_rows(x, rows, V, tok, 4, los, ent, top, tlp, ws, 256), los, ent, top, tlp)
    assert not moved(lambda: dels.dels_score_rows(x, rows, V, tok, 999, los, ent, top, tlp, ws, 256), los)   # refused
    assert dels.dels_score_rows(x, rows, V, tok, 4, los.data_ptr(), ent, top, tlp, ws, 256) == 0


def test_handles_under_inference_mode():
    first, _ = two_batches()
    rows, V = first.shape
    want = [t.clone() for t in dels.TokenScorer(rows, V, 4, device=DEV)(first)[1:]]
    with torch.inference_mode():
        sc = dels.TokenScorer(rows, V, 4, device=DEV)
        for a, b in zip(sc(first)[1:], want):
            assert torch.equal(a, b)
    for a, b in zip(sc(first)[1:], want):
        assert torch.equal(a, b)


@pytest.mark.parametrize("n", [7, 8, 9, 40])
def test_weights_gradients_by_the_steps_last_row_or_by_a_launch(n):
    """Both sides of the step's choice, and the engine's, which is always the launch: the same sums in the same order."""
    c = Case(12, 3001, torch.float32, 205, True, n=n)
    ids, t = teacher(c, 9, 3, True, 1.0)
    short, long, kw = c.dev("short"), c.dev("long"), c.kwargs()
    ids, t = ids.to(DEV), t.to(DEV)
    d = dels.Distiller(12, 3001, 9, torch.float32, n_weights=n, tail=True, device=DEV)
    for _ in range(3):                                        # (the count of the rows starts anew)
        _, _, ga, gb = d.step(short, ids, t, long=long, **kw)
        leaves = [kw["alpha"].requires_grad_(), kw["beta"].requires_grad_()]
        loss = dels.distill_loss(short, ids, t, long=long, tail=True, **kw)
        want = torch.autograd.grad(loss.sum(), leaves)
        kw = {k: v.detach() for k, v in kw.items()}
        assert torch.equal(ga, want[0]) and torch.equal(gb, want[1])


def test_a_step_with_many_weights_takes_no_serial_time():
    """The gradients of 20000 weights, one after another by one CTA, take some 40 ms; with a CTA each, microseconds."""
    rows, V, n = 16, 4096, 20000
    long, short = torch.randn(rows, V, device=DEV), torch.randn(rows, V, device=DEV)
    ids = torch.arange(rows * 4, dtype=torch.int32, device=DEV).view(rows, 4)
    lp = torch.full((rows, 4), -2.0, device=DEV)
    prior = torch.zeros(V, device=DEV)
    d = dels.Distiller(rows, V, 4, torch.float32, n_weights=n, tail=True, device=DEV)
    w = torch.ones(n, device=DEV)
    kw = dict(long=long, log_prior=prior, alpha=w, beta=w)
    for _ in range(3):
        _, _, ga, gb = d.step(short, ids, lp, **kw)
    assert (ga[rows:] == 0).all() and (gb[rows:] == 0).all() and (ga[:rows] != 0).any()
    ms = []
    for _ in range(5):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        d.step(short, ids, lp, **kw)
        b.record()
        torch.cuda.synchronize()
        ms.append(a.elapsed_time(b))
    assert min(ms) < 4.0, ms
