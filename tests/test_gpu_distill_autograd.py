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
