"""distill_loss and the handles around the library's calls (no GPU needed: the calls are stubbed
and the structures take host tensors): what backward() passes, what is refused, what is marked as written."""
import os

import pytest
import torch
from torch.utils.checkpoint import checkpoint

import paper_2607_07409_gb300 as dels

ROWS, V, K = 4, 24, 3


class Stub:
    """The library, but for the calls that launch: they keep the structures they were given."""

    def __init__(self, real):
        self.real, self.seen = real, []

    def __getattr__(self, name):
        return getattr(self.real, name)

    def dels_distill_loss(self, x, rows, v, t, loss, state, *rest):
        self.seen.append(("loss", x._obj, t._obj, state))
        return 0

    def dels_distill_grad(self, x, rows, v, t, up, state, *rest):
        self.seen.append(("grad", x._obj, t._obj, state))
        return 0


def host_rows(rows, v, long=None, short=None, log_prior=None, alpha=None, beta=None, temperature=1.0):
    x = dels.Rows()
    for name, t in (("long", long), ("short", short)):
        if t is not None:
            setattr(x, name + "_logits", t.data_ptr())
            setattr(x, name + "_stride", t.stride(0))
    for name, t in (("log_prior", log_prior), ("alpha", alpha), ("beta", beta)):
        if t is not None:
            setattr(x, name, t.data_ptr())
            x.n_weights = alpha.numel()
    x.temperature = temperature
    return x


def host_teacher(rows, ids, logprob, row_weight=None, tail=False):
    return dels.Teacher(ids.data_ptr(), logprob.data_ptr(), ids.shape[1], int(tail),
                        None if row_weight is None else row_weight.data_ptr())


@pytest.fixture
def stub(monkeypatch):
    if not os.path.exists(dels.library_path()):
        from paper_2607_07409_gb300 import build
        build.build()
    s = Stub(dels.lib())
    monkeypatch.setattr(dels, "lib", lambda: s)
    monkeypatch.setattr(dels, "rows_of", host_rows)
    monkeypatch.setattr(dels, "teacher_of", host_teacher)
    monkeypatch.setattr(dels, "_stream", lambda stream: None)
    monkeypatch.setattr(dels, "_current_device", lambda: -1, raising=False)    # a host tensor's get_device()
    return s


def inputs():
    return dict(short=torch.randn(ROWS, V), ids=torch.arange(ROWS * K, dtype=torch.int32).view(ROWS, K),
                logprob=torch.full((ROWS, K), -2.0), long=torch.randn(ROWS, V), log_prior=torch.zeros(V),
                alpha=torch.ones(2), beta=torch.ones(2), row_weight=torch.ones(ROWS))


def addresses(x, t):
    return dict(short=x.short_logits, long=x.long_logits, log_prior=x.log_prior, alpha=x.alpha, beta=x.beta, ids=t.ids,
                logprob=t.logprob, row_weight=t.row_weight)


def loss_of(v, **kw):
    v = dict(v)
    return dels.distill_loss(v.pop("short"), v.pop("ids"), v.pop("logprob"), **v, **kw)


def test_backward_takes_the_tensors_that_hooks_give_back(stub):
    """Hooks may give other tensors back than were saved (a copy from the host, one made again), whose rows may lie
    further apart; the first ones may be gone by then."""
    v = inputs()
    for name in ("short", "alpha", "beta"):
        v[name].requires_grad_()
    given = {}                                                # what unpack gave for the tensor saved from an address

    def pack(t):
        return t.data_ptr(), t.detach()

    def unpack(packed):
        at, t = packed
        if t.shape == (ROWS, V):
            wide = torch.zeros(ROWS, V + 5)
            wide[:, :V] = t
            new = wide[:, :V]
        else:
            new = t.clone()
        given[at] = new
        return new

    with torch.autograd.graph.saved_tensors_hooks(pack, unpack):
        loss = loss_of(v, tail=True, temperature=2.0)
    loss.sum().backward()
    (_, x0, t0, state0), (_, x1, t1, state1) = stub.seen
    for name, at in addresses(x0, t0).items():
        assert at == v[name].data_ptr(), name
    for name, at in addresses(x1, t1).items():
        assert at == given[v[name].data_ptr()].data_ptr(), name
    assert state1 == given[state0].data_ptr()
    assert x1.short_stride == x1.long_stride == V + 5
    assert x1.temperature == 2.0 and t1.tail == 1 and x1.n_weights == 2 and t1.k == K


def test_backward_under_checkpoint_takes_the_rows_made_again(stub):
    v = inputs()
    h, w = torch.randn(ROWS, 6), torch.randn(V, 6, requires_grad=True)
    made = []

    def head(h):
        made.append(h @ w.T)                                  # (kept here, so that the two differ in address)
        return loss_of(dict(v, short=made[-1]))

    checkpoint(head, h, use_reentrant=False).sum().backward()
    assert [kind for kind, *_ in stub.seen] == ["loss", "loss", "grad"] and len(made) == 2
    assert stub.seen[0][1].short_logits == made[0].data_ptr()
    assert stub.seen[2][1].short_logits == made[1].data_ptr() != made[0].data_ptr()


@pytest.mark.parametrize("name", ["long", "log_prior", "logprob", "row_weight"])
def test_tensors_without_a_gradient_may_not_require_one(stub, name):
    v = inputs()
    v["short"].requires_grad_()
    v[name].requires_grad_()
    with pytest.raises(ValueError, match=name):
        loss_of(v)
    assert not stub.seen
    with torch.no_grad():                                     # nothing is recorded: nothing is lost
        loss_of(v)
    loss_of(dict(v, **{name: v[name].detach()})).sum().backward()
    assert [kind for kind, *_ in stub.seen] == ["loss", "loss", "grad"] and v["short"].grad is not None


def test_tensors_of_another_device_than_the_current_one_are_refused(stub, monkeypatch):
    """The library launches on the current device, on its stream."""
    v = inputs()
    loss_of(dict(v, short=v["short"].requires_grad_()))
    calls = len(stub.seen)
    sc = dels.TokenScorer.__new__(dels.TokenScorer)
    sc.rows, sc.V, sc.top_k, sc._dev = ROWS, V, 0, -1
    d = dels.Distiller.__new__(dels.Distiller)
    d.rows, d.V, d.k, d.dtype, d.n_weights, d.tail, d.temperature, d._dev = ROWS, V, K, torch.float32, 2, False, 1.0, -1
    for o in (sc, d):
        o._own, o._call = [0] * 5, lambda *a: pytest.fail("the library was called")
    d._loss, d._grad_w, d._state, d._grad, d.ws_bytes = v["long"], (), v["long"], v["long"], 0
    monkeypatch.setattr(dels, "_current_device", lambda: 0)
    for call in (lambda: loss_of(v), lambda: sc(v["long"]), lambda: d.step(v["short"], v["ids"], v["logprob"]),
                 lambda: d.loss(v["short"], v["ids"], v["logprob"])):
        with pytest.raises(ValueError, match="current device"):
            call()
    assert len(stub.seen) == calls
    with torch.autograd.graph.saved_tensors_hooks(lambda t: t.clone(), lambda t: t):
        monkeypatch.setattr(dels, "_current_device", lambda: -1)
        loss = loss_of(v)
    monkeypatch.setattr(dels, "_current_device", lambda: 0)
    with pytest.raises(ValueError, match="current device"):
        loss.sum().backward()
