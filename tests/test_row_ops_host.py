"""Host-side checks of the scoring and distillation entry points (no GPU needed):
bad arguments are refused before a device is touched."""
import ctypes
import os

import pytest
import torch


@pytest.fixture(scope="module")
def dels():
    import paper_2607_07409_gb300 as m
    if not os.path.exists(m.library_path()):
        from paper_2607_07409_gb300 import build
        build.build()
    m.lib()
    return m


def rows(dels, **kw):
    x = dels.Rows()
    x.long_logits, x.dtype, x.temperature = 4096, 0, 1.0
    for k, v in kw.items():
        setattr(x, k, v)
    return ctypes.byref(x)


def teacher(dels, **kw):
    t = dels.Teacher()
    t.ids, t.logprob, t.k = 16, 32, 4
    for k, v in kw.items():
        setattr(t, k, v)
    return ctypes.byref(t)


WS = 1 << 12   # an aligned address that is never read on the host


def score(dels, x, R=2, V=8, tok=64, K=2, lp=64, ent=64, ids=64, tlp=64, ws=WS, n=256):
    return dels.lib().dels_score_rows(x, R, V, tok, K, lp, ent, ids, tlp, ws, n, None)


def step(dels, x, t, R=2, V=8, loss=64, grad=4096, ld=0, ga=None, gb=None, ws=WS, n=1 << 20):
    return dels.lib().dels_distill_step(x, R, V, t, loss, grad, ld, ga, gb, ws, n, None)


def test_sizes(dels):
    assert dels.dels_score_workspace_bytes(3, 100) >= 4
    assert dels.dels_score_workspace_bytes(-1, 100) == 0 and dels.dels_score_workspace_bytes(1, 0) == 0
    assert dels.dels_score_workspace_bytes(1, (1 << 30) + 1) == 0
    assert dels.dels_distill_state_bytes(0) == 0 and dels.dels_distill_state_bytes(5) % 16 == 0
    assert dels.dels_distill_workspace_bytes(5, 100) >= 256 + dels.dels_distill_state_bytes(5)
    assert dels.dels_distill_workspace_bytes(5, (1 << 22) + 1) == 0


@pytest.mark.parametrize("code,kw,args", [
    (-3, dict(dtype=5), {}),
    (-2, {}, dict(R=-1)), (-2, {}, dict(V=0)), (-2, {}, dict(V=(1 << 30) + 1)),
    (-2, {}, dict(K=-1)), (-2, {}, dict(K=257)),
    (-2, dict(temperature=0.0), {}), (-2, dict(temperature=-1.0), {}), (-2, dict(temperature=float("nan")), {}),
    (-2, dict(temperature=float("inf")), {}), (-2, dict(temperature=1e-42), {}),
    (-2, dict(long_stride=7), {}), (-2, dict(long_stride=-8), {}), (-2, dict(short_logits=4096, short_stride=3), {}),
    (-2, dict(short_logits=4096, alpha=16, n_weights=0), {}), (-2, dict(n_weights=-1), {}),
    (-1, dict(long_logits=None), {}), (-1, {}, dict(tok=None)), (-1, {}, dict(ids=None)), (-1, {}, dict(tlp=None)),
    (-4, dict(long_logits=4098), {}), (-4, dict(log_prior=2), {}), (-4, {}, dict(ent=66)), (-4, {}, dict(ws=WS + 4)),
    (-5, {}, dict(ws=None)), (-5, {}, dict(n=255)),
    (0, {}, dict(R=0)),
])
def test_score_refusals(dels, code, kw, args):
    assert score(dels, rows(dels, **kw), **args) == code


def test_score_needs_rows_and_takes_none(dels):
    assert score(dels, None) == -1


@pytest.mark.parametrize("code,kw,tk,args", [
    (-3, dict(dtype=-1), {}, {}),
    (-2, {}, {}, dict(V=(1 << 22) + 1)), (-2, {}, {}, dict(R=-3)), (-2, {}, dict(k=0), {}), (-2, {}, dict(k=257), {}),
    (-2, {}, {}, dict(ld=7)),
    (-1, dict(short_logits=None), {}, {}), (-1, {}, dict(ids=None), {}), (-1, {}, dict(logprob=None), {}),
    (-1, {}, {}, dict(loss=None)), (-1, {}, {}, dict(grad=None)),
    (-1, {}, {}, dict(ga=64)),                                   # no alpha to have a gradient
    (-1, dict(beta=16, n_weights=1), {}, dict(gb=64)),           # beta without a prior
    (-4, {}, dict(ids=18), {}), (-4, {}, dict(row_weight=1), {}), (-4, {}, {}, dict(grad=4098)),
    (-4, dict(alpha=16, n_weights=1), {}, dict(ga=66)), (-4, {}, {}, dict(ws=WS + 8)),
    (-5, {}, {}, dict(ws=None)), (-5, {}, {}, dict(n=256)),
])
def test_distill_refusals(dels, code, kw, tk, args):
    kw = dict(dict(short_logits=8192), **kw)
    assert step(dels, rows(dels, **kw), teacher(dels, **tk), **args) == code


def test_distill_needs_its_structures(dels):
    assert step(dels, None, teacher(dels)) == -1
    assert step(dels, rows(dels, short_logits=8192), None) == -1


def test_binding_refuses_host_tensors(dels):
    x = torch.zeros(2, 8)
    with pytest.raises(ValueError):
        dels.rows_of(2, 8, x)
    with pytest.raises(ValueError):
        dels.rows_of(2, 8)
    with pytest.raises(ValueError):
        dels.teacher_of(2, torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, 3))
