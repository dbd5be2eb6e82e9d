"""Drafting and sampled verification with a 4-bit vocabulary matrix, against the oracle with the weights it stands for:
the parity rules and tolerances of the bf16 heads, whose features are rounded the same way."""
import numpy as np
import pytest
import torch

import oracle
import synth
import paper_2607_07409_gb300 as dels
from parity import LP_TOL_BF16, check_draft, record
from test_gpu_sampling import _check_verify, _learned_weights, _verify_raw

pytestmark = pytest.mark.gpu

DEV = "cuda:0"

HEADS = {
    "gru": synth.HeadSpec("gru", "bf16", 64, 128, 48),
    "mlp": synth.HeadSpec("mlp", "bf16", 48, 80, 80, window=2, n_layers=1),
    "mlp2": synth.HeadSpec("mlp", "bf16", 64, 96, 96, window=3, n_layers=2),
    "xfmr": synth.HeadSpec("xfmr", "bf16", 64, 256, 64, n_heads=4, max_pos=16),
    "markov": synth.HeadSpec("markov", "bf16", 0, 0, 272),
    "wide": synth.HeadSpec("markov", "bf16", 0, 0, 1040),
}


def quantised(w, group, zeros):
    """Codes, scales and zero points of W [V, K], and the matrix they stand for."""
    V, K = w.shape
    groups = -(-K // group)
    x = torch.zeros(V, groups * group)
    x[:, :K] = w.float().cpu()
    x = x.view(V, groups, group)
    if zeros:
        lo, hi = x.amin(-1), x.amax(-1)
        scale = ((hi - lo) / 15).clamp(min=1e-6).to(torch.bfloat16)
        zero = torch.round(-lo / scale.float()).clamp(0, 15)
    else:
        scale = (x.abs().amax(-1) / 7).clamp(min=1e-6).to(torch.bfloat16)
        zero = torch.full_like(scale, 8, dtype=torch.float32)
    codes = (torch.round(x / scale.float()[..., None]) + zero[..., None]).clamp(0, 15)
    stands = ((codes - zero[..., None]) * scale.float()[..., None]).view(V, -1)[:, :K].contiguous()
    codes = codes.to(torch.uint8).view(V, -1)[:, :K].contiguous()
    return codes, scale, zero.to(torch.uint8) if zeros else None, stands


def setup(kind, B, n, V, ldt, group=32, zeros=False, table=False):
    w = synth.stress(synth.Workload(kind + "4", B=B, n=n, V=V, logit_dtype=ldt, head=HEADS[kind], weight=0.5, seed=B + n))
    d = synth.make_inputs(w, device=DEV, target=False)
    W = {k[5:]: v for k, v in d.items() if k.startswith("head.")}
    codes, scale, zero, stands = quantised(W["w_vocab"], group, zeros)
    m = dels.pack_w4(codes.to(DEV), scale.to(DEV), None if zero is None else zero.to(DEV), group=group)
    W4 = dict(W, w_vocab=m)
    if table:
        W4["input_table"] = dels.gru_input_table(w.head, W, V)
    ref = {k: v.cpu() for k, v in dict(W, w_vocab=stands).items()}
    return w, d, W4, ref, oracle.make_head(w.head, ref)


CASES = [("gru", 1, 5, 1024, "bf16", 32, False, False), ("gru", 5, 4, 5000, "f32", 64, True, True),
         ("gru", 40, 3, 3008, "bf16", 32, True, True), ("mlp", 3, 6, 2056, "f32", 32, False, False),
         ("mlp2", 9, 4, 24008, "bf16", 64, True, False), ("xfmr", 8, 4, 4096, "f32", 128, True, False),
         ("xfmr", 17, 3, 1000, "bf16", 32, False, False), ("markov", 1, 8, 50008, "f32", 128, True, False),
         ("markov", 64, 2, 24008, "bf16", 64, False, False), ("markov", 100, 3, 2008, "f32", 32, True, False),
         ("markov", 128, 2, 1032, "bf16", 128, False, False), ("gru", 2, 1, 1024, "bf16", 32, False, True),
         # several tiles for every group of warps
         ("markov", 5, 2, 100008, "bf16", 128, True, False), ("markov", 2, 2, 100008, "f32", 32, False, False),
         ("gru", 12, 2, 100008, "bf16", 64, False, True), ("mlp", 20, 2, 60008, "bf16", 32, True, False),
         ("markov", 64, 2, 60008, "f32", 64, False, False),
         # tiles that several groups share
         ("wide", 1, 3, 3008, "bf16", 64, True, False), ("wide", 7, 2, 24008, "f32", 32, False, False),
         ("wide", 12, 2, 5000, "bf16", 128, True, False), ("wide", 40, 2, 2008, "f32", 64, False, False)]


@pytest.mark.parametrize("case", CASES, ids=lambda c: f"{c[0]}-{c[1]}-{c[3]}-{c[5]}")
def test_draft(case):
    w, d, W, _, head = setup(*case)
    prior = dels.dels_prior_from_counts(d["counts"]).to(DEV)
    dr = dels.Drafter(w.head, W, w.B, w.n, w.V)
    tok, lp, gap = dr(d["long"], prior, 0.5, 0.3)
    assert dr.status() == 0
    info = check_draft(tok.cpu().numpy(), lp.cpu().numpy(), gap.cpu().numpy(), head, d["long"].cpu(),
                       oracle.log_prior(d["counts"]), 0.5, 0.3, LP_TOL_BF16)
    record(f"4-bit {case}", info)
    a, b = _learned_weights(w.n)
    tok, lp, gap = dr(d["long"], prior, a, b)
    check_draft(tok.cpu().numpy(), lp.cpu().numpy(), gap.cpu().numpy(), head, d["long"].cpu(),
                oracle.log_prior(d["counts"]), np.array(a), np.array(b), LP_TOL_BF16)


@pytest.mark.parametrize("case", CASES, ids=lambda c: f"{c[0]}-{c[1]}-{c[3]}-{c[5]}")
def test_sampled_draft_and_its_verification(case):
    w, d, W, ref, head = setup(*case)
    prior = dels.dels_prior_from_counts(d["counts"]).to(DEV)
    a, b = _learned_weights(w.n)
    dr = dels.Drafter(w.head, W, w.B, w.n, w.V)
    tok, lp, gap, state = dr.sample(d["long"], prior, a, b, 23, 7)
    assert dr.status() == 0
    tok, lp, gap = tok.cpu().numpy(), lp.cpu().numpy(), gap.cpu().numpy()
    check_draft(tok, lp, gap, head, d["long"].cpu(), oracle.log_prior(d["counts"]), np.array(a), np.array(b),
                LP_TOL_BF16, sample=(23, 7))
    target = synth.make_target_logits(w, d["long"], device=DEV)
    acc, bonus, bgap, st = _verify_raw(w, d, W, a, b, tok, lp, state, target, prior)
    assert st == 0
    _check_verify(w, d, ref, a, b, tok, acc, bonus, bgap, target, 23, 7, LP_TOL_BF16)


def test_non_finite_logits_flag_their_request():
    w, d, W, _, head = setup("markov", 5, 3, 2008, "f32")
    prior = dels.dels_prior_from_counts(d["counts"]).to(DEV)
    dr = dels.Drafter(w.head, W, w.B, w.n, w.V)
    want = [t.clone() for t in dr(d["long"], prior, 0.5, 0.3)]
    for bad, at in [(float("nan"), 77), (float("inf"), 2007), (-float("inf"), slice(None))]:
        long = d["long"].clone()
        long[3, 1, at] = bad
        tok, lp, _ = dr(long, prior, 0.5, 0.3)
        assert dr.status() == dels.DELS_STATUS_NONFINITE
        assert tok[3, 1] == -1 and torch.isnan(lp[3, 1])
        keep = [0, 1, 2, 4]
        assert torch.equal(tok[keep], want[0][keep]) and torch.equal(lp[keep], want[1][keep])


def test_masked_logits():
    """-inf and the lowest value in the long logits: never drafted, and no part of the log-probabilities."""
    w, d, W, _, head = setup("mlp", 4, 4, 2056, "f32")
    prior = dels.dels_prior_from_counts(d["counts"]).to(DEV)
    long = d["long"].clone()
    long[:, :, 1000:] = -float("inf")
    long[:, :, :200] = torch.finfo(torch.float32).min
    dr = dels.Drafter(w.head, W, w.B, w.n, w.V)
    tok, lp, gap = dr(long, prior, 0.5, 0.3)
    assert dr.status() == 0 and ((tok >= 200) & (tok < 1000)).all()
    check_draft(tok.cpu().numpy(), lp.cpu().numpy(), gap.cpu().numpy(), head, long.cpu(), oracle.log_prior(d["counts"]),
                0.5, 0.3, LP_TOL_BF16)


def test_a_captured_block_replays():
    w, d, W, _, head = setup("gru", 5, 4, 5000, "f32", 64, True, True)
    prior = dels.dels_prior_from_counts(d["counts"]).to(DEV)
    dr = dels.Drafter(w.head, W, w.B, w.n, w.V)
    long = d["long"].clone()
    one = [t.clone() for t in dr(long, prior, 0.5, 0.3)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = dr(long, prior, 0.5, 0.3)
    for t in out:
        t.zero_()
    graph.replay()
    graph.replay()
    assert all(torch.equal(a, b) for a, b in zip(one, out))
    long.mul_(0.5)
    graph.replay()
    two = [t.clone() for t in out]
    assert all(torch.equal(a, b) for a, b in zip(two, dr(long, prior, 0.5, 0.3)))


def test_refusals():
    w, d, W, _, _ = setup("markov", 2, 2, 1024, "f32")
    prior = dels.dels_prior_from_counts(d["counts"]).to(DEV)
    other = setup("markov", 2, 2, 1032, "f32")[2]["w_vocab"]
    dr = dels.Drafter(w.head, dict(W, w_vocab=other), w.B, w.n, w.V)
    with pytest.raises(dels.DelsError):        # of another vocabulary
        dr(d["long"], prior, 0.5, 0.3)
    import dataclasses
    for spec in (dataclasses.replace(w.head, d_rank=288), dataclasses.replace(w.head, wdtype="f32")):
        with pytest.raises(dels.DelsError):    # of another feature width; a float32 head
            dels.Drafter(spec, W, w.B, w.n, w.V)
