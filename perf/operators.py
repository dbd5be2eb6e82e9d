"""Cases of the row operators over the vocabulary: scoring and distillation.

Scoring gives the log-probability of one token of each row, the row's entropy
and its most likely alternatives, of plain logit rows or of the fused rows
``l = l_L + alpha l_S - beta l_P``. Distillation takes a teacher's top ids and
log-probabilities of each row (what scoring the target's rows gives) and
returns the Kullback-Leibler loss of the fused student rows, the gradient of
the local head's logits ``l_S`` and those of the fusion weights. Kinds:

* ``score``     one call of ``TokenScorer``
* ``loss``      the loss alone, as an evaluation takes it (``Distiller.loss``)
* ``step``      loss and gradients in one call, as a training step takes them (``Distiller.step``)
* ``autograd``  loss and gradients through ``distill_loss`` and PyTorch's engine, under a gradient of the losses

Where ``own`` is false the same values come from elementary float32 torch
operations. Logit rows are N(0, 3) with one likely token 0.5 to 8 above the
rest, as a language model's rows have; the last columns of a padded vocabulary
are -inf; the local head's logits are N(0, 1); a teacher's row is the
drafter's plus N(0, 2).
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}


def _score(rows, V, dtype, top_k, **kw):
    return dict(dict(kind="score", rows=rows, V=V, dtype=dtype, top_k=top_k, fused=False, n=1, pad=0, pitch=0,
                     temperature=1.0, left_out=False), **kw)


def _distill(kind, rows, V, dtype, top_k, **kw):
    return dict(dict(kind=kind, rows=rows, V=V, dtype=dtype, top_k=top_k, fused=True, n=1, pad=0, tail=True,
                     temperature=1.0, left_out=False), **kw)


def listed():
    return [
        # The smallest call: scoring one toy block of 8 float32 positions. Launches and latency.
        dict(_score(8, 1024, "f32", 8), name="score_tiny"),
        # One token of one request while it is served: its log-probability and 20 alternatives.
        dict(_score(1, 151936, "bf16", 20, pad=256), name="score_one_token"),
        # The drafted tokens of 8 requests under the fused rows that drew them, float32 logits.
        dict(_score(128, 151936, "f32", 8, fused=True, n=16), name="score_fused_b8"),
        # A teacher's table: the 64 most likely tokens of the target's rows for 64 blocks of 16.
        dict(_score(1024, 151936, "bf16", 64, pad=256), name="score_teacher_b64"),
        # A ragged batch of log-probabilities at temperature 0.7: odd vocabulary, padded prompt positions left out.
        dict(_score(297, 50257, "bf16", 5, left_out=True, temperature=0.7), name="score_ragged"),
        # Distilling a toy float32 head, 8 positions.
        dict(_distill("step", 8, 1024, "f32", 16, n=8), name="step_tiny"),
        # The training step of a head on 64 blocks of 16, bf16 logits: 64 teacher entries and the rest as one.
        dict(_distill("step", 1024, 151936, "bf16", 64, n=16, pad=256), name="step_b64"),
        # The same for float32 logits of an odd vocabulary at temperature 2, the teacher's entries renormalised,
        # prompt positions left out.
        dict(_distill("step", 297, 32003, "f32", 17, n=11, tail=False, temperature=2.0, left_out=True),
             name="step_ragged"),
        # A short sequence's step: 16 positions of one block, full vocabulary.
        dict(_distill("step", 16, 151936, "bf16", 128, n=16), name="step_one_block"),
        # Evaluating a plain student (no drafter beside it) on 32 blocks of 8.
        dict(_distill("loss", 256, 128256, "bf16", 32, fused=False, tail=False), name="loss_plain"),
        # A training loop that goes through autograd: forward, then the gradient of a weighted sum of the losses.
        dict(_distill("autograd", 256, 151936, "f32", 32, n=16), name="autograd_b16"),
    ]


# ------------------------------------------------------------------ drawing

def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["score", "score", "step", "step", "loss", "autograd"])
    V = rng.choice([32000, 32003, 50257, 128256, 151936, _log_int(rng, 1000, 151936), _log_int(rng, 1000, 151936)])
    dtype = rng.choice(["f32", "bf16"])
    most = 1024 * 151936 // (V * (2 if dtype == "f32" else 1))
    rows = _log_int(rng, 1, min(most, 4096))
    n = rng.choice([1, 7, 8, 16])
    pad = rng.choice([0, 0, 64, V // 500])
    if kind == "score":
        # odd pitches too: a row of another alignment than the one before it
        pitch = rng.choice([0, 0, V + rng.randint(1, 128)])
        return _score(rows, V, dtype, rng.choice([0, 1, 5, 20, 64, 128]), fused=rng.random() < 0.4, n=n, pad=pad,
                      pitch=pitch, temperature=rng.choice([1.0, 0.7, 1.5]), left_out=rng.random() < 0.3)
    # a block of 7 to 16 positions at the least
    n = rng.choice([7, 8, 11, 16])
    return _distill(kind, max(n, rows), V, dtype, _log_int(rng, 2, 128), fused=rng.random() < 0.8, n=n, pad=pad,
                    tail=rng.random() < 0.5, temperature=rng.choice([1.0, 1.5, 2.0]), left_out=rng.random() < 0.3)


# ------------------------------------------------------------------- inputs

def _gen(seed, salt):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 1009 + salt)
    return g


def _empty(c, pitch=0):
    """[rows, V] logits, or the first V columns of wider rows."""
    x = torch.empty(c["rows"], pitch or c["V"], dtype=TORCH[c["dtype"]], device=DEV)
    return x[:, :c["V"]] if pitch else x


def _logits(c, seed):
    """Logit rows with one likely token each, the padded columns at -inf."""
    g, rows, V = _gen(seed, 1), c["rows"], c["V"]
    live = V - c["pad"]
    ids = torch.randint(0, live, (rows,), generator=g, device=DEV)
    x = _empty(c, c.get("pitch", 0))
    step = max(1, (1 << 27) // V)
    for i in range(0, rows, step):               # in pieces: float32 temporaries stay small
        k = min(rows, i + step)
        r = torch.randn(k - i, V, generator=g, device=DEV).mul_(3.0)
        top = r.amax(-1, keepdim=True) + 0.5 + 7.5 * torch.rand(k - i, 1, generator=g, device=DEV)
        r.scatter_(1, ids[i:k, None], top)
        r[:, live:] = -math.inf
        x[i:k] = r.to(x.dtype)
    return x, ids


def _normal(c, seed, salt, pitch=0):
    g, x = _gen(seed, salt), _empty(c, pitch)
    step = max(1, (1 << 27) // c["V"])
    for i in range(0, c["rows"], step):
        k = min(c["rows"], i + step)
        x[i:k] = torch.randn(k - i, c["V"], generator=g, device=DEV).to(x.dtype)
    return x


def _log_prior(V, seed):
    """log of a Zipf(1.1) unigram law over a shuffled vocabulary, add-one smoothed."""
    rank = torch.randperm(V, generator=_gen(seed, 3), device=DEV).double()
    q = (rank + 1.0).pow(-1.1)
    n = torch.floor(q / q.sum() * 1e7) + 1.0
    return torch.log(n / n.sum()).float().contiguous()


def _teacher(c, long, seed):
    """A teacher's table of each row, its K most likely ids and their log-probabilities: float32 [rows, K].
    Every fifth row of more than one entry has one fewer (an id of -1)."""
    g, K, V, rows = _gen(seed, 4), c["top_k"], c["V"], c["rows"]
    ids = torch.empty(rows, K, dtype=torch.int32, device=DEV)
    lp = torch.empty(rows, K, dtype=torch.float32, device=DEV)
    step = max(1, (1 << 27) // V)
    for i in range(0, rows, step):
        k = min(rows, i + step)
        r = (long[i:k].float() + torch.randn(k - i, V, generator=g, device=DEV).mul_(2.0)) / c["temperature"]
        v, at = r.topk(K, -1)
        lp[i:k] = v - torch.logsumexp(r, -1, keepdim=True)
        ids[i:k] = at.to(torch.int32)
    if K > 1:
        ids[::5, -1] = -1
        lp[::5, -1] = -math.inf
    return ids, lp


def _inputs(c, seed):
    s = {"case": dict(c)}
    rows, n = c["rows"], c["n"]
    long, ids = _logits(c, seed)
    s["logits"], s["short"], s["prior"], s["alpha"], s["beta"] = long, None, None, None, None
    if c["fused"]:
        s["short"] = _normal(c, seed, 2, c.get("pitch", 0))
        s["prior"] = _log_prior(c["V"], seed)
        at = torch.arange(n, device=DEV, dtype=torch.float32) / n
        s["alpha"], s["beta"] = 0.5 - 0.2 * at, 0.3 + 0.1 * at     # weights of their own for each position
    g = _gen(seed, 5)
    skip = torch.arange(rows, device=DEV) % 8 == 7 if c["left_out"] else torch.zeros(rows, dtype=torch.bool, device=DEV)
    if c["kind"] == "score":
        # the given token: the likely one three times out of four
        other = torch.randint(0, c["V"] - c["pad"], (rows,), generator=g, device=DEV)
        tok = torch.where(torch.rand(rows, generator=g, device=DEV) < 0.75, ids, other)
        s["tokens"] = torch.where(skip, torch.full_like(tok, -1), tok).to(torch.int32)
        return s
    s["ids"], s["teacher"] = _teacher(c, long, seed)
    live = (~skip).float()
    s["weight"] = live / live.sum().clamp(min=1.0)
    s["grad_loss"] = torch.rand(rows, generator=g, device=DEV) + 0.5
    if not c["fused"]:                                  # a plain student: its logits are what is learned
        s["short"], s["logits"] = long, None
    return s


def prepare(case, seed):
    c, s = case, _inputs(case, seed)
    if own:
        import paper_2607_07409_gb300 as dels
        s["dels"] = dels
        if c["kind"] == "score":
            s["handle"] = dels.TokenScorer(c["rows"], c["V"], c["top_k"], device=DEV)
        elif c["kind"] != "autograd":
            s["handle"] = dels.Distiller(c["rows"], c["V"], c["top_k"], s["short"].dtype, n_weights=c["n"],
                                         tail=c["tail"], temperature=c["temperature"], device=DEV)
    if c["kind"] == "autograd":
        s["leaves"] = [s[k].requires_grad_() for k in ("short", "alpha", "beta") if s[k] is not None]
    return s


# ---------------------------------------------------------------------- run

def run(s):
    c = s["case"]
    if not own:
        with torch.no_grad():
            return _plain_score(s) if c["kind"] == "score" else _plain_distill(s)
    if c["kind"] == "score":
        return s["handle"](s["logits"], s["tokens"], short=s["short"], log_prior=s["prior"], alpha=s["alpha"],
                           beta=s["beta"], temperature=c["temperature"])
    if c["kind"] == "autograd":
        loss = s["dels"].distill_loss(s["short"], s["ids"], s["teacher"], long=s["logits"], log_prior=s["prior"],
                                      alpha=s["alpha"], beta=s["beta"], row_weight=s["weight"], tail=c["tail"],
                                      temperature=c["temperature"])
        grads = torch.autograd.grad(loss, s["leaves"], s["grad_loss"])
        return (loss.detach(),) + tuple(grads)
    call = s["handle"].step if c["kind"] == "step" else s["handle"].loss
    return call(s["short"], s["ids"], s["teacher"], long=s["logits"], log_prior=s["prior"], alpha=s["alpha"],
                beta=s["beta"], row_weight=s["weight"])


def _at(w, rows):
    """Per-position weights for each row, as a column."""
    return w[torch.arange(rows, device=w.device) % w.numel()].unsqueeze(1)


def _fused32(s):
    """The fused rows in float32, rounded after every operation."""
    c = s["case"]
    if not c["fused"]:
        return (s["logits"] if s["logits"] is not None else s["short"]).float()
    x = s["logits"].float() + _at(s["alpha"], c["rows"]) * s["short"].float()
    return x - _at(s["beta"], c["rows"]) * s["prior"]


def _log_q32(x, T):
    """log softmax(x / T): the largest entry is held out of the sum, whose logarithm is then one of 1 + rest."""
    top, at = x.max(-1, keepdim=True)
    z = (x - top) / T
    return z - torch.log1p(torch.exp(z).scatter_(1, at, 0.0).sum(-1, keepdim=True))


def _plain_score(s):
    c, tok = s["case"], s["tokens"].long()
    V, K = c["V"], c["top_k"]
    x = _fused32(s)
    lq = _log_q32(x, c["temperature"])
    out = (tok < 0)
    lp = lq.gather(1, tok.clamp(min=0).unsqueeze(1)).squeeze(1).masked_fill(out, 0.0)
    ent = -torch.where(lq > -math.inf, torch.exp(lq) * lq, torch.zeros_like(lq)).sum(-1)
    ent = ent.masked_fill(out, 0.0)
    if K == 0:
        return lp, ent, None, None
    # one integer key an entry: the order of the values, then the lower index first
    bits = (x + 0.0).view(torch.int32)
    key = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long() * (1 << 32)
    key += (V - 1 - torch.arange(V, device=x.device))
    top = key.topk(min(K, V), -1).values
    ids = V - 1 - (top & 0xFFFFFFFF)
    if K > V:
        ids = torch.cat([ids, ids.new_full((ids.shape[0], K - V), -1)], 1)
    tlp = lq.gather(1, ids.clamp(min=0)).masked_fill(ids < 0, -math.inf)
    none = (tlp == -math.inf) | out.unsqueeze(1)
    return lp, ent, ids.masked_fill(none, -1).to(torch.int32), tlp.masked_fill(none, -math.inf)


def _plain_distill(s):
    c = s["case"]
    rows, V, T = c["rows"], c["V"], c["temperature"]
    ids, t = s["ids"].long(), s["teacher"]
    listed_ = (ids >= 0) & (t > -math.inf)
    at = ids.clamp(min=0)
    x = _fused32(s)
    lq = _log_q32(x, T)
    q_at = lq.gather(1, at)
    zero = torch.zeros_like(t)
    if c["tail"]:
        log_p = t
    else:
        z = torch.where(listed_, t, torch.full_like(t, -math.inf)) / T
        log_p = z - z.amax(-1, keepdim=True)
        log_p = log_p - torch.log(torch.exp(log_p).sum(-1, keepdim=True))
    p = torch.where(listed_, torch.exp(log_p), zero)
    loss = torch.where(p > 0, p * (log_p - q_at), zero).sum(-1)
    q = torch.exp(lq)
    w = s["weight"] * s["grad_loss"] if c["kind"] == "autograd" else s["weight"]
    if c["tail"]:
        inside = torch.zeros_like(lq).scatter_add_(1, at, listed_.float()) > 0
        # what the largest entry leaves of 1, to all its digits, without the other entries
        first, k = p.max(-1, keepdim=True)
        rest = -torch.expm1(torch.where(first > 0, log_p.gather(1, k), torch.full_like(first, -math.inf))).squeeze(1)
        rest = (rest - p.scatter(1, k, 0.0).sum(-1)).clamp(min=0.0)
        q_rest, q_in = (torch.where(m, torch.zeros_like(q), q).sum(-1) for m in (inside, ~inside))
        has = (rest > 0) & (q_rest > 0)
        safe = torch.where(has, q_rest, torch.ones_like(q_rest))
        # logarithms of shares next to 1 from what they lack of it
        log_rest = torch.where(rest > 0.5, torch.log1p(-p.sum(-1)), torch.log(rest.clamp(min=1e-30)))
        loss = loss + torch.where(has, rest * (log_rest + torch.log1p(q_in / safe)), torch.zeros_like(loss))
        mass = p.sum(-1) + torch.where(has, rest, torch.zeros_like(rest))
        off = torch.where(has, rest / safe, torch.zeros_like(rest))
        g = q * torch.where(inside, mass.unsqueeze(1), (mass - off).unsqueeze(1))
    else:
        g = q
    loss = loss * s["weight"]
    if c["kind"] == "loss":
        return loss
    g = g.scatter_add(1, at, -p) * (w / T).unsqueeze(1)
    if not c["fused"]:
        return (loss, g.to(s["short"].dtype)) if c["kind"] == "autograd" else (loss, g.to(s["short"].dtype), None, None)
    n = s["alpha"].numel()
    at_n = torch.arange(rows, device=x.device) % n
    ga = torch.zeros_like(s["alpha"]).index_add_(0, at_n, (g * s["short"].float()).sum(-1))
    # a row's gradient sums to zero: a constant in the prior drops out, and is taken out before float32 sums
    gb = torch.zeros_like(s["beta"]).index_add_(0, at_n, -(g * (s["prior"] - s["prior"].mean())).sum(-1))
    return loss, (g * _at(s["alpha"], rows)).to(s["short"].dtype), ga, gb


# --------------------------------------------------------------------- work

def work(case):
    """Bytes: each logit read once, the prior and the teacher's table once, the outputs written once.
    Operations: per element the fusion (4), the exponent and its sums (6), and for a gradient 6 more."""
    c = case
    rows, V, s = c["rows"], c["V"], SIZE[c["dtype"]]
    cells = rows * V
    reads = cells * s * (2 if c["fused"] else 1) + (4 * V if c["fused"] else 0)
    flops = cells * (10 if c["fused"] else 6)
    if c["kind"] == "score":
        return {"bytes": reads + rows * (12 + 8 * c["top_k"]), "flops": flops}
    extra = rows * (8 + 8 * c["top_k"])
    if c["kind"] == "loss":
        return {"bytes": reads + extra, "flops": flops}
    return {"bytes": reads + cells * s + extra, "flops": flops + 6 * cells}


# -------------------------------------------------------------------- exact

def exact(case, seed):
    """The definitions in float64, a piece of the rows at a time."""
    c, s = case, _inputs(case, seed)
    rows, V, T, K = c["rows"], c["V"], c["temperature"], c["top_k"]
    step = max(1, (1 << 26) // V)
    out = []
    n = c["n"]
    ga, gb = (torch.zeros(n, dtype=torch.float64, device=DEV) for _ in range(2))
    for i in range(0, rows, step):
        r = slice(i, min(rows, i + step))
        pos = torch.arange(r.start, r.stop, device=DEV) % n
        x = s["logits"][r].double() if s["logits"] is not None else s["short"][r].double()
        if c["fused"]:
            al, be = s["alpha"].double()[pos, None], s["beta"].double()[pos, None]
            x = x + al * s["short"][r].double() - be * s["prior"].double()
        lq = torch.log_softmax(x / T, -1)
        if c["kind"] == "score":
            tok = s["tokens"][r].long()
            dead = tok < 0
            lp = torch.where(dead, 0.0, lq.gather(1, tok.clamp(min=0)[:, None])[:, 0])
            ent = torch.where(dead, 0.0, torch.special.entr(lq.exp()).sum(-1))
            top = lq.topk(min(K, V), -1).values if K else None
            if K:
                top = torch.nn.functional.pad(top, (0, K - top.shape[1]), value=-math.inf)
                top = torch.where(dead[:, None], torch.full_like(top, -math.inf), top)
            out.append((lp, ent) + ((top,) if K else ()))
            continue
        ids, t, w = s["ids"][r].long(), s["teacher"][r].double(), s["weight"][r].double()
        ok = (ids >= 0) & (t > -math.inf)
        t = torch.where(ok, t, torch.full_like(t, -math.inf))
        p = t.exp() if c["tail"] else torch.softmax(t / T, -1)
        target = torch.zeros_like(lq).scatter_add_(1, ids.clamp(min=0), torch.where(ok, p, torch.zeros_like(p)))
        inside = torch.zeros_like(lq).scatter_add_(1, ids.clamp(min=0), ok.double()) > 0
        term = torch.where(inside, torch.special.xlogy(target, target) - target * lq, torch.zeros_like(lq))
        loss = torch.where(inside & (target > 0), term, torch.zeros_like(term)).sum(-1)
        grad = lq.exp()
        if c["tail"]:
            rest = (1.0 - p.sum(-1)).clamp(min=0.0)
            log_rest_q = torch.logsumexp(torch.where(inside, torch.full_like(lq, -math.inf), lq), -1)
            has = (rest > 0) & (log_rest_q > -math.inf)
            safe = torch.where(has, log_rest_q, torch.zeros_like(log_rest_q))
            loss = loss + torch.where(has, torch.special.xlogy(rest, rest) - rest * safe, torch.zeros_like(rest))
            share = torch.where(has, rest / safe.exp(), torch.zeros_like(rest))
            mass = p.sum(-1) + torch.where(has, rest, torch.zeros_like(rest))
            grad = grad * torch.where(inside, mass[:, None], (mass - share)[:, None])
        loss = loss * w
        if c["kind"] == "loss":
            out.append((loss,))
            continue
        if c["kind"] == "autograd":
            w = w * s["grad_loss"][r].double()
        grad = (grad - target) * (w / T)[:, None]
        if c["fused"]:
            ga.index_add_(0, pos, (grad * s["short"][r].double()).sum(-1))
            gb.index_add_(0, pos, -(grad * s["prior"].double()).sum(-1))
            grad = grad * al
        out.append((loss, grad))
    got = [torch.cat(x) for x in zip(*out)]
    if c["kind"] == "score":
        return (got[0], got[1], None, got[2]) if K else (got[0], got[1], None, None)
    if c["kind"] == "loss":
        return got[0]
    if c["fused"]:
        return got[0], got[1], ga, gb
    return (got[0], got[1]) if c["kind"] == "autograd" else (got[0], got[1], None, None)
