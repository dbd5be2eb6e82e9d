"""Cases of the operators beside drafting with random numbers of the caller's own: products with 4-bit
vocabulary weights, probabilities of rows, and verification against given probabilities.

* ``w4``      logits of a head's features through a vocabulary matrix held in 4 bits (``W4Matrix``):
  ``y[b, v] = sum_k s[v, k / G] (c[v, k] - z[v, k / G]) x[b, k]`` with codes ``c`` of 0 to 15 and a scale
  (and, or 8, a zero point) for each group of ``G`` inputs
* ``probs``   the probabilities of plain or fused rows, ``softmax((l_L + alpha l_S - beta l_P) / T)`` (``RowProbs``)
* ``verify``  speculative sampling with given numbers (``BlockVerifier``): ``x_j`` is kept while
  ``u_j q_j(x_j) < p_j(x_j)``; then a token from ``max(0, p - q)`` at the first that is not, or from the last row
  of ``p``: the lowest ``v`` whose cumulated weight exceeds ``u_n`` times the whole. Without ``q`` the drafted
  tokens have probability 1 (a greedy drafter); with ``n = 0`` it draws a token of each row.

Where ``own`` is false the same values come from elementary torch operations, in float32 (the comparisons and
the cumulated sums of the verification in float64: they lie next to borders). Logit rows are N(0, 3) with one likely
token 0.5 to 8 above the rest; the local head's logits and features are N(0, 1); weights N(0, 0.02) before their
rounding to 4 bits; the target's rows are the drafter's plus N(0, 1), and drafted tokens are drawn from the drafter's.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}


def _w4(B, V, K, group, **kw):
    return dict(dict(kind="w4", B=B, V=V, K=K, group=group, zeros=False, x="bf16", out="f32"), **kw)


def _probs(rows, V, dtype, **kw):
    return dict(dict(kind="probs", rows=rows, V=V, dtype=dtype, out="f32", fused=False, n=1, pad=0, pitch=0,
                     temperature=1.0), **kw)


def _verify(B, n, V, **kw):
    return dict(dict(kind="verify", B=B, n=n, V=V, dtype="f32", draft="f32", ragged=False, pitch=0), **kw)


def listed():
    return [
        # The smallest product: one position of the toy head, its 128 features to 1024 tokens. Latency.
        dict(_w4(1, 1024, 128, 32), name="w4_tiny"),
        # One request while it drafts: the 1024-wide MLP head's feature to the full vocabulary.
        dict(_w4(1, 151936, 1024, 64), name="w4_one_token"),
        # 8 requests, the 2560-wide transformer head, groups of 128 with zero points.
        dict(_w4(8, 151936, 2560, 128, zeros=True), name="w4_b8"),
        # 64 requests, the GRU head's rank of 256, fine groups, bf16 logits.
        dict(_w4(64, 151936, 256, 32, out="bf16"), name="w4_b64"),
        # Odd sizes and float32 features: 5 requests, a vocabulary of 32003, 1000 inputs.
        dict(_w4(5, 32003, 1000, 64, zeros=True, x="f32"), name="w4_ragged"),
        # The rows of one toy block.
        dict(_probs(8, 1024, "f32", fused=True, n=8), name="probs_tiny"),
        # The target's rows of 64 blocks of 16 (and the token after each) at temperature 0.8, a padded vocabulary.
        dict(_probs(64 * 17, 151936, "bf16", pad=256, temperature=0.8), name="probs_target_b64"),
        # The drafter's fused rows of 8 requests, float32 logits.
        dict(_probs(128, 151936, "f32", fused=True, n=16), name="probs_fused_b8"),
        # One request's block of 8, a small vocabulary. Latency.
        dict(_verify(1, 8, 32000), name="verify_one"),
        # 64 blocks of 16 over the full vocabulary.
        dict(_verify(64, 16, 151936), name="verify_b64"),
        # A greedy drafter's blocks of up to 7, bf16 probabilities of an odd vocabulary in wider rows.
        dict(_verify(29, 7, 50257, dtype="bf16", draft="none", ragged=True, pitch=50304), name="verify_ragged"),
        # No draft: one token of each of 64 rows.
        dict(_verify(64, 0, 151936), name="draw_b64"),
    ]


# ------------------------------------------------------------------ drawing

def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["w4", "probs", "verify"])
    V = rng.choice([32000, 32003, 50257, 128256, 151936, _log_int(rng, 1000, 151936), _log_int(rng, 1000, 151936)])
    if kind == "w4":
        K = rng.choice([128, 256, 1024, 2560, 4096, _log_int(rng, 100, 4096), _log_int(rng, 100, 4096)])
        V = min(V, 151936 * 2560 // K)
        B = min(_log_int(rng, 1, 64), max(1, 8 * 151936 * 2560 // (V * K)))
        return _w4(B, V, K, rng.choice([32, 64, 128]), zeros=rng.random() < 0.5, x=rng.choice(["bf16", "bf16", "f32"]),
                   out=rng.choice(["f32", "bf16"]))
    if kind == "probs":
        dtype, out = rng.choice(["f32", "bf16"]), rng.choice(["f32", "f32", "bf16"])
        rows = _log_int(rng, 1, min(4096, 64 * 17 * 151936 // (2 * V)))
        # odd pitches too: a row of another alignment than the one before it
        return _probs(rows, V, dtype, out=out, fused=rng.random() < 0.5, n=rng.choice([1, 7, 8, 16]),
                      pad=rng.choice([0, 0, 64, V // 500]), pitch=rng.choice([0, 0, V + rng.randint(1, 128)]),
                      temperature=rng.choice([1.0, 0.7, 1.5]))
    n = rng.choice([0, 1, 4, 7, 8, 16])
    B = _log_int(rng, 1, min(256, 64 * 17 * 151936 // (V * (n + 1))))
    return _verify(B, n, V, dtype=rng.choice(["f32", "f32", "bf16"]), draft=rng.choice(["f32", "f32", "bf16", "none"]),
                   ragged=rng.random() < 0.5, pitch=rng.choice([0, 0, V + rng.randint(1, 128)]))


# ------------------------------------------------------------------- inputs

def _gen(seed, salt):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 1013 + salt)
    return g


def _normal(shape, seed, salt):
    return torch.randn(*shape, generator=_gen(seed, salt), device=DEV)


def _logits(rows, V, seed, pad=0):
    """Float32 logit rows with one likely token each, the padded columns at -inf."""
    g = _gen(seed, 1)
    x = torch.randn(rows, V, generator=g, device=DEV).mul_(3.0)
    ids = torch.randint(0, V - pad, (rows, 1), generator=g, device=DEV)
    x.scatter_(1, ids, x.amax(-1, keepdim=True) + 0.5 + 7.5 * torch.rand(rows, 1, generator=g, device=DEV))
    x[:, V - pad:] = -math.inf
    return x


def _stored(x, dtype, pitch):
    """The rows in this type, as the first columns of rows of `pitch` (0: dense)."""
    if not pitch:
        return x.to(TORCH[dtype])
    wide = torch.zeros(*x.shape[:-1], pitch, dtype=TORCH[dtype], device=DEV)
    wide[..., :x.shape[-1]] = x
    return wide[..., :x.shape[-1]]


def _log_prior(V, seed):
    """log of a Zipf(1.1) unigram law over a shuffled vocabulary, add-one smoothed."""
    rank = torch.randperm(V, generator=_gen(seed, 3), device=DEV).double()
    q = (rank + 1.0).pow(-1.1)
    n = torch.floor(q / q.sum() * 1e7) + 1.0
    return torch.log(n / n.sum()).float().contiguous()


def _codes(c, seed):
    """Codes [V, K] of 0 to 15, bf16 scales and uint8 zero points [V, groups] of rounded N(0, 0.02) weights."""
    V, K, G = c["V"], c["K"], c["group"]
    groups = -(-K // G)
    w = _normal((V, groups, G), seed, 2).mul_(0.02)
    if c["zeros"]:
        lo, hi = w.amin(-1, keepdim=True), w.amax(-1, keepdim=True)
        scale = ((hi - lo) / 15.0).to(torch.bfloat16)
        zero = torch.round(-lo / scale.float()).clamp_(0, 15)
    else:
        scale = (w.abs().amax(-1, keepdim=True) / 7.0).to(torch.bfloat16)
        zero = torch.full_like(scale, 8.0, dtype=torch.float32)
    codes = w.div_(scale.float()).add_(zero).round_().clamp_(0 if c["zeros"] else 1, 15).to(torch.uint8)
    codes = codes.reshape(V, groups * G)[:, :K].contiguous()
    return codes, scale.reshape(V, groups), zero.to(torch.uint8).reshape(V, groups) if c["zeros"] else None


def _inputs(c, seed):
    s = {"case": dict(c)}
    if c["kind"] == "w4":
        s["x"] = _normal((c["B"], c["K"]), seed, 4).to(TORCH[c["x"]])
        s["codes"], s["scales"], s["zeros"] = _codes(c, seed)
        return s
    if c["kind"] == "probs":
        rows, V, n = c["rows"], c["V"], c["n"]
        s["logits"] = _stored(_logits(rows, V, seed, c["pad"]), c["dtype"], c["pitch"])
        s["short"], s["prior"], s["alpha"], s["beta"] = None, None, None, None
        if c["fused"]:
            s["short"] = _stored(_normal((rows, V), seed, 2), c["dtype"], c["pitch"])
            s["prior"] = _log_prior(V, seed)
            at = torch.arange(n, device=DEV, dtype=torch.float32) / n
            s["alpha"], s["beta"] = 0.5 - 0.2 * at, 0.3 + 0.1 * at
        return s
    B, n, V = c["B"], c["n"], c["V"]
    x = _logits(B * (n + 1), V, seed).view(B, n + 1, V)
    target = torch.softmax(x + _normal((B, n + 1, V), seed, 2), -1)
    s["target"] = _stored(target, c["dtype"], c["pitch"])
    x = x[:, :n]
    if c["draft"] == "none":
        s["draft"], tokens = None, x.argmax(-1)
    else:
        s["draft"] = _stored(torch.softmax(x, -1), c["draft"], c["pitch"])
        noise = torch.rand(B, n, V, generator=_gen(seed, 5), device=DEV).clamp_(min=1e-30)
        tokens = (x - torch.log(-torch.log(noise))).argmax(-1)
    s["tokens"] = tokens.to(torch.int32)
    g = _gen(seed, 6)
    s["uniforms"] = torch.rand(B, n + 1, generator=g, device=DEV)
    s["lengths"] = torch.randint(0, n + 1, (B,), generator=g, device=DEV, dtype=torch.int32) if c["ragged"] else None
    return s


def prepare(case, seed):
    c, s = case, _inputs(case, seed)
    if own:
        import paper_2607_07409_gb300 as dels
        if c["kind"] == "w4":
            s["handle"] = dels.pack_w4(s["codes"], s["scales"], s["zeros"], group=c["group"])
            s["out"] = torch.empty(c["B"], c["V"], dtype=TORCH[c["out"]], device=DEV)
        elif c["kind"] == "probs":
            s["handle"] = dels.RowProbs(c["rows"], c["V"], TORCH[c["out"]], device=DEV)
        else:
            s["handle"] = dels.BlockVerifier(c["B"], c["n"], c["V"], device=DEV)
    return s


# ---------------------------------------------------------------------- run

def run(s):
    c = s["case"]
    if own:
        if c["kind"] == "w4":
            return s["handle"].project(s["x"], out=s["out"])
        if c["kind"] == "probs":
            return s["handle"](s["logits"], short=s["short"], log_prior=s["prior"], alpha=s["alpha"], beta=s["beta"],
                               temperature=c["temperature"])
        return s["handle"](s["tokens"], s["target"], s["uniforms"], draft=s["draft"], lengths=s["lengths"])
    if c["kind"] == "w4":
        return _plain_w4(s)
    return _plain_probs(s) if c["kind"] == "probs" else _plain_verify(s)


def _plain_w4(s):
    c = s["case"]
    G, K = c["group"], c["K"]
    zero = 8.0 if s["zeros"] is None else s["zeros"].float().repeat_interleave(G, 1)[:, :K]
    w = (s["codes"].float() - zero) * s["scales"].float().repeat_interleave(G, 1)[:, :K]
    return (s["x"].float() @ w.T).to(TORCH[c["out"]])


def _at(w, rows):
    """Per-position weights for each row, as a column."""
    return w[torch.arange(rows, device=w.device) % w.numel()].unsqueeze(1)


def _plain_probs(s):
    c = s["case"]
    x = s["logits"].float()
    if c["fused"]:
        x = x + _at(s["alpha"], c["rows"]) * s["short"].float() - _at(s["beta"], c["rows"]) * s["prior"]
    e = torch.exp((x - x.amax(-1, keepdim=True)) / c["temperature"])
    return (e / e.sum(-1, keepdim=True)).to(TORCH[c["out"]])


def _plain_verify(s):
    c = s["case"]
    n, rows = c["n"], torch.arange(c["B"], device=DEV)
    p, q, u, at = s["target"], s["draft"], s["uniforms"].double(), s["tokens"].long()
    length = s["lengths"].long() if s["lengths"] is not None else torch.full_like(rows, n)
    p_at = p[:, :n].gather(2, at[..., None])[..., 0].double()
    q_at = q.gather(2, at[..., None])[..., 0].double() if q is not None else torch.ones_like(p_at)
    kept = (u[:, :n] * q_at < p_at) & (torch.arange(n, device=DEV) < length[:, None])
    accepted = kept.long().cumprod(1).sum(1)
    left = p[rows, accepted].double()
    w = left
    if n:
        first = accepted.clamp(max=n - 1)
        if q is not None:
            w = (left - q[rows, first].double()).clamp(min=0.0)
        else:
            w = left.scatter(1, at[rows, first][:, None], 0.0)
        keep = (accepted < length) & (w > 0).any(1)
        w = torch.where(keep[:, None], w, left)
    total = w.cumsum(1)
    bonus = (total <= u[:, n:] * total[:, -1:]).sum(1)
    return accepted.to(torch.int32), bonus.to(torch.int32)


# --------------------------------------------------------------------- work

def work(case):
    """Bytes: codes, scales, zero points, features and logits once; each logit and probability once; of a verification
    the one row of each kind that the draw reads. Operations: two for each weight and request; 10 (plain 6) for each
    logit; 4 for each entry of the rows that are drawn from."""
    c = case
    if c["kind"] == "w4":
        V, K, B = c["V"], c["K"], c["B"]
        groups = -(-K // c["group"])
        weights = V * (K / 2 + groups * (2.5 if c["zeros"] else 2))
        return {"bytes": weights + B * (K * SIZE[c["x"]] + V * SIZE[c["out"]]), "flops": 2 * V * K * B}
    if c["kind"] == "probs":
        cells = c["rows"] * c["V"]
        reads = cells * SIZE[c["dtype"]] * (2 if c["fused"] else 1) + (4 * c["V"] if c["fused"] else 0)
        return {"bytes": reads + cells * SIZE[c["out"]], "flops": cells * (10 if c["fused"] else 6)}
    cells = c["B"] * c["V"]
    reads = cells * (SIZE[c["dtype"]] + (SIZE[c["draft"]] if c["n"] and c["draft"] != "none" else 0))
    return {"bytes": reads + c["B"] * (4 * (4 * c["n"] + 1) + 8), "flops": 4 * cells}


# -------------------------------------------------------------------- exact

def exact(case, seed):
    """The definitions in float64, a piece at a time."""
    c, s = case, _inputs(case, seed)
    if c["kind"] == "w4":
        G, K = c["group"], c["K"]
        x = s["x"].double()
        y = torch.empty(c["B"], c["V"], dtype=torch.float64, device=DEV)
        step = max(1, (1 << 26) // K)
        of = torch.arange(K, device=DEV) // G
        for i in range(0, c["V"], step):
            w = s["codes"][i:i + step].double()
            w = w - (8.0 if s["zeros"] is None else s["zeros"][i:i + step].double()[:, of])
            y[:, i:i + step] = torch.einsum("bk,vk->bv", x, w * s["scales"][i:i + step].double()[:, of])
        return y
    if c["kind"] == "probs":
        out = []
        step = max(1, (1 << 26) // c["V"])
        for i in range(0, c["rows"], step):
            x = s["logits"][i:i + step].double()
            if c["fused"]:
                pos = torch.arange(i, i + x.shape[0], device=DEV) % c["n"]
                x = x + s["alpha"].double()[pos, None] * s["short"][i:i + step].double()
                x = x - s["beta"].double()[pos, None] * s["prior"].double()
            out.append(torch.log_softmax(x / c["temperature"], -1).exp())
        return torch.cat(out)
    accepted, bonus = [], []
    tokens, u = s["tokens"].tolist(), s["uniforms"].double().tolist()
    lengths = s["lengths"].tolist() if s["lengths"] is not None else [c["n"]] * c["B"]
    for b in range(c["B"]):
        a = 0
        while a < lengths[b]:
            t = tokens[b][a]
            q = float(s["draft"][b, a, t]) if s["draft"] is not None else 1.0
            if not u[b][a] * q < float(s["target"][b, a, t]):
                break
            a += 1
        w = s["target"][b, a].double()
        if a < lengths[b]:
            q = torch.zeros_like(w)
            if s["draft"] is not None:
                q = s["draft"][b, a].double()
            else:
                q[tokens[b][a]] = math.inf
            rest = torch.relu(w - q)
            w = rest if float(rest.max()) > 0 else w
        sums = torch.cumsum(w, 0)
        accepted.append(a)
        bonus.append(int(torch.searchsorted(sums, u[b][c["n"]] * sums[-1], right=True)))
    return (torch.tensor(accepted, dtype=torch.int32, device=DEV), torch.tensor(bonus, dtype=torch.int32, device=DEV))
