"""Trains a Markov head and the fusion's weights from a target model's logits, then drafts with them.

    python examples/distill_head.py [--steps N]

Every training step scores the target's rows (the K most likely tokens of each and their
log-probabilities: a teacher's table, 8 K bytes a row in place of V logits) and distils the
head from it through the fusion l = l_L + alpha_j l_S - beta_j l_P, with the gradient to the
head's logits and to the weights of each block position. Before and after the training the
head drafts blocks of new contexts; the target verifies them greedily and scores the drafted
tokens. The models are synthetic: a target whose next token depends on the context and, by a
hidden table of rank 16, on the token before it, and a drafter that knows the context only.
"""
import argparse
import sys
from pathlib import Path

import torch

sys.path.insert(0, str(Path(__file__).resolve().parent.parent))

import paper_2607_07409_gb300 as dels  # noqa: E402
from synth import HeadSpec  # noqa: E402

B, N, V, RANK, K = 64, 8, 8192, 64, 32


class Models:
    """The target and the drafter: contexts in, logits out."""

    def __init__(self, device, seed=0):
        self.g = torch.Generator(device).manual_seed(seed)
        self.device = device
        self.left = self.normal(V, 16)
        self.right = self.normal(V, 16) * 0.6
        self.common = -1.1 * torch.log(torch.randperm(V, generator=self.g, device=device) + 1.0)   # frequent tokens

    def normal(self, *shape):
        return torch.randn(*shape, generator=self.g, device=self.device)

    def context(self):
        """What the target makes of B contexts at N + 1 positions, and what the drafter does at N."""
        base = self.normal(B, N + 1, V) * 2.0
        return base, base[:, :N] + 0.5 * self.normal(B, N, V) + self.common

    def target(self, base, previous):
        """The target's rows [B, positions, V] after the tokens `previous` (-1: none)."""
        pair = self.left[previous.clamp(min=0)] @ self.right.T
        return base + self.common + pair * (previous >= 0)[..., None]

    def tokens(self):
        """Tokens before the positions 1 .. N - 1, by their frequency."""
        p = self.common.softmax(0).expand(B, V)
        return torch.multinomial(p, N - 1, replacement=True, generator=self.g)


def draft_and_verify(models, weights, alpha, beta, prior, contexts=8):
    """Mean accepted length, the target's mean log-probability of the drafted tokens and its mean entropy."""
    drafter = dels.Drafter(HeadSpec("markov", "f32", 0, 0, RANK), weights, B, N, V)
    scorer = dels.TokenScorer(B * N, V, device=models.device)
    code = dels.dtype_code(torch.float32)
    nbytes = dels.dels_verify_workspace_bytes(B, N, V, code)
    ws = torch.zeros(nbytes, dtype=torch.uint8, device=models.device)
    accepted, bonus = (torch.empty(B, dtype=torch.int32, device=models.device) for _ in range(2))
    total = torch.zeros(3, device=models.device)
    for _ in range(contexts):
        base, long = models.context()
        tokens, _, _ = drafter(long, prior, [0.0] + alpha.tolist(), [0.0] + beta.tolist())
        before = torch.cat([torch.full_like(tokens[:, :1], -1), tokens], 1).long()
        rows = models.target(base, before)
        status = dels.dels_verify_block(tokens, rows, code, B, N, V, accepted, bonus, None, ws, nbytes)
        if status != dels.DELS_OK:
            raise dels.DelsError(status, "dels_verify_block")
        logprob, entropy, _, _ = scorer(rows[:, :N].reshape(B * N, V), tokens.reshape(-1))
        total += torch.stack([accepted.float().mean(), logprob.mean(), entropy.mean()])
    assert drafter.status() == 0 and scorer.status() == 0
    return [float(x) / contexts for x in total]


def main(steps=300, device="cuda"):
    models = Models(torch.device(device))
    prior = models.common.log_softmax(0)
    emb = (models.normal(V, RANK) * 0.1).requires_grad_()
    w_vocab = (models.normal(V, RANK) * 0.1).requires_grad_()
    alpha = torch.full((N - 1,), 0.5, device=device).requires_grad_()
    beta = torch.full((N - 1,), 0.1, device=device).requires_grad_()
    optimizer = torch.optim.Adam([{"params": [emb, w_vocab], "lr": 2e-2}, {"params": [alpha, beta], "lr": 1e-2}])
    rows = B * (N - 1)
    teacher = dels.TokenScorer(rows, V, K, device=device)

    def drafts():
        weights = {"emb": emb.detach(), "w_vocab": w_vocab.detach()}
        return draft_and_verify(models, weights, alpha.detach(), beta.detach(), prior)

    names = "accepted length %.2f, log-probability under the target %.3f, its entropy %.3f"
    before = drafts()
    print("before:", names % tuple(before))
    losses = []
    for step in range(steps):
        base, long = models.context()
        previous = models.tokens()
        _, _, ids, logprob = teacher(models.target(base[:, 1:N], previous).reshape(rows, V))
        short = emb[previous.reshape(-1)] @ w_vocab.T           # row b (N - 1) + j - 1: weight j - 1
        loss = dels.distill_loss(short, ids, logprob, long=long[:, 1:].reshape(rows, V), log_prior=prior, alpha=alpha,
                                 beta=beta, tail=True).mean()
        optimizer.zero_grad()
        loss.backward()
        optimizer.step()
        losses.append(loss.detach())
        if step % 50 == 0 or step == steps - 1:
            print(f"step {step}: loss {float(losses[-1]):.4f}")
    after = drafts()
    print("after: ", names % tuple(after))
    print("alpha", [round(x, 2) for x in alpha.tolist()], "beta", [round(x, 2) for x in beta.tolist()])
    return before, after, [float(x) for x in losses]


if __name__ == "__main__":
    parser = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    parser.add_argument("--steps", type=int, default=300)
    main(parser.parse_args().steps)
