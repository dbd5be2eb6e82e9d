"""The verification from given numbers where it can go wrong: empty columns beside a border."""
from fractions import Fraction

import pytest
import torch

import paper_2607_07409_gb300 as dels

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
F32 = torch.float32


def draw(p, u, h=None):
    """One draw a row of p [B, V] with uniforms u: (columns, status), from outputs that held -9 before."""
    B, V = p.shape
    h = h or dels.BlockVerifier(B, 0, V, device=DEV)
    h.accept_len.fill_(-9)
    h.bonus.fill_(-9)
    _, bonus = h(None, p.view(B, 1, V), torch.as_tensor(u, dtype=F32).expand(B).reshape(B, 1).contiguous().to(DEV))
    return bonus.tolist(), h.status()


# ---------------------------------------------------------------- borders beside what has no weight

# Three weights whose sums in float64 depend on their order: (x1 + x2) + x0 = 1 + 2^-52, x2 + (x1 + x0) = 1 + 2^-51.
X0, X1, X2 = 1.0, 2.0 ** -53 * (1 + 2.0 ** -23), 2.0 ** -53


@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("V,step,more,u", [
    (32768, 4096, {4 * 4096: 1.0}, 0.5),                       # a CTA's slice a step: the fourth has none
    (32768, 256, {5 * 4096: 1.0}, 0.5),                        # a warp's run a step
    (524288, 256, {5 * 256: 2.0 ** -50, 6 * 65536: 3.0}, 0.25),          # a part of a run a step
])
def test_the_border_lies_where_there_is_weight(V, step, more, u, offset):
    """u times the whole comes out between two sums up to the same column, taken in two orders: the column is one
    with weight all the same, and it is written. Sums here take 16 float64 additions at most, 2^-49 of the whole: of the
    columns with weight those whose sums enclose u times the whole to that."""
    weights = {0: X0, step: X1, 2 * step: X2, **more}
    p = torch.zeros(1, V + offset, dtype=F32)
    for v, w in weights.items():
        p[0, offset + v] = w
    bonus, status = draw(p.to(DEV)[:, offset:], u)
    total = sum(map(Fraction, weights.values()))
    at, near, right = Fraction(u) * total, total * Fraction(2) ** -49, []
    upto = Fraction(0)
    for v, w in sorted(weights.items()):
        if upto - near <= at <= upto + Fraction(w) + near:
            right.append(v)
        upto += Fraction(w)
    assert status == 0 and bonus[0] in right
