"""Distillation of rows whose first columns say nothing of their largest: the references that the sums
are relative to then lie far below them. Bounds as in test_gpu_row_ops."""
import pytest
import torch

from test_gpu_row_ops import Case, check_distill, gen

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
