"""The expert sort and its way back at the ends of their 32-bit ranges."""
import pytest
import torch

from paper_2503_21135_b200 import operators as ops

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", [2147483553, 2 ** 31 - 1])
def test_pairs_up_to_two_to_the_31(T):
    E, step = 3, 1 << 27
    idx = torch.empty((T, 1), dtype=torch.int32, device="cuda")
    for i in range(0, T, step):
        n = min(step, T - i)
        idx[i:i + n, 0] = torch.arange(i, i + n, device="cuda") % E
    pos, perm = torch.full((T, 1), -7, dtype=torch.int32, device="cuda"), torch.full((T,), -7, dtype=torch.int32, device="cuda")
    off = torch.empty(E + 1, dtype=torch.int32, device="cuda")
    ops.dispatch(idx, E, out=(None, off, perm, pos))
    counts = [(T - e + E - 1) // E for e in range(E)]
    want = [sum(counts[:e]) for e in range(E + 1)]
    assert off.tolist() == want
    first = torch.tensor(want, device="cuda")
    for i in range(0, T, step):
        t = torch.arange(i, min(i + step, T), device="cuda")
        at = first[t % E] + t // E
        assert torch.equal(pos[i:i + step, 0].long(), at)
        assert torch.equal(perm[at].long(), t)


def test_rows_of_two_to_the_31_values():
    """One token: every run of eight columns up to the last is in the sum and in the gradients, and nothing else is touched."""
    d = 2 ** 31 - 8
    rows = torch.zeros((1, d), dtype=torch.bfloat16, device="cuda")
    rows[0, :8], rows[0, -8:] = 1.0, 2.0
    w = torch.tensor([[0.5]], device="cuda")
    s = ops.dispatch(torch.zeros((1, 1), dtype=torch.int32, device="cuda"), 1, rows)
    assert torch.equal(s.rows, rows)
    y = ops.combine(s.rows, s.pos, w)
    assert (y[0, :8] == 0.5).all() and (y[0, -8:] == 1.0).all() and int(torch.count_nonzero(y)) == 16
    d_rows, d_w = ops.combine_backward(rows, s.rows, s.pos, w)
    assert torch.equal(d_rows, y) and d_w.item() == 8 * 1.0 + 8 * 4.0
