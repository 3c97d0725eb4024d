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
