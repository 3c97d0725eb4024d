"""Products with groups whose zero-point is all there is: the quantizer gives a group of one value (a constant, zeros, a pruned or padded
row) scale 1 and codes 0, so that its zero-point may be far below its scale.

A row of zeros gives 0 exactly: its codes' sum is 0 and so is each product with its zero-point.  A row of such groups gives the sum over
the groups of m times the group's sum of x.  That sum's MMA steps cut off at most 17 * 2^-23 of the absolute values each, eight steps a
group; the additions over groups, warps and pieces are within 2^-23 each of what has been added, at most K / G + 32 of them.  So the
result is within (8 * 17 + K / G + 32) 2^-23 of sum |w x|, and its own half step."""
import pytest
import torch

from paper_2503_21135_b200 import binding
from paper_2503_21135_b200 import operators as ops

pytestmark = pytest.mark.gpu
VALUES = [0.0, 1e-5, 1e-4, 0.25, -1e-4, 2e-7, -3.0]

# few-token kernel with 8 and with 16 tokens, with clusters and without; tcgen05 kernel with 16, 32 and 64 tokens, ragged rows and tokens
SHAPES = [(1, 300, 4096), (8, 20000, 256), (12, 100, 640), (40, 130, 1088), (16, 14336, 4096), (31, 6401, 4096), (64, 4101, 4160), (130, 4099, 4096)]


def product(T, N, K, G, y_dtype):
    g = torch.Generator(device="cuda").manual_seed(T + N)
    w = (torch.randn((N, K), generator=g, device="cuda") * 0.02).bfloat16()
    w[5::7] = 0
    for i, v in enumerate(VALUES):
        w[6 + 7 * i] = v
    mixed = torch.tensor(VALUES, device="cuda")[torch.arange(K // G, device="cuda") % len(VALUES)].repeat_interleave(G).bfloat16()
    w[4::7] = mixed                                     # another constant in every group
    x = torch.randn((T, K), generator=g, device="cuda").bfloat16()
    codes, params = ops.quantize_linear(w, G)
    y = ops.linear(x, codes, params, y_dtype=binding.F32 if y_dtype == "f32" else binding.BF16)
    q = torch.stack([codes & 15, codes >> 4], 2).view(N, K)
    m = params[:, :, 1].double().repeat_interleave(G, 1)
    return x.double(), q, m, y


@pytest.mark.parametrize("y_dtype", ["f32", "bf16"])
@pytest.mark.parametrize("G", [64, 128])
@pytest.mark.parametrize("T,N,K", SHAPES)
def test_constant_and_empty_groups(T, N, K, G, y_dtype):
    K = K // G * G
    X, q, m, y = product(T, N, K, G, y_dtype)
    assert (y[:, 5::7] == 0).all()
    rows = [6 + 7 * i for i in range(len(VALUES))] + list(range(4, N, 7))
    assert (q[rows] == 0).all()
    ref, mag = X @ m[rows].T, X.abs() @ m[rows].abs().T
    tol = (8 * 17 + K / G + 32) * 2.0 ** -23 * mag + torch.finfo(y.dtype).eps / 2 * ref.abs()
    assert bool(((y[:, rows].double() - ref).abs() <= 1.01 * tol).all())


@pytest.mark.parametrize("T,N,K", [(1, 300, 4096), (12, 100, 640), (64, 4101, 4160)])
def test_infinite_activation(T, N, K):
    """A NaN makes the token's row NaN, an infinity makes it infinite or NaN, also where all weights have one sign."""
    G = 128 if K % 128 == 0 else 64
    g = torch.Generator(device="cuda").manual_seed(T)
    w = (torch.rand((N, K), generator=g, device="cuda") * 0.1 + 1.0).bfloat16()
    x = torch.randn((T, K), generator=g, device="cuda").bfloat16()
    x[0, 7] = float("inf")
    if T > 2:
        x[2, 9] = float("nan")
    y = ops.linear(x, *ops.quantize_linear(w, G))
    assert not torch.isfinite(y[0]).any() and (T <= 2 or torch.isnan(y[2]).all())
    assert torch.isfinite(y[[i for i in range(T) if i not in (0, 2)]]).all()
