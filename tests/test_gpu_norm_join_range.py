"""The norm join's gradient where a row's factor is far from 1: rows of zeros and rows near zero with a tiny eps, rows of large values.
The cube of the factor is then outside the range of fp32, the gradient is not.

Tolerance as for the gradient at ordinary factors: every term has fewer than 16 roundings and the row sums' terms at most 40 more, 256 u of
the absolute values put through the formulas, T u of the absolute sum for sums over T tokens, half a step of the result's type."""
import numpy as np
import pytest
import torch

from paper_2503_21135_b200 import operators as ops

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
A, B = 0.9, 0.7


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def gradients(r, y, d_n, w_post, w_pre, gate, eps, sign):
    """The formulas in 64 bits; sign = +1 with absolute values: the absolute values of their terms (r', factors from the signed ones)."""
    x = A * r + B * gate * w_post * y / np.sqrt((y * y).mean(1, keepdims=True) + eps)
    s_y, s_r = 1 / np.sqrt((y * y).mean(1, keepdims=True) + eps), 1 / np.sqrt((x * x).mean(1, keepdims=True) + eps)
    u, yn = w_pre * d_n, y * s_y
    if sign > 0:
        u, yn, w_post, w_pre, gate, d_n = (np.abs(v) for v in (u, yn, w_post, w_pre, gate, d_n))
        x = A * np.abs(r) + B * gate * w_post * yn
    xn = x * s_r
    G = s_r * (u + sign * xn * (u * xn).mean(1, keepdims=True))
    dz = B * gate * G
    v = dz * w_post
    d_y = s_y * (v + sign * yn * (v * yn).mean(1, keepdims=True))
    return dict(d_r=A * G, d_y=d_y, d_w_post=dz * yn, d_gate=B * w_post * yn * G, d_w_pre=d_n * xn)


@pytest.mark.parametrize("scale,eps", [(0.0, 1e-30), (1e-15, 1e-30), (1e-13, 1e-26), (1e13, 1e-6), (1e15, 1e-6)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("d", [64, 1024, 4096, 5000, 12296])
def test_gradient_at_far_factors(d, dtype, scale, eps):
    T = 5
    g = torch.Generator(device="cuda").manual_seed(d)

    def randn(*s):
        return torch.randn(s, generator=g, device="cuda")

    r, y = (randn(T, d) * scale).to(dtype), (randn(T, d) * scale).to(dtype)
    r[3], y[3] = 0, 0
    d_n = randn(T, d).to(dtype)
    how = dict(w_post=randn(d), gate=randn(d), w_pre=randn(d), res_scale=A, block_scale=B, eps=eps)
    _, _, stats = ops.norm_join(r, y, **how, want_stats=True)
    got = ops.norm_join_backward(d_n, None, r, y, stats, **how)
    args = [f64(t) for t in (r, y, d_n, how["w_post"], how["w_pre"], how["gate"])]
    eps32 = float(np.float32(eps))
    want, mag = gradients(*args, eps32, -1), gradients(*args, eps32, 1)
    for name, t in got.items():
        ref, m = want[name], mag[name]
        rows = T if t.dim() == 1 else 0
        if rows:
            ref, m = ref.sum(0), m.sum(0)
        assert torch.isfinite(t).all(), name
        tol = (256 + rows) * U * m + torch.finfo(t.dtype).eps / 2 * np.abs(ref) + 1e-37
        assert (np.abs(f64(t) - ref) <= 1.01 * tol).all(), name
