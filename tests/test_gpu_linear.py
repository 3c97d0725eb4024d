"""Products with a 4-bit matrix, against numpy in 64 bits; the quantizer against the oracle's, bit for bit.

Tolerance.  With C = sum_k (s (16 + q) + |m - 16 s|) |x| the absolute values that a result's sums see: a 16-wide MMA adds 16 exact
products and the accumulator, each cut off at no more than 2^-23 of the largest, so 17 * 2^-23 of the group's sum a step and 8 steps
a group; what follows (scale, zero-point, one addition a group of a warp's share, eight warps' sums) is within 2^-23 per addition of
C, at most K / 64 / 8 + 16 of them."""
import numpy as np
import pytest
import torch

import oracle
from paper_2503_21135_b200 import binding
from paper_2503_21135_b200 import operators as ops

pytestmark = pytest.mark.gpu


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def decoded(codes, params, G):
    c = codes.cpu().numpy()
    q = np.empty((c.shape[0], c.shape[1] * 2))
    q[:, 0::2], q[:, 1::2] = c & 15, c >> 4
    s, m = np.repeat(f64(params)[:, :, 0], G, 1), np.repeat(f64(params)[:, :, 1], G, 1)
    return q, s, m


def check(x, codes, params, G, y):
    q, s, m = decoded(codes, params, G)
    X = f64(x)
    ref = X @ (s * q + m).T
    C = np.abs(X) @ (np.abs(s) * (16 + q) + np.abs(m - 16 * s)).T
    K = X.shape[1]
    tol = (8 * 17 + K / 512 + 16) * 2.0 ** -23 * C + torch.finfo(y.dtype).eps / 2 * np.abs(ref)
    assert y.shape == ref.shape and (np.abs(f64(y) - ref) <= tol * 1.01).all()


def make(T, N, K, G, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed + T * 7 + N + K)
    w = (torch.randn((N, K), generator=g, device="cuda") * 0.02).bfloat16()
    if K >= 128:
        w[:, 5] *= 20
    x = torch.randn((T, K), generator=g, device="cuda").bfloat16()
    return w, x


@pytest.mark.parametrize("y_dtype", ["f32", "bf16"])
@pytest.mark.parametrize("G", [64, 128])
@pytest.mark.parametrize("T,N,K", [(1, 1, 128), (1, 16, 128), (1, 17, 384), (1, 4096, 4096), (2, 4099, 1408), (3, 100, 14336), (8, 33, 256),
                                   (9, 200, 1152), (16, 1000, 2048), (17, 257, 640), (31, 48, 4096), (33, 300, 1024), (64, 1408, 2048),
                                   (65, 130, 512), (130, 520, 896), (500, 64, 256), (0, 64, 256), (1, 40000, 128), (7, 15, 16384)])
def test_linear(T, N, K, G, y_dtype):
    w, x = make(T, N, K, G)
    codes, params = ops.quantize_linear(w, G)
    y = ops.linear(x, codes, params, y_dtype=binding.F32 if y_dtype == "f32" else binding.BF16)
    check(x, codes, params, G, y)
    guard = torch.full((T + 1, N), 5.0, dtype=y.dtype, device="cuda")   # nothing behind the last row is written
    out = ops.linear(x, codes, params, y_dtype=binding.F32 if y_dtype == "f32" else binding.BF16, out=guard[:T])
    assert torch.equal(out, y) and (guard[T] == 5.0).all()


# Matrices and token counts behind the few-token kernel's: token tiles of 16, 32 and 64, partly filled; rows that end inside a block of
# 256; a last step of 64 indices; blocks that one run of work holds, that two share, that all runs share.
MANY = [(9, 14393, 4096), (16, 4099, 14336), (17, 6401, 4096), (31, 4096, 8128), (33, 4101, 4160), (64, 257, 49216), (64, 13000, 1024),
        (65, 1000, 10304), (500, 1500, 1088), (4000, 250, 832), (20000, 130, 320), (20000, 700, 64), (65536, 33, 384)]


@pytest.mark.parametrize("y_dtype", ["f32", "bf16"])
@pytest.mark.parametrize("G", [64, 128])
@pytest.mark.parametrize("T,N,K", MANY)
def test_linear_many(T, N, K, G, y_dtype):
    """As above, but a result's groups are added up one behind the other (two roundings of 2^-24 each), then at most 32 pieces."""
    K = max(K // G, 1) * G
    w, x = make(T, N, K, G)
    codes, params = ops.quantize_linear(w, G)
    guard = torch.full((T + 1, N), 5.0, dtype=torch.float32 if y_dtype == "f32" else torch.bfloat16, device="cuda")
    y = ops.linear(x, codes, params, y_dtype=binding.F32 if y_dtype == "f32" else binding.BF16, out=guard[:T])
    assert ops.poll_linear_status() == 0
    q = torch.stack([codes & 15, codes >> 4], 2).view(N, K).double()
    s, m = params.double().repeat_interleave(G, 1).unbind(2)
    X = x.double()
    ref, C = X @ (s * q + m).T, X.abs() @ (s.abs() * (16 + q) + (m - 16 * s).abs()).T
    tol = (8 * 17 + K / G + 32) * 2.0 ** -23 * C + torch.finfo(y.dtype).eps / 2 * ref.abs()
    assert bool(((y.double() - ref).abs() <= tol * 1.01).all()) and bool((guard[T] == 5.0).all())
    assert torch.equal(ops.linear(x, codes, params, y_dtype=binding.F32 if y_dtype == "f32" else binding.BF16), y)


def test_non_finite_rows_many():
    """A token's infinity and NaN stay its own, in every tile."""
    w, x = make(70, 12000, 1024, 128)
    codes, params = ops.quantize_linear(w, 128)
    y = ops.linear(x, codes, params)
    want = y.clone()
    x[3, 17], x[64, 300], x[69] = float("inf"), float("nan"), 0
    y = ops.linear(x, codes, params)
    rest = [i for i in range(69) if i not in (3, 64)]
    assert torch.equal(y[rest], want[rest]) and (y[69] == 0).all()
    assert not torch.isfinite(y[3]).any() and torch.isnan(y[64]).all()


@pytest.mark.parametrize("G", [64, 128])
@pytest.mark.parametrize("N,K", [(1, 128), (5, 384), (129, 1408), (64, 4096)])
def test_quantizer_is_the_experts(N, K, G):
    w, _ = make(1, N, K, G)
    w[0, :G] = 0.25                     # a group of one value: its scale rounds to 0, so 1
    if N > 1:
        w[1, :G] = 0
    codes, params = ops.quantize_linear(w, G)
    q, _, _ = decoded(codes, params, G)
    ref_q, ref_s, ref_m = oracle.quantize(oracle.as_u16(w.cpu()), G, 4)
    assert np.array_equal(q.astype(np.uint8), ref_q)
    assert np.array_equal(params.cpu().view(torch.int16).numpy()[:, :, 0].view(np.uint16), ref_s)
    assert np.array_equal(params.cpu().view(torch.int16).numpy()[:, :, 1].view(np.uint16), ref_m)


def test_every_code_and_the_last_group():
    """One input index at a time: y is that column, exactly (a product and one addition of the zero-point, both representable)."""
    N, K, G = 32, 192, 64
    g = torch.Generator().manual_seed(3)
    q = torch.randint(0, 16, (N, K), generator=g)
    codes = (q[:, 0::2] | (q[:, 1::2] << 4)).to(torch.uint8).cuda()
    s = 2.0 ** torch.randint(-4, 3, (N, K // G), generator=g)
    m = torch.randint(-8, 8, (N, K // G), generator=g).float()
    params = torch.stack([s, m], 2).half().cuda()
    x = torch.eye(K).bfloat16().cuda()
    y = ops.linear(x, codes, params)
    want = (q.float() * s.repeat_interleave(G, 1) + m.repeat_interleave(G, 1)).t()
    assert torch.equal(y.cpu(), want)


def test_far_apart_magnitudes_and_non_finite_rows():
    w, x = make(5, 70, 512, 128)
    codes, params = ops.quantize_linear(w, 128)
    x[0] *= 1e30
    x[1] *= 1e-30
    x[2] = 0
    y = ops.linear(x, codes, params)
    check(x, codes, params, 128, y)
    assert (y[2] == 0).all()
    want = y.clone()
    x[3, 17], x[1, 300] = float("inf"), float("nan")
    y = ops.linear(x, codes, params)
    assert torch.equal(y[[0, 2, 4]], want[[0, 2, 4]])
    assert torch.isnan(y[1]).all() and not torch.isfinite(y[3]).any()


@pytest.mark.parametrize("T,N,K", [(8, 1000, 2048), (16, 14336, 4096), (40, 4352, 4096)])
def test_capture_and_streams(T, N, K):
    w, x = make(T, N, K, 128)
    codes, params = ops.quantize_linear(w, 128)
    want = ops.linear(x, codes, params)
    graphs, outs = [], []
    for _ in range(2):
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            outs.append(ops.linear(x, codes, params))
        graphs.append(gr)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(3):
        for gr, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                gr.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)


def test_refused_tensors():
    w, x = make(4, 64, 256, 128)
    codes, params = ops.quantize_linear(w, 128)
    for f in (lambda: ops.linear(x.float(), codes, params), lambda: ops.linear(x[:, :128], codes, params),
              lambda: ops.linear(x, codes[:60], params), lambda: ops.linear(x, codes.to(torch.int8), params),
              lambda: ops.linear(x, codes, params.float()), lambda: ops.linear(x, codes, params, y_dtype=3),
              lambda: ops.quantize_linear(w.float()), lambda: ops.quantize_linear(w, 32), lambda: ops.quantize_linear(w[:, :100])):
        with pytest.raises(ValueError):
            f()
    with pytest.raises(binding.DynamoError):
        ops.linear(x, codes, torch.zeros((64, 8, 2), dtype=torch.float16, device="cuda"))   # groups of 32
