"""Tokens sorted by expert and back, and the gradients, against numpy in 64 bits.

Tolerances: a sum of k terms in fp32 (each product and addition rounded once, off by at most 2^-24 of what has been summed) is
within (k + 1) 2^-24 of the terms' absolute sum, and twice that is allowed; a result's own rounding is off by at most
eps / 2 of the value.  A dot product of d terms: d 2^-24 of the terms' absolute sum, whatever the order."""
import numpy as np
import pytest
import torch

from paper_2503_21135_b200 import binding
from paper_2503_21135_b200 import operators as ops

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def make_idx(T, E, k, drop, seed):
    """Distinct experts a token, skewed; drop: some pairs and whole tokens outside the range."""
    rng = np.random.default_rng(seed)
    score = rng.standard_normal((T, E)) - 1.2 * np.log1p(rng.permutation(E))[None, :]
    idx = np.argsort(-score, axis=1, kind="stable")[:, :k].astype(np.int32)
    if drop == "some":
        idx[rng.random((T, k)) < 0.2] = -1
        idx[::5] = E + 3
        idx[3::7, 0] = -2147483648
    elif drop == "all":
        idx[:] = -1
    return idx


def sorted_pairs(idx, E):
    flat = idx.ravel().astype(np.int64)
    keep = (flat >= 0) & (flat < E)
    pairs = np.flatnonzero(keep)
    order = pairs[np.argsort(flat[pairs], kind="stable")]
    pos = np.full(flat.size, -1, np.int64)
    pos[order] = np.arange(order.size)
    offsets = np.concatenate([[0], np.cumsum(np.bincount(flat[pairs], minlength=E))])
    return offsets, order, pos.reshape(idx.shape)


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


SHAPES = [(0, 8, 2, 64), (1, 1, 1, 8), (1, 8, 2, 4096), (2, 5, 3, 72), (7, 64, 6, 2048), (33, 8, 8, 264), (256, 256, 8, 64),
          (1000, 8, 2, 1408), (2047, 64, 6, 512), (2500, 60, 7, 40), (5000, 256, 8, 8), (9001, 16, 2, 16), (40000, 3, 1, 24),
          (700000, 4, 1, 8)]


@pytest.mark.parametrize("drop", ["none", "some", "all"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,E,k,d", SHAPES)
def test_dispatch(T, E, k, d, dtype, drop):
    if T > 10000 and (drop == "all" or dtype == "f32"):
        drop = "none"
    idx = make_idx(T, E, k, drop, T + E)
    g = torch.Generator(device="cuda").manual_seed(T + 1)
    x = torch.randn((T, d), generator=g, device="cuda").to(DT[dtype])
    rows = torch.full((T * k, d), 77.0, dtype=DT[dtype], device="cuda")
    off = torch.full((E + 1,), -7, dtype=torch.int32, device="cuda")
    perm = torch.full((T * k,), -7, dtype=torch.int32, device="cuda")
    pos = torch.full((T, k), -7, dtype=torch.int32, device="cuda")
    r = ops.dispatch(torch.from_numpy(idx).cuda(), E, x, out=(rows, off, perm, pos))
    ref_off, ref_perm, ref_pos = sorted_pairs(idx, E)
    n = ref_perm.size
    assert np.array_equal(r.offsets.cpu().numpy(), ref_off)
    assert np.array_equal(r.perm.cpu().numpy()[:n], ref_perm) and (r.perm.cpu().numpy()[n:] == -7).all()
    assert np.array_equal(r.pos.cpu().numpy(), ref_pos)
    assert torch.equal(r.rows[:n], x[torch.from_numpy(ref_perm // k).cuda()])
    assert (r.rows[n:] == 77.0).all()
    alone = ops.dispatch(torch.from_numpy(idx).cuda(), E)
    assert alone.rows is None and torch.equal(alone.pos, r.pos) and torch.equal(alone.offsets, r.offsets)
    assert torch.equal(alone.perm[:n], r.perm[:n])


def routed(T, E, k, d, dtype, drop, seed):
    idx = make_idx(T, E, k, drop, seed)
    _, order, pos = sorted_pairs(idx, E)
    g = torch.Generator(device="cuda").manual_seed(seed)
    rows = torch.randn((T * k, d), generator=g, device="cuda").to(DT[dtype])
    rows[order.size:] = float("nan")          # nothing has written there
    w = torch.rand((T, k), generator=g, device="cuda")
    post = torch.from_numpy(pos.astype(np.int32)).cuda()
    w[post < 0] = float("inf")                # nor has anybody looked at these
    return rows, post, w, pos, order.size


@pytest.mark.parametrize("weights", [True, False])
@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("dtype,drop", [("bf16", "none"), ("bf16", "some"), ("f32", "some"), ("f32", "all")])
@pytest.mark.parametrize("T,E,k,d", [(0, 8, 2, 64), (1, 8, 2, 4096), (5, 5, 5, 8), (37, 64, 6, 2048), (130, 16, 4, 72),
                                     (1000, 8, 3, 1408), (3000, 256, 8, 24), (333, 9, 7, 520), (64, 3, 1, 16384)])
def test_combine(T, E, k, d, dtype, drop, out, weights):
    rows, post, w, pos, n = routed(T, E, k, d, dtype, drop, T + k)
    y = ops.combine(rows, post, w if weights else None, y_dtype=binding.BF16 if out == "bf16" else binding.F32)
    assert y.dtype == DT[out] and y.shape == (T, d)
    kept = (pos >= 0)[:, :, None]
    terms = np.where(kept, f64(rows)[np.maximum(pos, 0)], 0.0)
    if weights:
        terms = terms * np.where(kept, f64(w)[:, :, None], 0.0)
    ref, mag = terms.sum(1), np.abs(terms).sum(1)
    tol = torch.finfo(DT[out]).eps / 2 * np.abs(ref) + 2 * (k + 1) * 2.0 ** -24 * mag
    assert (np.abs(f64(y) - ref) <= tol * 1.01).all()
    if not weights:
        assert torch.equal(ops.dispatch_backward(rows, post), ops.combine(rows, post))
    if T:
        assert torch.equal(y, ops.combine(rows, post, w if weights else None,
                                          y_dtype=binding.BF16 if out == "bf16" else binding.F32))


@pytest.mark.parametrize("dy_type", ["bf16", "f32"])
@pytest.mark.parametrize("dtype,drop", [("bf16", "none"), ("bf16", "some"), ("f32", "some"), ("f32", "all")])
@pytest.mark.parametrize("T,E,k,d", [(0, 8, 2, 64), (1, 8, 2, 4096), (5, 5, 5, 8), (37, 64, 6, 2048), (131, 16, 4, 1024),
                                     (1000, 8, 3, 1408), (777, 256, 8, 264), (64, 3, 1, 16384)])
def test_combine_backward(T, E, k, d, dtype, drop, dy_type):
    rows, post, w, pos, n = routed(T, E, k, d, dtype, drop, T + k + 1)
    g = torch.Generator(device="cuda").manual_seed(5)
    dy = torch.randn((T, d), generator=g, device="cuda").to(DT[dy_type])
    d_rows = torch.full_like(rows, 77.0)
    got, d_w = ops.combine_backward(dy, rows, post, w, d_rows=d_rows)
    assert got is d_rows and (d_rows[n:] == 77.0).all()
    R, D, W = f64(rows), f64(dy), f64(w)
    ref = np.zeros((n, d))
    ref_w, mag_w = np.zeros((T, k)), np.zeros((T, k))
    for j in range(k):
        t = np.flatnonzero(pos[:, j] >= 0)
        ref[pos[t, j]] = W[t, j][:, None] * D[t]
        ref_w[t, j] = (R[pos[t, j]] * D[t]).sum(1)
        mag_w[t, j] = np.abs(R[pos[t, j]] * D[t]).sum(1)
    tol = (torch.finfo(DT[dtype]).eps / 2 + 2.0 ** -23) * np.abs(ref)
    assert (np.abs(f64(d_rows[:n]) - ref) <= tol * 1.01).all()
    assert (np.abs(f64(d_w) - ref_w) <= d * 2.0 ** -24 * mag_w + 1e-30).all()
    assert (f64(d_w)[pos < 0] == 0).all()
    ones, none = ops.combine_backward(dy, rows, post, want_d_w=False)
    assert none is None and torch.equal(ones[:n], torch.from_numpy(D).cuda()[torch.from_numpy(
        np.repeat(np.arange(T), k)[np.argsort(np.where(pos < 0, T * k, pos).ravel(), kind="stable")][:n]).cuda()].to(rows.dtype))


def test_gradients_against_differences():
    """The loss's difference along a direction, in 64 bits, against the gradients (fp32 rows: relative 1e-6 of the terms)."""
    T, E, k, d = 50, 8, 3, 64
    idx = make_idx(T, E, k, "some", 1)
    g = torch.Generator(device="cuda").manual_seed(9)
    x, dx = (torch.randn((T, d), generator=g, device="cuda") for _ in range(2))
    w, dw = (torch.rand((T, k), generator=g, device="cuda") for _ in range(2))
    dy = torch.randn((T, d), generator=g, device="cuda")
    r = ops.dispatch(torch.from_numpy(idx).cuda(), E, x)
    rows = torch.nan_to_num(r.rows)
    d_rows, d_w = ops.combine_backward(dy, rows, r.pos, w)
    d_x = ops.dispatch_backward(d_rows, r.pos)
    kept = f64(r.pos) >= 0

    def loss(X, W):
        return (f64(dy) * (X[:, None, :] * np.where(kept, W, 0.0)[:, :, None]).sum(1)).sum()

    h = 1e-4
    diff = (loss(f64(x) + h * f64(dx), f64(w) + h * f64(dw)) - loss(f64(x) - h * f64(dx), f64(w) - h * f64(dw))) / (2 * h)
    terms_x, terms_w = f64(d_x) * f64(dx), f64(d_w) * f64(dw)
    assert abs(terms_x.sum() + terms_w.sum() - diff) <= 1e-5 * (np.abs(terms_x).sum() + np.abs(terms_w).sum())


def test_same_expert_twice_and_wild_positions():
    idx = torch.tensor([[2, 2], [0, 2], [2, 2]], dtype=torch.int32, device="cuda")
    x = torch.arange(24, dtype=torch.float32, device="cuda").view(3, 8)
    r = ops.dispatch(idx, 4, x)
    assert r.pos.tolist() == [[1, 2], [0, 3], [4, 5]] and r.offsets.tolist() == [0, 1, 1, 6, 6]
    pos = torch.tensor([[6, 0], [1 << 30, -9], [5, 2147483647]], dtype=torch.int32, device="cuda")
    y = ops.combine(r.rows, pos)
    assert torch.equal(y, torch.stack([r.rows[0], torch.zeros(8, device="cuda"), r.rows[5]]))


def test_capture_streams_and_repetition():
    T, E, k, d = 3000, 64, 6, 256
    idxs = [torch.from_numpy(make_idx(T, E, k, "some", s)).cuda() for s in (1, 2)]
    xs = [torch.randn((T, d), device="cuda") for _ in range(2)]
    w = torch.rand((T, k), device="cuda")

    def step(idx, x):
        r = ops.dispatch(idx, E, x)
        y = ops.combine(r.rows, r.pos, w)
        d_rows, d_w = ops.combine_backward(y, r.rows, r.pos, w)
        return y, d_w, ops.dispatch_backward(d_rows, r.pos)

    want = [step(i, x) for i, x in zip(idxs, xs)]
    torch.cuda.synchronize()
    # two graphs over the same inputs' buffers, replayed on two streams at once
    idx, x = idxs[0].clone(), xs[0].clone()
    graphs, outs = [], []
    for _ in range(2):
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            outs.append(step(idx, x))
        graphs.append(gr)
    for i in (1, 0):
        idx.copy_(idxs[i])
        x.copy_(xs[i])
        torch.cuda.synchronize()
        streams = [torch.cuda.Stream() for _ in range(2)]
        for gr, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                gr.replay()
        torch.cuda.synchronize()
        for out in outs:
            assert all(torch.equal(a, b) for a, b in zip(out, want[i]))


def test_refused_tensors():
    idx = torch.zeros((4, 2), dtype=torch.int32, device="cuda")
    x = torch.zeros((4, 64), device="cuda")
    for f in (lambda: ops.dispatch(idx.long(), 8, x), lambda: ops.dispatch(idx, 8, x[:3]), lambda: ops.dispatch(idx, 8, x.half()),
              lambda: ops.dispatch(idx, 8, x.t()), lambda: ops.dispatch(idx[:, ::2], 8, x),
              lambda: ops.combine(x, idx), lambda: ops.combine(x, idx, torch.zeros(4, 1, device="cuda")),
              lambda: ops.combine(torch.zeros(8, 64, device="cuda"), idx, y_dtype=7),
              lambda: ops.combine_backward(x[:3], torch.zeros(8, 64, device="cuda"), idx)):
        with pytest.raises(ValueError):
            f()
    for f in (lambda: ops.dispatch(idx, 300, x), lambda: ops.dispatch(idx, 1, x), lambda: ops.dispatch(idx, 8, x[:, :12].contiguous()),
              lambda: ops.dispatch(idx, 8, torch.zeros(4 * 64 + 2, device="cuda")[2:].view(4, 64))):
        with pytest.raises(binding.DynamoError):
            f()
