"""The operators around the layer in a row, as a decoder block uses them: the layer with the join behind it, blocks one behind the
other, experts of one's own between dispatch and combine, and the gradients through all of it.

The calls are the same kernels as by themselves, so the block is compared with its parts bit for bit.  The chains are compared with
64 bits by stages: every stage's result against the reference of the inputs that it had, within the bounds of the single operators'
tests, so that no bound has to be carried through a product."""
import numpy as np
import pytest
import torch

from helpers import make_gpu_layer, make_inputs
from paper_2503_21135_b200 import binding
from paper_2503_21135_b200 import operators as ops
from paper_2503_21135_b200 import workloads as wl

pytestmark = pytest.mark.gpu
CFG = wl.CONFIGS["tiny"]
U = 2.0 ** -24


@pytest.fixture(scope="module")
def layer():
    wg, wu, wd, bits, pool, sets = make_inputs(CFG)
    gpu = make_gpu_layer(CFG, wg, wu, wd, bits, pool, max_tokens=256)
    gpu.set_channel_switch(sets)
    w_r, bias = wl.router_weights(CFG)
    return gpu, w_r.cuda(), bias.cuda()


def stream(T, r_dtype, gate, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed + T)
    d = CFG.d_model

    def randn(*s, dtype=torch.bfloat16, scale=1.0):
        return (torch.randn(s, generator=g, device="cuda") * scale).to(dtype)

    r = randn(T, d, dtype=r_dtype)
    how = dict(w_post=randn(d), w_pre=randn(d), gate={"none": None, "channel": randn(d), "token": randn(T, 1, dtype=torch.float32)}[gate],
               res_scale=0.9, block_scale=0.7, eps=1e-5)
    return r, how


@pytest.mark.parametrize("r_dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("y_dtype", [binding.BF16, binding.F32])
@pytest.mark.parametrize("T,gate", [(0, "none"), (1, "token"), (7, "channel"), (64, "none"), (200, "token")])
def test_block_is_its_parts(layer, T, gate, y_dtype, r_dtype):
    gpu, w_r, bias = layer
    r, how = stream(T, r_dtype, gate)
    _, n = ops.norm_join(r)
    y = gpu.forward_router(n, w_r, bias, y_dtype)
    want_r, want_n = ops.norm_join(r, y, **how)
    y_own = torch.empty_like(y)
    before = gpu.kernel_launches()
    r_out, n_out = gpu.forward_block(r, n, w_r, bias, y_dtype=y_dtype, y=y_own, **how)
    assert gpu.poll_status() == 0 and (gpu.kernel_launches() > before) == (T > 0)
    assert torch.equal(y_own, y) and torch.equal(r_out, want_r) and torch.equal(n_out, want_n)
    only_r, none = gpu.forward_block(r, n, w_r, bias, y_dtype=y_dtype, **{**how, "w_pre": None}, pre_norm=False)
    assert torch.equal(only_r, want_r) and none is None
    got = gpu.forward_block(r, n, w_r, bias, y_dtype=y_dtype, in_place=True, **how)
    assert got[0] is r and got[1] is n and torch.equal(r, want_r) and torch.equal(n, want_n)


def test_blocks_in_a_row_captured(layer):
    """Three blocks in place, as a graph: the same bits as one call after the other, on every replay."""
    gpu, w_r, bias = layer
    r0, how = stream(33, torch.bfloat16, "channel")
    r, n = r0.clone(), torch.empty_like(r0)

    def blocks():
        ops.norm_join(r, n_out=n)
        for _ in range(3):
            gpu.forward_block(r, n, w_r, bias, in_place=True, **how)

    blocks()
    want_r, want_n = r.clone(), n.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        blocks()
    for _ in range(3):
        r.copy_(r0)
        graph.replay()
        assert torch.equal(r, want_r) and torch.equal(n, want_n)
    assert gpu.poll_status() == 0


def test_block_refusals(layer):
    gpu, w_r, bias = layer
    r, how = stream(4, torch.bfloat16, "none")
    _, n = ops.norm_join(r)
    for f in (lambda: gpu.forward_block(r, n.float(), w_r, bias), lambda: gpu.forward_block(r, n, w_r[:4], bias),
              lambda: gpu.forward_block(r, n, w_r, bias, w_post=how["w_post"].float(), w_pre=how["w_pre"]),
              lambda: gpu.forward_block(r, n, w_r, bias, gate=how["w_post"][:, None]), lambda: gpu.forward_block(r, n, w_r, bias, post_norm=False, w_post=how["w_post"])):
        with pytest.raises(AssertionError):
            f()
    empty = binding.DynamoLayer.from_config(CFG, max_tokens=8)
    with pytest.raises(binding.DynamoError):
        empty.forward_block(r, n, w_r, bias)             # a layer without weights
    big, _ = stream(300, torch.bfloat16, "none")
    with pytest.raises(binding.DynamoError):
        gpu.forward_block(big, big.clone(), w_r, bias)   # more tokens than the layer has room for


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


@pytest.mark.parametrize("T,E,k,d,G,scale", [(1, 4, 2, 256, 64, 1.0), (37, 8, 2, 512, 128, 1.0), (150, 5, 3, 192, 64, 30.0)])
def test_experts_of_ones_own(T, E, k, d, G, scale):
    """Routing, dispatch, a 4-bit product an expert, combine, join.  With scores of a wide range most tokens go to few experts and
    others get no token; a third of the pairs is dropped."""
    g = torch.Generator(device="cuda").manual_seed(T)
    r = torch.randn((T, d), generator=g, device="cuda").bfloat16()
    logits = torch.randn((T, E), generator=g, device="cuda") * scale
    w = [(torch.randn((d, d), generator=g, device="cuda") * 0.05).bfloat16() for _ in range(E)]
    idx = torch.empty((T, k), dtype=torch.int32, device="cuda")
    tw = torch.empty((T, k), device="cuda")
    off = torch.empty(E + 1, dtype=torch.int32, device="cuda")
    perm = torch.empty(T * k, dtype=torch.int32, device="cuda")
    assert binding.dynamo_route_permute_static(logits.data_ptr(), T, E, k, 1, idx.data_ptr(), tw.data_ptr(), off.data_ptr(),
                                               perm.data_ptr(), torch.cuda.current_stream().cuda_stream) == 0
    _, n = ops.norm_join(r)
    s = ops.dispatch(idx, E, n)
    assert torch.equal(s.offsets, off) and torch.equal(s.perm, perm)      # the library's own sort
    idx[:, k - 1][torch.rand(T, generator=g, device="cuda") < 0.3] = -1
    s = ops.dispatch(idx, E, n)
    o = s.offsets.tolist()
    assert torch.equal(s.rows[:o[-1]], n[(s.perm[:o[-1]] // k).long()])
    out = torch.full((T * k, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    for e in range(E):
        codes, params = ops.quantize_linear(w[e], G)
        ops.linear(s.rows[o[e]:o[e + 1]], codes, params, y_dtype=binding.BF16, out=out[o[e]:o[e + 1]])
        q = np.stack([codes.cpu().numpy() & 15, codes.cpu().numpy() >> 4], 2).reshape(d, d)
        sc, m = (np.repeat(f64(params)[:, :, i], G, 1) for i in (0, 1))
        X = f64(s.rows[o[e]:o[e + 1]])
        ref, C = X @ (sc * q + m).T, np.abs(X) @ (np.abs(sc) * (16 + q) + np.abs(m - 16 * sc)).T
        assert (np.abs(f64(out[o[e]:o[e + 1]]) - ref) <= 1.01 * ((8 * 17 + d / 512 + 16) * 2 * U * C + 2.0 ** -8 * np.abs(ref))).all()
    y = ops.combine(out, s.pos, tw, y_dtype=binding.F32)      # rows behind the last pair are NaN and read by nobody
    pos, W, rows = s.pos.cpu().numpy(), f64(tw), f64(out)
    terms = np.where((pos >= 0)[:, :, None], W[:, :, None] * rows[np.maximum(pos, 0)], 0.0)
    assert (np.abs(f64(y) - terms.sum(1)) <= 2 * (k + 1) * U * np.abs(terms).sum(1)).all()
    r_out, n_out = ops.norm_join(r, y, eps=1e-5, res_scale=0.5)
    Y = f64(y)
    z = Y / np.sqrt((Y * Y).mean(1, keepdims=True) + 1e-5)
    ref = 0.5 * f64(r) + z
    R = 0.5 * np.abs(f64(r)) + np.abs(z)
    assert (np.abs(f64(r_out) - ref) <= 64 * U * R + 2.0 ** -8 * np.abs(ref)).all()
    ref_n = ref / np.sqrt((ref * ref).mean(1, keepdims=True) + 1e-5)
    near = 64 * U * (1 + np.linalg.norm(R, axis=1) / np.linalg.norm(ref, axis=1))[:, None] * np.abs(ref_n) + 64 * U * R * np.abs(ref_n / ref)
    assert (np.abs(f64(n_out) - ref_n) <= near + 2.0 ** -8 * np.abs(ref_n)).all()


def test_gradients_through_a_row():
    """Dispatch, one matrix an expert (torch's product), combine, join, all in fp32, and the gradients of a weighted sum of both results:
    against automatic differentiation in 64 bits.  What each operator adds is within 256 u of the absolute terms; as the references
    are well away from cancellation only in the norm, the gradients are compared by their 2-norms: 2000 u, of which torch's fp32
    products (sums of 96 terms, 96 u each way) take the larger part; and against differences of the 64-bit loss along the gradient."""
    T, E, k, d = 41, 5, 2, 96
    g = torch.Generator().manual_seed(9)

    def randn(*s):
        return torch.randn(s, generator=g)

    x, r, W = randn(T, d), randn(T, d), randn(E, d, d) * 0.1
    w_post, w_pre, gate = randn(d), randn(d), randn(T, 1)
    idx = torch.stack([torch.randperm(E, generator=g)[:k] for _ in range(T)]).int()
    idx[::6, 1] = -1
    tw = torch.rand((T, k), generator=g)
    c_n, c_r = randn(T, d), randn(T, d)
    leaves64 = [t.double().requires_grad_() for t in (x, r, W, tw, w_post, w_pre, gate)]

    def loss64(x, r, W, tw, w_post, w_pre, gate):
        keep = (idx >= 0).double()
        y = (torch.einsum("td,tkde->tke", x, W[idx.clamp(min=0).long()]) * (tw * keep)[:, :, None]).sum(1)
        z = y * torch.rsqrt((y * y).mean(1, keepdim=True) + 1e-5) * w_post
        ro = 0.9 * r + 0.7 * gate * z
        n = ro * torch.rsqrt((ro * ro).mean(1, keepdim=True) + 1e-5) * w_pre
        return (n * c_n).sum() + (ro * c_r).sum()

    L = loss64(*leaves64)
    want = torch.autograd.grad(L, leaves64)
    eps = 1e-6
    for leaf, gr in zip(leaves64, want):     # the reference itself, along the gradient
        args = [t.detach() for t in leaves64]
        i = next(j for j, t in enumerate(leaves64) if t is leaf)
        v = gr / gr.norm()
        up, down = list(args), list(args)
        up[i], down[i] = args[i] + eps * v, args[i] - eps * v
        assert abs(float(loss64(*up) - loss64(*down)) / (2 * eps) - float(gr.norm())) <= 1e-5 * float(gr.norm())

    X, R, WW, TW, WP, WQ, GT, CN, CR = (t.cuda() for t in (x, r, W, tw, w_post, w_pre, gate, c_n, c_r))
    s = ops.dispatch(idx.cuda(), E, X)
    o = s.offsets.tolist()
    rows = torch.zeros((T * k, d), device="cuda")
    for e in range(E):
        rows[o[e]:o[e + 1]] = s.rows[o[e]:o[e + 1]] @ WW[e]
    y = ops.combine(rows, s.pos, TW)
    how = dict(w_post=WP, gate=GT, w_pre=WQ, res_scale=0.9, block_scale=0.7, eps=1e-5)
    ro, n, stats = ops.norm_join(R, y, n_dtype=binding.F32, want_stats=True, **how)
    loss = float((n.double() * CN.double()).sum() + (ro.double() * CR.double()).sum())
    assert abs(loss - float(L.detach())) <= 2000 * U * float((n * CN).abs().sum() + (ro * CR).abs().sum())
    gj = ops.norm_join_backward(CN, CR, R, y, stats, **how)
    d_rows, d_w = ops.combine_backward(gj["d_y"], rows, s.pos, TW)
    d_in, d_W = torch.zeros((T * k, d), device="cuda"), torch.zeros_like(WW)
    for e in range(E):
        d_in[o[e]:o[e + 1]] = d_rows[o[e]:o[e + 1]] @ WW[e].T
        d_W[e] = s.rows[o[e]:o[e + 1]].T @ d_rows[o[e]:o[e + 1]]
    got = (ops.dispatch_backward(d_in, s.pos), gj["d_r"], d_W, d_w, gj["d_w_post"], gj["d_w_pre"], gj["d_gate"])
    for a, b, name in zip(got, want, ("x", "r", "W", "tw", "w_post", "w_pre", "gate")):
        diff = float((a.cpu().double().reshape(b.shape) - b).norm())
        assert diff <= 2000 * U * float(b.norm()), (name, diff / float(b.norm()))
