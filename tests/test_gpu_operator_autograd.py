"""The operators around the layer are not differentiable by themselves: a tensor whose gradient is wanted is refused, and a tensor that a
call writes counts as changed."""
import pytest
import torch

from helpers import make_gpu_layer, make_inputs
from paper_2503_21135_b200 import binding
from paper_2503_21135_b200 import operators as ops
from paper_2503_21135_b200 import workloads as wl

pytestmark = pytest.mark.gpu


def setup():
    idx = torch.tensor([[0, 1], [1, 2], [2, 0]], dtype=torch.int32, device="cuda")
    x = torch.randn((3, 64), device="cuda")
    s = ops.dispatch(idx, 3, x)
    return idx, x, s


def calls():
    """name -> (floating-point inputs, call on them)."""
    idx, x, s = setup()
    stats = ops.norm_join(x, x, want_stats=True)[2]
    vec = torch.ones(64, device="cuda")
    codes, params = ops.quantize_linear(x.bfloat16(), 64)
    w = torch.rand((3, 2), device="cuda")
    return {"dispatch": ([x], lambda a: ops.dispatch(idx, 3, a)),
            "combine": ([s.rows, w], lambda a, b: ops.combine(a, s.pos, b)),
            "dispatch_backward": ([s.rows], lambda a: ops.dispatch_backward(a, s.pos)),
            "combine_backward": ([x, s.rows, w], lambda a, b, c: ops.combine_backward(a, b, s.pos, c)),
            "norm_join": ([x, x.clone(), vec, vec.clone(), vec.clone()],
                          lambda a, b, c, e, f: ops.norm_join(a, b, w_post=c, gate=e, w_pre=f)),
            "norm_join_backward": ([x, x.clone(), x.clone(), x.clone(), stats, vec, vec.clone(), vec.clone()],
                                   lambda a, b, c, e, f, p, q, h: ops.norm_join_backward(a, b, c, e, f, w_post=p, gate=q, w_pre=h)),
            "quantize_linear": ([x.bfloat16()], lambda a: ops.quantize_linear(a, 64)),
            "linear": ([x.bfloat16(), params], lambda a, b: ops.linear(a, codes, b))}


NAMES = ["dispatch", "combine", "dispatch_backward", "combine_backward", "norm_join", "norm_join_backward", "quantize_linear", "linear"]


@pytest.mark.parametrize("name", NAMES)
def test_a_wanted_gradient_is_refused(name):
    inputs, call = calls()[name]
    want = call(*inputs)
    for i in range(len(inputs)):
        args = [t.detach().requires_grad_(j == i) for j, t in enumerate(inputs)]
        with pytest.raises(ValueError, match="gradient"):
            call(*args)
        with torch.no_grad():
            got = call(*args)
        with torch.inference_mode():
            call(*args)
        flat = [v.values() if isinstance(v, dict) else v if isinstance(v, tuple) else [v] for v in (got, want)]
        assert all(a is None and b is None or torch.equal(a, b) for a, b in zip(*flat))


def test_a_given_output_that_wants_a_gradient_is_refused():
    idx, x, s = setup()
    out = torch.zeros((3, 64), device="cuda", requires_grad=True)
    with pytest.raises(ValueError, match="gradient"):
        ops.combine(s.rows, s.pos, out=out)
    with torch.no_grad():
        ops.combine(s.rows, s.pos, out=out)


@pytest.fixture(scope="module")
def block():
    """A layer, its router, and a stream of four tokens."""
    cfg = wl.CONFIGS["tiny"]
    wg, wu, wd, bits, pool, sets = make_inputs(cfg)
    gpu = make_gpu_layer(cfg, wg, wu, wd, bits, pool, max_tokens=16)
    gpu.set_channel_switch(sets)
    w_r, bias = (t.cuda() for t in wl.router_weights(cfg))
    r, n = (torch.randn((4, cfg.d_model), device="cuda").bfloat16() for _ in range(2))
    w = torch.ones(cfg.d_model, dtype=torch.bfloat16, device="cuda")
    return gpu, w_r, bias, r, n, w


def test_block_forward(block):
    gpu, w_r, bias, r, n, w = block
    want = gpu.forward_block(r, n, w_r, bias, w_post=w)
    p = torch.nn.Parameter(w)
    with pytest.raises(ValueError, match="gradient"):
        gpu.forward_block(r, n, w_r, bias, w_post=p)
    with pytest.raises(ValueError, match="gradient"):
        gpu.forward_block(r, n, torch.nn.Parameter(w_r), bias)
    with torch.no_grad():
        got = gpu.forward_block(r, n, w_r, bias, w_post=p)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_written_tensors_count_as_changed():
    idx, x, s = setup()
    codes, params = ops.quantize_linear(x.bfloat16(), 64)
    r, n = torch.zeros_like(x), torch.zeros((3, 64), dtype=torch.bfloat16, device="cuda")
    y, out, d_rows = torch.zeros((3, 3), device="cuda"), torch.zeros_like(x), torch.zeros_like(s.rows)
    for written, call in ((list(s), lambda: ops.dispatch(idx, 3, x, out=tuple(s))), ([out], lambda: ops.combine(s.rows, s.pos, out=out)),
                          ([out], lambda: ops.dispatch_backward(s.rows, s.pos, out=out)),
                          ([d_rows], lambda: ops.combine_backward(x, s.rows, s.pos, d_rows=d_rows)),
                          ([r, n], lambda: ops.norm_join(r, x, r_out=r, n_out=n)),
                          ([y], lambda: ops.linear(x.bfloat16(), codes, params, out=y))):
        before = [t._version for t in written]
        call()
        assert [t._version for t in written] == [v + 1 for v in before]
    # what autograd kept of a tensor that a call then wrote is not used for a gradient
    leaf = torch.ones((3, 64), device="cuda", requires_grad=True)
    loss = (leaf * out).sum()
    ops.combine(s.rows, s.pos, out=out)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()


def test_inference_tensors_can_be_given():
    """They have no version to count; torch keeps none of them for a gradient."""
    idx, x, s = setup()
    with torch.inference_mode():
        out = torch.zeros((3, 64), device="cuda")
    ops.combine(s.rows, s.pos, out=out)
    assert torch.equal(out, ops.combine(s.rows, s.pos))


def test_block_writes_count(block):
    gpu, w_r, bias, r, n, w = block
    r, n = r.clone(), n.clone()
    y = torch.empty_like(r)
    before = [t._version for t in (r, n, y)]
    gpu.forward_block(r, n, w_r, bias, w_post=w, y=y, y_dtype=binding.BF16)
    assert [t._version for t in (r, n, y)] == [before[0], before[1], before[2] + 1]
    gpu.forward_block(r, n, w_r, bias, w_post=w, y=y, y_dtype=binding.BF16, in_place=True)
    assert [t._version for t in (r, n, y)] == [before[0] + 1, before[1] + 1, before[2] + 2]
