"""Refusals of the operators around the layer: everything is checked on the host before any launch (no GPU needed; the
pointers are made up and never followed)."""
import ctypes

import pytest
import torch

from paper_2503_21135_b200 import binding, build
from paper_2503_21135_b200 import operators as ops

OK, NULL, SHAPE, ALIGN, SMALL, TOKENS, ARG = 0, 1, 2, 4, 5, 10, 13
P = 1 << 20   # an aligned address


@pytest.fixture(scope="module")
def lib():
    build.build_library()
    return binding.load()


def _bytes(f, *a):
    n = ctypes.c_size_t(77)
    return f(*a, ctypes.byref(n)), n.value


def test_dispatch_refusals(lib):
    good = dict(idx=P, T=64, E=8, k=2, x=P, d=64, dt=0, off=P, perm=P, pos=P, rows=P, ws=None, nb=0)

    def call(**kw):
        a = {**good, **kw}
        return lib.dynamo_dispatch(a["idx"], a["T"], a["E"], a["k"], a["x"], a["d"], a["dt"], a["off"], a["perm"], a["pos"],
                                   a["rows"], a["ws"], a["nb"], None)

    for kw, st in ((dict(E=0), SHAPE), (dict(E=257), SHAPE), (dict(k=0), SHAPE), (dict(k=9, E=16), SHAPE), (dict(k=3, E=2), SHAPE),
                   (dict(T=-1), TOKENS), (dict(T=1 << 30), TOKENS), (dict(d=4), SHAPE), (dict(d=12), SHAPE), (dict(d=0), SHAPE),
                   (dict(dt=2), SHAPE), (dict(idx=None), NULL), (dict(off=None), NULL), (dict(perm=None), NULL),
                   (dict(pos=None), NULL), (dict(rows=None), NULL), (dict(x=None), NULL), (dict(x=P + 8), ALIGN),
                   (dict(rows=P + 4), ALIGN), (dict(T=100000, ws=None), NULL), (dict(T=100000, ws=P, nb=16), SMALL),
                   (dict(T=100000, ws=P + 16, nb=1 << 30), ALIGN)):
        assert call(**kw) == st, kw
    assert _bytes(lib.dynamo_dispatch_workspace_bytes, 64, 8, 2) == (OK, 0)
    st, n = _bytes(lib.dynamo_dispatch_workspace_bytes, 100000, 256, 8)
    assert st == OK and n >= 256 * 4
    assert lib.dynamo_dispatch_workspace_bytes(64, 8, 2, None) == NULL


def test_combine_refusals(lib):
    def fwd(rows=P, dt=0, pos=P, w=P, T=4, k=2, d=64, y=P, ydt=1):
        return lib.dynamo_combine(rows, dt, pos, w, T, k, d, y, ydt, None)

    def bwd(dy=P, dydt=0, rows=P, dt=0, pos=P, w=P, T=4, k=2, d=64, dr=P, dw=P):
        return lib.dynamo_combine_backward(dy, dydt, rows, dt, pos, w, T, k, d, dr, dw, None)

    for kw, st in ((dict(k=0), SHAPE), (dict(k=9), SHAPE), (dict(d=7), SHAPE), (dict(dt=5), SHAPE), (dict(T=-1), TOKENS),
                   (dict(T=1 << 30), TOKENS), (dict(rows=None), NULL), (dict(pos=None), NULL), (dict(rows=P + 2), ALIGN)):
        assert fwd(**kw) == st and bwd(**kw) == st, kw
    assert fwd(ydt=2) == SHAPE and fwd(y=None) == NULL and fwd(y=P + 8) == ALIGN
    assert fwd(T=0, rows=None, pos=None, y=None) == OK and bwd(T=0, dy=None, rows=None, pos=None, dr=None) == OK
    assert bwd(dydt=2) == SHAPE and bwd(dy=None) == NULL and bwd(dr=None) == NULL and bwd(dr=P + 8) == ALIGN


def _desc(**kw):
    base = dict(d=64, y_dtype=0, r_dtype=0, n_dtype=0, w_dtype=1, gate_kind=0, post_norm=1, pre_norm=1, res_scale=1.0,
                block_scale=1.0, eps=1e-6)
    base.update(kw)
    return binding.JoinDesc(**base)


BAD_DESC = [(dict(d=0), SHAPE), (dict(d=20), SHAPE), (dict(d=16392), SHAPE), (dict(y_dtype=2), SHAPE), (dict(r_dtype=-1), SHAPE),
            (dict(n_dtype=3), SHAPE), (dict(w_dtype=9), SHAPE), (dict(gate_kind=3), ARG), (dict(eps=0.0), ARG), (dict(eps=-1.0), ARG),
            (dict(eps=float("nan")), ARG), (dict(res_scale=float("inf")), ARG), (dict(block_scale=float("nan")), ARG)]


def test_norm_join_refusals(lib):
    def fwd(desc=None, r=P, y=P, wp=P, gate=None, wq=P, T=4, ro=P, no=P, st=None, **kw):
        D = _desc(**kw) if desc is None else desc
        return lib.dynamo_norm_join_forward(ctypes.byref(D) if D else None, r, y, wp, gate, wq, T, ro, no, st, None)

    def bwd(dn=P, dro=P, r=P, y=P, st=P, wp=P, gate=None, wq=P, T=4, dr=P, dy=P, dwp=P, dg=None, dwq=P, ws=P, nb=1 << 30, **kw):
        D = _desc(**kw)
        return lib.dynamo_norm_join_backward(ctypes.byref(D), dn, dro, r, y, st, wp, gate, wq, T, dr, dy, dwp, dg, dwq, ws, nb, None)

    for kw, st in BAD_DESC:
        assert fwd(**kw) == st and bwd(**kw) == st, kw
        assert _bytes(lib.dynamo_norm_join_workspace_bytes, ctypes.byref(_desc(**kw)), 4)[0] == st
    assert fwd(T=-1) == TOKENS and bwd(T=-1) == TOKENS and fwd(desc=False) == NULL
    assert fwd(r=None) == NULL and fwd(ro=None) == NULL and fwd(no=None) == NULL and fwd(gate_kind=1) == NULL
    assert fwd(y=None, pre_norm=0) == ARG and fwd(T=0, r=None) == OK
    for kw in (dict(r=P + 8), dict(y=P + 8), dict(wp=P + 4), dict(wq=P + 8), dict(ro=P + 8), dict(no=P + 8), dict(st=P + 4),
               dict(gate=P + 4, gate_kind=1)):
        assert fwd(**kw) == ALIGN, kw
    for kw in (dict(dn=P + 8), dict(dro=P + 8), dict(dr=P + 8), dict(dy=P + 8), dict(ws=P + 16), dict(st=P + 4)):
        assert bwd(**kw) == ALIGN, kw
    assert bwd(dn=None) == NULL and bwd(st=None) == NULL and bwd(r=None) == NULL and bwd(ws=None) == NULL
    assert bwd(nb=8) == SMALL
    # gradients of what is not there
    assert bwd(post_norm=0) == ARG and bwd(pre_norm=0) == ARG and bwd(dg=P) == ARG
    assert bwd(y=None, dwp=None) == ARG and bwd(pre_norm=0, dwq=None, dro=None) == NULL


def test_block_refusals(lib):
    """What the layer refuses and what the join refuses, before either is launched; a layer without weights comes last."""
    st, ctx = binding.dynamo_create(binding.LayerDesc(256, 512, 8, 0, 2, 64, 16, 16, 64, 1))
    assert st == OK
    good = dict(d=256, ydt=1, rdt=0, ndt=0, wdt=0, kind=0, post=1, pre=1, a=1.0, b=1.0, eps=1e-6, ctx=ctx, r=P, n=P, w=P, wp=P, gate=None, wq=P,
                T=4, y=P, ro=P, no=P, st=None)

    def call(desc=True, **kw):
        a = {**good, **kw}
        D = binding.JoinDesc(*(a[k] for k in ("d", "ydt", "rdt", "ndt", "wdt", "kind", "post", "pre", "a", "b", "eps")))
        return lib.dynamo_moe_block_forward(a["ctx"], ctypes.byref(D) if desc else None, a["r"], a["n"], a["w"], None, a["wp"], a["gate"],
                                            a["wq"], a["T"], a["y"], a["ro"], a["no"], a["st"], None, None)

    for kw, want in ((dict(ctx=None), NULL), (dict(desc=False), NULL), (dict(d=264), SHAPE), (dict(y=None), NULL), (dict(r=None), NULL),
                     (dict(ro=None), NULL), (dict(no=None), NULL), (dict(kind=1), NULL), (dict(kind=7), ARG), (dict(eps=0.0), ARG),
                     (dict(a=float("inf")), ARG), (dict(ydt=5), SHAPE), (dict(wp=P + 2), ALIGN), (dict(st=P + 4), ALIGN), (dict(T=-1), TOKENS),
                     (dict(), 9)):
        assert call(**kw) == want, kw
    assert binding.dynamo_destroy(ctx) == OK


def test_linear_refusals(lib):
    def quant(w=P, N=8, K=128, G=64, c=P, p=P):
        return lib.dynamo_linear_quantize(w, N, K, G, c, p, None)

    def fwd(x=P, T=1, N=8, K=128, G=64, c=P, p=P, y=P, ydt=0, ws=None, nb=0):
        return lib.dynamo_linear_forward(x, T, N, K, G, c, p, y, ydt, ws, nb, None)

    for kw, st in ((dict(N=0), SHAPE), (dict(K=0), SHAPE), (dict(K=96), SHAPE), (dict(K=192, G=128), SHAPE), (dict(G=32), SHAPE),
                   (dict(c=None), NULL), (dict(p=None), NULL), (dict(c=P + 8), ALIGN), (dict(p=P + 4), ALIGN)):
        assert quant(**kw) == st and fwd(**kw) == st, kw
    assert _bytes(lib.dynamo_linear_workspace_bytes, 1, 64, 256, 64) == (OK, 0)
    assert _bytes(lib.dynamo_linear_workspace_bytes, 64, 8192, 8192, 64)[1] >= 64 * 8192 * 2
    assert _bytes(lib.dynamo_linear_workspace_bytes, 64, 64, 200, 64)[0] == SHAPE
    assert _bytes(lib.dynamo_linear_workspace_bytes, -1, 64, 256, 64)[0] == TOKENS
    assert quant(w=None) == NULL and quant(w=P + 2) == ALIGN
    assert fwd(x=None) == NULL and fwd(y=None) == NULL and fwd(x=P + 8) == ALIGN and fwd(ydt=7) == SHAPE
    big = dict(T=40, N=8192, K=8192)
    assert fwd(**big) == NULL and fwd(ws=P, nb=8, **big) == SMALL and fwd(ws=P + 16, nb=1 << 30, **big) == ALIGN
    assert fwd(T=16, N=8, K=(1 << 24) + 64) == SHAPE and fwd(T=65536, N=1 << 24, K=1 << 24, ws=P, nb=1 << 40) == TOKENS
    assert fwd(T=-1) == TOKENS and fwd(T=binding.LINEAR_MAX_TOKENS + 1) == TOKENS and fwd(T=0, x=None, y=None) == OK


def test_host_tensors_are_refused():
    x, idx = torch.zeros(4, 64), torch.zeros(4, 2, dtype=torch.int32)
    for f in (lambda: ops.dispatch(idx, 8, x), lambda: ops.combine(x, idx), lambda: ops.combine_backward(x, x, idx),
              lambda: ops.norm_join(x), lambda: ops.norm_join_backward(x, x, x, None, x), lambda: ops.quantize_linear(x),
              lambda: ops.linear(x, idx, x)):
        with pytest.raises(ValueError):
            f()
