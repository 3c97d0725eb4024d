"""Norm behind a block, gate, residual scale and norm in front of the next, and the gradient, against numpy in 64 bits.

Tolerances (u = 2^-24, half a step of fp32).  A row's sum of squares: additions of positive terms in chains of at most
8 V + 10 < 32 a thread and warp and 5 more across warps, so within 40 u; halved by the root, with rsqrt's own 2^-22 (4 u): a row factor is
within 24 u of its value.  A product behind it has at most four more roundings: z within 28 u, r' within 32 u of
R = |res_scale r| + |block_scale g z|.  s_r differs by the same share of its own sum's error, and by at most
32 u |R|_2 / |r'|_2 through r'; n = r' s_r w.  TOL = 64 u covers the constants.  The gradient's row sums add at most 40 u of the
absolute terms' sum, and each of its terms has fewer than 16 roundings and factors within 24 u: 256 u of the absolute values
put through the same formula.  Sums over T tokens: T u of the absolute terms' sum more.  A stored result is off by eps / 2 more."""
import numpy as np
import pytest
import torch

from paper_2503_21135_b200 import binding
from paper_2503_21135_b200 import operators as ops

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
CODE = {"bf16": binding.BF16, "f32": binding.F32}
U = 2.0 ** -24
A, B, EPS = 0.9, 0.7, 1e-5


def f64(t):
    return None if t is None else t.detach().cpu().to(torch.float64).numpy()


def half_step(name):
    return torch.finfo(DT[name]).eps / 2


def make(T, d, y_type, r_type, w_type, gate, post, pre, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed + T * 31 + d)

    def randn(*s, dtype=torch.float32, scale=1.0):
        return (torch.randn(s, generator=g, device="cuda") * scale).to(dtype)

    y, r = randn(T, d, dtype=DT[y_type], scale=0.3), randn(T, d, dtype=DT[r_type])
    if T > 2:
        y[1] = 0          # a block that gives nothing
        y[2], r[2] = 0, 0
    w_post = randn(d, dtype=DT[w_type]) if post == "weight" else None
    w_pre = randn(d, dtype=DT[w_type]) if pre == "weight" else None
    gt = {"none": None, "channel": randn(d, dtype=DT[w_type]), "token": randn(T, 1)}[gate]
    return r, y, dict(w_post=w_post, gate=gt, w_pre=w_pre, post_norm=post != "off", pre_norm=pre != "off", res_scale=A,
                      block_scale=B, eps=EPS)


def reference(r, y, how):
    """r', n, factors and the absolute values R of r' in 64 bits."""
    r, y = f64(r), f64(y)
    s_y = np.ones((r.shape[0], 1))
    if y is None:
        x, R = r, np.abs(r)
    else:
        if how["post_norm"]:
            s_y = 1 / np.sqrt((y * y).mean(1, keepdims=True) + EPS)
        z = y * s_y * (1.0 if how["w_post"] is None else f64(how["w_post"]))
        if how["gate"] is not None:
            z = z * f64(how["gate"])
        x, R = A * r + B * z, np.abs(A * r) + np.abs(B * z)
    s_r = np.ones_like(s_y)
    if how["pre_norm"]:
        s_r = 1 / np.sqrt((x * x).mean(1, keepdims=True) + EPS)
    n = x * s_r * (1.0 if how["w_pre"] is None else f64(how["w_pre"]))
    return x, n, s_y, s_r, R


WIDTHS = [8, 64, 256, 264, 512, 520, 1024, 1408, 2048, 4096, 4104, 8192, 16384]
CASES = [(T, d) for d in WIDTHS for T in (1, 5)] + [(0, 64), (3000, 64), (1500, 264), (1300, 1024), (700, 4096), (300, 8200), (450, 12296)]
OPTIONS = [("bf16", "bf16", "f32", "channel", "weight", "weight", "bf16"), ("f32", "f32", "bf16", "token", "weight", "weight", "f32"),
           ("f32", "bf16", "f32", "none", "ones", "ones", "bf16"), ("bf16", "f32", "bf16", "channel", "off", "weight", "bf16"),
           ("bf16", "bf16", "bf16", "token", "weight", "off", "bf16")]


@pytest.mark.parametrize("y_type,r_type,w_type,gate,post,pre,n_type", OPTIONS)
@pytest.mark.parametrize("T,d", CASES)
def test_forward(T, d, y_type, r_type, w_type, gate, post, pre, n_type):
    r, y, how = make(T, d, y_type, r_type, w_type, gate, post, pre)
    r_out, n, stats = ops.norm_join(r, y, **how, n_dtype=CODE[n_type], want_stats=True)
    x, ref_n, s_y, s_r, R = reference(r, y, how)
    tol_x = 64 * U * R
    assert r_out.dtype == DT[r_type] and (np.abs(f64(r_out) - x) <= tol_x + half_step(r_type) * np.abs(x)).all()
    st = f64(stats)
    through = np.sqrt((R * R).sum(1, keepdims=True) / np.maximum((x * x).sum(1, keepdims=True), 1e-30)) if T else s_r
    assert (np.abs(st[:, :1] - s_y) <= 64 * U * s_y).all()
    assert (np.abs(st[:, 1:] - s_r) <= 64 * U * (1 + through) * s_r).all()
    if pre == "off":
        assert n is None
    else:
        w = 1.0 if how["w_pre"] is None else np.abs(f64(how["w_pre"]))
        tol_n = s_r * w * (tol_x + np.abs(x) * 64 * U * (1 + through))
        assert n.dtype == DT[n_type] and (np.abs(f64(n) - ref_n) <= tol_n + half_step(n_type) * np.abs(ref_n) + 1e-30).all()
    # in place, and again: the same bits
    r2 = r.clone()
    again = ops.norm_join(r2, y, **how, n_dtype=CODE[n_type], r_out=r2)
    assert again[0] is r2 and torch.equal(r2, r_out) and (n is None or torch.equal(again[1], n))


@pytest.mark.parametrize("r_type,n_type", [("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("T,d", [(1, 4096), (5, 8), (130, 1408), (33, 16384)])
def test_norm_in_front_alone(T, d, r_type, n_type):
    r, _, how = make(T, d, "bf16", r_type, "f32", "none", "off", "weight")
    how.update(post_norm=True)
    r_out, n, stats = ops.norm_join(r, **how, n_dtype=CODE[n_type], want_stats=True)
    x, ref_n, _, s_r, _ = reference(r, None, how)
    assert r_out is r
    assert (np.abs(f64(n) - ref_n) <= 128 * U * np.abs(ref_n) + half_step(n_type) * np.abs(ref_n) + 1e-30).all()
    d_n = torch.randn((T, d), device="cuda").to(DT[n_type])
    g = ops.norm_join_backward(d_n, None, r, None, stats, **how)
    w = f64(how["w_pre"])
    u = w * f64(d_n)
    G = s_r * u - x * s_r ** 3 / d * (u * x).sum(1, keepdims=True)
    mag = s_r * np.abs(u) + np.abs(x) * s_r ** 3 / d * np.abs(u * x).sum(1, keepdims=True)
    assert g["d_y"] is None and g["d_gate"] is None
    assert (np.abs(f64(g["d_r"]) - G) <= 256 * U * mag + half_step(r_type) * np.abs(G)).all()
    terms = f64(d_n) * x * s_r
    assert (np.abs(f64(g["d_w_pre"]) - terms.sum(0)) <= (256 + T) * U * np.abs(terms).sum(0) + 1e-30).all()


@pytest.mark.parametrize("upstream", [True, False])
@pytest.mark.parametrize("y_type,r_type,w_type,gate,post,pre,n_type", OPTIONS)
@pytest.mark.parametrize("T,d", CASES)
def test_backward(T, d, y_type, r_type, w_type, gate, post, pre, n_type, upstream):
    if not upstream and (pre == "off" or T > 100):
        pytest.skip("a gradient has to come from somewhere; the long cases run once")
    r, y, how = make(T, d, y_type, r_type, w_type, gate, post, pre, 3)
    _, _, stats = ops.norm_join(r, y, **how, want_stats=True)
    g = torch.Generator(device="cuda").manual_seed(17)
    d_n = torch.randn((T, d), generator=g, device="cuda").to(DT[n_type]) if pre != "off" else None
    d_ro = torch.randn((T, d), generator=g, device="cuda").to(DT[r_type]) if upstream else None
    got = ops.norm_join_backward(d_n, d_ro, r, y, stats, **how)
    x, _, s_y, s_r, R = reference(r, y, how)
    Y = f64(y)
    wp = 1.0 if how["w_post"] is None else f64(how["w_post"])
    wq = 1.0 if how["w_pre"] is None else f64(how["w_pre"])
    k = 1.0 if gate == "none" else f64(how["gate"])
    zero = np.zeros((T, d))
    dn, dro = zero if d_n is None else f64(d_n), zero if d_ro is None else f64(d_ro)
    u, yn = wq * dn, Y * s_y
    z = yn * wp

    def through(dro, u, x, k, z, yn, wp, dn, sign):
        """The formulas; with absolute values and sign = +1 the absolute values of their terms."""
        G = dro + s_r * u + sign * x * s_r ** 3 / d * (u * x).sum(1, keepdims=True)
        dz = B * k * G
        v = dz * wp
        dy = s_y * (v + sign * yn * (v * yn).mean(1, keepdims=True)) if how["post_norm"] else dz
        return G, dz, dy, B * z * G

    G, dz, dy, dg = through(dro, u, x, k, z, yn, wp, dn, -1)
    mG, mz, my, mg = through(np.abs(dro), np.abs(u), R, np.abs(k), np.abs(z), np.abs(yn), np.abs(wp), np.abs(dn), 1)
    tol = 256 * U
    assert (np.abs(f64(got["d_r"]) - A * G) <= tol * mG + half_step(r_type) * np.abs(A * G) + 1e-30).all()
    assert (np.abs(f64(got["d_y"]) - dy) <= tol * my + half_step(y_type) * np.abs(dy) + 1e-30).all()
    for name, terms, mags, there in (("d_w_post", dz * yn, mz * np.abs(yn), how["w_post"] is not None),
                                     ("d_w_pre", dn * x * s_r, np.abs(dn) * R * s_r, how["w_pre"] is not None),
                                     ("d_gate", dg, mg, gate == "channel")):
        if there:
            assert got[name].dtype == torch.float32
            assert (np.abs(f64(got[name]) - terms.sum(0)) <= (256 + T) * U * mags.sum(0) + 1e-30).all(), name
        elif name != "d_gate" or gate == "none":
            assert got[name] is None
    if gate == "token":
        assert got["d_gate"].shape == (T, 1)
        # the row's sum: at most d additions
        assert (np.abs(f64(got["d_gate"]) - dg.sum(1, keepdims=True)) <= tol * mg.sum(1, keepdims=True) + 1e-30).all()
    again = ops.norm_join_backward(d_n, d_ro, r, y, stats, **how)
    assert all(a is None and b is None or torch.equal(a, b) for a, b in zip(got.values(), again.values()))


def test_gradient_against_differences():
    """Central differences of the definition in 64 bits along one direction of every input; fp32 tensors, so the gradients
    are within 1e-5 of the terms' absolute sum (256 u), and the differences' own error is h^2 = 1e-8 of the same."""
    T, d = 6, 128
    r, y, how = make(T, d, "f32", "f32", "f32", "channel", "weight", "weight", 5)
    y[1:3] = torch.randn((2, d), device="cuda")
    _, _, stats = ops.norm_join(r, y, **how, n_dtype=binding.F32, want_stats=True)
    d_n, d_ro = torch.randn((T, d), device="cuda"), torch.randn((T, d), device="cuda")
    got = ops.norm_join_backward(d_n, d_ro, r, y, stats, **how)
    names = {"d_r": r, "d_y": y, "d_w_post": how["w_post"], "d_gate": how["gate"], "d_w_pre": how["w_pre"]}
    step = {n: torch.randn_like(t) for n, t in names.items()}
    h = 1e-4

    def loss(sign):
        moved = {n: t.double() + sign * h * step[n].double() for n, t in names.items()}
        x, n, *_ = reference(moved["d_r"], moved["d_y"], {**how, "w_post": moved["d_w_post"], "gate": moved["d_gate"], "w_pre": moved["d_w_pre"]})
        return (n * f64(d_n)).sum() + (x * f64(d_ro)).sum()

    terms = [f64(got[n]) * f64(step[n]) for n in names]
    total, mag = sum(t.sum() for t in terms), sum(np.abs(t).sum() for t in terms)
    assert abs(total - (loss(1) - loss(-1)) / (2 * h)) <= 2e-5 * mag


def test_non_finite_rows_stay_in_their_rows():
    r, y, how = make(40, 512, "bf16", "bf16", "f32", "channel", "weight", "weight")
    want = ops.norm_join(r, y, **how)
    y[7, 3], r[9, 100] = float("nan"), float("inf")
    r_out, n = ops.norm_join(r, y, **how)
    other = [i for i in range(40) if i not in (7, 9)]
    assert torch.equal(r_out[other], want[0][other]) and torch.equal(n[other], want[1][other])
    assert torch.isnan(n[7]).all() and torch.isnan(n[9]).any()


def test_capture_with_two_graphs():
    r, y, how = make(300, 2048, "bf16", "bf16", "f32", "channel", "weight", "weight")
    d_n, d_ro = torch.randn((2, 300, 2048), device="cuda").bfloat16()

    def step():
        r_out, n, stats = ops.norm_join(r, y, **how, want_stats=True)
        return [r_out, n] + list(ops.norm_join_backward(d_n, d_ro, r, y, stats, **how).values())

    want = step()
    graphs, outs = [], []
    for _ in range(2):
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            outs.append(step())
        graphs.append(gr)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for gr, s in zip(graphs, streams):
        with torch.cuda.stream(s):
            gr.replay()
    torch.cuda.synchronize()
    for out in outs:
        assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_refused_tensors():
    r, y, how = make(4, 64, "bf16", "bf16", "f32", "channel", "weight", "weight")
    s = torch.zeros((4, 2), device="cuda")
    bad = [dict(how, w_post=how["w_post"].half()), dict(how, w_post=how["w_post"][:32]), dict(how, gate=how["gate"].bfloat16()),
           dict(how, gate=torch.zeros((3, 1), device="cuda")), dict(how, pre_norm=False), dict(how, post_norm=False)]
    for kw in bad:
        with pytest.raises(ValueError):
            ops.norm_join(r, y, **kw)
        with pytest.raises(ValueError):
            ops.norm_join_backward(y, y, r, y, s, **kw)
    for f in (lambda: ops.norm_join(r, y[:2], **how), lambda: ops.norm_join(r.t(), y, **how), lambda: ops.norm_join(r, **how),
              lambda: ops.norm_join(r, y, **how, n_dtype=5), lambda: ops.norm_join(r, y, **how, r_out=r.float()),
              lambda: ops.norm_join_backward(None, y, r, y, s, **how), lambda: ops.norm_join_backward(y, y, r, y, s[:2], **how)):
        with pytest.raises(ValueError):
            f()
    with pytest.raises(binding.DynamoError):
        ops.norm_join(r, y, **dict(how, eps=0.0))
    with pytest.raises(binding.DynamoError):
        ops.norm_join(torch.zeros((2, 12), device="cuda"))
