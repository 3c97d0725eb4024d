"""The operators that stand around the MoE layer of a decoder block, as cases that can be timed.

``dispatch`` / ``combine``: tokens sorted by expert and back with the routing weights applied, and their gradients;
``norm``: the norms after and before a block, fused with its gate and residual scale, and the gradient;
``linear``: products of a few token rows with a 4-bit matrix that has group scales.

Keys of a case: ``op`` (``dispatch``, ``dispatch_grad``, ``combine``, ``combine_grad``, ``norm``, ``norm_grad``,
``linear``); ``tokens``.  Routing: ``experts``, ``top_k``, ``width``, ``dtype``, ``drop`` (a tenth of the pairs and every
16th token reach no expert).  Norms: ``width``, ``dtype`` (of the block's output and its gradient), ``stream`` (of the residual
stream and its gradient), ``gate`` (``none``, ``channel``, ``token``), ``post`` (a norm behind the block).  Linear: ``rows`` x ``cols``
of the matrix, ``group``, ``dtype`` (of the result).
"""
import math

import torch

own = False

_DT = {"bf16": torch.bfloat16, "f32": torch.float32}
_EPS = 1e-6
_RES_SCALE, _BLOCK_SCALE = 0.9, 0.7
_DROP, _DROP_EVERY = 0.1, 16


def _route(name, op, tokens, experts, top_k, width, dtype="bf16", drop=False):
    c = {"op": op, "tokens": tokens, "experts": experts, "top_k": top_k, "width": width, "dtype": dtype, "drop": drop}
    return {**c, "name": name} if name else c


def _norm(name, op, tokens, width, dtype="bf16", stream="bf16", gate="none", post=True):
    c = {"op": op, "tokens": tokens, "width": width, "dtype": dtype, "stream": stream, "gate": gate, "post": post}
    return {**c, "name": name} if name else c


def _linear(name, tokens, rows, cols, group=128, dtype="bf16"):
    c = {"op": "linear", "tokens": tokens, "rows": rows, "cols": cols, "group": group, "dtype": dtype}
    return {**c, "name": name} if name else c


def listed():
    return [
        # a small decode batch on its way to eight experts: launches and latency
        _route("dispatch_8", "dispatch", 8, 8, 2, 4096),
        # a long prompt on its way to eight experts
        _route("dispatch_4096", "dispatch", 4096, 8, 2, 4096),
        # training with a capacity limit: gradient of the sort, many small experts, 32-bit rows, odd number of tokens
        _route("dispatch_grad_2047", "dispatch_grad", 2047, 64, 6, 2048, "f32", True),
        # many small experts' results back to a decode batch
        _route("combine_64", "combine", 64, 64, 6, 2048),
        # the same for several prompts together
        _route("combine_8192", "combine", 8192, 64, 6, 2048),
        # training: gradients of rows and routing weights, some pairs beyond the experts' capacity
        _route("combine_grad_4096", "combine_grad", 4096, 8, 2, 4096, "bf16", True),
        # one user's token between two blocks
        _norm("norm_1", "norm", 1, 4096, "f32", "bf16", "channel"),
        # a long prompt between two blocks, gate per channel
        _norm("norm_4096", "norm", 4096, 4096, "bf16", "bf16", "channel"),
        # training between two blocks: both norms' weights and the channels' gate have gradients
        _norm("norm_grad_4096", "norm_grad", 4096, 4096, "bf16", "bf16", "channel"),
        # training in 32 bits, gate per token, odd sizes
        _norm("norm_grad_1021", "norm_grad", 1021, 1408, "f32", "f32", "token"),
        # one user's token through a projection of 4-bit weights
        _linear("linear_1", 1, 4096, 4096),
        # a full decode batch through a wide projection, finer groups, 32-bit result
        _linear("linear_64", 64, 4096, 14336, 64, "f32"),
    ]


_COST = 235e6   # of the largest listed case


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(lo * (hi / lo) ** rng.random()))))


def _cost(c):
    w = work(c)
    return max(w["bytes"], w["flops"] / 50)


def draw(rng):
    """Sizes over their logarithm, every operator, direction, type and option; tokens are halved until the case costs no
    more than the largest listed one."""
    kind = rng.choice(["route", "norm", "linear"])
    if kind == "route":
        experts, top_k = rng.choice([(8, 2), (8, 1), (16, 2), (60, 4), (64, 6), (64, 8), (160, 6), (256, 8), (5, 3)])
        c = _route(None, rng.choice(["dispatch", "dispatch_grad", "combine", "combine_grad"]), _log_int(rng, 1, 20000), experts,
                   top_k, 8 * _log_int(rng, 8, 1024), rng.choice(["bf16", "bf16", "f32"]), rng.random() < 0.4)
    elif kind == "norm":
        c = _norm(None, rng.choice(["norm", "norm_grad"]), _log_int(rng, 1, 20000), 8 * _log_int(rng, 8, 2048),
                  rng.choice(["bf16", "f32"]), rng.choice(["bf16", "f32"]), rng.choice(["none", "channel", "token"]),
                  rng.random() < 0.7)
    else:
        group = rng.choice([64, 128])
        c = _linear(None, _log_int(rng, 1, 100), _log_int(rng, 60, 15000), group * _log_int(rng, 1, 14336 // group), group,
                    rng.choice(["bf16", "f32"]))
    while _cost(c) > _COST:
        c["tokens"] = c["tokens"] // 2
    return c


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 7919 + 13)
    return g


def _sorted_pairs(idx, n_experts):
    """offsets [E + 1], perm [T k] (-1 behind the last pair) and pos [T, k] (-1: the pair reaches no expert)."""
    flat = idx.reshape(-1).long()
    n = flat.numel()
    keep = (flat >= 0) & (flat < n_experts)
    key = torch.where(keep, flat, n_experts)
    sorted_key, order = torch.sort(key, stable=True)
    place = torch.arange(n, device=idx.device)
    offsets = torch.searchsorted(sorted_key, torch.arange(n_experts + 1, device=idx.device))
    perm = torch.where(sorted_key < n_experts, order, -1)
    pos = torch.empty_like(order)
    pos[order] = torch.where(sorted_key < n_experts, place, -1)
    return offsets.int(), perm.int(), pos.view(idx.shape).int()


def prepare(case, seed):
    g, dev, T = _gen(seed), "cuda", case["tokens"]

    def randn(*shape, dtype=torch.float32, scale=1.0):
        return (torch.randn(shape, generator=g, device=dev) * scale).to(dtype)

    s = {"case": case}
    if case["op"] == "linear":
        N, K, G = case["rows"], case["cols"], case["group"]
        w = randn(N, K // G, G, scale=0.02)
        lo, hi = w.amin(2), w.amax(2)
        scale, zero = ((hi - lo) / 15).half(), lo.half()
        q = ((w - zero.float()[:, :, None]) / scale.float()[:, :, None]).round().clamp(0, 15).to(torch.uint8).view(N, K)
        s["codes"] = q[:, 0::2] | (q[:, 1::2] << 4)
        s["params"] = torch.stack([scale, zero], 2).contiguous()
        s["x"] = randn(T, K, dtype=torch.bfloat16)
        return s
    d, dt = case["width"], _DT[case["dtype"]]
    if case["op"] in ("norm", "norm_grad"):
        rt = _DT[case["stream"]]
        s["y"], s["r"] = randn(T, d, dtype=dt, scale=0.3), randn(T, d, dtype=rt)
        s["w_post"] = (1 + randn(d, scale=0.1)) if case["post"] else None
        s["w_pre"] = 1 + randn(d, scale=0.1)
        s["gate"] = {"none": None, "channel": randn(d, scale=0.5), "token": torch.sigmoid(randn(T, 1))}[case["gate"]]
        if case["op"] == "norm_grad":
            # the loss's gradients of the normed output and of the stream, and what the forward kept of its rows
            s["d_n"], s["d_r_out"] = randn(T, d, dtype=torch.bfloat16), randn(T, d, dtype=rt)
            s["stats"] = _norm_plain(s)[2]
        return s
    E, k = case["experts"], case["top_k"]
    popularity = -1.2 * torch.log(1.0 + torch.randperm(E, generator=g, device=dev).float())
    idx = torch.topk(randn(T, E) + popularity, k, dim=1).indices.int()
    if case["drop"]:
        idx[torch.rand((T, k), generator=g, device=dev) < _DROP] = -1
        idx[5::_DROP_EVERY] = -1
    offsets, perm, pos = _sorted_pairs(idx, E)
    if case["op"] == "dispatch":
        s["idx"], s["x"] = idx, randn(T, d, dtype=dt)
        # the buffers that the program's experts read; rows behind the last pair stay zero
        s["out"] = (torch.zeros((T * k, d), dtype=dt, device=dev), torch.empty_like(offsets), torch.full_like(perm, -1),
                    torch.empty_like(pos))
        return s
    rows = randn(T * k, d, dtype=dt)
    rows[perm < 0] = math.nan   # nothing has written there
    s["rows"], s["pos"] = rows, pos
    if case["op"] != "dispatch_grad":
        w = torch.softmax(randn(T, k), 1)
        s["w"] = torch.where(pos >= 0, w, math.nan)
    if case["op"] == "combine_grad":
        s["dy"] = randn(T, d, dtype=dt)
        s["d_rows"] = torch.zeros((T * k, d), dtype=dt, device=dev)
    return s


def _norm_plain(s):
    """r_out, n and the row factors [T, 2], in 32 bits."""
    z = s["y"].float()
    s_y = torch.ones(z.shape[0], 1, device=z.device)
    if s["w_post"] is not None:
        s_y = torch.rsqrt((z * z).mean(1, keepdim=True) + _EPS)
        z = z * s_y * s["w_post"]
    if s["gate"] is not None:
        z = z * s["gate"]
    r_out = _RES_SCALE * s["r"].float() + _BLOCK_SCALE * z
    s_r = torch.rsqrt((r_out * r_out).mean(1, keepdim=True) + _EPS)
    return r_out, r_out * s_r * s["w_pre"], torch.cat([s_y, s_r], 1)


def _norm_grad_plain(s):
    c, y, d_n = s["case"], s["y"].float(), s["d_n"].float()
    s_y, s_r = s["stats"][:, :1], s["stats"][:, 1:]
    yn = y * s_y
    z = yn * s["w_post"] if c["post"] else yn
    gate = 1.0 if s["gate"] is None else s["gate"]
    r_out = _RES_SCALE * s["r"].float() + _BLOCK_SCALE * gate * z
    rn = r_out * s_r
    u = d_n * s["w_pre"]
    G = s["d_r_out"].float() + s_r * (u - rn * (u * rn).mean(1, keepdim=True))
    dz = _BLOCK_SCALE * gate * G
    out = {"d_r": (_RES_SCALE * G).to(s["r"].dtype), "d_w_pre": (d_n * rn).sum(0)}
    if c["post"]:
        v = dz * s["w_post"]
        out["d_y"] = (s_y * (v - yn * (v * yn).mean(1, keepdim=True))).to(s["y"].dtype)
        out["d_w_post"] = (dz * yn).sum(0)
    else:
        out["d_y"] = dz.to(s["y"].dtype)
    if c["gate"] != "none":
        terms = _BLOCK_SCALE * z * G
        out["d_gate"] = terms.sum(0) if c["gate"] == "channel" else terms.sum(1, keepdim=True)
    return out


def _plain(s):
    c = s["case"]
    op = c["op"]
    if op == "dispatch":
        offsets, perm, pos = _sorted_pairs(s["idx"], c["experts"])
        token = torch.div(perm.clamp(min=0), c["top_k"], rounding_mode="floor").long()
        rows = torch.where((perm >= 0)[:, None], s["x"][token], 0)
        return {"rows": rows, "offsets": offsets, "perm": perm, "pos": pos}
    if op in ("dispatch_grad", "combine"):
        at = s["pos"].long()
        terms = torch.where((at >= 0)[:, :, None], s["rows"].float()[at.clamp(min=0)], 0)
        if op == "combine":
            terms = terms * torch.where(at >= 0, s["w"], 0)[:, :, None]
        return {"y": terms.sum(1).to(s["rows"].dtype)}
    if op == "combine_grad":
        at, dy = s["pos"].long(), s["dy"].float()
        kept = at >= 0
        terms = torch.where(kept[:, :, None], s["rows"].float()[at.clamp(min=0)], 0)
        d_w = (terms * dy[:, None, :]).sum(2)
        d_rows = torch.zeros_like(s["d_rows"])
        d_rows[at[kept]] = (s["w"][:, :, None] * dy[:, None, :])[kept].to(d_rows.dtype)
        return {"d_rows": d_rows, "d_w": d_w}
    if op == "norm":
        r_out, n, _ = _norm_plain(s)
        return {"r_out": r_out.to(s["r"].dtype), "n": n.to(torch.bfloat16)}
    if op == "norm_grad":
        return _norm_grad_plain(s)
    N, K, G = c["rows"], c["cols"], c["group"]
    q = torch.stack([s["codes"] & 15, s["codes"] >> 4], 2).view(N, K // G, G).float()
    w = (q * s["params"][:, :, :1].float() + s["params"][:, :, 1:].float()).view(N, K)
    return {"y": (s["x"].float() @ w.t()).to(_DT[c["dtype"]])}


def _calls(s):
    from paper_2503_21135_b200 import binding
    from paper_2503_21135_b200 import operators as ops

    c = s["case"]
    op = c["op"]
    if op == "dispatch":
        r = ops.dispatch(s["idx"], c["experts"], s["x"], out=s["out"])
        return {"rows": r.rows, "offsets": r.offsets, "perm": r.perm, "pos": r.pos}
    if op == "dispatch_grad":
        return {"y": ops.dispatch_backward(s["rows"], s["pos"])}
    if op == "combine":
        return {"y": ops.combine(s["rows"], s["pos"], s["w"])}
    if op == "combine_grad":
        d_rows, d_w = ops.combine_backward(s["dy"], s["rows"], s["pos"], s["w"], d_rows=s["d_rows"])
        return {"d_rows": d_rows, "d_w": d_w}
    if op in ("norm", "norm_grad"):
        how = dict(w_post=s["w_post"], gate=s["gate"], w_pre=s["w_pre"], post_norm=c["post"], res_scale=_RES_SCALE,
                   block_scale=_BLOCK_SCALE, eps=_EPS)
        if op == "norm":
            r_out, n = ops.norm_join(s["r"], s["y"], **how)
            return {"r_out": r_out, "n": n}
        grads = ops.norm_join_backward(s["d_n"], s["d_r_out"], s["r"], s["y"], s["stats"], **how)
        return {name: g for name, g in grads.items() if g is not None}
    return {"y": ops.linear(s["x"], s["codes"], s["params"], y_dtype=binding.BF16 if c["dtype"] == "bf16" else binding.F32)}


def run(state):
    return _calls(state) if own else _plain(state)


def work(case):
    T, op = case["tokens"], case["op"]
    if op == "linear":
        N, K, G = case["rows"], case["cols"], case["group"]
        return {"bytes": N * K / 2 + 4.0 * N * K / G + 2.0 * T * K + T * N * (2.0 if case["dtype"] == "bf16" else 4.0),
                "flops": 2.0 * T * N * K}
    d, b = case["width"], 2.0 if case["dtype"] == "bf16" else 4.0
    if op in ("norm", "norm_grad"):
        rb = 2.0 if case["stream"] == "bf16" else 4.0
        vectors = 4.0 * d * (1 + case["post"] + (case["gate"] == "channel")) + 4.0 * T * (case["gate"] == "token")
        if op == "norm":
            return {"bytes": T * d * (b + 2 * rb + 2) + vectors, "flops": 10.0 * T * d}
        return {"bytes": T * d * (2 * b + 3 * rb + 2) + 2 * vectors + 8.0 * T, "flops": 30.0 * T * d}
    k, E = case["top_k"], case["experts"]
    pairs = T * k * ((1 - _DROP) * (1 - 1 / _DROP_EVERY) if case["drop"] else 1.0)
    if op == "dispatch":
        return {"bytes": T * d * b + pairs * d * b + 12.0 * T * k + 4.0 * (E + 1), "flops": 0.0}
    if op == "combine_grad":
        return {"bytes": T * d * b + 2 * pairs * d * b + 12.0 * T * k, "flops": 3 * pairs * d}
    return {"bytes": pairs * d * b + T * d * b + (8.0 if op == "combine" else 4.0) * T * k, "flops": 2 * pairs * d}


def exact(case, seed):
    """Definitions in 64 bits: loops over experts and choices, gradients by automatic differentiation."""
    s, op = prepare(case, seed), case["op"]
    if op == "linear":
        N, K, G, T = case["rows"], case["cols"], case["group"], case["tokens"]
        codes = torch.empty((N, K), dtype=torch.float64, device="cuda")
        codes[:, 0::2], codes[:, 1::2] = (s["codes"] % 16).double(), (s["codes"] // 16).double()
        x, y = s["x"].double(), torch.zeros((T, N), dtype=torch.float64, device="cuda")
        for i in range(K // G):
            xi = x[:, i * G:(i + 1) * G]
            y += (xi @ codes[:, i * G:(i + 1) * G].t()) * s["params"][:, i, 0].double()
            y += xi.sum(1, keepdim=True) * s["params"][:, i, 1].double()
        return {"y": y}
    if op in ("norm", "norm_grad"):
        leaf = lambda t: None if t is None else t.double().requires_grad_(True)  # noqa: E731
        v = {n: leaf(s[n]) for n in ("y", "r", "w_post", "w_pre", "gate")}

        def rms(a, w):
            return a / (a.pow(2).sum(1, keepdim=True) / case["width"] + _EPS).sqrt() * w

        z = rms(v["y"], v["w_post"]) if case["post"] else v["y"]
        if case["gate"] != "none":
            z = z * v["gate"]
        r_out = v["r"] * _RES_SCALE + z * _BLOCK_SCALE
        n = rms(r_out, v["w_pre"])
        if op == "norm":
            return {"r_out": r_out.detach(), "n": n.detach()}
        ((n * s["d_n"].double()).sum() + (r_out * s["d_r_out"].double()).sum()).backward()
        return {"d_" + name: t.grad for name, t in v.items() if t is not None}
    T, k, E = case["tokens"], case["top_k"], case["experts"]
    if op == "dispatch":
        flat = s["idx"].reshape(-1)
        lists = [(flat == e).nonzero().reshape(-1) for e in range(E)]
        order = torch.cat(lists)
        rows = torch.zeros((T * k, case["width"]), dtype=torch.float64, device="cuda")
        rows[: order.numel()] = s["x"].double()[order // k]
        return {"rows": rows, "offsets": None, "perm": None, "pos": None}
    y = torch.zeros((T, case["width"]), dtype=torch.float64, device="cuda")
    if op == "combine_grad":
        dy = s["dy"].double()
        d_rows = torch.zeros((T * k, case["width"]), dtype=torch.float64, device="cuda")
        d_w = torch.zeros((T, k), dtype=torch.float64, device="cuda")
        for j in range(k):
            t = (s["pos"][:, j] >= 0).nonzero().reshape(-1)
            at = s["pos"][t, j].long()
            d_rows[at] = dy[t] * s["w"][t, j].double().unsqueeze(1)
            d_w[t, j] = torch.linalg.vecdot(dy[t], s["rows"][at].double())
        return {"d_rows": d_rows, "d_w": d_w}
    for j in range(k):
        t = (s["pos"][:, j] >= 0).nonzero().reshape(-1)
        term = s["rows"][s["pos"][t, j].long()].double()
        y[t] += term * s["w"][t, j].double().unsqueeze(1) if op == "combine" else term
    return {"y": y}
