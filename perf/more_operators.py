"""Cases for timing and checking the operators around a layer's experts when the layer is trained: the norm before it
(layer norm or root-mean-square norm, with the residual sum, forward and backward), its tokens sorted by expert and
brought back with the router's weights (and the gradients of both), and the orthogonalised update of its matrices.

With `own` false `run` computes an operator in its plain form (elementary torch operations in 32 bits); with `own` true
it calls paper_2508_02322_b200.  `exact` states the same outputs in 64 bits from the definitions.
"""
import math

import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-6
# the polynomial a s + b s^3 + c s^5 that each orthogonalising step applies to the singular values
COEFFICIENTS = (3.4445, -4.7750, 2.0315)
STEPS = 5


# ------------------------------------------------------------------------------------------------ cases
def _norm(name, op, rows, d, dtype, rms, residual, bias, w_f32=False, pad=0):
    return {"name": name, "op": op, "rows": rows, "d": d, "dtype": dtype, "rms": rms, "residual": residual, "bias": bias,
            "w_f32": w_f32, "pad": pad}


def _moe(name, op, tokens, k, experts, d, dtype, weights=True, add=False, dropped=0.0):
    return {"name": name, "op": op, "tokens": tokens, "k": k, "experts": experts, "d": d, "dtype": dtype, "weights": weights,
            "add": add, "dropped": dropped}


def _ortho(name, n, rows, cols, step, tall, dtype, pad=0):
    return {"name": name, "op": "ortho", "n": n, "rows": rows, "cols": cols, "step": step, "tall": tall, "dtype": dtype,
            "pad": pad}


def listed():
    return [
        # one decoded token before a layer of the 57B shape: latency
        _norm("norm_decode_1", "norm_forward", 1, 3584, "bf16", True, True, False),
        # a training batch of that shape: the residual stream is read, added to, written and normalised
        _norm("norm_train_16384", "norm_forward", 16384, 3584, "bf16", True, True, False),
        # gradients of a small fp32 batch through a layer norm with bias, an odd number of rows
        _norm("norm_backward_1001", "norm_backward", 1001, 2048, "f32", False, False, True, True, 4),
        # gradients of that training batch, the residual stream's own gradient added
        _norm("norm_backward_16384", "norm_backward", 16384, 3584, "bf16", True, True, False),
        # a decoded batch sorted to 64 experts: latency
        _moe("dispatch_decode_64", "dispatch", 64, 8, 64, 3584, "bf16"),
        # a training batch sorted to 64 experts: bound by writing every row eight times
        _moe("dispatch_train_16384", "dispatch", 16384, 8, 64, 3584, "bf16"),
        # a ragged prompt back from 64 experts, some (token, expert) pairs beyond an expert's capacity left out
        _moe("combine_prompt_777", "combine", 777, 6, 64, 2048, "bf16", True, True, 0.07),
        # a training batch back from its experts, added to what the shared expert gave
        _moe("combine_train_16384", "combine", 16384, 8, 64, 3584, "bf16", True, True),
        # gradients of a ragged batch in fp32 through two experts a token
        _moe("combine_backward_1023", "combine_backward", 1023, 2, 8, 4096, "f32", True, False, 0.02),
        # gradients of a training batch by the experts' rows and by the router's weights
        _moe("combine_backward_16384", "combine_backward", 16384, 8, 64, 3584, "bf16"),
        # updates of the three matrices of a sliced expert: 845 micro-experts of width 2048, the last matrix tall
        _ortho("ortho_sliced_expert", 3, 845, 2048, 0, 1, "f32", 3),
        # updates of the gate matrices of 16 sliced experts, each of another height, and of a down matrix
        _ortho("ortho_layer_16", 16, 1408, 2048, 37, 1, "bf16"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


MAX_NORM = 16384 * 3584
MAX_MOE = 16384 * 9 * 3584
MAX_ORTHO = 16 * 1200 * 1200 * 2048


def draw(rng):
    op = rng.choice(["norm_forward", "norm_backward", "dispatch", "combine", "combine_backward", "ortho"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op.startswith("norm"):
        d = rng.choice([1, 8, 8, 64]) * _log_int(rng, 32, 200)
        rows = min(_log_int(rng, 1, 65536), MAX_NORM // (d * (2 if dtype == "f32" else 1)))
        rms = rng.random() < 0.5
        return {"op": op, "rows": rows, "d": d, "dtype": dtype, "rms": rms, "residual": rng.random() < 0.5,
                "bias": not rms and rng.random() < 0.7, "w_f32": rng.random() < 0.5, "pad": rng.choice([0, 0, 1, 8, 24])}
    if op == "ortho":
        while True:
            rows, cols, n = _log_int(rng, 48, 3584), _log_int(rng, 48, 3584), _log_int(rng, 1, 16)
            short = min(rows, cols)
            if n * short * short * max(rows, cols) <= MAX_ORTHO:
                break
        return {"op": op, "n": n, "rows": rows, "cols": cols, "step": rng.choice([0, 0, rows // (2 * n)]),
                "tall": rng.choice([0, 0, n // 2]), "dtype": dtype, "pad": rng.choice([0, 0, 3, 8])}
    k = rng.choice([1, 2, 4, 6, 8])
    d = rng.choice([1, 8, 8, 64]) * _log_int(rng, 32, 100)
    tokens = min(_log_int(rng, 1, 65536), MAX_MOE // ((k + 1) * d * (2 if dtype == "f32" else 1)))
    return {"op": op, "tokens": tokens, "k": k, "experts": max(k, _log_int(rng, 4, 256)), "d": d, "dtype": dtype,
            "weights": rng.random() < 0.8, "add": op == "combine" and rng.random() < 0.5,
            "dropped": rng.choice([0.0, 0.0, 0.03, 0.3])}


def _shapes(case):
    """Rows and columns of each matrix of an orthogonalising call: `step` fewer rows from one to the next, the last
    `tall` of them turned (as a down matrix lies)."""
    wide = [(case["rows"] - case["step"] * i, case["cols"]) for i in range(case["n"])]
    cut = case["n"] - case["tall"]
    return wide[:cut] + [(c, r) for r, c in wide[cut:]]


def work(case):
    """What one pass cannot do without: every input read once, every output written once; multiply-adds count two, and
    a symmetric product half of them."""
    if case["op"] == "ortho":
        size = 2 if case["dtype"] == "bf16" else 4
        flops = moved = 0
        for r, c in _shapes(case):
            m, n = min(r, c), max(r, c)
            flops += STEPS * (m * m * n + m * m * m + 2 * m * m * n)
            moved += r * c * (size + 2)
        return {"bytes": moved, "flops": flops}
    size = 2 if case["dtype"] == "bf16" else 4
    if case["op"].startswith("norm"):
        n, w = case["rows"] * case["d"], 4 if case["w_f32"] else size
        stats = case["rows"] * (4 if case["rms"] else 8)
        if case["op"] == "norm_forward":
            return {"bytes": n * size * (4 if case["residual"] else 2) + stats + case["d"] * w * (2 if case["bias"] else 1),
                    "flops": 6 * n}
        return {"bytes": n * size * (4 if case["residual"] else 3) + stats + case["d"] * (w + 4 * (2 if case["bias"] else 1)),
                "flops": 12 * n}
    t, pairs = case["tokens"], case["tokens"] * case["k"]
    d, kept = case["d"], case["tokens"] * case["k"] * (1.0 - case["dropped"])
    if case["op"] == "dispatch":
        return {"bytes": (t + kept) * d * size + pairs * 8 + 4 * (case["experts"] + 1), "flops": 0}
    w = 4 * pairs if case["weights"] else 0
    if case["op"] == "combine":
        return {"bytes": (kept + t * (2 if case["add"] else 1)) * d * size + pairs * 4 + w, "flops": 2 * kept * d}
    return {"bytes": (t + kept * (2 if case["weights"] else 1)) * d * size + pairs * 4 + 2 * w, "flops": 3 * kept * d}


# ------------------------------------------------------------------------------------------------ inputs
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _padded(values, pad, dtype):
    """`values` [rows, n] as the left part of rows that are `pad` elements longer."""
    rows, n = values.shape
    buf = torch.zeros((rows, n + pad), dtype=dtype, device=DEV)
    buf[:, :n] = values
    return buf[:, :n]


def _norm_inputs(case, seed):
    g = _gen(seed)
    rows, d, dt = case["rows"], case["d"], DTYPES[case["dtype"]]
    wt = torch.float32 if case["w_f32"] else dt
    rnd = lambda *s: torch.randn(s, device=DEV, generator=g)
    # hidden states: tokens of different size, a few channels that stand out, and a mean that is not zero
    channel = torch.ones(d, device=DEV)
    channel[torch.randint(0, d, (4,), device=DEV, generator=g)] = 12.0
    x = rnd(rows, d) * channel * torch.exp(0.5 * rnd(rows, 1)) + 0.3
    s = {"case": case, "x": _padded(x, case["pad"], dt), "weight": (1.0 + 0.2 * rnd(d)).to(wt),
         "bias": (0.1 * rnd(d)).to(wt) if case["bias"] else None}
    if case["op"] == "norm_forward":
        s["residual"] = _padded(rnd(rows, d) * 0.5, case["pad"], dt) if case["residual"] else None
        return s
    z = s["x"].double()
    mean = torch.zeros(rows, device=DEV, dtype=torch.float64) if case["rms"] else z.mean(1)
    var = (z - mean[:, None]).pow(2).mean(1)
    s["mean"] = None if case["rms"] else mean.float()
    s["rstd"] = (var + EPS).rsqrt().float()
    s["dy"] = _padded(rnd(rows, d) * 0.02, case["pad"], dt)
    s["d_sum"] = _padded(rnd(rows, d) * 0.02, case["pad"], dt) if case["residual"] else None
    return s


def _routing(case, g):
    """Distinct experts per token, some experts taken far more often than others; dropped pairs have index -1."""
    t, k, e = case["tokens"], case["k"], case["experts"]
    score = torch.rand((t, e), device=DEV, generator=g).log().neg().log().neg() + torch.randn(e, device=DEV, generator=g) * 0.7
    top, idx = score.topk(k, dim=1)
    w = torch.softmax(top, dim=1)
    idx = idx.int()
    if case["dropped"]:
        idx = torch.where(torch.rand((t, k), device=DEV, generator=g) < case["dropped"], -1, idx)
    return idx, w


def _moe_inputs(case, seed):
    g = _gen(seed)
    t, d, dt = case["tokens"], case["d"], DTYPES[case["dtype"]]
    idx, w = _routing(case, g)
    s = {"case": case, "idx": idx, "w": w if case["weights"] else None}
    pairs = t * case["k"]
    if case["op"] == "dispatch":
        s["x"] = torch.randn((t, d), device=DEV, generator=g).to(dt)
        # rows behind the last kept pair stay what they were
        s["out"] = torch.zeros((pairs, d), dtype=dt, device=DEV)
        return s
    s["rows"] = _plain_sort(idx, case["experts"])[0]
    s["y"] = torch.randn((pairs, d), device=DEV, generator=g).to(dt)
    s["add"] = torch.randn((t, d), device=DEV, generator=g).to(dt) if case["add"] else None
    if case["op"] == "combine_backward":
        s["dy"] = (torch.randn((t, d), device=DEV, generator=g) * 0.02).to(dt)
        s["out"] = torch.zeros((pairs, d), dtype=dt, device=DEV)
    return s


def _ortho_inputs(case, seed):
    """Gradients as training makes them: the product of a batch's gradients, of which a few directions dominate, and its
    hidden states."""
    g = _gen(seed)
    mats = []
    for r, c in _shapes(case):
        tokens = 2 * min(r, c)
        left = torch.randn((tokens, r), device=DEV, generator=g) * torch.exp(torch.randn(r, device=DEV, generator=g) * 0.5)
        right = torch.randn((tokens, c), device=DEV, generator=g) * torch.linspace(0, -2, c, device=DEV).exp()
        mats.append(_padded(left.t() @ right * (1e-3 / tokens), case["pad"], DTYPES[case["dtype"]]))
    return {"case": case, "updates": mats}


def _inputs(case, seed):
    if case["op"] == "ortho":
        return _ortho_inputs(case, seed)
    return _norm_inputs(case, seed) if case["op"].startswith("norm") else _moe_inputs(case, seed)


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        import paper_2508_02322_b200 as P
        # scratch that a program keeps beside its weights
        if case["op"] == "ortho":
            s["workspace"] = P.alloc_workspace(P.camera_orthogonalize_workspace_bytes(s["updates"]), DEV)
        if case["op"] == "dispatch":
            s["workspace"] = P.alloc_workspace(P.camera_moe_dispatch_workspace_bytes(case["tokens"], case["k"], case["experts"]), DEV)
        if case["op"] == "norm_backward":
            s["workspace"] = P.alloc_workspace(P.camera_norm_backward_workspace_bytes(case["rows"], case["d"]), DEV)
    return s


# ------------------------------------------------------------------------------------------------ plain forms
def _plain_norm_forward(s):
    c = s["case"]
    z, out = s["x"].float(), {}
    if c["residual"]:
        out["sum"] = (z + s["residual"].float()).to(s["x"].dtype)       # what the next layer reads; the norm is of this
        z = out["sum"].float()
    if not c["rms"]:
        out["mean"] = z.mean(1)
        z = z - out["mean"][:, None]
    out["rstd"] = (z.pow(2).mean(1) + EPS).rsqrt()
    y = z * out["rstd"][:, None] * s["weight"].float()
    if c["bias"]:
        y = y + s["bias"].float()
    out["y"] = y.to(s["x"].dtype)
    return out


def _plain_norm_backward(s):
    c = s["case"]
    z, dy, rstd = s["x"].float(), s["dy"].float(), s["rstd"][:, None]
    if not c["rms"]:
        z = z - s["mean"][:, None]
    xh = z * rstd
    g = dy * s["weight"].float()
    dx = g - xh * (g * xh).mean(1, keepdim=True)
    if not c["rms"]:
        dx = dx - g.mean(1, keepdim=True)
    dx = dx * rstd
    if c["residual"]:
        dx = dx + s["d_sum"].float()
    out = {"x": dx.to(s["x"].dtype), "weight": (dy * xh).sum(0)}
    if c["bias"]:
        out["bias"] = dy.sum(0)
    return out


def _plain_sort(idx, experts):
    """The row each (token, slot) pair gets when pairs are sorted by expert (by token and slot within one; -1: dropped),
    the pairs in that order, and where each expert's rows begin."""
    flat = idx.reshape(-1).long()
    key = torch.where((flat >= 0) & (flat < experts), flat, experts)
    key, order = key.sort(stable=True)
    rows = torch.empty_like(flat)
    rows[order] = torch.where(key < experts, torch.arange(flat.numel(), device=DEV), -1)
    offsets = torch.searchsorted(key, torch.arange(experts + 1, device=DEV))
    return rows.int().reshape(idx.shape), order, offsets.int()


def _plain_dispatch(s):
    c = s["case"]
    rows, order, offsets = _plain_sort(s["idx"], c["experts"])
    kept = torch.arange(order.numel(), device=DEV) < offsets[-1]
    x = torch.where(kept[:, None], s["x"][order // c["k"]], s["out"])
    return {"x": x, "rows": rows, "offsets": offsets}


def _plain_combine(s):
    got = s["y"][s["rows"].clamp_min(0).long()].float()
    w = (s["rows"] >= 0).float() if s["w"] is None else torch.where(s["rows"] >= 0, s["w"], 0.0)
    y = (got * w[:, :, None]).sum(1)
    if s["add"] is not None:
        y = y + s["add"].float()
    return y.to(s["y"].dtype)


def _plain_combine_backward(s):
    rows, dy = s["rows"], s["dy"].float()
    t, k = rows.shape
    w = torch.ones((t, k), device=DEV) if s["w"] is None else s["w"]
    kept = rows >= 0
    d = torch.cat([s["out"], s["out"][:1]])                         # dropped pairs write to a row that is cut off
    at = torch.where(kept, rows, t * k).long()
    d[at.reshape(-1)] = (w[:, :, None] * dy[:, None, :]).to(d.dtype).reshape(t * k, -1)
    out = {"y": d[:t * k]}
    if s["w"] is not None:
        dot = (s["y"][rows.clamp_min(0).long()].float() * dy[:, None, :]).sum(2)
        out["weights"] = torch.where(kept, dot, 0.0)
    return out


def _plain_ortho_one(u):
    a, b, c = COEFFICIENTS
    x = u.float()
    turned = x.shape[0] > x.shape[1]
    x = x.t() if turned else x
    x = x / (x.norm() + 1e-7)
    for _ in range(STEPS):
        gram = x @ x.t()
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    return (x.t() if turned else x).bfloat16()


# ------------------------------------------------------------------------------------------------ one pass
PLAIN = {"norm_forward": _plain_norm_forward, "norm_backward": _plain_norm_backward, "dispatch": _plain_dispatch,
         "combine": _plain_combine, "combine_backward": _plain_combine_backward,
         "ortho": lambda s: [_plain_ortho_one(u) for u in s["updates"]]}


def run(state):
    s, c = state, state["case"]
    if not own:
        return PLAIN[c["op"]](s)
    import paper_2508_02322_b200 as P
    if c["op"] == "norm_forward":
        return P.camera_norm_forward(s["x"], s["weight"], s["bias"], residual=s["residual"], eps=EPS, rms=c["rms"])
    if c["op"] == "norm_backward":
        return P.camera_norm_backward(s["dy"], s["x"], s["rstd"], s["mean"], s["weight"], d_sum=s["d_sum"], want_bias=c["bias"],
                                      workspace=s["workspace"])
    if c["op"] == "dispatch":
        return P.camera_moe_dispatch(s["x"], s["idx"], c["experts"], out=s["out"], workspace=s["workspace"])
    if c["op"] == "combine":
        return P.camera_moe_combine(s["y"], s["rows"], s["w"], add=s["add"])
    if c["op"] == "combine_backward":
        return P.camera_moe_combine_backward(s["dy"], s["y"], s["rows"], s["w"], want_weights=c["weights"], out=s["out"])
    return P.camera_orthogonalize(s["updates"], steps=STEPS, coefficients=COEFFICIENTS, workspace=s["workspace"])


# ------------------------------------------------------------------------------------------------ 64 bits
def _exact_norm(case, s):
    z = s["x"].double()
    out = {}
    forward = case["op"] == "norm_forward"
    if forward and case["residual"]:
        out["sum"] = z + s["residual"].double()
        z = out["sum"].to(s["x"].dtype).double()
    w, b = s["weight"].double(), s["bias"].double() if case["bias"] else None
    if forward:
        if case["rms"]:
            out["rstd"] = (z.square().mean(1) + EPS) ** -0.5
            out["y"] = z * out["rstd"][:, None] * w
        else:
            out["mean"] = z.mean(1)
            out["rstd"] = (z.var(1, unbiased=False) + EPS) ** -0.5
            out["y"] = torch.nn.functional.layer_norm(z, (case["d"],), w, b, EPS)
        return out
    # the gradient of the formula, from the statistics that the forward pass kept
    leaf = [z.requires_grad_(), w.requires_grad_()] + ([b.requires_grad_()] if b is not None else [])
    if case["rms"]:
        y = leaf[0] * (leaf[0].square().mean(1, keepdim=True) + EPS) ** -0.5 * leaf[1]
    else:
        y = torch.nn.functional.layer_norm(leaf[0], (case["d"],), leaf[1], leaf[2] if b is not None else None, EPS)
    grads = torch.autograd.grad(y, leaf, s["dy"].double())
    out = {"x": grads[0] + s["d_sum"].double() if case["residual"] else grads[0], "weight": grads[1]}
    if b is not None:
        out["bias"] = grads[2]
    return out


def _exact_moe(case, s):
    t, k = case["tokens"], case["k"]
    if case["op"] == "dispatch":
        return {"x": _plain_dispatch(s)["x"].double(), "rows": None, "offsets": None}
    parts = []
    y = torch.zeros((t * k + 1, case["d"]), dtype=torch.float64, device=DEV) if case["op"] == "combine_backward" else None
    for a in range(0, t, 1024):
        rows = s["rows"][a:a + 1024].long()
        kept = (rows >= 0).double()
        w = kept if s["w"] is None else s["w"][a:a + 1024].double() * kept
        got = s["y"][rows.clamp_min(0)].double()
        if y is None:
            part = torch.einsum("tkd,tk->td", got, w)
            parts.append(part + s["add"][a:a + 1024].double() if s["add"] is not None else part)
        else:
            dy = s["dy"][a:a + 1024].double()
            y[torch.where(rows >= 0, rows, t * k)] = torch.einsum("td,tk->tkd", dy, w)
            parts.append(torch.einsum("tkd,td->tk", got, dy) * kept)
    if y is None:
        return torch.cat(parts)
    out = {"y": y[:t * k]}
    if s["w"] is not None:
        out["weights"] = torch.cat(parts)
    return out


def _exact_ortho(case, s):
    """Through the singular values: each goes through the polynomial, STEPS times."""
    a, b, c = COEFFICIENTS
    out = []
    for u in s["updates"]:
        x = u.double()
        flip = x.shape[0] > x.shape[1]
        x = x.t() if flip else x
        # x = V diag(s) W^T, and V from x x^T: p(x) = V diag(p(s) / s) V^T x
        lam, v = torch.linalg.eigh(x @ x.t())
        sv = lam.clamp_min(0.0).sqrt() / (torch.linalg.norm(x) + 1e-7)
        factor = torch.ones_like(sv) / (torch.linalg.norm(x) + 1e-7)
        for _ in range(STEPS):
            step = a + b * sv ** 2 + c * sv ** 4
            sv, factor = sv * step, factor * step
        y = v @ (factor[:, None] * (v.t() @ x))
        out.append(y.t() if flip else y)
    return out


def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "ortho":
        return _exact_ortho(case, s)
    return _exact_norm(case, s) if case["op"].startswith("norm") else _exact_moe(case, s)
