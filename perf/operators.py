"""Cases for timing and checking the recovery operators: the gated feed-forward block of one expert (forward, and
forward with backward), the log-probabilities of given tokens with entropy and top alternatives, and the distillation
loss against a teacher's top log-probabilities with its gradient.

Together they are the steps around a layer that was sliced: the full model's top log-probabilities are read off once,
the sliced block is trained against them, and the result is evaluated by the log-probabilities of a text's tokens.

With `own` false `run` computes an operator in its plain form (elementary torch operations in 32 bits); with `own` true
it calls paper_2508_02322_b200.  `exact` states the same outputs in 64 bits from the definitions.
"""
import math

import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ------------------------------------------------------------------------------------------------ cases
def _ffn(name, op, tokens, d_model, d_ff, down_ld=0):
    return {"name": name, "op": op, "tokens": tokens, "d_model": d_model, "d_ff": d_ff, "down_ld": down_ld or d_ff}


def _logprobs(name, rows, vocab, dtype, top_n, temperature=1.0, masked=False, pad=0):
    return {"name": name, "op": "logprobs", "rows": rows, "vocab": vocab, "dtype": dtype, "top_n": top_n,
            "temperature": temperature, "masked": masked, "pad": pad}


def _distill(name, mode, rows, vocab, dtype, k, temperature=1.0, tail=False, pad=0):
    return {"name": name, "op": "distill", "mode": mode, "rows": rows, "vocab": vocab, "dtype": dtype, "k": k,
            "temperature": temperature, "tail": tail, "pad": pad}


def listed():
    return [
        # one token through one routed expert of the 57B shape: the latency of decoding
        _ffn("ffn_decode_1", "ffn_forward", 1, 3584, 2560),
        # a batch of decoded tokens through the shared expert of that shape: bound by reading its weights
        _ffn("ffn_decode_24", "ffn_forward", 24, 3584, 20480),
        # a prompt through an expert that lost a fifth of its micro-experts and kept the width of its W_down buffer
        _ffn("ffn_prompt_777_sliced", "ffn_forward", 777, 2048, 1127, 1408),
        # calibration tokens through the shared expert: bound by the tensor cores
        _ffn("ffn_prompt_4096", "ffn_forward", 4096, 3584, 20480),
        # a recovery step on a sliced expert, an odd number of tokens and of micro-experts
        _ffn("ffn_train_1001_sliced", "ffn_train", 1001, 2048, 845, 848),
        # a recovery step on a whole routed expert
        _ffn("ffn_train_8192", "ffn_train", 8192, 3584, 2560),
        # the sampled token of one decode step, with its alternatives
        _logprobs("logprobs_decode_1", 1, 151936, "bf16", 8),
        # a decoded batch under a grammar's mask, fp32 logits at a temperature
        _logprobs("logprobs_decode_40_masked", 40, 50257, "f32", 20, 0.7, True, 3),
        # perplexity of a text: log-probabilities and entropies only
        _logprobs("logprobs_text_4095", 4095, 151936, "bf16", 0),
        # the teacher's top log-probabilities for a training batch
        _logprobs("logprobs_teacher_2048", 2048, 151936, "bf16", 64, 2.0),
        # validation loss of a small batch, fp32 logits of an odd width
        _distill("distill_loss_250", "forward", 250, 32003, "f32", 32, 1.0, True, 5),
        # a training step: loss and gradient from one call
        _distill("distill_step_4096", "step", 4096, 151936, "bf16", 64, 2.0, True),
    ]


def _log_int(rng, lo, hi):
    while True:
        v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
        if v != 3072:
            return max(lo, min(hi, v))


MAX_FFN_FORWARD = 6 * 4096 * 3584 * 20480
MAX_FFN_TRAIN = 18 * 8192 * 3584 * 2560
MAX_LOGITS = 4096 * 151936


def draw(rng):
    op = rng.choice(["ffn_forward", "ffn_train", "logprobs", "distill"])
    if op.startswith("ffn"):
        cap, per = (MAX_FFN_FORWARD, 6) if op == "ffn_forward" else (MAX_FFN_TRAIN, 18)
        while True:
            tokens = _log_int(rng, 1 if op == "ffn_forward" else 16, 8192)
            d_model = 8 * _log_int(rng, 64, 512)
            d_ff = _log_int(rng, 256, 20480)
            down_ld = (d_ff + 7) // 8 * 8 + rng.choice([0, 0, 8, 64])
            if per * tokens * d_model * d_ff <= cap and 3072 not in (d_model, down_ld):
                break
        return {"op": op, "tokens": tokens, "d_model": d_model, "d_ff": d_ff, "down_ld": down_ld}
    vocab = _log_int(rng, 1000, 152064)
    rows = _log_int(rng, 1, 16384)
    rows = max(1, min(rows, MAX_LOGITS // vocab))
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if dtype == "f32":
        rows = max(1, rows // 2)
    pad = rng.choice([0, 0, 1, 8, 61])
    temperature = rng.choice([1.0, 1.0, round(rng.uniform(0.5, 3.0), 3)])
    if op == "logprobs":
        return {"op": op, "rows": rows, "vocab": vocab, "dtype": dtype, "top_n": rng.choice([0, 1, 5, 20, 64]),
                "temperature": temperature, "masked": rng.random() < 0.3, "pad": pad}
    return {"op": op, "mode": rng.choice(["forward", "backward", "step", "step"]), "rows": rows, "vocab": vocab,
            "dtype": dtype, "k": rng.choice([1, 8, 20, 33, 64]), "temperature": temperature,
            "tail": rng.random() < 0.5, "pad": pad}


def work(case):
    """What one pass cannot do without: every input read once, every output written once; multiply-adds count two."""
    if case["op"].startswith("ffn"):
        t, d, f = case["tokens"], case["d_model"], case["d_ff"]
        if case["op"] == "ffn_forward":
            return {"bytes": 2 * (3 * d * f + 2 * t * d), "flops": 6 * t * d * f}
        return {"bytes": 2 * (6 * d * f + 4 * t * d), "flops": 18 * t * d * f}
    size = 2 if case["dtype"] == "bf16" else 4
    rows, n = case["rows"], case["rows"] * case["vocab"]
    if case["op"] == "logprobs":
        # per logit: the maximum, a multiply-add, the exponential, its sum, the entropy's sum
        return {"bytes": n * size + rows * (16 + 8 * case["top_n"]), "flops": 7 * n}
    if case["mode"] == "forward":
        return {"bytes": n * size + rows * (8 * case["k"] + 12), "flops": 5 * n}
    per = 4 if case["mode"] == "backward" else 9
    return {"bytes": 2 * n * size + rows * (8 * case["k"] + 16), "flops": per * n}


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


def _ffn_inputs(case, seed):
    g = _gen(seed)
    t, d, f, ld = case["tokens"], case["d_model"], case["d_ff"], case["down_ld"]
    rnd = lambda *s: torch.randn(s, device=DEV, generator=g)
    x = rnd(t, d)
    s = {"case": case, "d_ff": f,
         "x": (x / x.pow(2).mean(1, keepdim=True).sqrt()).bfloat16(),
         "w_gate": (rnd(f, d) * 0.02).bfloat16(), "w_up": (rnd(f, d) * 0.02).bfloat16(),
         "w_down": (rnd(d, ld) * 0.02).bfloat16()}
    if case["op"] == "ffn_train":
        s["dy"] = (rnd(t, d) * 0.01).bfloat16()
    return s


def _logits(case, g):
    """Raw scores of a language model: a broad bell, and per row a few tokens that stand out."""
    rows, vocab = case["rows"], case["vocab"]
    z = torch.randn((rows, vocab), device=DEV, generator=g).mul_(1.5)
    n_out = 12
    idx = torch.randint(0, vocab, (rows, n_out), device=DEV, generator=g)
    up = torch.rand((rows, n_out), device=DEV, generator=g) * 24.0
    z.scatter_reduce_(1, idx, up, "amax")       # a token drawn twice takes the larger value, whatever the order
    return z, idx


def _logprobs_inputs(case, seed):
    g = _gen(seed)
    rows, vocab = case["rows"], case["vocab"]
    z, idx = _logits(case, g)
    targets = torch.randint(0, vocab, (rows,), device=DEV, generator=g)
    likely = torch.rand((rows,), device=DEV, generator=g) < 0.7
    targets = torch.where(likely, idx[:, 0], targets)
    if case["masked"]:
        allowed = torch.rand((vocab,), device=DEV, generator=g) < 0.7
        keep = z.gather(1, targets[:, None])
        z.masked_fill_(~allowed[None, :], -math.inf)
        z.scatter_(1, targets[:, None], keep)
    return {"case": case, "logits": _padded(z, case["pad"], DTYPES[case["dtype"]]), "targets": targets}


def _distill_inputs(case, seed):
    g = _gen(seed)
    rows, k, tau = case["rows"], case["k"], case["temperature"]
    teacher, _ = _logits(case, g)
    idx = torch.empty((rows, k), dtype=torch.int32, device=DEV)
    logprob = torch.empty((rows, k), dtype=torch.float32, device=DEV)
    for r in range(0, rows, 512):
        z = teacher[r:r + 512] / tau
        top, i = z.topk(k, dim=1)
        idx[r:r + 512] = i.int()
        logprob[r:r + 512] = top - torch.logsumexp(z, 1, keepdim=True)
    student = teacher
    student += torch.randn(student.shape, device=DEV, generator=g) * 0.7
    s = {"case": case, "logits": _padded(student, case["pad"], DTYPES[case["dtype"]]), "idx": idx, "logprob": logprob}
    if case["mode"] != "forward":
        # the mean over the tokens that count; a few belong to the prompt and carry no loss
        weight = torch.full((rows,), 1.0 / rows, device=DEV)
        weight[torch.rand((rows,), device=DEV, generator=g) < 0.05] = 0.0
        s["d_loss"] = weight
    if case["mode"] == "backward":
        s["lse"] = torch.empty(rows, device=DEV)
        s["log_tail"] = torch.empty(rows, device=DEV)
        for r in range(0, rows, 512):
            z = s["logits"][r:r + 512].float() / tau
            s["lse"][r:r + 512] = torch.logsumexp(z, 1)
            z.scatter_(1, idx[r:r + 512].long(), -math.inf)
            s["log_tail"][r:r + 512] = torch.logsumexp(z, 1)
    return s


def prepare(case, seed):
    if case["op"].startswith("ffn"):
        s = _ffn_inputs(case, seed)
        if own:
            import paper_2508_02322_b200 as P
            ffn = P.Ffn(s["w_gate"], s["w_up"], s["w_down"], d_ff=case["d_ff"])
            train = case["op"] == "ffn_train"
            s["ffn"] = ffn
            s["workspace"] = P.alloc_workspace(P.camera_ffn_workspace_bytes(ffn, case["tokens"], backward=train), DEV)
            s["saved"] = P.alloc_workspace(P.camera_ffn_saved_bytes(ffn, case["tokens"]), DEV) if train else None
        return s
    if case["op"] == "logprobs":
        return _logprobs_inputs(case, seed)
    return _distill_inputs(case, seed)


# ------------------------------------------------------------------------------------------------ plain forms
def _plain_ffn_forward(s):
    f = s["d_ff"]
    x, wg, wu, wd = s["x"].float(), s["w_gate"].float(), s["w_up"].float(), s["w_down"][:, :f].float()
    g, u = x @ wg.t(), x @ wu.t()
    h = g * torch.sigmoid(g) * u
    return (h @ wd.t()).bfloat16()


def _plain_ffn_train(s):
    f = s["d_ff"]
    x, wg, wu, wd = s["x"].float(), s["w_gate"].float(), s["w_up"].float(), s["w_down"][:, :f].float()
    dy = s["dy"].float()
    g, u = x @ wg.t(), x @ wu.t()
    sig = torch.sigmoid(g)
    act = g * sig
    h = act * u
    y = h @ wd.t()
    dh = dy @ wd
    du = dh * act
    dg = dh * u * (sig + act * (1 - sig))
    dx = dg @ wg + du @ wu
    return {"y": y.bfloat16(), "dx": dx.bfloat16(), "dw_gate": (dg.t() @ x).bfloat16(), "dw_up": (du.t() @ x).bfloat16(),
            "dw_down": (dy.t() @ h).bfloat16()}


def _top_lowest_index(z, n):
    """Indices of the n largest values of each row of fp32 z, by decreasing value, ties by increasing index: the top n
    of 64-bit keys that hold the value's order above the reversed index."""
    bits = (z + 0.0).view(torch.int32).long()
    order = torch.where(bits < 0, -(bits & 0x7fffffff), bits)
    key = order * (1 << 24) + ((1 << 24) - 1 - torch.arange(z.shape[1], device=z.device))
    return key.topk(n, dim=1).indices


def _plain_logprobs(s):
    c = s["case"]
    z = s["logits"].float()
    zt = z / c["temperature"]
    m = zt.amax(1, keepdim=True)
    e = torch.exp(zt - m)
    total = e.sum(1, keepdim=True)
    lse = m + torch.log(total)
    out = {"logprob": zt.gather(1, s["targets"][:, None]).squeeze(1) - lse.squeeze(1)}
    p = e / total
    out["entropy"] = lse.squeeze(1) - (p * torch.where(e > 0, zt, 0.0)).sum(1)
    if c["top_n"]:
        i = _top_lowest_index(z, c["top_n"])
        out["top_idx"] = i.int()
        out["top_logprob"] = zt.gather(1, i) - lse
    return out


def _plain_distill(s):
    c = s["case"]
    z = s["logits"].float() / c["temperature"]
    idx = s["idx"].long()
    lp = s["logprob"]
    top = z.gather(1, idx)
    if c["mode"] == "backward":
        lse, log_tail = s["lse"][:, None], s["log_tail"][:, None]
    else:
        m = z.amax(1, keepdim=True)
        e = torch.exp(z - m)
        lse = m + torch.log(e.sum(1, keepdim=True))
        e.scatter_(1, idx, 0.0)
        log_tail = m + torch.log(e.sum(1, keepdim=True))
    log_q = top - lse
    out = {}
    if c["tail"]:
        p = torch.exp(lp)
        rest = (1 - p.sum(1, keepdim=True)).clamp_min(0.0)
        loss = (p * (lp - log_q)).sum(1)
        log_rest = torch.log(rest.clamp_min(1e-38))
        loss = loss + (rest * (log_rest - (log_tail - lse))).squeeze(1)
    else:
        p = torch.exp(lp - lp.amax(1, keepdim=True))
        p = p / p.sum(1, keepdim=True)
        loss = (p * (torch.log(p) - log_q)).sum(1)
    if c["mode"] != "backward":
        out["loss"] = loss
    if c["mode"] == "step":
        out["loss"] = torch.where(s["d_loss"] == 0, 0.0, out["loss"])
    if c["mode"] != "forward":
        q = torch.exp(z - lse)
        at_top = q.gather(1, idx) - p
        if c["tail"]:
            # a token outside the list moves only the rest's share: q_v (1 - rest / (1 - Q))
            q = q * (1 - rest * torch.exp(lse - log_tail))
        q.scatter_(1, idx, at_top)
        q *= (s["d_loss"] / c["temperature"])[:, None]
        out["d_logits"] = q.to(s["logits"].dtype)
    return out


# ------------------------------------------------------------------------------------------------ one pass
def run(state):
    c = state["case"]
    if not own:
        if c["op"] == "ffn_forward":
            return _plain_ffn_forward(state)
        if c["op"] == "ffn_train":
            return _plain_ffn_train(state)
        return _plain_logprobs(state) if c["op"] == "logprobs" else _plain_distill(state)
    import paper_2508_02322_b200 as P
    if c["op"] == "ffn_forward":
        return P.camera_ffn_forward(state["ffn"], state["x"], workspace=state["workspace"])
    if c["op"] == "ffn_train":
        y = P.camera_ffn_forward(state["ffn"], state["x"], saved=state["saved"], workspace=state["workspace"])
        grads = P.camera_ffn_backward(state["ffn"], state["x"], state["dy"], state["saved"], workspace=state["workspace"])
        return {"y": y, "dx": grads["x"], "dw_gate": grads["w_gate"], "dw_up": grads["w_up"],
                "dw_down": grads["w_down"][:, :c["d_ff"]]}
    if c["op"] == "logprobs":
        return P.camera_token_logprobs(state["logits"], state["targets"], top_n=c["top_n"], temperature=c["temperature"])
    kw = dict(temperature=c["temperature"], tail=c["tail"])
    if c["mode"] == "forward":
        return {"loss": P.camera_distill_forward(state["logits"], state["idx"], state["logprob"], **kw)["loss"]}
    if c["mode"] == "backward":
        return {"d_logits": P.camera_distill_backward(state["logits"], state["idx"], state["logprob"], state["d_loss"],
                                                      state["lse"], state["log_tail"], **kw)}
    loss, d_logits = P.camera_distill_step(state["logits"], state["idx"], state["logprob"], state["d_loss"], **kw)
    return {"loss": loss, "d_logits": d_logits}


# ------------------------------------------------------------------------------------------------ 64 bits
def _exact_ffn(case, s):
    f = case["d_ff"]
    train = case["op"] == "ffn_train"
    leaf = [s["x"].double(), s["w_gate"].double(), s["w_up"].double(), s["w_down"][:, :f].double()]
    for t in leaf:
        t.requires_grad_(train)
    x, wg, wu, wd = leaf
    y = (torch.nn.functional.silu(x @ wg.t()) * (x @ wu.t())) @ wd.t()
    if not train:
        return y
    grads = torch.autograd.grad(y, leaf, s["dy"].double())
    return {"y": y.detach(), "dx": grads[0], "dw_gate": grads[1], "dw_up": grads[2], "dw_down": grads[3]}


def _exact_logprobs(case, s):
    rows, n = case["rows"], case["top_n"]
    parts = []
    for r in range(0, rows, 256):
        z = s["logits"][r:r + 256].double()
        lp = torch.log_softmax(z / case["temperature"], 1)
        part = {"logprob": lp.gather(1, s["targets"][r:r + 256, None]).squeeze(1),
                "entropy": -torch.xlogy(lp.exp(), lp.exp()).sum(1)}
        if n:
            part["top_idx"] = z.sort(dim=1, descending=True, stable=True).indices[:, :n]
            part["top_logprob"] = lp.gather(1, part["top_idx"])
            part["top_idx"] = part["top_idx"].int()
        parts.append(part)
    return {k: torch.cat([p[k] for p in parts]) for k in parts[0]}


def _exact_distill(case, s):
    tau = float(case["temperature"])
    parts = []
    for r in range(0, case["rows"], 256):
        sl = slice(r, r + 256)
        z = s["logits"][sl].double()
        want = case["mode"] != "forward"
        z.requires_grad_(want)
        idx = s["idx"][sl].long()
        lq = torch.log_softmax(z / tau, 1)
        lp = s["logprob"][sl].double()
        listed_lq = lq.gather(1, idx)
        if case["tail"]:
            rest = (1 - lp.exp().sum(1)).clamp_min(0.0)
            outside = torch.logsumexp(lq.scatter(1, idx, -math.inf), 1)
            loss = (lp.exp() * (lp - listed_lq)).sum(1) + torch.xlogy(rest, rest) - rest * outside
        else:
            lp = torch.log_softmax(lp, 1)
            loss = (lp.exp() * (lp - listed_lq)).sum(1)
        part = {}
        if case["mode"] != "backward":
            part["loss"] = loss.detach()
            if case["mode"] == "step":
                part["loss"] = part["loss"] * (s["d_loss"][sl] != 0)
        if want:
            part["d_logits"] = torch.autograd.grad(loss, z, s["d_loss"][sl].double())[0]
        parts.append(part)
    return {k: torch.cat([p[k] for p in parts]) for k in parts[0]}


def exact(case, seed):
    if case["op"].startswith("ffn"):
        return _exact_ffn(case, _ffn_inputs(case, seed))
    if case["op"] == "logprobs":
        return _exact_logprobs(case, _logprobs_inputs(case, seed))
    return _exact_distill(case, _distill_inputs(case, seed))
