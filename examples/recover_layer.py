"""Train the experts that a slicing left of a whole MoE layer (norm, router, experts, residual) with orthogonalised updates.

    python examples/recover_layer.py [--prune 0.4] [--steps 60] [--tokens 1024]

A layer of routed gated experts is scored on calibration tokens and its micro-experts of least energy are cut out over all
experts; what is left (experts of different heights) is trained so that the layer's output follows the whole layer's:

  camera_score_layer, camera_select_prune, camera_sub_index, camera_compact_weights     the sliced experts
  camera_norm_forward, camera_moe_dispatch, camera_ffn_forward, camera_moe_combine      the layer's output
  camera_moe_combine_backward, camera_ffn_backward, camera_moe_dispatch_backward, camera_norm_backward     its gradients
  camera_orthogonalize                                                                  the update of the experts' matrices

The experts' matrices are what is trained; the gradients of the norm's weight and of the router come out of the same backward
pass and are left unused here.  Weights and hidden states are synthetic (random); the router and its gradient are plain matrix
products.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2508_02322_b200 as P  # noqa: E402


class Block:
    """x + MoE(norm(x)): a norm's weight, a router and gated experts, with what a backward pass needs kept in between."""

    def __init__(self, norm_weight, w_router, experts, top_k, tokens):
        self.norm_weight, self.w_router, self.experts, self.top_k = norm_weight, w_router, experts, top_k
        dev, d = w_router.device, w_router.shape[1]
        n = tokens * top_k
        widest = max(experts, key=lambda f: f.d_ff)
        # an expert may be given any number of the pairs: buffers for all of them
        self.workspace = P.alloc_workspace(P.camera_ffn_workspace_bytes(widest, n, backward=True), dev)
        self.saved = [P.alloc_workspace(P.camera_ffn_saved_bytes(f, n), dev) for f in experts]
        self.y_sorted = torch.empty(n, d, dtype=torch.bfloat16, device=dev)

    def route(self, h):
        """Top k experts of each token, their probabilities over the sum of the kept ones, and all probabilities."""
        p = torch.softmax(h.float() @ self.w_router.float().t(), 1)
        top, idx = p.topk(self.top_k, 1)
        return idx.int(), (top / top.sum(1, keepdim=True)).contiguous(), p

    def forward(self, x):
        norm = P.camera_norm_forward(x, self.norm_weight, rms=True)
        idx, w, p = self.route(norm["y"])
        s = P.camera_moe_dispatch(norm["y"], idx, len(self.experts))
        ends = s["offsets"].tolist()                    # the host's loop over experts needs their rows
        for e, ffn in enumerate(self.experts):
            a, b = ends[e], ends[e + 1]
            if b > a:
                P.camera_ffn_forward(ffn, s["x"][a:b], y=self.y_sorted[a:b], saved=self.saved[e], workspace=self.workspace)
        y = P.camera_moe_combine(self.y_sorted, s["rows"], w, add=x)
        self.kept = x, norm, idx.long(), w, p, s, ends
        return y

    def backward(self, dy):
        """Gradients given dy: a dict with x, norm, router and experts (a list of dicts, None where no token went)."""
        x, norm, idx, w, p, s, ends = self.kept
        back = P.camera_moe_combine_backward(dy, self.y_sorted, s["rows"], w)
        dx_sorted, grads = torch.empty_like(s["x"]), []
        for e, ffn in enumerate(self.experts):
            a, b = ends[e], ends[e + 1]
            grads.append(P.camera_ffn_backward(ffn, s["x"][a:b], back["y"][a:b], self.saved[e], out={"x": dx_sorted[a:b]},
                                               workspace=self.workspace) if b > a else None)
        # w = top / sum of top, top = softmax(logits): both plain
        kept = p.gather(1, idx)
        total = kept.sum(1, keepdim=True)
        dw = back["weights"]
        dp = torch.zeros_like(p).scatter_(1, idx, (dw - (dw * w).sum(1, keepdim=True)) / total)
        dz = p * (dp - (p * dp).sum(1, keepdim=True))
        from_router = (dz @ self.w_router.float()).to(x.dtype)
        dh = P.camera_moe_dispatch_backward(dx_sorted, s["rows"], add=from_router)
        back_norm = P.camera_norm_backward(dh, x, norm["rstd"], None, self.norm_weight, d_sum=dy)
        return {"x": back_norm["x"], "norm": back_norm["weight"], "router": dz.t() @ norm["y"].float(), "experts": grads}


def slice_layer(norm_weight, w_router, w_gate, w_up, w_down, x, top_k, prune):
    """The layer's experts without the micro-experts of least energy on x, as P.Ffn over buffers of the original size."""
    layer = P.Layer(w_router, w_gate, w_up, w_down, top_k=top_k)
    energy = P.camera_score_layer(layer, P.camera_norm_forward(x, norm_weight, rms=True)["y"], 0.95)
    keep = P.camera_select_prune(energy, prune)
    sub, counts = P.camera_sub_index(keep, P.expert_offsets_tensor(layer), [1])
    out = P.camera_compact_weights(layer, sub, counts, 1)
    kept = counts.sum(1).tolist()
    return [P.Ffn(out["w_gate"][e], out["w_up"][e], out["w_down"][e], d_ff=f) for e, f in enumerate(kept) if f > 0], kept


def recover(d_model=256, d_ff=512, n_experts=8, top_k=2, tokens=1024, prune=0.4, steps=60, lr=0.001, momentum=0.9, rank=16, seed=0, device="cuda", log=print):
    g = torch.Generator(device=device).manual_seed(seed)
    rnd = lambda *s: torch.randn(s, device=device, generator=g)
    strength = lambda: torch.exp(rnd(d_ff, 1) * 0.7)
    w_gate = [(rnd(d_ff, d_model) * d_model ** -0.5 * 1.5).bfloat16() for _ in range(n_experts)]
    w_up = [(rnd(d_ff, d_model) * d_model ** -0.5 * strength()).bfloat16() for _ in range(n_experts)]
    w_down = [(rnd(d_model, d_ff) * d_ff ** -0.5).bfloat16() for _ in range(n_experts)]
    w_router = (rnd(n_experts, d_model) * d_model ** -0.5).bfloat16()
    norm_weight = (1 + 0.1 * rnd(d_model)).bfloat16()
    # hidden states lie near a few directions, which is why the remaining micro-experts can stand in for the others
    basis = rnd(rank, d_model)
    data = lambda: (rnd(tokens, rank) @ basis * rank ** -0.5).bfloat16()

    teacher = Block(norm_weight, w_router, [P.Ffn(*m) for m in zip(w_gate, w_up, w_down)], top_k, tokens)
    experts, kept = slice_layer(norm_weight, w_router, w_gate, w_up, w_down, data(), top_k, prune)
    if len(experts) < n_experts:
        raise ValueError("the slicing left an expert without micro-experts: prune less")
    student = Block(norm_weight.clone(), w_router, experts, top_k, tokens)
    log(f"{n_experts * d_ff} micro-experts, {sum(kept)} kept ({min(kept)} to {max(kept)} an expert)")

    views = [m for f in experts for m in (f.w_gate[:f.d_ff], f.w_up[:f.d_ff], f.w_down[:, :f.d_ff])]
    master = [v.float() for v in views]
    velocity = [torch.zeros_like(m) for m in master]
    scratch = P.alloc_workspace(P.camera_orthogonalize_workspace_bytes(velocity), device)
    losses = []
    for step in range(steps):
        x = data()
        target = teacher.forward(x).float()
        off = student.forward(x).float() - target
        losses.append(float(off.pow(2).mean()))
        grads = student.backward((off * (2.0 / off.numel()) * tokens).bfloat16())      # times tokens: within bf16's ease
        flat = [None if gr is None else t for gr, f in zip(grads["experts"], experts)
                for t in ((None,) * 3 if gr is None else (gr["w_gate"], gr["w_up"], gr["w_down"][:, :f.d_ff]))]
        for v, t in zip(velocity, flat):
            v.mul_(momentum)
            if t is not None:
                v.add_(t)
        updates = P.camera_orthogonalize(velocity, workspace=scratch)
        for m, v, o in zip(master, views, updates):
            # an orthogonal matrix's elements are sqrt(1 / longer side) in size: brought to the size of the weights' own
            m.sub_(o.float(), alpha=lr * (1 - step / steps) * max(m.shape) ** 0.5)
            v.copy_(m)
        if step % 20 == 0:
            log(f"step {step:3d}  squared error {losses[-1]:.5f}")
    assert P.camera_read_status(scratch) == 0 and P.camera_read_status(student.workspace) == 0
    log(f"squared error {losses[0]:.5f} -> {losses[-1]:.5f}")
    return {"kept": kept, "losses": losses, "student": student, "velocity": velocity, "updates": updates}


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--prune", type=float, default=0.4)
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--tokens", type=int, default=1024)
    a = ap.parse_args()
    recover(prune=a.prune, steps=a.steps, tokens=a.tokens)
