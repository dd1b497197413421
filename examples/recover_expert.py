"""Slice a feed-forward expert with CAMERA-P and train what is left against the whole one.

    python examples/recover_expert.py [--prune 0.4] [--steps 100] [--tokens 2048]

One gated expert (as a layer of one shared expert) is scored on calibration tokens, the micro-experts of least energy are
cut out, and the sliced expert is trained so that a language-model head behind it predicts what it predicted with the
whole expert:

  camera_score_layer, camera_select_prune, camera_sub_index, camera_compact_weights    the sliced expert
  camera_ffn_forward + head + camera_token_logprobs                                    the teacher's top log-probabilities
  camera_ffn_forward + head + camera_distill_step + camera_ffn_backward                a training step
  camera_token_logprobs                                                                evaluation

Weights, hidden states and the head are synthetic (random); the head and its gradient are plain matrix products.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2508_02322_b200 as P  # noqa: E402


def slice_expert(w_gate, w_up, w_down, x, prune_ratio):
    """The expert without the micro-experts of least energy on x, as a P.Ffn over buffers of the original size."""
    layer = P.Layer(None, [w_gate], [w_up], [w_down], top_k=0, n_shared=1)
    energy = P.camera_score_layer(layer, x, 0.95)
    keep = P.camera_select_prune(energy, prune_ratio)
    sub, counts = P.camera_sub_index(keep, P.expert_offsets_tensor(layer), [1])
    out = P.camera_compact_weights(layer, sub, counts, 1)
    kept = int(counts.sum())
    return P.Ffn(out["w_gate"][0], out["w_up"][0], out["w_down"][0], d_ff=kept)


def recover(d_model=512, d_ff=2048, vocab=8192, tokens=2048, prune=0.4, steps=100, lr=3e-4, rank=16, top=64, temperature=1.0, seed=0,
            device="cuda", log=print):
    g = torch.Generator(device=device).manual_seed(seed)
    rnd = lambda *s: torch.randn(s, device=device, generator=g)
    # micro-experts of very different weight, as trained experts have them
    strength = torch.exp(rnd(d_ff, 1) * 0.7)
    w_gate, w_up = (rnd(d_ff, d_model) * d_model ** -0.5 * 1.5).bfloat16(), (rnd(d_ff, d_model) * d_model ** -0.5 * strength).bfloat16()
    w_down = (rnd(d_model, d_ff) * d_ff ** -0.5).bfloat16()
    head = (rnd(vocab, d_model) * 0.25).bfloat16()
    # hidden states lie near a few directions, which is why the remaining micro-experts can stand in for the others
    basis = rnd(rank, d_model)
    data = lambda: (lambda x: (x / x.pow(2).mean(1, keepdim=True).sqrt()).bfloat16())(rnd(tokens, rank) @ basis)
    calib_x, eval_x = data(), data()

    teacher = P.Ffn(w_gate, w_up, w_down)
    student = slice_expert(w_gate, w_up, w_down, calib_x, prune)
    f = student.d_ff
    log(f"{d_ff} micro-experts, {f} kept")

    workspace = P.alloc_workspace(P.camera_ffn_workspace_bytes(teacher, tokens, backward=True), device)
    saved = P.alloc_workspace(P.camera_ffn_saved_bytes(student, tokens), device)
    logits_of = lambda ffn, x, **kw: P.camera_ffn_forward(ffn, x, workspace=workspace, **kw) @ head.t()

    eval_logits = logits_of(teacher, eval_x)
    targets = torch.distributions.Categorical(logits=eval_logits.float()).sample()
    eval_lists = P.camera_token_logprobs(eval_logits, targets, top_n=top, temperature=temperature)

    def evaluate():
        z = logits_of(student, eval_x)
        own = P.camera_token_logprobs(z, targets)
        kl = P.camera_distill_forward(z, eval_lists["top_idx"], eval_lists["top_logprob"], temperature=temperature, tail=True)
        return float(kl["loss"].mean()), float(torch.exp(-own["logprob"].mean()))

    teacher_ppl = float(torch.exp(-eval_lists["logprob"].mean()))
    before = evaluate()
    log(f"perplexity: teacher {teacher_ppl:.2f}, sliced {before[1]:.2f}; divergence {before[0]:.4f}")

    names = {"w_gate": student.w_gate[:f], "w_up": student.w_up[:f], "w_down": student.w_down}
    master = {k: v.float() for k, v in names.items()}
    optimizer = torch.optim.Adam(master.values(), lr=lr)
    d_loss = torch.full((tokens,), 1.0 / tokens, device=device)
    for step in range(steps):
        x = data()                                   # fresh tokens, and what the whole expert makes of them
        lists = P.camera_token_logprobs(logits_of(teacher, x), top_n=top, temperature=temperature, entropy=False)
        z = logits_of(student, x, saved=saved)
        loss, d_logits = P.camera_distill_step(z, lists["top_idx"], lists["top_logprob"], d_loss, temperature=temperature,
                                               tail=True, d_logits=z)
        dy = d_logits @ head
        grads = P.camera_ffn_backward(student, x, dy, saved, want_x=False, workspace=workspace)
        for k, m in master.items():
            m.grad = grads[k].float()
        master["w_down"].grad[:, f:] = 0.0           # the columns behind the sliced ones hold nothing
        optimizer.step()
        for k, v in names.items():
            v.copy_(master[k])
        if step % 20 == 0:
            log(f"step {step:3d}  divergence {float(loss.mean()):.4f}")
    assert P.camera_read_status(workspace) == 0
    after = evaluate()
    log(f"perplexity: teacher {teacher_ppl:.2f}, recovered {after[1]:.2f}; divergence {after[0]:.4f}")
    return {"teacher_ppl": teacher_ppl, "before": before, "after": after, "kept": f}


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--prune", type=float, default=0.4)
    ap.add_argument("--steps", type=int, default=100)
    ap.add_argument("--tokens", type=int, default=2048)
    a = ap.parse_args()
    recover(prune=a.prune, steps=a.steps, tokens=a.tokens)
