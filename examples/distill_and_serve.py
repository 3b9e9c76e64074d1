"""Distils a 4-bit teacher into a small student with 4-bit AdamW, then serves the student from 4-bit weights.

    python examples/distill_and_serve.py [--steps 200]

The teacher is a frozen output head kept in 4 bits (lpmm.w4_quantize). For every batch of hidden states it answers with its top
logits and their log-sum-exp (lpmm.w4_matvec); the student, a two-layer network on the same states, gets its loss and the gradient
of its logits from them (lpmm.distill_grad), and its parameters take a step with 4-bit optimizer states (lpmm.adamw4_step, which
also writes the bfloat16 copy that the next forward pass uses). At the end the student's matrices are quantized too and answer
single states. Synthetic data; needs a CUDA device.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2309_01507_b200 import lpmm                           # noqa: E402
from paper_2309_01507_b200.workloads import TensorSpec           # noqa: E402


def main(steps: int = 200, hidden: int = 256, width: int = 512, vocab: int = 4000, tokens: int = 256, top: int = 64, tau: float = 2.0,
         device: str = "cuda") -> dict:
    gen = torch.Generator(device=device)
    gen.manual_seed(0)
    randn = lambda *shape: torch.randn(*shape, generator=gen, device=device)      # noqa: E731

    # the frozen teacher: logits = states @ W^T, W in 4 bits with a scale per 64 columns
    teacher = lpmm.w4_quantize(randn(vocab, hidden) * (2.5 / hidden ** 0.5), group=64, scale_dtype=torch.bfloat16)

    # the student: fp32 masters for the optimizer, bfloat16 copies for the model
    specs = [TensorSpec("up", width, hidden, 2), TensorSpec("head", vocab, width, 2)]
    params = [randn(width, hidden) / hidden ** 0.5, randn(vocab, width) * (0.1 / width ** 0.5)]
    copies = [p.bfloat16() for p in params]
    state = lpmm.state_init(lpmm.default_config(), specs, device=device)

    losses = []
    for step in range(1, steps + 1):
        states = randn(tokens, hidden).bfloat16()
        weights = (torch.rand(tokens, generator=gen, device=device) > 0.1).float()      # a tenth of the positions is padding
        weights /= weights.sum()

        answers = lpmm.w4_matvec(teacher, states, out_dtype=torch.float32)
        top_logits, top_ids = torch.topk(answers, top, dim=1)
        lse = torch.logsumexp(answers / tau, dim=1)

        inner = torch.nn.functional.silu(states @ copies[0].T)
        logits = inner @ copies[1].T
        loss, dlogits = lpmm.distill_grad(logits, top_ids, top_logits, temperature=tau, teacher_lse=lse, weights=weights, out=logits)
        losses.append(loss.sum())

        dinner = (dlogits @ copies[1]).float()
        pre = (states @ copies[0].T).float()
        gate = torch.sigmoid(pre)
        grads = [(dinner * (gate * (1 + pre * (1 - gate)))).bfloat16().T @ states, dlogits.T @ inner]
        lpmm.adamw4_step(state, params, [g.contiguous() for g in grads], lr=3e-3, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.0,
                         step=step, params_bf16=copies)

    # the student in service: 4-bit matrices, one state at a time
    served = [lpmm.w4_quantize(c, group=32, zero_points=True, scale_dtype=torch.bfloat16) for c in copies]
    same = close = 0
    for _ in range(50):
        x = randn(hidden).bfloat16()
        y4 = lpmm.w4_matvec(served[1], torch.nn.functional.silu(lpmm.w4_matvec(served[0], x)), out_dtype=torch.float32)
        y16 = (torch.nn.functional.silu(x @ copies[0].T) @ copies[1].T).float()
        same += int(y4.argmax() == y16.argmax())
        close += float(torch.nn.functional.cosine_similarity(y4, y16, dim=0)) / 50
    first, last = float(losses[0]), float(torch.stack(losses[-10:]).mean())
    full = sum(p.numel() * 2 for p in params)
    small = sum(m.codes.numel() + 3 * m.scales.numel() for m in served)
    print(f"distillation loss {first:.4f} -> {last:.4f} in {steps} steps; the 4-bit student ({small / full:.2f} of the bf16 bytes) agrees "
          f"with the bf16 one on {same} of 50 best entries, cosine {close:.4f}")
    return {"first": first, "last": last, "same": same, "cosine": close}


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=200)
    main(ap.parse_args().steps)
