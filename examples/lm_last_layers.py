"""The end of a language model's training step on the library's operators: residual add + norm, head with
cross entropy, distillation from a teacher's top logits, and the way back.

    python examples/lm_last_layers.py [--steps 60]

A small model (embedding -> residual add + norm -> head, the head's weight its own) learns a random successor
table: token t is followed by table[t].  A teacher that knows the table hands over its top logits; the head's loss is
fused with its product, so its logits exist only for the distillation term.  Gradients are combined by hand, as the
library has no tape: dL/dhidden from the head (and from the distillation through the logits' product), then the norm's
backward, whose result is the gradient of the embedding rows.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_1810_10962_b200 import lm  # noqa: E402


def main(argv=None) -> float:
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--tokens", type=int, default=512)
    ap.add_argument("--vocabulary", type=int, default=1000)
    ap.add_argument("--width", type=int, default=256)
    ap.add_argument("--lr", type=float, default=0.5)
    ap.add_argument("--temperature", type=float, default=2.0)
    a = ap.parse_args(argv)
    gen = torch.Generator(device="cuda").manual_seed(1)
    V, D, K = a.vocabulary, a.width, 4
    embedding = torch.randn(V, D, device="cuda", generator=gen)           # fp32 masters, bf16 operands
    head = torch.randn(V, D, device="cuda", generator=gen) * 0.02
    gain = torch.ones(D, device="cuda")
    table = torch.randperm(V, device="cuda", generator=gen)
    loss = 0.0
    for step in range(a.steps):
        tokens = torch.randint(0, V, (a.tokens,), device="cuda", generator=gen)
        target = table[tokens].clone()
        target[::16] = -100                                               # tokens that carry no loss
        count = int((target >= 0).sum())
        # forward: residual add + norm, head + cross entropy
        x = embedding[tokens].bfloat16()
        residual = torch.zeros_like(x)
        hidden, h, rstd = lm.rms_norm_forward(x, residual, gain, 1e-5)
        w = head.bfloat16()
        losses, lse = lm.linear_cross_entropy_forward(hidden, w, target)
        # the way back: head, distillation (its logits are a plain product), norm
        dloss = torch.full((a.tokens,), 1.0 / count, device="cuda")
        dhidden, dw = lm.linear_cross_entropy_backward(hidden, w, target, lse, dloss)
        logits = hidden @ w.t()
        index = (table[tokens][:, None] + torch.arange(K, device="cuda")) % V      # the teacher's short list
        teacher = torch.tensor([8.0, 2.0, 1.0, 0.0], device="cuda").expand(a.tokens, K).contiguous()
        soft, dlogits = lm.topk_distillation_step(logits, teacher, index, dloss * 0.1, a.temperature)
        dhidden = dhidden + dlogits @ w
        dw = dw + dlogits.t() @ hidden
        dx, dgain = lm.rms_norm_backward(dhidden, h, gain, rstd)
        embedding.index_add_(0, tokens, dx.float(), alpha=-a.lr * D ** 0.5)
        head -= a.lr * D ** 0.5 * dw.float()
        gain -= a.lr * 0.1 * dgain
        loss = float(losses.sum()) / count
        if step % 10 == 0 or step == a.steps - 1:
            print(f"step {step:3d}  cross entropy {loss:.4f}  distillation {float(soft.mean()):.4f}")
    # answering: the last token's hidden row in 8 bits, as an 8-bit product would take it
    q, scales, _, _ = lm.rms_norm_forward_fp8(embedding[tokens[:1]].bfloat16(), None, gain, 1e-5)
    guess = int(((q.float() * scales) @ head.t()).argmax())
    print(f"token {int(tokens[0])} -> {guess}, the table says {int(table[tokens[0]])}")
    return loss


if __name__ == "__main__":
    main()
