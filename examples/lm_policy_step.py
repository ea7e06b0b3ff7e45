"""A policy-gradient step of a small attention model on the library's operators: norm + rotation of the heads, residual
add + norm, log probabilities and entropy of sampled tokens, the way back through all of them, clipping.

    python examples/lm_policy_step.py [--steps 60]

The model sees a token and answers with another one, sampled from its distribution; it is rewarded where the answer is the
token that a hidden table asks for.  Products and the attention itself are plain torch; gradients are combined by hand, as
the library has no tape.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_1810_10962_b200 import lm  # noqa: E402

EPS = 1e-6


def make_parameters(vocabulary, width, heads, kv_heads, head_dim, generator):
    normal = lambda *shape: torch.randn(*shape, device="cuda", generator=generator)  # noqa: E731
    return {"embedding": normal(vocabulary, width), "qkv": normal((heads + 2 * kv_heads) * head_dim, width) * width ** -0.5,
            "q_weight": torch.ones(head_dim, device="cuda"), "k_weight": torch.ones(head_dim, device="cuda"),
            "out": normal(width, heads * head_dim) * (heads * head_dim) ** -0.5, "gain": torch.ones(width, device="cuda"),
            "head": normal(vocabulary, width) * 0.02}


def tables(positions, rotary):
    angle = torch.arange(positions, dtype=torch.float64, device="cuda")[:, None] * 10000.0 ** (
        -torch.arange(0, rotary, 2, dtype=torch.float64, device="cuda") / rotary)
    return torch.cos(angle).float(), torch.sin(angle).float()


class Step:
    """Forward pass up to the logits, then log probabilities and gradients of chosen tokens."""

    def __init__(self, parameters, shape, cos_sin, dtype):
        self.p, (self.heads, self.kv_heads, self.head_dim), self.cos_sin, self.dtype = parameters, shape, cos_sin, dtype

    def forward(self, tokens):
        p, Hq, Hk, D = {n: v.to(self.dtype) if v.dim() == 2 else v for n, v in self.p.items()}, self.heads, self.kv_heads, self.head_dim
        B, S = tokens.shape
        self.tokens, self.cast = tokens, p
        self.x = p["embedding"][tokens]
        self.packed = (self.x @ p["qkv"].t()).view(B, S, Hq + 2 * Hk, D)
        self.position = torch.arange(S, device="cuda").expand(B, S).contiguous()
        self.rotation = (self.packed[:, :, :Hq], self.packed[:, :, Hq: Hq + Hk], p["q_weight"], p["k_weight"], *self.cos_sin,
                         self.position, EPS)
        q, k = lm.head_norm_rotary_forward(*self.rotation)
        # attention, causal, each key head shared by Hq / Hk query heads
        self.q = q.view(B, S, Hk, Hq // Hk, D).float()
        self.k, self.v = k.float(), self.packed[:, :, Hq + Hk:].float()
        score = torch.einsum("bshgd,bthd->bhgst", self.q, self.k) * D ** -0.5
        hidden = torch.ones(S, S, dtype=torch.bool, device="cuda").triu(1)
        self.weights = score.masked_fill(hidden, float("-inf")).softmax(-1)
        self.mixed = torch.einsum("bhgst,bthd->bshgd", self.weights, self.v).reshape(B, S, Hq * D).to(self.dtype)
        y, self.h, self.rstd = lm.rms_norm_forward(self.mixed @ p["out"].t(), self.x, p["gain"], EPS)
        self.y = y
        return y @ p["head"].t()

    def backward(self, dlogits):
        """Gradients of all parameters."""
        p, Hq, Hk, D = self.cast, self.heads, self.kv_heads, self.head_dim
        B, S = self.tokens.shape
        flat = lambda t: t.reshape(B * S, -1)  # noqa: E731
        grads = {"head": flat(dlogits).t() @ flat(self.y)}
        dh, grads["gain"] = lm.rms_norm_backward(dlogits @ p["head"], self.h, p["gain"], self.rstd)
        grads["out"] = flat(dh).t() @ flat(self.mixed)
        dmixed = (dh @ p["out"]).view(B, S, Hk, Hq // Hk, D).float()
        dv = torch.einsum("bhgst,bshgd->bthd", self.weights, dmixed)
        dweights = torch.einsum("bshgd,bthd->bhgst", dmixed, self.v)
        dscore = self.weights * (dweights - (self.weights * dweights).sum(-1, keepdim=True)) * D ** -0.5
        dq = torch.einsum("bhgst,bthd->bshgd", dscore, self.k).reshape(B, S, Hq, D).to(self.dtype)
        dk = torch.einsum("bhgst,bshgd->bthd", dscore, self.q).to(self.dtype)
        dq, dk, grads["q_weight"], grads["k_weight"] = lm.head_norm_rotary_backward(dq, dk.contiguous(), *self.rotation)
        dpacked = torch.cat([dq, dk, dv.to(self.dtype)], 2)
        grads["qkv"] = flat(dpacked).t() @ flat(self.x)
        dx = flat(dpacked) @ p["qkv"] + flat(dh)
        grads["embedding"] = torch.zeros_like(self.p["embedding"]).index_add_(0, self.tokens.flatten(), dx.float())
        return {n: grads[n] for n in self.p}


def main(argv=None) -> float:
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--batch", type=int, default=32)
    ap.add_argument("--length", type=int, default=16)
    ap.add_argument("--vocabulary", type=int, default=40)
    ap.add_argument("--width", type=int, default=128)
    ap.add_argument("--lr", type=float, default=1.0)
    ap.add_argument("--entropy", type=float, default=0.01)
    ap.add_argument("--max-norm", type=float, default=1.0)
    a = ap.parse_args(argv)
    gen = torch.Generator(device="cuda").manual_seed(2)
    shape, V = (4, 2, 32), a.vocabulary
    parameters = make_parameters(V, a.width, *shape, gen)
    step_of = Step(parameters, shape, tables(a.length, 32), torch.bfloat16)
    table = torch.randperm(V, device="cuda", generator=gen)
    rate = 0.0
    for step in range(a.steps):
        tokens = torch.randint(0, V, (a.batch, a.length), device="cuda", generator=gen)
        logits = step_of.forward(tokens)
        answers = torch.multinomial(logits.float().softmax(-1).view(-1, V), 1, generator=gen).view_as(tokens)
        reward = (answers == table[tokens]).float()
        logprob, entropy, lse = lm.token_log_probs_forward(logits, answers)
        count = tokens.numel()
        dlogprob = -(reward - reward.mean()) / count                      # of the loss, to be made small
        dentropy = torch.full_like(entropy, -a.entropy / count)
        grads = step_of.backward(lm.token_log_probs_backward(logits, answers, lse, entropy, dlogprob, dentropy))
        norm = lm.clip_gradients(list(grads.values()), a.max_norm)
        for name, g in grads.items():
            parameters[name] -= a.lr * g.float()
        rate = float(reward.mean())
        if step % 10 == 0 or step == a.steps - 1:
            print(f"step {step:3d}  rewarded {rate:.3f}  entropy {float(entropy.mean()):.3f}  gradient norm {float(norm):.3f}")
    # what an interface would show for the last answer: its log probability and the alternatives
    logprob, _, _, top, index = lm.token_log_probs_forward_top(logits[-1:, -1], answers[-1:, -1], 3)
    print(f"answer {int(answers[-1, -1])} at {float(logprob):.2f}; most likely", [(int(i), round(float(v), 2)) for i, v in zip(index[0], top[0])])
    return rate


if __name__ == "__main__":
    main()
