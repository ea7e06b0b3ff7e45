"""Token log probabilities, heads' norm + rotation, residual add + norm and clipping together in one training step; what the
binding refuses; calls side by side."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu


def example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "lm_policy_step.py")
    spec = importlib.util.spec_from_file_location("lm_policy_step", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def plain_loss(p, shape, cos, sin, tokens, answers, dlogprob, dentropy):
    """The same step in 64 bits: the sum of both outputs times their gradients."""
    Hq, Hk, D = shape
    B, S = tokens.shape

    def norm(x, w):
        return x / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-6) * w

    def turned(x):
        a, b = x[..., : D // 2], x[..., D // 2:]
        c, s = cos.double()[:S, None], sin.double()[:S, None]
        return torch.cat([a * c - b * s, b * c + a * s], -1)

    x = p["embedding"][tokens]
    packed = (x @ p["qkv"].T).view(B, S, Hq + 2 * Hk, D)
    q, k = turned(norm(packed[:, :, :Hq], p["q_weight"])), turned(norm(packed[:, :, Hq: Hq + Hk], p["k_weight"]))
    k, v = (t.repeat_interleave(Hq // Hk, 2) for t in (k, packed[:, :, Hq + Hk:]))
    score = torch.einsum("bshd,bthd->bhst", q, k) * D ** -0.5
    score = score.masked_fill(torch.ones(S, S, dtype=torch.bool, device="cuda").triu(1), float("-inf"))
    mixed = torch.einsum("bhst,bthd->bshd", score.softmax(-1), v).reshape(B, S, -1)
    logits = norm(mixed @ p["out"].T + x, p["gain"]) @ p["head"].T
    logq = logits.log_softmax(-1)
    logp = torch.where(answers >= 0, logq.gather(-1, answers.clamp(min=0)[..., None])[..., 0], 0.0)
    entropy = -(logq.exp() * logq).sum(-1)
    return logits, (logp * dlogprob.double() + entropy * dentropy.double()).sum()


def test_a_step_against_64_bits():
    from paper_1810_10962_b200 import lm
    module = example()
    g = torch.Generator(device="cuda").manual_seed(5)
    shape, V, B, S = (6, 2, 32), 57, 3, 21
    parameters = module.make_parameters(V, 96, *shape, g)
    for name in ("q_weight", "k_weight", "gain"):
        parameters[name] += 0.2 * torch.randn(parameters[name].shape, device="cuda", generator=g)
    parameters["head"] *= 20
    cos, sin = module.tables(S, 32)
    tokens, answers = (torch.randint(0, V, (B, S), device="cuda", generator=g) for _ in range(2))
    answers[0, ::4] = -100
    dlogprob, dentropy = (torch.randn(B, S, device="cuda", generator=g) / (B * S) for _ in range(2))
    step = module.Step(parameters, shape, (cos, sin), torch.float32)
    matmul = torch.backends.cuda.matmul.allow_tf32
    torch.backends.cuda.matmul.allow_tf32 = False
    try:
        logits = step.forward(tokens)
        logprob, entropy, lse = lm.token_log_probs_forward(logits, answers)
        grads = step.backward(lm.token_log_probs_backward(logits, answers, lse, entropy, dlogprob, dentropy))
    finally:
        torch.backends.cuda.matmul.allow_tf32 = matmul
    leaves = {n: v.double().requires_grad_() for n, v in parameters.items()}
    want_logits, loss = plain_loss(leaves, shape, cos, sin, tokens, answers, dlogprob, dentropy)
    loss.backward()
    # some ten products and norms one after another, each good to 2^-24 sqrt(its length <= 192) of its norm, some to twice that
    tolerance = 10 * 2 * 192 ** 0.5 * 2.0 ** -24
    off = lambda got, want: float((got.double() - want).norm() / want.norm())  # noqa: E731
    assert off(logits, want_logits.detach()) < tolerance
    for name, leaf in leaves.items():
        assert off(grads[name], leaf.grad) < 4 * tolerance, name           # there and back, and sums of both signs
    total = sum(float(leaf.grad.square().sum()) for leaf in leaves.values()) ** 0.5
    outs = [torch.empty_like(t) for t in grads.values()]
    norm = lm.clip_gradients(list(grads.values()), 0.5 * total, outs)
    assert abs(float(norm) - total) < 4 * tolerance * total
    for got, leaf in zip(outs, leaves.values()):
        assert off(got, leaf.grad * 0.5) < 8 * tolerance


def test_example_runs():
    rate = example().main(["--steps", "12"])
    assert 0.0 <= rate <= 1.0


def test_binding_refuses_tensors_that_do_not_fit():
    from paper_1810_10962_b200 import bns, lm
    c = lambda *s, dtype=torch.bfloat16: torch.zeros(*s, dtype=dtype, device="cuda")  # noqa: E731
    z, token, vector = c(4, 64), c(4, dtype=torch.int64), c(4, dtype=torch.float32)
    q, k, w, t, at = c(3, 4, 32), c(3, 2, 32), c(32, dtype=torch.float32), c(5, 8, dtype=torch.float32), c(3, dtype=torch.int64)
    bad = [
        lambda: lm.token_log_probs_forward(z, c(5, dtype=torch.int64)),
        lambda: lm.token_log_probs_forward(z, c(4, dtype=torch.float32)),
        lambda: lm.token_log_probs_forward(z.t(), c(64, dtype=torch.int64)),
        lambda: lm.token_log_probs_forward(z.half(), token),
        lambda: lm.token_log_probs_forward(z, c(8, dtype=torch.int64)[::2]),
        lambda: lm.token_log_probs_backward(z, token, vector, vector, c(4)),
        lambda: lm.token_log_probs_backward(z, token, c(3, dtype=torch.float32), vector, vector),
        lambda: lm.token_log_probs_backward(z, token, vector, None, vector, vector),
        lambda: lm.head_norm_rotary_forward(q, k.float(), w, w, t, t, at, 1e-6),
        lambda: lm.head_norm_rotary_forward(q, c(3, 2, 16), w, w, t, t, at, 1e-6),
        lambda: lm.head_norm_rotary_forward(q, c(2, 2, 32), w, w, t, t, at, 1e-6),
        lambda: lm.head_norm_rotary_forward(q, c(1, 3, 2, 32), w, w, t, t, at, 1e-6),
        lambda: lm.head_norm_rotary_forward(q, k, c(32), w, t, t, at, 1e-6),
        lambda: lm.head_norm_rotary_forward(q, k, w, None, t, t, at, 1e-6),
        lambda: lm.head_norm_rotary_forward(q, k, w, w, t.bfloat16(), t, at, 1e-6),
        lambda: lm.head_norm_rotary_forward(q, k, w, w, t, t[:4], at, 1e-6),
        lambda: lm.head_norm_rotary_forward(q, k, w, w, t, t, at[:2], 1e-6),
        lambda: lm.head_norm_rotary_forward(q[..., ::2], None, w[:16].clone(), None, t, t, at, 1e-6),
        lambda: lm.head_norm_rotary_forward(c(3, 32), None, w, None, t, t, at, 1e-6),
        lambda: lm.head_norm_rotary_backward(q[:2], k, q, k, w, w, t, t, at, 1e-6),
        lambda: lm.head_norm_rotary_backward(q, None, q, k, w, w, t, t, at, 1e-6),
        lambda: lm.head_norm_rotary_backward(q.transpose(0, 1).contiguous().transpose(0, 1), k, q, k, w, w, t, t, at, 1e-6),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(TypeError):
            call()
            pytest.fail(f"call {i} was not refused")
    for call in (lambda: lm.token_log_probs_forward_top(z, token, 65), lambda: lm.token_log_probs_forward(z, token, 0.0),
                 lambda: lm.token_log_probs_forward_top(z[:, :8].contiguous(), token, 9),
                 lambda: lm.head_norm_rotary_forward(q, k, w, w, t, t, at, 0.0),
                 lambda: lm.head_norm_rotary_forward(q, k, w, w, c(5, 17, dtype=torch.float32), c(5, 17, dtype=torch.float32), at, 1e-6)):
        with pytest.raises(bns.BnsError) as err:
            call()
        assert err.value.status == -2
    with pytest.raises(bns.BnsError) as err:
        lm.head_norm_rotary_backward(q, k, q, k, w, w, t, t, at, 1e-6, workspace=c(64, dtype=torch.uint8))
    assert err.value.status == -7


def test_calls_side_by_side_on_two_streams():
    """Two streams at once, each with its own tensors: the same bits as one after the other."""
    from paper_1810_10962_b200 import lm
    g = torch.Generator(device="cuda").manual_seed(7)
    cases = []
    for seed in range(2):
        z = torch.randn(300, 20011, device="cuda", generator=g).bfloat16()
        q = torch.randn(2, 500, 10, 128, device="cuda", generator=g).bfloat16()
        w = torch.ones(128, device="cuda")
        t = torch.randn(500, 64, device="cuda", generator=g)
        grads = [torch.randn(n, device="cuda", generator=g) for n in (300_000, 17, 5000)]
        cases.append((z, torch.randint(0, 20011, (300,), device="cuda", generator=g), q, w, t, torch.arange(500, device="cuda").expand(2, 500).contiguous(),
                      lm.GradientList(grads, [torch.empty_like(x) for x in grads])))

    def run(case):
        z, token, q, w, t, at, both = case
        out = [*lm.token_log_probs_forward_top(z, token, 20)]
        out.append(lm.token_log_probs_backward(z, token, out[2], out[1], out[0], out[1]))
        rest = (q[:, :, :8], q[:, :, 8:], w, w, t, t, at, 1e-6)
        turned = lm.head_norm_rotary_forward(*rest)
        out += [*turned, *lm.head_norm_rotary_backward(*turned, *rest), both.clip(0.1), *both.out]
        return out

    want = [[t.clone() for t in run(c)] for c in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    for _ in range(5):
        got = []
        for case, stream in zip(cases, streams):
            with torch.cuda.stream(stream):
                got.append(run(case))
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert all(torch.equal(x, y) for x, y in zip(a, b))
