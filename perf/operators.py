"""Cases of the language-model operators: what a training or serving program has in hand, and one pass.

Three operators, each in every direction a program calls it:

* ``norm``     residual add + root-mean-square norm: forward, forward with 8-bit output and scales
               (one per row or per 128 columns), forward + backward;
* ``head``     linear head + softmax cross entropy over the vocabulary: forward, forward + backward;
* ``distill``  divergence from a teacher's top logits: forward, backward, loss and gradient in one call.

``own`` chooses between the plain form (elementary torch operations in 32 bits, rounded once at the end) and the
framework's calls.  ``exact`` states the same definitions in 64 bits.
"""
import math

import torch

own = False

EPS = 1e-5
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "bf16": 2}


# --------------------------------------------------------------------------------------------- the cases
def listed():
    return [
        # one token of one request while answering: the block's norm feeding an 8-bit product
        dict(name="norm_token_fp8", op="norm", do="fp8", T=1, D=4096, dtype="bf16", group=0, residual=True),
        # a long prompt, 8-bit output with one scale per 128 columns
        dict(name="norm_prompt_fp8", op="norm", do="fp8", T=8192, D=8192, dtype="bf16", group=128, residual=True),
        # a training step's norm, forward and backward
        dict(name="norm_train", op="norm", do="train", T=8192, D=4096, dtype="bf16", group=0, residual=True),
        # the same in fp32 at a ragged batch and a width that is no multiple of a vector, first norm (no residual)
        dict(name="norm_train_ragged", op="norm", do="train", T=1531, D=2050, dtype="f32", group=0, residual=False),
        # a few answer tokens (fine-tuning on short answers): the head's weight is the whole cost
        dict(name="head_few_train", op="head", do="train", T=24, V=32768, D=1024, dtype="bf16", ignored=0.0),
        # evaluation: loss only, a vocabulary that is no multiple of anything, prompt tokens left out
        dict(name="head_eval", op="head", do="fwd", T=2048, V=50257, D=2048, dtype="bf16", ignored=0.3),
        # fp32 training at ragged sizes
        dict(name="head_train_f32", op="head", do="train", T=1021, V=32003, D=1000, dtype="f32", ignored=0.1),
        # a large model's training step on one GPU
        dict(name="head_train_large", op="head", do="train", T=4096, V=131072, D=4096, dtype="bf16", ignored=0.05),
        # a few tokens against a teacher's short list
        dict(name="distill_few", op="distill", do="step", T=8, V=32768, K=16, dtype="bf16", tau=2.0),
        # a training step: loss and gradient of a batch
        dict(name="distill_train", op="distill", do="step", T=4096, V=131072, K=64, dtype="bf16", tau=2.0),
        # evaluation in fp32, odd vocabulary
        dict(name="distill_eval_odd", op="distill", do="fwd", T=2047, V=50257, K=33, dtype="f32", tau=1.0),
        # the gradient alone, the loss's weight known only later; odd vocabulary, so rows start anywhere
        dict(name="distill_bwd_odd", op="distill", do="bwd", T=1024, V=65537, K=128, dtype="bf16", tau=4.0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "head", "distill"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op == "norm":
        T, D = _log(rng, 1, 8192), _log(rng, 64, 8192)
        if rng.random() < 0.5:      # whole 16-byte vectors
            D = max(80, D // 40 * 40)
        do = rng.choice(["fwd", "fp8", "train"])
        return dict(op=op, do=do, T=T, D=D, dtype=dtype, group=rng.choice([0, 128]) if do == "fp8" else 0,
                    residual=rng.random() < 0.8)
    if op == "head":
        T, V, D = _log(rng, 1, 4096), _log(rng, 1000, 131072), _log(rng, 64, 4096)
        if rng.random() < 0.7:
            D = max(80, D // 40 * 40)
        return dict(op=op, do=rng.choice(["fwd", "train"]), T=T, V=V, D=D, dtype=dtype,
                    ignored=rng.choice([0.0, 0.1, 0.5]))
    T, V = _log(rng, 1, 4096), _log(rng, 1000, 131072)
    if rng.random() < 0.5:
        V = max(1000, V // 64 * 64)
    if dtype == "f32":
        T = max(1, T // 2)
    return dict(op=op, do=rng.choice(["fwd", "bwd", "step"]), T=T, V=V, K=_log(rng, 1, 256), dtype=dtype,
                tau=rng.choice([1.0, 2.0, 4.0]))


# --------------------------------------------------------------------------------------------- inputs
def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, device="cuda", generator=gen)

    def uniform(*shape):
        return torch.rand(*shape, device="cuda", generator=gen)

    return {"case": case, **{"norm": _prepare_norm, "head": _prepare_head, "distill": _prepare_distill}[case["op"]](
        case, normal, uniform)}


def _prepare_norm(case, normal, uniform):
    T, D, dtype = case["T"], case["D"], DTYPES[case["dtype"]]
    # a block's output joins a residual stream that has grown over the layers and has a few large columns
    stream = normal(T, D) * (1.0 + 20.0 * (uniform(D) > 0.995)) * 2.0
    state = {"x": normal(T, D).to(dtype), "residual": stream.to(dtype) if case["residual"] else None,
             "weight": 1.0 + 0.2 * normal(D)}
    if not case["residual"]:
        state["x"] = stream.to(dtype)
    if case["do"] == "train":
        state["dy"] = (normal(T, D) * 1e-2).to(dtype)
        state["dh"] = (normal(T, D) * 1e-2).to(dtype)
    return state


def _prepare_head(case, normal, uniform):
    T, V, D, dtype = case["T"], case["V"], case["D"], DTYPES[case["dtype"]]
    w = normal(V, D) * 0.02
    target = (uniform(T) * V).long().clamp_(max=V - 1)
    # a trained model's hidden rows lean towards their target's row, some strongly
    lean = uniform(T, 1) * (12.0 / (0.02 * D))
    x = normal(T, D) * min(1.0, 64.0 / math.sqrt(D)) + lean * (w[target] / 0.02)
    left_out = uniform(T) < case["ignored"]
    target = torch.where(left_out, torch.full_like(target, -100), target)
    state = {"x": x.to(dtype), "w": w.to(dtype), "target": target}
    if case["do"] == "train":   # the mean over the tokens that count
        state["dloss"] = (target >= 0).float() / (target >= 0).sum().clamp(min=1)
    return state


def _prepare_distill(case, normal, uniform):
    T, V, K, dtype = case["T"], case["V"], case["K"], DTYPES[case["dtype"]]
    z = normal(T, V) * 2.0
    # K distinct places a row, spread over the vocabulary; the student agrees with the teacher in part
    base = (uniform(T, 1) * V).long()
    step = 1 + (uniform(T, 1) * (V // K - 1)).long()
    index = (base + step * torch.arange(K, device="cuda")) % V
    teacher = torch.sort(normal(T, K) * 3.0 + 8.0, dim=1, descending=True).values
    z.scatter_add_(1, index, teacher * uniform(T, K))
    # lists of different lengths; now and then a token without any
    length = torch.where(uniform(T) < 0.1, (uniform(T) * (K + 1)).long(), torch.full((T,), K, device="cuda"))
    index = torch.where(torch.arange(K, device="cuda") < length[:, None], index, torch.full_like(index, -1)).int()
    state = {"z": z.to(dtype), "teacher": teacher, "index": index, "dloss": uniform(T) / T}
    if case["do"] == "bwd":     # what the forward call left
        state["lse"] = torch.logsumexp(state["z"].float() / case["tau"], dim=1)
    return state


# --------------------------------------------------------------------------------------------- one pass
def run(state):
    case = state["case"]
    if own:
        return {"norm": _own_norm, "head": _own_head, "distill": _own_distill}[case["op"]](case, state)
    return {"norm": _plain_norm, "head": _plain_head, "distill": _plain_distill}[case["op"]](case, state)


def _own_norm(case, state):
    from paper_1810_10962_b200 import lm
    x, residual, weight = state["x"], state["residual"], state["weight"]
    if case["do"] == "fp8":
        q, scales, h, rstd = lm.rms_norm_forward_fp8(x, residual, weight, EPS, group=case["group"])
        return {"q": q, "scales": scales, "h": h, "rstd": rstd}
    y, h, rstd = lm.rms_norm_forward(x, residual, weight, EPS)
    if case["do"] == "fwd":
        return {"y": y, "h": h, "rstd": rstd}
    dx, dweight = lm.rms_norm_backward(state["dy"], h, weight, rstd, dh=state["dh"])
    return {"y": y, "h": h, "rstd": rstd, "dx": dx, "dweight": dweight}


def _plain_norm(case, state):
    x, residual, weight = state["x"], state["residual"], state["weight"]
    s = x.float() if residual is None else x.float() + residual.float()
    h = s.to(x.dtype)
    rstd = torch.rsqrt((s * s).mean(dim=1) + EPS)
    y = s * rstd[:, None] * weight
    if case["do"] == "fp8":
        T, D = s.shape
        group = case["group"] or D
        groups = -(-D // group)
        parts = torch.nn.functional.pad(y, (0, groups * group - D)).view(T, groups, group)
        amax = parts.abs().amax(dim=2)
        scales = torch.where(amax > 0, amax / 448.0, torch.ones_like(amax))
        q = (parts / scales[:, :, None]).view(T, groups * group)[:, :D].to(torch.float8_e4m3fn)
        return {"q": q, "scales": scales, "h": h, "rstd": rstd}
    out = {"y": y.to(x.dtype), "h": h, "rstd": rstd}
    if case["do"] == "train":
        dy, xhat = state["dy"].float(), h.float() * rstd[:, None]
        wdy = dy * weight
        c = (wdy * xhat).mean(dim=1, keepdim=True)
        out["dx"] = (rstd[:, None] * (wdy - xhat * c) + state["dh"].float()).to(x.dtype)
        out["dweight"] = (dy * xhat).sum(dim=0)
    return out


def _own_head(case, state):
    from paper_1810_10962_b200 import lm
    x, w, target = state["x"], state["w"], state["target"]
    loss, lse = lm.linear_cross_entropy_forward(x, w, target)
    if case["do"] == "fwd":
        return {"loss": loss, "lse": lse}
    dx, dw = lm.linear_cross_entropy_backward(x, w, target, lse, state["dloss"])
    return {"loss": loss, "lse": lse, "dx": dx, "dw": dw}


def _plain_head(case, state):
    x, w, target = state["x"].float(), state["w"].float(), state["target"]
    z = x @ w.T
    top = z.amax(dim=1, keepdim=True)
    lse = top[:, 0] + torch.log(torch.exp(z - top).sum(dim=1))
    counts = target >= 0
    at = target.clamp(min=0)[:, None]
    loss = torch.where(counts, lse - z.gather(1, at)[:, 0], torch.zeros_like(lse))
    if case["do"] == "fwd":
        return {"loss": loss, "lse": lse}
    g = (state["dloss"] * counts)[:, None]
    G = torch.exp(z - lse[:, None]) * g
    G.scatter_add_(1, at, -g)
    return {"loss": loss, "lse": lse, "dx": (G @ w).to(state["x"].dtype), "dw": (G.T @ x).to(state["w"].dtype)}


def _own_distill(case, state):
    from paper_1810_10962_b200 import lm
    z, teacher, index, tau = state["z"], state["teacher"], state["index"], case["tau"]
    if case["do"] == "fwd":
        loss, lse = lm.topk_distillation_forward(z, teacher, index, tau)
        return {"loss": loss, "lse": lse}
    if case["do"] == "bwd":
        return {"dz": lm.topk_distillation_backward(z, teacher, index, state["lse"], state["dloss"], tau)}
    loss, dz = lm.topk_distillation_step(z, teacher, index, state["dloss"], tau)
    return {"loss": loss, "dz": dz}


def _plain_distill(case, state):
    tau, z = case["tau"], state["z"].float() / case["tau"]
    there = state["index"] >= 0
    any_there = there.any(dim=1)
    at = state["index"].clamp(min=0).long()
    a = torch.where(there, state["teacher"] / tau, torch.full_like(state["teacher"], -math.inf))
    a = a - torch.where(any_there, a.amax(dim=1), torch.zeros_like(a[:, 0]))[:, None]
    e = torch.exp(a)
    total = torch.where(any_there, e.sum(dim=1), torch.ones_like(e[:, 0]))[:, None]
    p = e / total
    out = {}
    if case["do"] == "bwd":
        lse = state["lse"]
    else:
        top = z.amax(dim=1)
        lse = top + torch.log(torch.exp(z - top[:, None]).sum(dim=1))
        terms = p * ((a - torch.log(total)) - (z.gather(1, at) - lse[:, None]))
        out["loss"] = tau * tau * torch.where(there, terms, torch.zeros_like(terms)).sum(dim=1)
        if case["do"] == "fwd":
            return {"loss": out["loss"], "lse": lse}
    g = (state["dloss"] * tau * any_there)[:, None]
    dz = torch.exp(z - lse[:, None]) * g
    dz.scatter_add_(1, at, -g * p)
    out["dz"] = dz.to(state["z"].dtype)
    return out


# --------------------------------------------------------------------------------------------- what it cannot do without
def work(case):
    b = BYTES[case["dtype"]]
    T = case["T"]
    if case["op"] == "norm":
        D = case["D"]
        read = T * D * b * (2 if case["residual"] else 1) + 4 * D
        write = T * D * b + 4 * T                              # h, rstd
        if case["do"] == "fp8":
            write += T * D + 4 * T * (-(-D // case["group"]) if case["group"] else 1)
        else:
            write += T * D * b
        flops = 6 * T * D
        if case["do"] == "train":                              # dy and dh; h may still be on the chip
            read, write, flops = read + 2 * T * D * b, write + T * D * b + 4 * D, flops + 9 * T * D
        return {"bytes": read + write, "flops": flops}
    V = case["V"]
    if case["op"] == "head":
        D = case["D"]
        bytes_, flops = (T + V) * D * b + 16 * T, 2 * T * V * D
        if case["do"] == "train":                              # gradients out; the logits' second product is not counted
            bytes_, flops = bytes_ + (T + V) * D * b + 4 * T, flops + 4 * T * V * D
        return {"bytes": bytes_, "flops": flops}
    bytes_, flops = T * V * b + T * case["K"] * 8 + 8 * T, 4 * T * V
    if case["do"] != "fwd":
        bytes_ += T * V * b
    return {"bytes": bytes_, "flops": flops}


# --------------------------------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    state = prepare(case, seed)
    return {"norm": _exact_norm, "head": _exact_head, "distill": _exact_distill}[case["op"]](case, state)


def _e4m3(v):
    """The nearest value with three bits of fraction, exponents from -6 up, ties to even."""
    _, exponent = torch.frexp(v)
    quantum = torch.ldexp(torch.ones_like(v), (exponent - 1).clamp(min=-6) - 3)
    return torch.round(v / quantum) * quantum


def _exact_norm(case, state):
    h = state["x"].double()
    if state["residual"] is not None:
        h = h + state["residual"].double()
    weight = state["weight"].double()
    T, D = h.shape
    rstd = 1.0 / torch.sqrt(torch.einsum("td,td->t", h, h) / D + EPS)
    xhat = h * rstd.unsqueeze(1)
    y = xhat * weight
    if case["do"] == "fp8":
        group = case["group"] if case["group"] else D
        scales, q = [], torch.empty_like(y)
        for at in range(0, D, group):
            part = y[:, at:at + group]
            scale = part.abs().max(dim=1).values / 448.0
            scale[scale == 0] = 1.0
            scales.append(scale)
            q[:, at:at + group] = _e4m3(part / scale.unsqueeze(1))
        return {"q": q, "scales": torch.stack(scales, dim=1), "h": h, "rstd": rstd}
    out = {"y": y, "h": h, "rstd": rstd}
    if case["do"] == "train":
        dxhat = state["dy"].double() * weight
        inner = torch.einsum("td,td->t", dxhat, xhat) / D
        out["dx"] = rstd.unsqueeze(1) * (dxhat - inner.unsqueeze(1) * xhat) + state["dh"].double()
        out["dweight"] = torch.einsum("td,td->d", state["dy"].double(), xhat)
    return out


def _exact_head(case, state):
    x, w, target = state["x"].double(), state["w"].double(), state["target"]
    rows = torch.nonzero(target >= 0)[:, 0]
    z = torch.matmul(x, w.transpose(0, 1))
    lse = torch.logsumexp(z, dim=1)
    loss = torch.zeros_like(lse)
    loss[rows] = lse[rows] - z[rows, target[rows]]
    if case["do"] == "fwd":
        return {"loss": loss, "lse": lse}
    q = torch.exp(z.sub_(lse.unsqueeze(1)))
    q[rows, target[rows]] -= 1.0
    weight = torch.zeros_like(lse)
    weight[rows] = state["dloss"].double()[rows]
    q.mul_(weight.unsqueeze(1))
    return {"loss": loss, "lse": lse, "dx": torch.matmul(q, w), "dw": torch.matmul(q.transpose(0, 1), x)}


def _exact_distill(case, state):
    tau = case["tau"]
    z = state["z"].double().div_(tau)
    T, V = z.shape
    there = state["index"] >= 0
    lse = torch.logsumexp(z, dim=1)
    logp = (state["teacher"].double() / tau).masked_fill(~there, -math.inf)
    logp = torch.where(there, logp - torch.logsumexp(logp, dim=1, keepdim=True), torch.full_like(logp, -math.inf))
    p = torch.exp(logp)
    at = torch.where(there, state["index"], torch.zeros_like(state["index"])).long()
    if case["do"] != "bwd":
        logq = torch.gather(z, 1, at) - lse.unsqueeze(1)
        loss = tau ** 2 * torch.where(there & (p > 0), p * (logp - logq), torch.zeros_like(p)).sum(dim=1)
        if case["do"] == "fwd":
            return {"loss": loss, "lse": lse}
    q = z.sub_(lse.unsqueeze(1)).exp_()
    q.scatter_add_(1, at, -p)
    q[~there.any(dim=1)] = 0.0
    dz = q.mul_((state["dloss"].double() * tau).unsqueeze(1))
    return {"dz": dz} if case["do"] == "bwd" else {"loss": loss, "dz": dz}
