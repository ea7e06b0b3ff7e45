"""Cases of more language-model operators: what a training or serving program has in hand, and one pass.

Three operators, each in every direction a program calls it:

* ``logp``    log probabilities of given tokens with the distribution's entropy: forward, forward with the top
              alternatives, forward + backward;
* ``rotary``  root-mean-square norm of each head of queries and keys with the rotation by position in the same pass:
              forward, forward + backward;
* ``clip``    global norm over many gradients: the norm alone, the norm and the clipped gradients.

``own`` chooses between the plain form (elementary torch operations in 32 bits, rounded once at the end) and the
framework's calls.  ``exact`` states the same definitions in 64 bits.
"""
import math

import torch

own = False

EPS = 1e-6
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "bf16": 2}


# --------------------------------------------------------------------------------------------- the cases
def listed():
    return [
        # one answer token of one request, with the 20 alternatives that a serving interface shows
        dict(name="logp_token_top", op="logp", do="top", T=1, V=131072, K=20, dtype="bf16", tau=1.0, allowed=1.0, ignored=0.0),
        # a serving batch under a grammar: most of the vocabulary masked with -inf
        dict(name="logp_masked_top", op="logp", do="top", T=64, V=50257, K=5, dtype="f32", tau=0.7, allowed=0.01, ignored=0.0),
        # a prompt's tokens scored, odd vocabulary, so rows start anywhere
        dict(name="logp_prompt_top", op="logp", do="top", T=2047, V=50257, K=10, dtype="bf16", tau=1.0, allowed=1.0,
             ignored=0.0),
        # a policy-gradient step of a large model: log probability and entropy of the batch, and the logits' gradient
        dict(name="logp_train", op="logp", do="train", T=4096, V=131072, K=0, dtype="bf16", tau=1.0, allowed=1.0, ignored=0.3),
        # the same in fp32 at ragged sizes, sampled at a temperature
        dict(name="logp_train_odd", op="logp", do="train", T=509, V=32003, K=0, dtype="f32", tau=1.3, allowed=1.0,
             ignored=0.1),
        # one answer token: its heads out of the packed projection
        dict(name="rotary_token", op="rotary", do="fwd", B=1, S=1, Hq=32, Hk=8, D=128, R=128, dtype="bf16", pairs="halves",
             order="packed"),
        # a long prompt
        dict(name="rotary_prompt", op="rotary", do="fwd", B=1, S=8192, Hq=32, Hk=8, D=128, R=128, dtype="bf16", pairs="halves",
             order="packed"),
        # a training step, forward and backward
        dict(name="rotary_train", op="rotary", do="train", B=4, S=4096, Hq=32, Hk=8, D=128, R=128, dtype="bf16",
             pairs="halves", order="packed"),
        # fp32, part of a narrow head turned, neighbouring elements paired, heads before positions in memory, ragged lengths
        dict(name="rotary_train_odd", op="rotary", do="train", B=3, S=517, Hq=12, Hk=12, D=80, R=32, dtype="f32",
             pairs="neighbours", order="heads"),
        # the gradients of a small adapter: a few dozen matrices, launch latency is the cost
        dict(name="clip_adapter", op="clip", do="clip", layers=12, D=1024, F=16, V=0, dtype="bf16", above=True),
        # a small model in fp32, odd widths, gradients below the limit
        dict(name="clip_small", op="clip", do="clip", layers=12, D=750, F=2050, V=50257, dtype="f32", above=False),
        # a large model's gradients, matrices in bf16 and norms' weights in fp32
        dict(name="clip_large", op="clip", do="clip", layers=8, D=4096, F=14336, V=32768, dtype="bf16", above=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["logp", "rotary", "clip"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op == "logp":
        do = rng.choice(["fwd", "top", "top", "train"])
        T, V = _log(rng, 1, 4096), _log(rng, 1000, 131072)
        if rng.random() < 0.5:      # whole 16-byte vectors
            V = max(1000, V // 64 * 64)
        if dtype == "f32":
            T = max(1, T // 2)
        if do == "top":             # the plain form sorts
            T = max(1, min(T, (2047 * 50257) // V))
        return dict(op=op, do=do, T=T, V=V, K=_log(rng, 1, 64) if do == "top" else 0, dtype=dtype,
                    tau=rng.choice([0.7, 1.0, 1.3]), allowed=rng.choice([1.0, 1.0, 0.1]), ignored=rng.choice([0.0, 0.3]))
    if op == "rotary":
        D = rng.choice([32, 64, 72, 80, 96, 128, 128, 128, 192, 256])
        Hk = rng.choice([1, 2, 4, 8, 12])
        Hq = Hk * rng.choice([1, 2, 4])
        B = rng.choice([1, 1, 2, 3, 8])
        most = 16384 * 40 * 128 // ((Hq + Hk) * D * B)
        S = min(_log(rng, 1, 16384), most) if dtype == "bf16" else min(_log(rng, 1, 16384), most // 2)
        return dict(op=op, do=rng.choice(["fwd", "train"]), B=B, S=max(1, S), Hq=Hq, Hk=Hk, D=D,
                    R=rng.choice([D, D, D // 8 * 4]), dtype=dtype, pairs=rng.choice(["halves", "halves", "neighbours"]),
                    order=rng.choice(["packed", "dense", "heads"]))
    D = _log(rng, 64, 4096)
    if rng.random() < 0.7:
        D = max(64, D // 64 * 64)
    adapter = rng.random() < 0.3
    return dict(op=op, do=rng.choice(["norm", "clip", "clip"]), layers=_log(rng, 1, 24) if D <= 2048 else _log(rng, 1, 6), D=D,
                F=_log(rng, 4, 64) if adapter else _log(rng, D, 3 * D), V=0 if adapter else _log(rng, 1000, 50000),
                dtype=dtype, above=rng.random() < 0.7)


# --------------------------------------------------------------------------------------------- inputs
def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, device="cuda", generator=gen)

    def uniform(*shape):
        return torch.rand(*shape, device="cuda", generator=gen)

    return {"case": case, **{"logp": _prepare_logp, "rotary": _prepare_rotary, "clip": _prepare_clip}[case["op"]](
        case, normal, uniform)}


def _prepare_logp(case, normal, uniform):
    T, V, dtype = case["T"], case["V"], DTYPES[case["dtype"]]
    z = normal(T, V).mul_(2.0)
    token = (uniform(T) * V).long().clamp_(max=V - 1)
    # some places of each row stand out, the given token often among them
    places = (uniform(T, 8) * V).long().clamp_(max=V - 1)
    token = torch.where(uniform(T) < 0.7, places[:, 0], token)
    z.scatter_add_(1, places, 6.0 + 3.0 * normal(T, 8))
    if case["allowed"] < 1.0:       # masked places, never fewer than the alternatives asked for
        keep = uniform(T, V) < case["allowed"]
        keep.scatter_(1, token[:, None], True)
        keep[:, : case["K"]] = True
        z.masked_fill_(~keep, -math.inf)
    token = torch.where(uniform(T) < case["ignored"], torch.full_like(token, -100), token)
    state = {"z": z.to(dtype), "token": token}
    if case["do"] == "train":       # advantages of either sign, an entropy bonus
        state["dlogp"], state["dentropy"] = -normal(T) / T, torch.full((T,), -0.01 / T, device="cuda")
    return state


def _prepare_rotary(case, normal, uniform):
    B, S, Hq, Hk, D, R, dtype = (case[k] for k in ("B", "S", "Hq", "Hk", "D", "R", "dtype"))
    dtype = DTYPES[dtype]
    spread = 1.0 + 10.0 * (uniform(D) > 0.97)       # a few large columns
    if case["order"] == "packed":                   # queries, keys and values of one projection
        qkv = (normal(B, S, Hq + 2 * Hk, D) * spread).to(dtype)
        q, k = qkv[:, :, :Hq], qkv[:, :, Hq: Hq + Hk]
    elif case["order"] == "dense":
        q, k = (normal(B, S, Hq, D) * spread).to(dtype), (normal(B, S, Hk, D) * spread).to(dtype)
    else:                                           # heads before positions
        q, k = ((normal(B, H, S, D) * spread).to(dtype).transpose(1, 2) for H in (Hq, Hk))
    # documents one after another: positions start again at a place of each row's own; the tables are the program's, made once
    table = max(2 * S, 64)
    start = (uniform(B, 1) * (table - S)).long()
    position = start + torch.arange(S, device="cuda")
    angle = torch.arange(table, device="cuda", dtype=torch.float64)[:, None] * 10000.0 ** (
        -torch.arange(0, R, 2, device="cuda", dtype=torch.float64) / R)
    state = {"q": q, "k": k, "q_weight": 1.0 + 0.2 * normal(D), "k_weight": 1.0 + 0.2 * normal(D), "position": position,
             "cos": torch.cos(angle).float(), "sin": torch.sin(angle).float()}
    if case["do"] == "train":
        state["dq"], state["dk"] = (normal(B, S, Hq, D) * 1e-2).to(dtype), (normal(B, S, Hk, D) * 1e-2).to(dtype)
    return state


def _sizes(case):
    """(elements, fp32 whatever the case's type) of every gradient: a layer's two norms and its matrices, the embedding."""
    D, F = case["D"], case["F"]
    small = F < D and case["V"] == 0                # an adapter: F is its rank
    layer = [(D * F, False), (F * D, False)] * 2 if small else [
        (D, True), (D * D, False), (D * D // 2, False), (D * D, False), (D, True), (F * D, False), (F * D, False), (D * F, False)]
    return layer * case["layers"] + ([(case["V"] * D, False), (D, True)] if case["V"] else [])


def _prepare_clip(case, normal, uniform):
    sizes, dtype = _sizes(case), DTYPES[case["dtype"]]
    # gradients live in one buffer for each type, every tensor on a 128-byte boundary
    room = {}
    places = []
    for n, wide in sizes:
        kind = torch.float32 if wide else dtype
        places.append((kind, room.get(kind, 0), n))
        room[kind] = room.get(kind, 0) + -(-n // 64) * 64
    flat = {kind: torch.zeros(n, dtype=kind, device="cuda") for kind, n in room.items()}
    out = {kind: torch.zeros_like(f) for kind, f in flat.items()}
    grads, outs = ([buffers[kind][at: at + n] for kind, at, n in places] for buffers in (flat, out))
    scale = 0.1 + uniform(len(grads))
    total = sum(n for n, _ in sizes)
    level = 4.0 if case["above"] else 0.2           # the norm, about
    for i, g in enumerate(grads):
        part = normal(min(g.numel(), 1 << 24)).mul_(scale[i] * level / math.sqrt(total))
        for at in range(0, g.numel(), part.numel()):
            g[at: at + part.numel()].copy_(part[: g.numel() - at])
    state = {"grads": grads, "outs": outs, "flat": flat, "out": out, "max_norm": 1.0}
    if own:
        from paper_1810_10962_b200 import lm
        state["list"] = lm.GradientList(grads, outs)
    return state


# --------------------------------------------------------------------------------------------- one pass
def run(state):
    case = state["case"]
    if own:
        return {"logp": _own_logp, "rotary": _own_rotary, "clip": _own_clip}[case["op"]](case, state)
    return {"logp": _plain_logp, "rotary": _plain_rotary, "clip": _plain_clip}[case["op"]](case, state)


def _own_logp(case, state):
    from paper_1810_10962_b200 import lm
    z, token, tau = state["z"], state["token"], case["tau"]
    if case["do"] == "top":
        logp, entropy, lse, top, index = lm.token_log_probs_forward_top(z, token, case["K"], tau)
        return {"logp": logp, "entropy": entropy, "lse": lse, "top": top, "index": index}
    logp, entropy, lse = lm.token_log_probs_forward(z, token, tau)
    out = {"logp": logp, "entropy": entropy, "lse": lse}
    if case["do"] == "train":
        out["dz"] = lm.token_log_probs_backward(z, token, lse, entropy, state["dlogp"], state["dentropy"], tau)
    return out


def _plain_logp(case, state):
    tau, token = case["tau"], state["token"]
    z = state["z"].float() / tau
    most = z.amax(dim=1, keepdim=True)
    z = z - most
    p = torch.exp(z)
    total = p.sum(dim=1, keepdim=True)
    logs = torch.log(total)
    p = p / total
    z = z - logs                                    # log probabilities
    given = token >= 0
    at = token.clamp(min=0)[:, None]
    logp = torch.where(given, z.gather(1, at)[:, 0], torch.zeros_like(z[:, 0]))
    entropy = -torch.where(p > 0, p * z, torch.zeros_like(p)).sum(dim=1)
    out = {"logp": logp, "entropy": entropy, "lse": (most + logs)[:, 0]}
    if case["do"] == "top":
        index = torch.sort(state["z"].float(), dim=1, descending=True, stable=True).indices[:, : case["K"]]
        out["top"], out["index"] = z.gather(1, index), index.int()
    if case["do"] == "train":
        g = (state["dlogp"] * given)[:, None]
        dz = -p * (g + state["dentropy"][:, None] * torch.where(p > 0, z + entropy[:, None], torch.zeros_like(z)))
        dz.scatter_add_(1, at, g)
        out["dz"] = (dz / tau).to(state["z"].dtype)
    return out


def _own_rotary(case, state):
    from paper_1810_10962_b200 import lm
    rest = (state["q"], state["k"], state["q_weight"], state["k_weight"], state["cos"], state["sin"], state["position"], EPS)
    neighbours = case["pairs"] == "neighbours"
    q, k = lm.head_norm_rotary_forward(*rest, interleaved=neighbours)
    out = {"q": q, "k": k}
    if case["do"] == "train":
        out["dq"], out["dk"], out["dq_weight"], out["dk_weight"] = lm.head_norm_rotary_backward(
            state["dq"], state["dk"], *rest, interleaved=neighbours)
    return out


def _turn(x, cos, sin, R, neighbours):
    """The first R elements of every head turned, pair by pair."""
    out = x.clone()
    first, second = (slice(0, R, 2), slice(1, R, 2)) if neighbours else (slice(0, R // 2), slice(R // 2, R))
    a, b = x[..., first], x[..., second]
    out[..., first] = a * cos - b * sin
    out[..., second] = b * cos + a * sin
    return out


def _plain_rotary(case, state):
    R, neighbours = case["R"], case["pairs"] == "neighbours"
    cos, sin = state["cos"][state["position"]][:, :, None], state["sin"][state["position"]][:, :, None]
    out = {}
    for name in ("q", "k"):
        x, weight = state[name].float(), state[name + "_weight"]
        rstd = torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + EPS)
        xhat = x * rstd
        out[name] = _turn(xhat * weight, cos, sin, R, neighbours).to(state[name].dtype)
        if case["do"] == "train":
            dy = _turn(state["d" + name].float(), cos, -sin, R, neighbours)
            wdy = dy * weight
            c = (wdy * xhat).mean(dim=-1, keepdim=True)
            out["d" + name] = (rstd * (wdy - xhat * c)).to(state[name].dtype)
            out["d" + name + "_weight"] = (dy * xhat).sum(dim=2).sum(dim=1).sum(dim=0)
    return out


def _own_clip(case, state):
    if case["do"] == "norm":
        return {"norm": state["list"].norm()}
    return {"norm": state["list"].clip(state["max_norm"]), **{str(kind): o for kind, o in state["out"].items()}}


def _plain_clip(case, state):
    squares = [g.float().square().sum(dtype=torch.float64) for g in state["grads"]]
    norm = torch.sqrt(torch.stack(squares).sum()).float()
    if case["do"] == "norm":
        return {"norm": norm}
    factor = torch.where(norm <= state["max_norm"], torch.ones_like(norm), state["max_norm"] / norm)
    for g, o in zip(state["grads"], state["outs"]):
        o.copy_(g.float() * factor)
    return {"norm": norm, **{str(kind): o for kind, o in state["out"].items()}}


# --------------------------------------------------------------------------------------------- what it cannot do without
def work(case):
    b = BYTES[case["dtype"]]
    if case["op"] == "logp":
        T, V = case["T"], case["V"]
        bytes_, flops = T * V * b + 8 * T + 12 * T + 8 * T * case["K"], 6 * T * V
        if case["do"] == "train":                              # the logits may still be on the chip
            bytes_, flops = bytes_ + T * V * b + 8 * T, flops + 8 * T * V
        return {"bytes": bytes_, "flops": flops}
    if case["op"] == "rotary":
        D, R, tokens = case["D"], case["R"], case["B"] * case["S"]
        values = tokens * (case["Hq"] + case["Hk"]) * D
        shared = tokens * 8 + min(tokens, 2 * case["S"]) * R * 4 + 8 * D        # positions, the tables' rows, weights
        bytes_, flops = 2 * values * b + shared, 8 * values
        if case["do"] == "train":                              # incoming gradients read, gradients written
            bytes_, flops = bytes_ + 2 * values * b + 8 * D, flops + 14 * values
        return {"bytes": bytes_, "flops": flops}
    bytes_ = sum(n * (4 if wide else b) for n, wide in _sizes(case))
    values = sum(n for n, _ in _sizes(case))
    if case["do"] == "norm":
        return {"bytes": bytes_ + 4, "flops": 2 * values}
    return {"bytes": 2 * bytes_ + 4, "flops": 3 * values}


# --------------------------------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    state = prepare(case, seed)
    return {"logp": _exact_logp, "rotary": _exact_rotary, "clip": _exact_clip}[case["op"]](case, state)


def _exact_logp(case, state):
    tau, token, T = case["tau"], state["token"], case["T"]
    z = state["z"].double().div_(tau)
    lse = torch.logsumexp(z, dim=1)
    rows = torch.nonzero(token >= 0)[:, 0]
    logp = torch.zeros_like(lse)
    logp[rows] = z[rows, token[rows]] - lse[rows]
    out = {"logp": logp, "lse": lse}
    if case["do"] == "top":
        # the largest, the lowest place first among equals: places are taken one after another
        left = z.clone()
        index = torch.empty(T, case["K"], dtype=torch.int32, device=z.device)
        place = torch.arange(z.shape[1], device=z.device)
        for k in range(case["K"]):
            top = left.max(dim=1, keepdim=True).values
            at = torch.where(left == top, place, torch.full_like(place, z.shape[1])).min(dim=1, keepdim=True).values
            index[:, k] = at[:, 0].int()
            left.scatter_(1, at, -math.inf)
        del left
        out["index"] = index
        out["top"] = torch.gather(z, 1, index.long()) - lse.unsqueeze(1)
    logq = z.sub_(lse.unsqueeze(1))
    q = torch.exp(logq)
    logq.masked_fill_(q == 0, 0.0)
    out["entropy"] = -torch.einsum("tv,tv->t", q, logq)
    if case["do"] == "train":
        weight = torch.zeros_like(lse)
        weight[rows] = state["dlogp"].double()[rows]
        # of the entropy: -q (log q + H); of the log probability: 1 at the token, less q
        logq.add_(out["entropy"].unsqueeze(1)).mul_(state["dentropy"].double().unsqueeze(1)).add_(weight.unsqueeze(1))
        dz = logq.mul_(q).neg_()
        dz[rows, token[rows]] += weight[rows]
        out["dz"] = dz.div_(tau)
    return out


def _exact_rotary(case, state):
    D, R = case["D"], case["R"]
    position = state["position"]
    # the rotation as a complex product of the table's values
    turn = torch.complex(state["cos"].double(), state["sin"].double())[position].unsqueeze(2)
    order = torch.arange(R, device=position.device)
    order = order.view(R // 2, 2) if case["pairs"] == "neighbours" else order.view(2, R // 2).T
    out = {}

    def turned(x, by):
        y = x.clone()
        pair = torch.complex(x[..., order[:, 0]], x[..., order[:, 1]]) * by
        y[..., order[:, 0]], y[..., order[:, 1]] = pair.real, pair.imag
        return y

    for name in ("q", "k"):
        x, weight = state[name].double(), state[name + "_weight"].double()
        rstd = 1.0 / torch.sqrt(torch.einsum("bshd,bshd->bsh", x, x) / D + EPS).unsqueeze(-1)
        xhat = x * rstd
        out[name] = turned(xhat * weight, turn)
        if case["do"] == "train":
            dn = turned(state["d" + name].double(), turn.conj())
            inner = torch.einsum("bshd,bshd->bsh", dn * weight, xhat).unsqueeze(-1) / D
            out["d" + name] = rstd * (dn * weight - inner * xhat)
            out["d" + name + "_weight"] = torch.einsum("bshd,bshd->d", dn, xhat)
    return out


def _exact_clip(case, state):
    norm = math.sqrt(math.fsum(float(torch.linalg.vector_norm(g.double())) ** 2 for g in state["grads"]))
    out = {"norm": torch.tensor(norm, dtype=torch.float64, device="cuda")}
    if case["do"] == "clip":
        factor = min(1.0, state["max_norm"] / norm) if norm > 0 else 1.0
        out.update({str(kind): f.double() * factor for kind, f in state["flat"].items()})
    return out
