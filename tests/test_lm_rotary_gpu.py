"""Norm + rotation of queries' and keys' heads, and its gradient, against the definition in 64 bits.

u = 2^-24 is fp32's rounding.  A lane adds up at most 32 squares of a head in a row and five joins follow; a gradient of a
weight is a sum over positions and heads whose longest chain of additions is some 200 at these sizes."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
STORE = {torch.float32: U, torch.bfloat16: 2.0 ** -8}
TYPES = [torch.bfloat16, torch.float32]
EPS = 1e-6


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def tables(P, R):
    angle = torch.arange(P, device="cuda", dtype=torch.float64)[:, None] * 100.0 ** (-torch.arange(0, R, 2, device="cuda", dtype=torch.float64) / R)
    return torch.cos(angle).float(), torch.sin(angle).float()


def case(B, S, Hq, Hk, D, R, dtype, seed, order="dense", P=50):
    g = gen(seed)
    randn = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    if order == "packed":
        qkv = (randn(B, S, Hq + 2 * Hk, D) * 2).to(dtype)
        q, k = qkv[:, :, :Hq], qkv[:, :, Hq: Hq + Hk]
    elif order == "heads":
        q, k = ((randn(B, H, S, D) * 2).to(dtype).transpose(1, 2) for H in (Hq, Hk))
    elif order == "odd":            # addresses and strides that are multiples of nothing
        room = (randn(B, S, Hq + Hk, D + 3) * 2).to(dtype)
        q, k = room[:, :, :Hq, 1: D + 1], room[:, :, Hq:, 2: D + 2]
    else:
        q, k = (randn(B, S, Hq, D) * 2).to(dtype), (randn(B, S, Hk, D) * 2).to(dtype)
    cos, sin = tables(P, R)
    position = torch.randint(0, P, (B, S), device="cuda", generator=g)
    weights = 1 + 0.3 * randn(D), 1 + 0.3 * randn(D)
    grads = randn(B, S, Hq, D).to(dtype), randn(B, S, Hk, D).to(dtype)
    return q, k, *weights, cos, sin, position, grads


def pairs(x, R, interleaved):
    return (x[..., 0:R:2], x[..., 1:R:2]) if interleaved else (x[..., : R // 2], x[..., R // 2: R])


def turned(x, c, s, R, interleaved):
    y = x.clone()
    a, b = pairs(x, R, interleaved)
    ya, yb = pairs(y, R, interleaved)
    ya.copy_(a * c - b * s)
    yb.copy_(b * c + a * s)
    return y


def reference(x, w, cos, sin, position, dy, interleaved):
    """(y, dx, dw) and what their terms add up to in magnitude."""
    R, D = 2 * cos.shape[1], x.shape[-1]
    there = ((position >= 0) & (position < cos.shape[0]))[:, :, None, None]
    at = position.clamp(0, cos.shape[0] - 1)
    c, s = cos.double()[at][:, :, None], sin.double()[at][:, :, None]
    x, w, dy = torch.where(there, x.double(), torch.ones_like(x, dtype=torch.float64)), w.double(), torch.where(there, dy.double(), 0.0)
    rstd = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS)
    n = x * rstd
    y = torch.where(there, turned(n * w, c, s, R, interleaved), 0.0)
    y_size = torch.where(there, turned((n * w).abs(), c.abs(), -s.abs(), R, interleaved).abs() + turned((n * w).abs(), c.abs(), s.abs(), R, interleaved).abs(), 0.0)
    d = turned(dy, c, -s, R, interleaved)
    d_size = turned(dy.abs(), c.abs(), -s.abs(), R, interleaved).abs() + turned(dy.abs(), c.abs(), s.abs(), R, interleaved).abs()
    wd, wd_size = w * d, w.abs() * d_size
    dx = rstd * (wd - n * (wd * n).mean(-1, keepdim=True))
    dx_size = rstd * (wd_size + n.abs() * (wd_size * n.abs()).mean(-1, keepdim=True))
    return (y, dx, (d * n).sum((0, 1, 2))), (y_size, dx_size, (d_size * n.abs()).sum((0, 1, 2)))


def within(got, want, tol, what):
    off = (got.double() - want).abs()
    bad = ~(off <= tol)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {float((off / tol).nan_to_num(math.inf).max()):.3g} times the bound"


def check(q, k, qw, kw, cos, sin, position, grads, interleaved):
    from paper_1810_10962_b200 import lm
    rest = (q, k, qw, kw, cos, sin, position, EPS, interleaved)
    outs = lm.head_norm_rotary_forward(*rest)
    dq, dk, dqw, dkw = lm.head_norm_rotary_backward(*grads, *rest)
    for x, w, y, dy, dx, dw, name in ((q, qw, outs[0], grads[0], dq, dqw, "q"), (k, kw, outs[1], grads[1], dk, dkw, "k")):
        (want_y, want_dx, want_dw), (y_size, dx_size, dw_size) = reference(x, w, cos, sin, position, dy, interleaved)
        assert y.is_contiguous() and y.shape == x.shape and y.dtype == x.dtype
        within(y, want_y, 32 * U * y_size + STORE[x.dtype] * want_y.abs() + 1e-38, name)
        within(dx, want_dx, 96 * U * dx_size + STORE[x.dtype] * want_dx.abs() + 1e-38, "d" + name)
        within(dw, want_dw, 200 * U * dw_size + 1e-38, f"d{name}_weight")


# every vector width and both numbers of vectors a lane holds; rests that end within a pair; one head, many heads
SHAPES = [(1, 1, 1, 1, 2, 2), (1, 3, 2, 1, 5, 4), (2, 7, 3, 2, 33, 16), (1, 64, 4, 4, 64, 64), (2, 33, 8, 2, 72, 72), (2, 33, 6, 3, 72, 36),
          (3, 17, 12, 12, 80, 32), (1, 100, 5, 1, 96, 96), (2, 60, 32, 8, 128, 128), (1, 9, 40, 40, 128, 64), (1, 31, 7, 1, 192, 128),
          (2, 20, 4, 2, 250, 100), (1, 40, 16, 1, 256, 256), (1, 5, 3, 2, 576, 64), (1, 6, 2, 1, 1024, 1024), (1, 3, 1, 1, 1023, 1022), (1, 4, 2, 2, 1020, 8)]


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,S,Hq,Hk,D,R", SHAPES)
def test_norm_and_rotation(B, S, Hq, Hk, D, R, dtype, interleaved):
    check(*case(B, S, Hq, Hk, D, R, dtype, 3 + D + S), interleaved)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("order", ["packed", "heads", "odd"])
@pytest.mark.parametrize("B,S,Hq,Hk,D,R", [(2, 19, 8, 2, 128, 128), (3, 11, 5, 5, 80, 40), (1, 300, 3, 1, 66, 66)])
def test_orders_of_memory(B, S, Hq, Hk, D, R, order, dtype):
    check(*case(B, S, Hq, Hk, D, R, dtype, 5 + D, order), False)


def test_many_positions():
    """More positions than a launch of the gradient has warps for."""
    check(*case(2, 5000, 2, 1, 64, 64, torch.bfloat16, 9, P=5000), False)


def test_padding():
    """Positions outside the tables: zeros come out, whatever is there, and nothing reaches the weights' gradients."""
    from paper_1810_10962_b200 import lm
    for dtype in TYPES:
        q, k, qw, kw, cos, sin, position, grads = case(2, 21, 4, 2, 64, 32, dtype, 11)
        for at, p in (((0, 3), -1), ((1, 20), -100), ((1, 0), cos.shape[0]), ((0, 20), 2 ** 40)):
            position[at] = p
            q[at] = math.nan
            grads[0][at] = math.inf
        outs = lm.head_norm_rotary_forward(q, k, qw, kw, cos, sin, position, EPS)
        dq, dk, dqw, dkw = lm.head_norm_rotary_backward(*grads, q, k, qw, kw, cos, sin, position, EPS)
        for t in (*outs, dq, dk):
            assert bool((t[0, 3] == 0).all()) and bool((t[1, 20] == 0).all()) and bool((t[1, 0] == 0).all()) and bool(t.isfinite().all())
        assert bool(dqw.isfinite().all())
        check(q, k, qw, kw, cos, sin, position, grads, False)
        narrow = position.clamp(-1, 1000).int()
        for a, b in zip(lm.head_norm_rotary_forward(q, k, qw, kw, cos, sin, narrow, EPS), outs):
            assert torch.equal(a, b)


def test_queries_alone_and_three_dimensions():
    from paper_1810_10962_b200 import lm
    q, k, qw, kw, cos, sin, position, grads = case(1, 30, 6, 2, 96, 48, torch.float32, 13)
    both = lm.head_norm_rotary_forward(q, k, qw, kw, cos, sin, position, EPS)
    alone, none = lm.head_norm_rotary_forward(q[0], None, qw, None, cos, sin, position[0], EPS)
    assert none is None and torch.equal(alone, both[0][0])
    dq, dk, dqw, dkw = lm.head_norm_rotary_backward(grads[0][0], None, q[0], None, qw, None, cos, sin, position[0], EPS)
    assert dk is None and dkw is None
    within(dqw, reference(q, qw, cos, sin, position, grads[0], False)[0][2], 200 * U * reference(q, qw, cos, sin, position, grads[0], False)[1][2], "dq_weight")


def test_keys_without_heads():
    from paper_1810_10962_b200 import lm
    q, k, qw, kw, cos, sin, position, grads = case(2, 5, 3, 1, 64, 64, torch.bfloat16, 14)
    none = k[:, :, :0]
    torch.full((64,), 7.0, device="cuda")                    # what a new tensor would find
    outs = lm.head_norm_rotary_forward(q, none, qw, kw, cos, sin, position, EPS)
    assert outs[1].shape == (2, 5, 0, 64) and torch.equal(outs[0], lm.head_norm_rotary_forward(q, None, qw, None, cos, sin, position, EPS)[0])
    got = lm.head_norm_rotary_backward(grads[0], outs[1], q, none, qw, kw, cos, sin, position, EPS)
    assert bool((got[3] == 0).all()) and torch.equal(got[0], lm.head_norm_rotary_backward(grads[0], None, q, None, qw, None, cos, sin, position, EPS)[0])


def test_heads_of_zeros_and_of_large_values():
    q, k, qw, kw, cos, sin, position, grads = case(1, 4, 2, 2, 64, 64, torch.float32, 15)
    q[0, 0] = 0
    q[0, 1] *= 1e15
    k[0, 2] *= 1e-12
    check(q, k, qw, kw, cos, sin, position, grads, False)


def test_broadcast_inputs():
    """Heads that are one head seen several times: the strides say so, the gradients are of each."""
    q, k, qw, kw, cos, sin, position, grads = case(2, 9, 4, 1, 64, 64, torch.bfloat16, 17)
    check(q, k.expand(2, 9, 4, 64), qw, kw, cos, sin, position, (grads[0], grads[0]), False)


def test_without_positions():
    from paper_1810_10962_b200 import lm
    q, k, qw, kw, cos, sin, position, grads = case(2, 9, 4, 1, 64, 64, torch.bfloat16, 19)
    none = lambda t: t[:, :0]  # noqa: E731
    outs = lm.head_norm_rotary_forward(none(q), none(k), qw, kw, cos, sin, none(position).contiguous(), EPS)
    assert outs[0].shape == (2, 0, 4, 64)
    got = lm.head_norm_rotary_backward(*outs, none(q), none(k), qw, kw, cos, sin, none(position).contiguous(), EPS)
    assert bool((got[2] == 0).all()) and bool((got[3] == 0).all())


@pytest.mark.parametrize("interleaved", [False, True])
def test_gradient_against_differences(interleaved):
    from paper_1810_10962_b200 import lm
    q, k, qw, kw, cos, sin, position, grads = case(1, 5, 2, 1, 32, 16, torch.float32, 21)
    step = 2.0 ** -6

    def value(q, k, qw, kw):
        outs = lm.head_norm_rotary_forward(q, k, qw, kw, cos, sin, position, EPS, interleaved)
        return sum(float((o.double() * g.double()).sum()) for o, g in zip(outs, grads))

    got = lm.head_norm_rotary_backward(*grads, q, k, qw, kw, cos, sin, position, EPS, interleaved)
    inputs = [q, k, qw, kw]
    g = gen(23)
    for i, d in enumerate(got):
        e = torch.randn(inputs[i].shape, device="cuda", generator=g)
        e /= e.norm()
        moved = [[t + (sign * step * e if j == i else 0) for j, t in enumerate(inputs)] for sign in (1, -1)]
        want = (value(*moved[0]) - value(*moved[1])) / (2 * step)
        # 480 values of order 1: some 1e-5 in the sum; third derivatives along a unit direction are below 100
        assert abs(float((d.double() * e.double()).sum()) - want) < 1e-5 / step + 100 * step ** 2 / 6


def test_streams_graphs_and_the_same_bits():
    from paper_1810_10962_b200 import lm
    q, k, qw, kw, cos, sin, position, grads = case(2, 700, 8, 2, 128, 128, torch.bfloat16, 25, "packed")

    def all_of():
        rest = (q, k, qw, kw, cos, sin, position, EPS)
        return (*lm.head_norm_rotary_forward(*rest), *lm.head_norm_rotary_backward(*grads, *rest))

    want = all_of()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = all_of()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = all_of()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_past_32_bit_offsets():
    from paper_1810_10962_b200 import lm
    S, H, D = 140_000, 120, 128                              # 2.15e9 elements
    q = torch.ones(1, S, H, D, dtype=torch.bfloat16, device="cuda")
    tail, _, qw, _, cos, sin, position, grads = case(1, 5, H, 1, D, 64, torch.bfloat16, 27)
    q[:, -5:] = tail
    at = torch.cat([torch.zeros(1, S - 5, dtype=torch.int64, device="cuda"), position], 1)
    out, _ = lm.head_norm_rotary_forward(q, None, qw, None, cos, sin, at, EPS)
    assert torch.equal(out[:, -5:], lm.head_norm_rotary_forward(tail, None, qw, None, cos, sin, position, EPS)[0])
    dq = lm.head_norm_rotary_backward(out, None, q, None, qw, None, cos, sin, at, EPS)[0]
    assert torch.equal(dq[:, -5:], lm.head_norm_rotary_backward(out[:, -5:].contiguous(), None, tail, None, qw, None, cos, sin, position, EPS)[0])
