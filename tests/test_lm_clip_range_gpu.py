"""Clipping where the factor leaves fp32's normal range, and norms beyond fp32: a value is off by the store's rounding, the factor's
(u = 2^-24) and the norm's (14 u, half of what a sum of fp32 squares over a batch has), or half of the smallest step."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
STORE = {torch.float32: U, torch.bfloat16: 2.0 ** -8}
HALF_STEP = {torch.float32: 2.0 ** -150, torch.bfloat16: 2.0 ** -134}
TYPES = [torch.bfloat16, torch.float32]


def make(sizes, scale, types, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [(torch.randn(n, device="cuda", generator=g).clamp_(-3, 3) * scale).to(types[i % len(types)]) for i, n in enumerate(sizes)]


def check(grads, outs, max_norm):
    from paper_1810_10962_b200 import lm
    before = [g.double() for g in grads]
    want = math.sqrt(math.fsum(float(g.square().sum()) for g in before))
    max_norm = float(torch.tensor(max_norm, dtype=torch.float32))       # what the call takes
    norm = float(lm.clip_gradients(grads, max_norm, outs))
    assert norm == math.inf if want > 3.5e38 else abs(norm - want) <= 14 * U * want
    factor = 1.0 if want <= max_norm else max_norm / want
    for g, o in zip(before, grads if outs is None else outs):
        exact = g * factor
        off = (o.double() - exact).abs()
        assert bool((off <= (STORE[o.dtype] + 16 * U) * exact.abs() + HALF_STEP[o.dtype]).all()), float((off / exact.abs()).nan_to_num(0).max())


LISTS = {"one": [1], "few": [5, 70_001, 999], "many": [130] * 1500, "large": [9_000_001, 3]}


@pytest.mark.parametrize("scale,max_norm", [(1e36, 1e-8), (1e33, 1e-8), (1e30, 1e-8), (1e36, 1e-2), (1e38, 1e-30), (1e20, 1e-20), (1e38, 1.0), (1e38, 1e30),
                                            (1e15, 1e-40)])
@pytest.mark.parametrize("sizes", LISTS.values(), ids=LISTS.keys())
@pytest.mark.parametrize("types", [(torch.float32,), (torch.bfloat16,), (torch.bfloat16, torch.float32)], ids=["f32", "bf16", "both"])
def test_factors_below_the_normal_range(types, sizes, scale, max_norm):
    grads = make(sizes, scale, types, 3)
    check(grads, [torch.ones_like(g) for g in grads], max_norm)
    check(grads, None, max_norm)


@pytest.mark.parametrize("dtype", TYPES)
def test_small_factors_at_any_address(dtype):
    room, other = make([9000], 1e36, (dtype,), 5)[0], torch.zeros(9000, dtype=dtype, device="cuda")
    grads = [room[1000 * i + i: 1000 * i + i + 900 + i] for i in range(8)]
    outs = [other[1000 * i + 3: 1000 * i + 3 + 900 + i] for i in range(8)]
    check(grads, outs, 1e-8)
    between = torch.ones(9000, dtype=torch.bool, device="cuda")
    for i in range(8):
        between[1000 * i + 3: 1000 * i + 3 + 900 + i] = False
    assert bool((other[between] == 0).all())


def test_norms_beyond_fp32_and_infinite_gradients():
    """A finite norm clips by its value; an infinite gradient makes finite ones zero, but for a limit that is infinite too."""
    from paper_1810_10962_b200 import lm
    grads = [torch.full((70_001,), 3e38, device="cuda"), torch.full((5000,), -3e38, dtype=torch.bfloat16, device="cuda")]
    for limit in (1.0, 1e-6, 3e38):
        check(grads, [torch.ones_like(g) for g in grads], limit)
    outs = [torch.ones_like(g) for g in grads]
    assert float(lm.clip_gradients(grads, math.inf, outs)) == math.inf and all(torch.equal(a, b) for a, b in zip(grads, outs))
    grads[0][77] = math.inf
    for limit in (1.0, 0.0, 1e-45):
        assert float(lm.clip_gradients(grads, limit, outs)) == math.inf
        assert bool(outs[0][77].isnan()) and int(outs[0].count_nonzero()) == 1 and not outs[1].any()
