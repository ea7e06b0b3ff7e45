"""The norm over many gradients and clipping against the definition in 64 bits.

u = 2^-24 is fp32's rounding.  Squares are added in fp32 over batches of at most 64, 16 in a row, the rest in 64 bits; the
norm has half their error and its own rounding.  A clipped value is rounded twice: the factor, and the store."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
STORE = {torch.float32: U, torch.bfloat16: 2.0 ** -8}


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def make(sizes, seed, scale=1.0, types=(torch.bfloat16, torch.float32)):
    g = gen(seed)
    return [(torch.randn(n, device="cuda", generator=g) * scale).to(types[i % len(types)]) for i, n in enumerate(sizes)]


def norm_of(grads):
    return math.sqrt(math.fsum(float(g.double().square().sum()) for g in grads))


def check(grads, max_norm):
    from paper_1810_10962_b200 import lm
    want = norm_of(grads)
    got = lm.gradient_norm(grads)
    assert got.shape == () and got.dtype == torch.float32
    assert abs(float(got) - want) <= 14 * U * want
    factor = 1.0 if want <= max_norm else max_norm / want
    before = [g.clone() for g in grads]
    outs = [torch.empty_like(g) for g in grads]
    assert torch.equal(lm.clip_gradients(grads, max_norm, outs), got)
    for g, o in zip(before, outs):
        off = (o.double() - g.double() * factor).abs()
        assert bool((off <= (STORE[g.dtype] + 16 * U) * g.double().abs() * factor + 1e-40).all())
        if factor == 1.0:
            assert torch.equal(o, g)
    assert all(torch.equal(a, b) for a, b in zip(grads, before))
    assert torch.equal(lm.clip_gradients(grads, max_norm), got)              # in place
    assert all(torch.equal(a, b) for a, b in zip(grads, outs))


LISTS = [[1], [7], [1, 1, 1], [8, 16, 24], [0, 5, 0, 130], [4097, 3, 100_000], [1000] * 64, [999] * 65, [1_000_003, 1, 250_000],
         [17] * 1000, [33, 0, 8] * 400, [5_000_000, 2_000_001]]


@pytest.mark.parametrize("max_norm", [1.0, 1e6])
@pytest.mark.parametrize("sizes", LISTS, ids=lambda s: f"{len(s)}x{max(s)}")
def test_norm_and_clipping(sizes, max_norm):
    check(make(sizes, 3 + len(sizes)), max_norm)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_odd_addresses(dtype):
    """Views at every phase of a 16-byte word, outputs at another phase than their gradients."""
    from paper_1810_10962_b200 import lm
    room, other = make([9000], 5, types=(dtype,))[0], torch.zeros(9000, dtype=dtype, device="cuda")
    grads = [room[1000 * i + i: 1000 * i + i + 900 + i] for i in range(8)]
    outs = [other[1000 * i + 3: 1000 * i + 3 + 900 + i] for i in range(8)]
    norm = lm.clip_gradients(grads, 0.5, outs)
    want = norm_of(grads)
    assert abs(float(norm) - want) <= 14 * U * want
    mask = torch.ones(9000, dtype=torch.bool, device="cuda")
    for i, (g, o) in enumerate(zip(grads, outs)):
        mask[1000 * i + 3: 1000 * i + 3 + 900 + i] = False
        want_o = g.double() * 0.5 / want
        assert bool(((o.double() - want_o).abs() <= (STORE[dtype] + 16 * U) * want_o.abs()).all())
    assert bool((other[mask] == 0).all())                                  # nothing between the outputs is touched


@pytest.mark.parametrize("scale", [1e-40, 1e-30, 1e-20, 1e15, 1e25, 1e36])
def test_squares_outside_the_range_of_fp32(scale):
    check(make([3000, 70_001], 7, scale, (torch.float32,)), 1.0)
    check([*make([3000], 8, scale, (torch.float32,)), torch.zeros(5000, device="cuda"), torch.zeros(70_001, device="cuda")], scale)


def test_zeros_and_limits():
    from paper_1810_10962_b200 import lm
    zeros = [torch.zeros(5000, device="cuda"), -torch.zeros(33, dtype=torch.bfloat16, device="cuda")]
    check(zeros, 1.0)
    check(zeros, 0.0)
    grads = make([300, 20], 9)
    outs = [torch.ones_like(g) for g in grads]
    lm.clip_gradients(grads, 0.0, outs)
    assert all(bool((o == 0).all()) for o in outs)
    lm.clip_gradients(grads, math.inf, outs)
    assert all(torch.equal(a, b) for a, b in zip(grads, outs))


@pytest.mark.parametrize("at", [0, 1, 4000, 4999])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_infinity_and_nan(dtype, at):
    from paper_1810_10962_b200 import lm
    for bad in (math.inf, -math.inf, math.nan):
        grads = make([5000, 10], 11, types=(dtype,))
        grads[0][at] = bad
        outs = [torch.ones_like(g) for g in grads]
        norm = lm.clip_gradients(grads, 1.0, outs)
        if bad != bad:
            assert bool(norm.isnan()) and all(bool(o.isnan().all()) for o in outs)
        else:
            assert norm == math.inf and bool(outs[0][at].isnan()) and bool((outs[1] == 0).all())
            assert int(outs[0].isnan().sum()) == 1


def test_orders_of_memory_and_no_gradients():
    from paper_1810_10962_b200 import lm
    g = torch.randn(64, 30, 5, device="cuda", generator=gen(13))
    views = [g.permute(2, 0, 1), make([100], 14)[0]]
    outs = [torch.empty_like(v) for v in views]
    norm = lm.clip_gradients(views, 1.0, outs)
    assert abs(float(norm) - norm_of(views)) <= 14 * U * norm_of(views)
    assert torch.allclose(outs[0], views[0] / norm, rtol=1e-6)
    assert float(lm.gradient_norm([])) == 0.0 and float(lm.clip_gradients([], 1.0)) == 0.0
    assert float(lm.gradient_norm([torch.empty(0, device="cuda")])) == 0.0


def test_refusals():
    from paper_1810_10962_b200 import bns, lm
    a = torch.randn(1000, device="cuda")
    with pytest.raises(TypeError):
        lm.clip_gradients([a, a], 1.0)                                     # scaled twice in place
    with pytest.raises(TypeError):
        lm.clip_gradients([a[:600], a[500:]], 1.0)
    with pytest.raises(TypeError):
        lm.clip_gradients([a[:500], a[500:]], 1.0, [a[500:], a[:500]])
    with pytest.raises(TypeError):
        lm.clip_gradients([a[:500]], 1.0, [a[1:501]])
    norm = lm.gradient_norm([a, a])                                         # read only: counted twice
    assert abs(float(norm) - math.sqrt(2) * norm_of([a])) <= 20 * U * norm_of([a])
    for bad in ([a.half()], [a.view(10, 100)[:, :50]], [a.cpu()], [a.long()]):
        with pytest.raises(TypeError):
            lm.gradient_norm(bad)
    with pytest.raises(bns.BnsError):
        lm.clip_gradients([a], -1.0)
    with pytest.raises(bns.BnsError):
        lm.clip_gradients([a], math.nan)
    with pytest.raises(bns.BnsError):
        lm.GradientList([a]).norm(torch.empty(16, dtype=torch.uint8, device="cuda"))


def test_a_list_used_again_streams_and_graphs():
    from paper_1810_10962_b200 import lm
    grads = make([50_000, 3, 999, 128], 17)
    outs = [torch.zeros_like(g) for g in grads]
    both = lm.GradientList(grads, outs)
    first = both.clip(1.0)
    want = [o.clone() for o in outs]
    for _ in range(5):
        assert torch.equal(both.norm(), first) and torch.equal(both.clip(1.0), first)
        assert all(torch.equal(a, b) for a, b in zip(outs, want))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = both.clip(1.0)
    side.synchronize()
    assert torch.equal(got, first)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both.clip(1.0)
    for g in grads:
        g.mul_(2)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(got, 2 * first)
    for a, b in zip(outs, want):
        assert torch.allclose(a.float(), b.float(), rtol=2 ** -7, atol=1e-9)


def test_past_32_bit_offsets():
    from paper_1810_10962_b200 import lm
    n = 2_200_000_001
    g = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    g[-3:] = torch.tensor([3.0, 4.0, 12.0], device="cuda")
    g[5] = 84.0
    norm = lm.clip_gradients([g], 8.5)
    assert float(norm) == 85.0
    assert torch.allclose(g[-3:].float(), torch.tensor([0.3, 0.4, 1.2], device="cuda"), rtol=2 ** -8)
    assert int((g != 0).sum()) == 4
