"""The language-model operators against plain statements of their definitions in 64 bits.

Tolerances are bounds, not fits: u = 2^-24 is fp32's rounding, 2^-8 the largest relative rounding of a bf16 store,
and every sum of n terms kept in fp32 may be off by its longest chain of additions times u times the sum of the terms'
magnitudes."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
STORE = {"f32": 2 * U, "bf16": 2.0 ** -8}
DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-5


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def randn(g, *shape, dtype="f32"):
    return torch.randn(*shape, device="cuda", generator=g).to(DTYPE[dtype])


def assert_within(got, want, tol, what):
    off = (got.double() - want).abs()
    bad = ~(off <= tol)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {float((off / tol).nan_to_num(math.inf).max()):.3g} times the bound"


# ----------------------------------------------------------------------------- root-mean-square norm
SHAPES = [(1, 1), (1, 64), (3, 7), (2, 128), (5, 130), (33, 1000), (7, 2050), (300, 513), (1, 4096), (700, 4096), (4, 8191),
          (9, 16384), (3, 16392), (2, 20001), (2, 40000)]


def norm_case(T, D, dtype, residual, seed):
    g = gen(seed)
    x = randn(g, T, D, dtype=dtype)
    r = (randn(g, T, D) * 3).to(DTYPE[dtype]) if residual else None
    w = 1 + 0.3 * randn(g, D)
    s = x.double() + (r.double() if residual else 0)
    rstd = 1 / torch.sqrt((s * s).mean(1) + EPS)
    return x, r, w, s, rstd


@pytest.mark.parametrize("residual", [True, False])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,D", SHAPES)
def test_norm_forward(T, D, dtype, residual):
    from paper_1810_10962_b200 import lm
    x, r, w, s, rstd = norm_case(T, D, dtype, residual, 11 + T + D)
    y, h, got = lm.rms_norm_forward(x, r, w, EPS)
    # a thread adds at most ceil(D / 1024) + 16 squares in a row, ten joins follow; half of it reaches the root
    u = (D / 1024 + 16 + 10 + 8) * U
    assert_within(got, rstd, u * rstd, "rstd")
    want = s * rstd[:, None] * w.double()
    assert_within(y, want, (u + 4 * U + STORE[dtype]) * want.abs() + 1e-38, "y")
    if residual:
        assert torch.equal(h, (x.float() + r.float()).to(x.dtype))
    else:
        assert h is x


def e4m3(v):
    _, e = torch.frexp(v)
    quantum = torch.ldexp(torch.ones_like(v), (e - 1).clamp(min=-6) - 3)
    return torch.round(v / quantum) * quantum


@pytest.mark.parametrize("group", [0, 128])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,D", SHAPES)
def test_norm_forward_fp8(T, D, dtype, group):
    from paper_1810_10962_b200 import lm
    x, r, w, s, rstd = norm_case(T, D, dtype, True, 23 + T + D)
    x[0, : min(D, 128)] = 0                     # a group (for narrow rows the row) of zeros
    r[0, : min(D, 128)] = 0
    s = x.double() + r.double()
    rstd = 1 / torch.sqrt((s * s).mean(1) + EPS)
    q, scales, h, got = lm.rms_norm_forward_fp8(x, r, w, EPS, group=group)
    u = (D / 1024 + 16 + 10 + 8) * U
    assert_within(got, rstd, u * rstd, "rstd")
    assert torch.equal(h, (x.float() + r.float()).to(x.dtype))
    y = s * rstd[:, None] * w.double()
    width = group or D
    n = -(-D // width)
    parts = torch.nn.functional.pad(y, (0, n * width - D)).view(T, n, width)
    amax = parts.abs().amax(2)
    want = torch.where(amax > 0, amax / 448, torch.ones_like(amax))
    assert scales.shape == (T, n)
    assert_within(scales, want, (u + 6 * U) * want, "scales")
    per = want.repeat_interleave(width, 1)[:, :D]
    value = q.double() * per
    # nearest e4m3: half of an ulp of 2^-3, or of the smallest quantum 2^-9 (both times the scale)
    assert_within(value, y, torch.maximum(y.abs() * 2.0 ** -4, per * 2.0 ** -10) * (1 + 1e-4), "q")
    # and only what lies within rounding of a tie may go the other way
    assert float((q.double() != e4m3(y / per)).float().mean()) <= max(2e-4, 1.5 / y.numel())


@pytest.mark.parametrize("with_dh", [True, False])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,D", SHAPES + [(3000, 256)])
def test_norm_backward(T, D, dtype, with_dh):
    from paper_1810_10962_b200 import lm
    g = gen(37 + T + D)
    h, dy = randn(g, T, D, dtype=dtype) * 2, randn(g, T, D, dtype=dtype)
    dh = randn(g, T, D, dtype=dtype) if with_dh else None
    w, rstd = 1 + 0.3 * randn(g, D), 0.1 + torch.rand(T, device="cuda", generator=g)
    dx, dw = lm.rms_norm_backward(dy, h, w, rstd, dh=dh)
    again = lm.rms_norm_backward(dy, h, w, rstd, dh=dh)
    assert torch.equal(dx, again[0]) and torch.equal(dw, again[1])          # a fixed order of summation
    rs, xhat, wdy = rstd.double()[:, None], h.double() * rstd.double()[:, None], w.double() * dy.double()
    c = (wdy * xhat).mean(1, keepdim=True)
    u = (D / 1024 + 16 + 10 + 8) * U
    want = rs * (wdy - xhat * c) + (dh.double() if with_dh else 0)
    tol = (6 * U * (rs * (wdy.abs() + (xhat * c).abs()) + (dh.double().abs() if with_dh else 0))
           + u * rs * xhat.abs() * (wdy * xhat).abs().mean(1, keepdim=True) + STORE[dtype] * want.abs())
    assert_within(dx, want, tol + 1e-38, "dx")
    blocks = min(T, 148 * 16)
    chain = T / 148 + blocks / 8 + 8 + 4
    assert_within(dw, (dy.double() * xhat).sum(0), chain * U * (dy.double() * xhat).abs().sum(0) + 1e-38, "dweight")


def test_norm_gradient_against_differences():
    from paper_1810_10962_b200 import lm
    g = gen(41)
    T, D = 6, 200
    x, r, w = randn(g, T, D), randn(g, T, D), 1 + 0.3 * randn(g, D)
    dy, dh = randn(g, T, D), randn(g, T, D)

    def value(x, w):
        y, h, _ = lm.rms_norm_forward(x, r, w, EPS)
        return float((y.double() * dy.double()).sum() + (h.double() * dh.double()).sum())

    _, h, rstd = lm.rms_norm_forward(x, r, w, EPS)
    dx, dweight = lm.rms_norm_backward(dy, h, w, rstd, dh=dh)
    step = 2.0 ** -7
    for k in range(4):
        ex, ew = randn(g, T, D), randn(g, D)
        # central differences: step^2 / 6 times the third derivative (of order 10 per row here), values off by some u
        # per element, divided by the step
        for got, plus, minus in (((dx.double() * ex.double()).sum(), value(x + step * ex, w), value(x - step * ex, w)),
                                 ((dweight.double() * ew.double()).sum(), value(x, w + step * ew), value(x, w - step * ew))):
            assert abs(float(got) - (plus - minus) / (2 * step)) < 0.02 * math.sqrt(T * D)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_norm_strided_rows_and_odd_addresses(dtype):
    from paper_1810_10962_b200 import lm
    g = gen(43)
    for T, D, pad, shift in ((5, 96, 32, 0), (5, 96, 7, 0), (4, 130, 6, 1), (6, 64, 3, 3)):
        store = [randn(g, T * (D + pad) + shift, dtype=dtype)[shift:].view(T, D + pad)[:, :D] for _ in range(4)]
        x, r, dy, dh = store
        w = 1 + 0.3 * randn(g, D)
        for a, b in zip(lm.rms_norm_forward(x, r, w, EPS), lm.rms_norm_forward(x.contiguous(), r.contiguous(), w, EPS)):
            assert torch.allclose(a.float(), b.float(), rtol=2 * STORE[dtype] + 1e-6, atol=0)
        for group in (0, 128):
            q, s, h, _ = lm.rms_norm_forward_fp8(x, r, w, EPS, group=group)
            q2, s2, h2, _ = lm.rms_norm_forward_fp8(x.contiguous(), r.contiguous(), w, EPS, group=group)
            assert torch.equal(h, h2) and torch.allclose(s, s2, rtol=1e-6) and torch.equal(q.float(), q2.float())
        rstd = torch.rand(T, device="cuda") + 0.5
        for a, b in zip(lm.rms_norm_backward(dy, x, w, rstd, dh=dh),
                        lm.rms_norm_backward(dy.contiguous(), x.contiguous(), w, rstd, dh=dh.contiguous())):
            assert torch.allclose(a.float(), b.float(), rtol=2 * STORE[dtype], atol=1e-5)


def test_norm_special_values():
    from paper_1810_10962_b200 import lm
    D = 256
    x = torch.ones(6, D, device="cuda")
    x[0] = 0
    x[1, 3] = math.inf
    x[2, 5] = math.nan
    x[3] *= 1e-30                               # squares underflow: eps decides
    x[4] *= 1e-25
    w = torch.ones(D, device="cuda")
    y, _, rstd = lm.rms_norm_forward(x, None, w, EPS)
    assert bool((y[0] == 0).all()) and math.isclose(float(rstd[0]), EPS ** -0.5, rel_tol=1e-6)
    assert float(rstd[1]) == 0 and bool(y[1, 3].isnan()) and float(y[1, 4]) == 0
    assert bool(y[2].isnan().all())
    assert torch.allclose(y[3], x[3] * EPS ** -0.5, rtol=1e-6)
    for group in (0, 128):
        q, s, _, _ = lm.rms_norm_forward_fp8(x, None, w, EPS, group=group)
        q = q.float()
        assert bool((q[0] == 0).all()) and bool((s[0] == 1).all())
        assert bool(q[1, :128].isnan().all()) and bool(s[1, 0].isnan())
        assert bool(q[2].isnan().all())
        assert bool((q[3:] == 448).all())       # all elements are the largest
        assert torch.allclose(s[4], torch.full_like(s[4], 1e-25 * EPS ** -0.5 / 448), rtol=1e-5)


def test_norm_without_rows():
    from paper_1810_10962_b200 import lm
    x, w = torch.empty(0, 64, device="cuda"), torch.ones(64, device="cuda")
    y, h, rstd = lm.rms_norm_forward(x, x.clone(), w, EPS)
    assert y.shape == (0, 64) and rstd.shape == (0,)
    dx, dw = lm.rms_norm_backward(y, h, w, rstd)
    assert dx.shape == (0, 64) and bool((dw == 0).all())


# ----------------------------------------------------------------------------- linear head + cross entropy
def head_case(T, V, D, dtype, seed, left_out=0.2, int64=True):
    g = gen(seed)
    x, w = randn(g, T, D, dtype=dtype), (randn(g, V, D) * (2 / math.sqrt(D))).to(DTYPE[dtype])
    target = torch.randint(0, V, (T,), device="cuda", generator=g)
    target[torch.rand(T, device="cuda", generator=g) < left_out] = -100
    dloss = torch.rand(T, device="cuda", generator=g) + 0.5
    return x, w, target if int64 else target.int(), dloss


def head_bounds(x, w, target, dloss, dtype):
    """Losses, log-sums, gradients in 64 bits, and how far fp32 sums may be from them."""
    xd, wd = x.double(), w.double()
    T, D = x.shape
    V = w.shape[0]
    z = xd @ wd.T
    # fp32 accumulation in steps of 16 terms of K; truncation counts as twice the rounding.  fp32 tensors: the terms'
    # six products, the three that are dropped below 2^-24 of the product each.
    pairs = 6 if dtype == "f32" else 1
    chain = lambda n: 2 * U * (pairs * n / 16 + 16)  # noqa: E731
    tz = float(((chain(D) + (4 * U if pairs == 6 else 0)) * (xd.abs() @ wd.abs().T)).max())
    lse = torch.logsumexp(z, 1)
    counts = target >= 0
    at = target.long().clamp(min=0)[:, None]
    loss = torch.where(counts, lse - z.gather(1, at)[:, 0], torch.zeros_like(lse))
    tl = 2 * tz + 8 * U * (1 + lse.abs() + z.abs().max())
    p = torch.exp(z - lse[:, None]) * (dloss.double() * counts)[:, None]
    G = p.clone()
    G.scatter_add_(1, at, -(dloss.double() * counts)[:, None])
    te = 2 * tz + 32 * U + 8 * U * float(lse.abs().max())      # of an exponential, relative
    tG = (2.0 ** -8 if dtype == "bf16" else 4 * U) * G.abs() + te * p
    bounds = []
    for A, tA, B, n in ((G, tG, wd, V), (G.T, tG.T, xd, T)):
        want = A @ B
        bounds.append((want, tA @ B.abs() + (chain(n) + (4 * U if pairs == 6 else 0)) * ((A.abs() + tA) @ B.abs())
                       + STORE[dtype] * 1.01 * want.abs() + 1e-30))
    return loss, lse, tl, bounds


def check_head(x, w, target, dloss, dtype):
    from paper_1810_10962_b200 import bns, lm
    want_loss, want_lse, tl, ((want_dx, tol_dx), (want_dw, tol_dw)) = head_bounds(x, w, target, dloss, dtype)
    loss, lse = lm.linear_cross_entropy_forward(x, w, target)
    assert_within(lse, want_lse, tl, "lse")
    assert_within(loss, want_loss, tl, "loss")
    assert bool((loss[target < 0] == 0).all())
    dx, dw = lm.linear_cross_entropy_backward(x, w, target, lse, dloss)
    again = lm.linear_cross_entropy_backward(x, w, target, lse, dloss)
    assert torch.equal(dx, again[0]) and torch.equal(dw, again[1])
    assert_within(dx, want_dx, tol_dx, "dx")
    assert_within(dw, want_dw, tol_dw, "dw")
    assert bns.wait_timeouts() == 0


HEADS = [(1, 2, 8), (1, 1, 1), (3, 255, 64), (128, 256, 64), (129, 257, 72), (5, 1000, 65), (64, 300, 127), (127, 513, 200),
         (300, 700, 136), (256, 2048, 320), (513, 1025, 33), (1, 5000, 256), (24, 9001, 512), (1000, 333, 1000), (2100, 400, 40)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,V,D", HEADS)
def test_head(T, V, D, dtype):
    check_head(*head_case(T, V, D, dtype, 100 + T + V + D, int64=(T + V) % 2 == 0), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,V,D,piece", [(70, 1500, 96, 512), (300, 1111, 100, 256), (2, 3000, 64, 1024), (1300, 900, 72, 300)])
def test_head_in_pieces_of_the_vocabulary(T, V, D, piece, dtype):
    from paper_1810_10962_b200 import bns
    try:
        bns.set_tuning("head_piece", piece)
        check_head(*head_case(T, V, D, dtype, 7 + T), dtype)
    finally:
        bns.set_tuning("head_piece", 0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pad_x,pad_w", [(8, 16), (3, 0), (0, 5), (1, 1)])
def test_head_strided_rows(pad_x, pad_w, dtype):
    from paper_1810_10962_b200 import lm
    T, V, D = 140, 600, 88
    x, w, target, dloss = head_case(T, V, D, dtype, 55)
    xs, ws = torch.full((T, D + pad_x), math.nan, device="cuda", dtype=x.dtype), torch.full((V, D + pad_w), math.nan, device="cuda", dtype=x.dtype)
    xs[:, :D], ws[:, :D] = x, w
    check_head(xs[:, :D], ws[:, :D], target, dloss, dtype)
    for a, b in zip(lm.linear_cross_entropy_forward(xs[:, :D], ws[:, :D], target), lm.linear_cross_entropy_forward(x, w, target)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("T", [1, 2, 3, 4, 7, 8, 9, 16, 17, 32, 33])
@pytest.mark.parametrize("V,D", [(1, 3), (7, 4), (1001, 130), (333, 1024), (6001, 36), (50, 1633), (35, 4100)])
def test_head_few_rows_fp32(T, V, D):
    check_head(*head_case(T, V, D, "f32", 300 + T + V, int64=T % 2 == 0), "f32")


@pytest.mark.parametrize("pad_x,pad_w", [(4, 8), (3, 0), (0, 5)])
@pytest.mark.parametrize("D", [88, 90])
def test_head_few_rows_strided(D, pad_x, pad_w):
    T, V = 6, 500
    x, w, target, dloss = head_case(T, V, D, "f32", 56)
    xs, ws = torch.full((T, D + pad_x), math.nan, device="cuda"), torch.full((V, D + pad_w), math.nan, device="cuda")
    xs[:, :D], ws[:, :D] = x, w
    check_head(xs[:, :D], ws[:, :D], target, dloss, "f32")


def test_head_few_rows_left_out():
    from paper_1810_10962_b200 import bns, lm
    x, w, target, dloss = head_case(5, 300, 20, "f32", 79, left_out=0.0)
    target[1], target[3] = -7, 300              # left out, the second as it is past the vocabulary
    workspace = torch.empty(lm.linear_cross_entropy_workspace_bytes(x, w, target), dtype=torch.uint8, device="cuda")
    loss, lse = lm.linear_cross_entropy_forward(x, w, target, workspace=workspace)
    assert bns.workspace_status(workspace) == lm.FLAG_BAD_TARGET
    assert bool((loss[[1, 3]] == 0).all()) and bool((loss[[0, 2, 4]] > 0).all())
    dloss[1] = math.nan
    lse[3] = math.nan
    dx, dw = lm.linear_cross_entropy_backward(x, w, target, lse, dloss)
    assert bool((dx[[1, 3]] == 0).all()) and bool((dx[[0, 2, 4]] != 0).any(1).all()) and bool(dw.isfinite().all())


def test_head_rows_left_out():
    from paper_1810_10962_b200 import bns, lm
    x, w, target, dloss = head_case(40, 500, 64, "bf16", 77)
    target[:] = -1
    loss, lse = lm.linear_cross_entropy_forward(x, w, target)
    assert bool((loss == 0).all()) and bool(lse.isfinite().all())
    dloss[:] = math.nan                         # of rows that are left out: ignored
    dx, dw = lm.linear_cross_entropy_backward(x, w, target, lse, dloss)
    assert bool((dx == 0).all()) and bool((dw == 0).all())
    # a target past the vocabulary is left out too, and told
    target[3], target[4] = 500, 499
    workspace = torch.empty(lm.linear_cross_entropy_workspace_bytes(x, w, target), dtype=torch.uint8, device="cuda")
    loss, _ = lm.linear_cross_entropy_forward(x, w, target, workspace=workspace)
    assert bns.workspace_status(workspace) == lm.FLAG_BAD_TARGET and float(loss[3]) == 0 and float(loss[4]) > 0
    target[3] = -5
    lm.linear_cross_entropy_forward(x, w, target, workspace=workspace)
    assert bns.workspace_status(workspace) == 0


def test_head_extreme_logits():
    """Logits of +-3e4: the sum of exponentials is one term, the loss of the largest is 0 and of another the difference."""
    from paper_1810_10962_b200 import lm
    T, V, D = 130, 300, 64
    x, w = torch.zeros(T, D, device="cuda", dtype=torch.bfloat16), torch.zeros(V, D, device="cuda", dtype=torch.bfloat16)
    x[:, 0], w[:, 0] = 128, -256
    w[7, 0] = 256
    target = torch.full((T,), 7, device="cuda")
    target[1] = 8
    loss, lse = lm.linear_cross_entropy_forward(x, w, target)
    assert bool((lse == 32768).all()) and float(loss[0]) == 0 and float(loss[1]) == 65536
    dx, dw = lm.linear_cross_entropy_backward(x, w, target, lse, torch.ones(T, device="cuda"))
    assert float(dx[0].float().abs().max()) == 0 and float(dx[1, 0]) == 512
    assert float(dw[7, 0]) == 128 and float(dw[8, 0]) == -128 and float(dw[9].float().abs().max()) == 0


def test_head_nan_and_infinity_travel():
    from paper_1810_10962_b200 import lm
    x, w, target, _ = head_case(20, 300, 64, "bf16", 5, left_out=0)
    x[2, 3] = math.nan
    loss, lse = lm.linear_cross_entropy_forward(x, w, target)
    assert bool(loss[2].isnan()) and bool(lse[2].isnan()) and int(loss.isnan().sum()) == 1


def test_head_without_rows():
    from paper_1810_10962_b200 import lm
    x, w = torch.empty(0, 64, device="cuda"), torch.randn(300, 64, device="cuda")
    target = torch.empty(0, dtype=torch.int64, device="cuda")
    loss, lse = lm.linear_cross_entropy_forward(x, w, target)
    dx, dw = lm.linear_cross_entropy_backward(x, w, target, lse, loss)
    assert loss.shape == (0,) and dx.shape == (0, 64) and bool((dw == 0).all())


def test_head_gradient_against_differences():
    from paper_1810_10962_b200 import lm
    x, w, target, dloss = head_case(50, 400, 48, "f32", 99)
    value = lambda x, w: float((lm.linear_cross_entropy_forward(x, w, target)[0].double() * dloss.double()).sum())  # noqa: E731
    _, lse = lm.linear_cross_entropy_forward(x, w, target)
    dx, dw = lm.linear_cross_entropy_backward(x, w, target, lse, dloss)
    g, step = gen(1), 2.0 ** -6
    for _ in range(4):
        ex, ew = randn(g, *x.shape), randn(g, *w.shape) * 0.1
        for got, plus, minus in (((dx.double() * ex.double()).sum(), value(x + step * ex, w), value(x - step * ex, w)),
                                 ((dw.double() * ew.double()).sum(), value(x, w + step * ew), value(x, w - step * ew))):
            # losses off by some 1e-6 a row over the step; the third derivative of a row's loss along ex is of order 10
            assert abs(float(got) - (plus - minus) / (2 * step)) < 50 * 1.5 * (2e-6 / step + 10 * step ** 2 / 6)


# ----------------------------------------------------------------------------- distillation
def distill_case(T, V, K, dtype, seed, int64=False, teacher="f32"):
    g = gen(seed)
    z = (randn(g, T, V) * 3).to(DTYPE[dtype])
    a = (randn(g, T, K) * 3).to(DTYPE[teacher])
    index = torch.randint(0, V, (T, K), device="cuda", generator=g)      # places may repeat
    index[torch.rand(T, K, device="cuda", generator=g) < 0.2] = -1
    if T > 2:
        index[T // 2] = -1                                                # a row without entries
    if K > 2:
        a[0, 1] = -math.inf
    return z, a, index if int64 else index.int(), torch.rand(T, device="cuda", generator=g) + 0.5


def distill_want(z, a, index, dloss, tau):
    zd = z.double() / tau
    V = z.shape[1]
    there = (index >= 0) & (index < V)
    ad = torch.where(there, a.double() / tau, torch.full((), -math.inf, device="cuda", dtype=torch.float64))
    some = (ad > -math.inf).any(1)
    ad[~some] = 0
    p = torch.softmax(ad, 1) * there * some[:, None]
    lse = torch.logsumexp(zd, 1)
    at = torch.where(there, index, torch.zeros_like(index)).long()
    terms = torch.where(p > 0, p * (torch.log(p) - zd.gather(1, at) + lse[:, None]), torch.zeros_like(p))
    loss, size = tau * tau * terms.sum(1), tau * tau * (p * (zd.gather(1, at).abs() + lse.abs()[:, None] + ad.nan_to_num(neginf=0).abs() + 1)).sum(1)
    q = torch.softmax(zd, 1) * some[:, None]      # not exp(z - lse): log V vanishes beside logits of 1e38 in 64 bits too
    share = torch.zeros_like(q).scatter_add_(1, at, p)
    scale = (dloss.double() * tau)[:, None]
    return loss, lse, (q - share) * scale, (q + share) * scale, size


def check_distill(z, a, index, dloss, tau, dtype):
    from paper_1810_10962_b200 import lm
    loss, lse, dz, size, terms = distill_want(z, a, index, dloss, tau)
    got_loss, got_lse = lm.topk_distillation_forward(z, a, index, tau)
    V = z.shape[1]
    # exponents: a multiply-add of a value up to max |z| / tau, then 2 ulp; sums: V / 4096 in a row in a thread, then joins
    top = float(z.double().abs().where(z.isfinite(), torch.zeros((), device="cuda", dtype=torch.float64)).max())
    ue = U * (8 + 4 * (top + 20) / tau) + U * (V / 4096 * 8 + 32)
    assert_within(got_lse, lse, ue + 4 * U * lse.abs(), "lse")
    assert_within(got_loss, loss, (2 * ue + 16 * U) * terms + 2 * ue * tau * tau, "loss")
    tol = 2 * ue * size + STORE[dtype] * dz.abs() + 1e-37
    step_loss, step_dz = lm.topk_distillation_step(z, a, index, dloss, tau)
    assert_within(step_loss, loss, (2 * ue + 16 * U) * terms + 2 * ue * tau * tau, "loss of the step")
    assert_within(step_dz, dz, tol, "dz of the step")
    assert_within(lm.topk_distillation_backward(z, a, index, got_lse, dloss, tau), dz, tol, "dz")
    empty = (index < 0).all(1)
    assert bool((got_loss[empty] == 0).all()) and bool((step_dz[empty] == 0).all())


DISTILLS = [(1, 1, 1), (1, 7, 3), (4, 100, 8), (3, 1000, 33), (5, 4099, 64), (9, 32768, 16), (2, 50257, 128), (6, 65537, 1024),
            (300, 2001, 20), (1, 131072, 64), (2, 250001, 5),
            (400, 33000, 9), (320, 50257, 40), (310, 131072, 8), (301, 140001, 12)]


@pytest.mark.parametrize("tau", [1.0, 2.5])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,V,K", DISTILLS)
def test_distillation(T, V, K, dtype, tau):
    check_distill(*distill_case(T, V, K, dtype, 300 + T + V, int64=V % 2 == 1, teacher="bf16" if K == 16 else "f32"), tau, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_distillation_strided_rows(dtype):
    z, a, index, dloss = distill_case(7, 1000, 12, dtype, 8)
    for pad in (24, 1, 3):
        store = torch.full((7, 1000 + pad), math.inf, device="cuda", dtype=z.dtype)
        store[:, :1000] = z
        check_distill(store[:, :1000], a, index, dloss, 1.0, dtype)
    z, a, index, dloss = distill_case(600, 1001, 5, dtype, 13)           # many rows
    store = torch.full((600, 1003), math.inf, device="cuda", dtype=z.dtype)
    store[:, :1001] = z
    check_distill(store[:, :1001], a, index, dloss, 1.0, dtype)


def test_distillation_masked_vocabulary():
    """Student logits of -inf (places that may not be chosen) carry nothing; a teacher's entry there costs infinity."""
    from paper_1810_10962_b200 import lm
    z, a, index, dloss = distill_case(4, 300, 6, "f32", 9)
    index = index.clamp(min=0) % 200
    z[:, 200:] = -math.inf
    check_distill(z, a, index, dloss, 1.0, "f32")
    index[1, 0] = 250
    a[1] = 0
    loss, lse = lm.topk_distillation_forward(z, a, index, 1.0)
    assert float(loss[1]) == math.inf and bool(loss[[0, 2, 3]].isfinite().all()) and bool(lse.isfinite().all())
    _, dz = lm.topk_distillation_step(z, a, index, dloss, 1.0)
    assert bool(dz.isfinite().all()) and math.isclose(float(dz[1, 250]), -float(dloss[1]) / 6, rel_tol=1e-5)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [300, 5001])
def test_distillation_logits_at_the_types_lowest_value(V, dtype):
    """Masked with the lowest finite value: where some logits are not, they carry nothing; where all are, the student is
    uniform."""
    from paper_1810_10962_b200 import lm
    z, a, index, dloss = distill_case(5, V, 6, dtype, 31)
    lowest = torch.finfo(z.dtype).min
    index = index.clamp(min=0)
    a[:] = 0
    z[1, V // 2:] = lowest
    index[1] = index[1] % (V // 2)
    z[3] = lowest
    loss, lse, dz, size, terms = distill_want(z, a, index, dloss, 1.0)
    got_loss, got_lse = lm.topk_distillation_forward(z, a, index, 1.0)
    step_loss, step_dz = lm.topk_distillation_step(z, a, index, dloss, 1.0)
    others = [0, 1, 2, 4]
    assert torch.allclose(got_loss[others].double(), loss[others], rtol=1e-4, atol=1e-5)
    assert torch.allclose(step_dz.double(), dz, rtol=2e-2 if dtype == "bf16" else 1e-4, atol=1e-7)
    assert float(got_lse[3]) == lowest and torch.equal(step_loss, got_loss)
    # six places of equal weight against a uniform student; the same place twice counts twice
    assert math.isclose(float(got_loss[3]), math.log(V / 6), rel_tol=1e-4)
    assert bool(lm.topk_distillation_backward(z, a, index, got_lse, dloss, 1.0).isfinite().all())


@pytest.mark.parametrize("tau", [0.5, 1.0, 3.0])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_distillation_teacher_at_the_types_lowest_value(dtype, tau):
    """Entries at the lowest finite value carry nothing beside others, and are of equal weight where there are only such."""
    from paper_1810_10962_b200 import lm
    V, K = 1200, 5
    g = gen(77)
    z = randn(g, 4, V).to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    a = randn(g, 4, K).to(z.dtype)
    a[1, 2:] = torch.finfo(a.dtype).min
    a[2] = torch.finfo(a.dtype).min
    index = torch.stack([torch.randperm(V, generator=g, device=g.device)[:K] for _ in range(4)]).to(torch.int32).to(z.device)
    dloss = torch.tensor([1.0, 2.0, -1.0, 0.5], device=z.device)
    p = torch.softmax(a.double() / tau, -1)
    log_q = torch.log_softmax(z.double() / tau, -1)
    terms = torch.where(p > 0, p * (p.clamp(min=1e-300).log() - log_q.gather(1, index.long())), torch.zeros_like(p))
    dz = log_q.exp().scatter_add(1, index.long(), -p) * (dloss.double() * tau)[:, None]
    loss, lse = lm.topk_distillation_forward(z, a, index, tau)
    step_loss, step_dz = lm.topk_distillation_step(z, a, index, dloss, tau)
    # exponents of some 20 at most, in fp32: 20 x 2^-23 an operation, few of them in a row
    assert torch.allclose(loss.double(), tau * tau * terms.sum(-1), rtol=2e-5, atol=2e-5 * tau * tau)
    assert torch.equal(step_loss, loss)
    for got in (step_dz, lm.topk_distillation_backward(z, a, index, lse, dloss, tau)):
        assert torch.allclose(got.double(), dz, rtol=2.0 ** -8 if dtype == "bf16" else 5e-5, atol=2e-6 * tau)


@pytest.mark.parametrize("tau", [0.7, 1.0])
@pytest.mark.parametrize("mask", [-1e4, -1e9, -1e10, -3e20, -1e38, 1e10])
def test_distillation_far_logits(mask, tau):
    """Masks of other sizes, for stretches of a row, for most of it and for a whole row; likewise among the teacher's values.
    As a positive number it is what the rest of the row vanishes beside."""
    from paper_1810_10962_b200 import lm
    V, K = 40000, 5
    g = gen(78)
    z, a = randn(g, 6, V), randn(g, 6, K)
    z[1, 7000:23001] = mask
    z[2, 3:V - 1] = mask
    z[3] = mask
    a[4, :3] = mask
    a[5] = mask
    index = torch.stack([torch.randperm(V, generator=g, device=g.device)[:K] for _ in range(6)]).to(torch.int32)
    index[:, 0] = 5                # masked in rows 2 and 3
    index[1:3, 1:] = torch.tensor([0, 1, 2, V - 1], device=index.device, dtype=torch.int32)
    dloss = torch.tensor([1.0, 2.0, -1.0, 0.5, 1.0, 1.0], device=z.device)
    p = torch.softmax(a.double() / tau, -1)
    log_q = torch.log_softmax(z.double() / tau, -1)
    terms = torch.where(p > 0, p * (p.clamp(min=1e-300).log() - log_q.gather(1, index.long())), torch.zeros_like(p))
    want = tau * tau * terms.sum(-1)
    dz = log_q.exp().scatter_add(1, index.long(), -p) * (dloss.double() * tau)[:, None]
    loss, lse = lm.topk_distillation_forward(z, a, index, tau)
    step_loss, step_dz = lm.topk_distillation_step(z, a, index, dloss, tau)
    # losses: differences of logits and a log-sum of some 20, and of a mask where an entry is masked
    assert torch.allclose(loss.double(), want, rtol=2e-5, atol=2e-5)
    assert torch.equal(step_loss, loss)
    assert torch.allclose(step_dz.double(), dz, rtol=1e-4, atol=2e-6)
    assert torch.allclose(lse.double(), torch.logsumexp(z.double() / tau, -1), rtol=1e-6, atol=2e-5)
    # the gradient from a log-sum in fp32 is as good as that number: the rows of usual size
    usual = lse.abs() < 1e3
    got = lm.topk_distillation_backward(z, a, index, lse, dloss, tau)
    assert torch.allclose(got[usual].double(), dz[usual], rtol=1e-4, atol=2e-6)
    assert bool(got.isfinite().all())


def test_distillation_places_outside_the_vocabulary_are_no_entries():
    from paper_1810_10962_b200 import lm
    z, a, index, dloss = distill_case(3, 100, 8, "f32", 10, int64=True)
    other = index.clone()
    other[index < 0] = 2 ** 40
    for x, y in zip(lm.topk_distillation_step(z, a, index, dloss, 1.0), lm.topk_distillation_step(z, a, other, dloss, 1.0)):
        assert torch.equal(x, y)


def test_distillation_gradient_against_differences():
    from paper_1810_10962_b200 import lm
    z, a, index, dloss = distill_case(10, 200, 9, "f32", 12)
    value = lambda z: float((lm.topk_distillation_forward(z, a, index, 2.0)[0].double() * dloss.double()).sum())  # noqa: E731
    _, dz = lm.topk_distillation_step(z, a, index, dloss, 2.0)
    g, step = gen(2), 2.0 ** -5
    for _ in range(4):
        e = randn(g, *z.shape)
        want = (value(z + step * e) - value(z - step * e)) / (2 * step)
        # loss per row some 4e-5 off at most; third derivative along e of order 1 at this temperature
        assert abs(float((dz.double() * e.double()).sum()) - want) < 10 * 1.5 * (1e-5 / step + 4 * step ** 2 / 6)


# ----------------------------------------------------------------------------- streams
def test_calls_go_to_the_current_stream_and_into_a_graph():
    from paper_1810_10962_b200 import lm
    x, w, target, dloss = head_case(60, 700, 64, "bf16", 21)
    want = lm.linear_cross_entropy_forward(x, w, target)
    want_grads = lm.linear_cross_entropy_backward(x, w, target, want[1], dloss)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = lm.linear_cross_entropy_forward(x, w, target)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = lm.linear_cross_entropy_forward(x, w, target)
        grads = lm.linear_cross_entropy_backward(x, w, target, got[1], dloss)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((*got, *grads), (*want, *want_grads)))


def test_example_learns():
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "lm_last_layers.py")
    spec = importlib.util.spec_from_file_location("lm_last_layers", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    first, last = module.main(["--steps", "1"]), module.main(["--steps", "40"])
    assert 6.0 < first < 8.0 and last < 0.5 * first       # log 1000 = 6.9 at the start


# ----------------------------------------------------------------------------- more than 2^31 elements
def test_norm_past_32_bit_offsets():
    from paper_1810_10962_b200 import lm
    T, D = 540_000, 4096                                     # 2.2e9 elements
    x = torch.empty(T, D, dtype=torch.bfloat16, device="cuda")
    x[-5:] = randn(gen(61), 5, D, dtype="bf16")
    x[:-5] = 1
    w = 1 + 0.3 * randn(gen(62), D)
    y, _, rstd = lm.rms_norm_forward(x, None, w, EPS)
    want = lm.rms_norm_forward(x[-5:].contiguous(), None, w, EPS)
    assert torch.equal(y[-5:], want[0]) and torch.equal(rstd[-5:], want[2])
    del y
    q, scales, _, _ = lm.rms_norm_forward_fp8(x, None, w, EPS, group=128)
    want_q = lm.rms_norm_forward_fp8(x[-5:].contiguous(), None, w, EPS, group=128)
    assert torch.equal(q[-5:].float(), want_q[0].float()) and torch.equal(scales[-5:], want_q[1])
    del q, scales
    dx, _ = lm.rms_norm_backward(x, x, w, rstd)
    assert torch.equal(dx[-5:], lm.rms_norm_backward(x[-5:].contiguous(), x[-5:].contiguous(), w, rstd[-5:].contiguous())[0])


def test_distillation_past_32_bit_offsets():
    from paper_1810_10962_b200 import lm
    T, V, K = 17_000, 131072, 8                              # 2.2e9 elements
    z = torch.zeros(T, V, dtype=torch.bfloat16, device="cuda")
    tail, a, index, dloss = distill_case(5, V, K, "bf16", 63)
    z[-5:] = tail
    full = lambda t: torch.cat([t[:1].expand(T - 5, *t.shape[1:]), t]).contiguous()  # noqa: E731
    loss, dz = lm.topk_distillation_step(z, full(a), full(index), full(dloss), 2.0)
    want_loss, want_dz = lm.topk_distillation_step(tail, a, index, dloss, 2.0)
    assert torch.allclose(loss[-5:], want_loss, rtol=1e-5, atol=1e-6)
    assert torch.allclose(dz[-5:].float(), want_dz.float(), rtol=2 ** -7, atol=1e-9)


def test_head_past_32_bit_offsets():
    from paper_1810_10962_b200 import lm
    T, V, D = 8, 1_100_000, 2048                             # 2.25e9 weights
    w = torch.zeros(V, D, dtype=torch.bfloat16, device="cuda")
    g = gen(64)
    x = randn(g, T, D, dtype="bf16")
    w[-300:] = (randn(g, 300, D) * 0.05).bfloat16()
    target = torch.randint(V - 300, V, (T,), device="cuda", generator=g)
    dloss = torch.rand(T, device="cuda", generator=g) + 0.5
    loss, lse = lm.linear_cross_entropy_forward(x, w, target)
    z = x.double() @ w[-300:].double().T
    want = torch.logsumexp(torch.cat([z, torch.full((T, 1), math.log(V - 300), device="cuda", dtype=torch.float64)], 1), 1)
    assert torch.allclose(lse.double(), want, rtol=1e-5)
    at = (target - (V - 300))[:, None]
    assert torch.allclose(loss.double(), want - z.gather(1, at)[:, 0], rtol=1e-5, atol=1e-5)
    _, dw = lm.linear_cross_entropy_backward(x, w, target, lse, dloss)
    G = torch.exp(z - want[:, None]) * dloss.double()[:, None]
    G.scatter_add_(1, at, -dloss.double()[:, None])
    assert_within(dw[-300:], G.T @ x.double(), 2.0 ** -7 * (G.abs().T @ x.double().abs()) + 1e-8, "dw")
