"""The head's products over many tiles a CTA pair, every element of every output against the definition in 64 bits.

Tolerances are bounds of the arithmetic that is built, u = 2^-24 being fp32's rounding:

* A sum on the tensor cores loses at most 2 u of the terms' magnitudes with every step of 16 terms.  Where it is taken in
  segments that count ends with the segment, and every segment adds one rounding u.
* bf16 tensors: products are exact.  fp32 tensors: two fp16 terms keep a value to 2^-22 of itself, the product of the
  two low terms is dropped, another 2^-22, so that a product is right to 3 2^-22 = 12 u; those with a low term are 2^-11 of it, and
  their whole chain counts 2^-11 of its length.
* G carries the error of its logit and of the log-sum, and 2^-8 (bf16) or 2^-22 (fp32) of itself for its own rounding."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
STORE = {"f32": 2 * U, "bf16": 2.0 ** -8}
DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}


def case(T, V, D, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(T, D, device="cuda", generator=g).to(DTYPE[dtype])
    w = (torch.randn(V, D, device="cuda", generator=g) * (2 / math.sqrt(D))).to(DTYPE[dtype])
    target = torch.randint(0, V, (T,), device="cuda", generator=g)
    target[torch.rand(T, device="cuda", generator=g) < 0.1] = -100
    return x, w, target, torch.rand(T, device="cuda", generator=g) + 0.5


def chain(n, dtype, segment, parts=0):
    """What a sum of n terms may be off by, as a part of the sum of the terms' magnitudes.  `parts`: additions of a split sum's
    parts, and of pieces of the vocabulary."""
    inside = 2 * U * (min(n, segment) / 16 + 2) + U * (n / segment + 2 + parts)
    if dtype == "bf16":
        return inside
    return inside + 12 * U + 2 * 2.0 ** -11 * 2 * U * (min(n, 4096) / 16 + 2)


def within(got, want, tol, what):
    bad = ~((got.double() - want).abs() <= tol)
    if bad.any():
        at = torch.nonzero(bad)
        raise AssertionError(f"{what}: {len(at)} of {bad.numel()} off, first at {at[0].tolist()}, last at {at[-1].tolist()}, worst "
                             f"{float(((got.double() - want).abs() / tol).nan_to_num(math.inf).max()):.3g} times the bound")


def check(x, w, target, dloss, dtype, segment_z, segment_out):
    from paper_1810_10962_b200 import bns, lm
    T, D = x.shape
    V = w.shape[0]
    loss, lse = lm.linear_cross_entropy_forward(x, w, target)
    dx, dw = lm.linear_cross_entropy_backward(x, w, target, lse, dloss)
    for _ in range(3):
        again = (*lm.linear_cross_entropy_forward(x, w, target), *lm.linear_cross_entropy_backward(x, w, target, lse, dloss))
        for a, b, what in zip(again, (loss, lse, dx, dw), ("loss", "lse", "dx", "dw")):
            assert torch.equal(a, b), f"{what} differs from call to call"
    assert bns.wait_timeouts() == 0

    wd = w.double()
    # rows of dw add up over blocks of rows; 2^28 logits at a time
    want_dw = torch.zeros(V, D, device="cuda", dtype=torch.float64)
    off_dw, size_dw = torch.zeros_like(want_dw), torch.zeros_like(want_dw)
    rows = max(1, 2 ** 28 // V)
    for first in range(0, T, rows):
        part = slice(first, min(T, first + rows))
        xd = x[part].double()
        counts = target[part] >= 0
        at = target[part].clamp(min=0)[:, None]
        z = xd @ wd.T
        tz = (xd.abs() @ wd.abs().T).mul_(chain(D, dtype, segment_z))
        want_lse = torch.logsumexp(z, 1)
        q = torch.exp(z - want_lse[:, None])
        t_lse = (q * tz).sum(1) + 8 * U * (1 + want_lse.abs()) + U * (V / 64 / 16 + 64)   # sums of exponentials: by thread, strip, row
        within(lse[part], want_lse, t_lse, f"lse from row {first}")
        z_at = z.gather(1, at)[:, 0]
        want_loss = torch.where(counts, want_lse - z_at, torch.zeros_like(z_at))
        within(loss[part], want_loss, t_lse + tz.gather(1, at)[:, 0] + 8 * U * z_at.abs(), f"loss from row {first}")
        g = (dloss[part].double() * counts)[:, None]
        # of an exponential, relative: its logit, the log-sum, the exponent's rounding, 2^x to 2 ulp, the factor
        tz.add_(t_lse[:, None] + 16 * U).add_((z - want_lse[:, None]).abs_().add_(want_lse.abs()[:, None]).mul_(4 * U))
        G = q.mul_(g)
        tG = tz.mul_(G)
        G.scatter_add_(1, at, -g)
        tG.add_(G.abs().mul_(STORE["bf16"] if dtype == "bf16" else 6 * U))
        want = G @ wd
        tol = (tG @ wd.abs()) * 1.01 + (G.abs() @ wd.abs()) * chain(V, dtype, segment_out, 70) + STORE[dtype] * 1.01 * want.abs() + 1e-30
        within(dx[part], want, tol, f"dx from row {first}")
        want_dw += G.T @ xd
        off_dw += tG.T @ xd.abs()
        size_dw += G.abs().T @ xd.abs()
    within(dw, want_dw, off_dw * 1.01 + size_dw * chain(T, dtype, segment_out, 70) + STORE[dtype] * 1.01 * want_dw.abs() + 1e-30, "dw")


# Products that give a CTA pair several tiles, with a number of rows whose last tile has warps without any: rows of dw
# (vocabulary % 256 in 1 ... 224) in the first two, rows of G (rows % 256 in 1 ... 224) in the others.
@pytest.mark.parametrize("T,V,D,dtype", [(192, 50304, 2048, "bf16"), (64, 50257, 4096, "bf16"), (4000, 20000, 64, "bf16"),
                                         (4000, 20000, 64, "f32"), (700, 30000, 512, "f32")])
def test_many_tiles(T, V, D, dtype):
    check(*case(T, V, D, dtype, T + V + D), dtype, 256 if dtype == "f32" else 512, 256 if dtype == "f32" else 1 << 40)


# fp32 sums that are long enough for a lost product of terms, or for segments that are too long, to pass the bound.
@pytest.mark.parametrize("T,V,D", [(300, 3001, 4100), (1021, 8003, 1000), (140, 20000, 2048)])
def test_long_fp32_sums(T, V, D):
    check(*case(T, V, D, "f32", T + V + D), "f32", 256, 256)


# Pieces of the vocabulary whose last one has fewer stages of K than dx's sum has parts: 4097 = 4 x 1024 + 1 in four parts, and
# 61464 = 15 x 4096 + 24 in two without any setting.
@pytest.mark.parametrize("T,V,D,piece", [(200, 4097, 64, 1024), (200, 2049, 64, 512), (41979, 61464, 64, 0)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_last_piece_shorter_than_the_parts(T, V, D, piece, dtype):
    from paper_1810_10962_b200 import bns
    try:
        bns.set_tuning("head_piece", piece)
        check(*case(T, V, D, dtype, T + V), dtype, 256 if dtype == "f32" else 512, 256 if dtype == "f32" else 1 << 40)
    finally:
        bns.set_tuning("head_piece", 0)


# A row that is sure of its target has loss 0, and one that is sure of another place the difference of the two logits, at any
# size of the logits.  A logit is one product with 1: exact, or in two fp16 terms right to 2^-22 = 4 u.  The exponents come from
# multiply-adds against one rounded reference, so what is left of it is 2^x and log2 near 0: a few 2^-22.
@pytest.mark.parametrize("logit", [17.3, 100.7, 1000.3, 29997.3, 3e8])
@pytest.mark.parametrize("T,V,D", [(1, 5, 3), (4, 40000, 8), (7, 2000, 130), (32, 900, 64), (33, 900, 64), (200, 5000, 72)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_loss_of_sure_rows(T, V, D, logit, dtype):
    from paper_1810_10962_b200 import lm
    x, w = (torch.zeros(n, D, device="cuda", dtype=DTYPE[dtype]) for n in (T, V))
    x[:, 0] = 1.0
    w[:, 0] = -logit / 2
    w[3, 0] = logit
    w[1, 0] = logit / 4
    target = torch.full((T,), 3, device="cuda")
    target[::3] = 1
    loss, lse = lm.linear_cross_entropy_forward(x, w, target)
    z = w[:, 0].double()
    want = torch.logsumexp(z, 0)
    terms = 4 * U if dtype == "f32" else 0
    assert bool(((lse.double() - want).abs() <= (4 * U + terms) * want.abs()).all())
    off = (loss.double() - (want - z[target])).abs()
    tol = 8 * 2.0 ** -22 + 8 * U * (want - z[target]).abs() + terms * torch.where(target == 3, 0.0, want.abs() + z[target].abs())
    assert bool((off <= tol).all()), f"{float((off / tol).max()):.3g} times the bound, loss off by {float(off.max()):.3g}"


# The gradient's logits are the statistics' logits, bit for bit, so that the gradient of a sure row vanishes like 1 - p and does
# not carry what the tensor cores lose of a logit (5e-4 of one at 60 and width 4096).  What is left of z - lse: the rounding of
# the log-sum, and that of two constants whose product is 1 up to u.
@pytest.mark.parametrize("T,V,D", [(100, 2500, 4096), (300, 2500, 4096), (300, 700, 1000), (9, 1500, 4096)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gradient_of_sure_rows(T, V, D, dtype):
    from paper_1810_10962_b200 import lm
    g = torch.Generator(device="cuda").manual_seed(T + D)
    w = (torch.randn(V, D, device="cuda", generator=g) * 0.02).to(DTYPE[dtype])
    target = torch.randperm(V, device="cuda", generator=g)[:T]
    x = (w[target].float() * (60 / w[target].float().square().sum(1, keepdim=True))).to(DTYPE[dtype])
    dloss = torch.ones(T, device="cuda")
    loss, lse = lm.linear_cross_entropy_forward(x, w, target)
    dx, dw = lm.linear_cross_entropy_backward(x, w, target, lse, dloss)
    z = x.double() @ w.double().T
    q = torch.softmax(z, 1)
    assert float(q.gather(1, target[:, None]).min()) > 1 - 1e-12
    G = q.scatter_add(1, target[:, None], -torch.ones(T, 1, device="cuda", dtype=torch.float64))
    tG = torch.zeros_like(G).scatter_(1, target[:, None], 6 * U * z.amax(1, keepdim=True) + 16 * U)
    for got, want, tol, what in ((dx, G @ w.double(), tG @ w.double().abs(), "dx"), (dw, G.T @ x.double(), tG.T @ x.double().abs(), "dw")):
        within(got, want, 1.02 * tol + 1e-12, what)


# The four places where the gradient call looks at its targets: few fp32 rows, the products' own warps, a kernel before them (over
# 1024 rows), and no rows at all.
@pytest.mark.parametrize("T,dtype", [(5, "f32"), (16, "f32"), (17, "f32"), (40, "bf16"), (1024, "bf16"), (1025, "bf16"), (3000, "f32")])
@pytest.mark.parametrize("int64", [True, False])
def test_gradient_call_tells_of_bad_targets(T, dtype, int64):
    from paper_1810_10962_b200 import bns, lm
    V, D = 300, 64
    x, w, target, dloss = case(T, V, D, dtype, 3)
    target = target if int64 else target.int()
    _, lse = lm.linear_cross_entropy_forward(x, w, target)
    workspace = torch.full((lm.linear_cross_entropy_workspace_bytes(x, w, target, backward=True),), 0xAB, dtype=torch.uint8, device="cuda")
    lm.linear_cross_entropy_backward(x, w, target, lse, dloss, workspace=workspace)
    assert bns.workspace_status(workspace) == 0
    for place in (0, T - 1, T // 2):
        bad = target.clone()
        bad[place] = V
        dx, _ = lm.linear_cross_entropy_backward(x, w, bad, lse, dloss, workspace=workspace)
        assert bns.workspace_status(workspace) == lm.FLAG_BAD_TARGET
        assert bool((dx[place] == 0).all())
    lm.linear_cross_entropy_backward(x[:0], w, target[:0], lse[:0], dloss[:0], workspace=workspace)
    assert bns.workspace_status(workspace) == 0
