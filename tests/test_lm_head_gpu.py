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


def chain(n, dtype, segment):
    """What a sum of n terms may be off by, as a part of the sum of the terms' magnitudes."""
    inside = 2 * U * (min(n, segment) / 16 + 2) + U * (n / segment + 70)     # 70: parts of a split sum, pieces
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

    xd, wd = x.double(), w.double()
    counts = target >= 0
    at = target.clamp(min=0)[:, None]
    z = xd @ wd.T
    tz = (xd.abs() @ wd.abs().T).mul_(chain(D, dtype, segment_z))
    want_lse = torch.logsumexp(z, 1)
    q = torch.exp(z - want_lse[:, None])
    t_lse = (q * tz).sum(1) + 8 * U * (1 + want_lse.abs()) + U * (V / 64 / 16 + 64)       # sums of exponentials: by thread, strip, row
    within(lse, want_lse, t_lse, "lse")
    z_at = z.gather(1, at)[:, 0]
    want_loss = torch.where(counts, want_lse - z_at, torch.zeros_like(z_at))
    within(loss, want_loss, t_lse + tz.gather(1, at)[:, 0] + 8 * U * z_at.abs(), "loss")
    g = (dloss.double() * counts)[:, None]
    # of an exponential, relative: its logit, the log-sum, the exponent's rounding, 2^x to 2 ulp, the factor
    tz.add_(t_lse[:, None] + 16 * U).add_((z - want_lse[:, None]).abs_().add_(want_lse.abs()[:, None]).mul_(4 * U))
    G = q.mul_(g)
    tG = tz.mul_(G)
    G.scatter_add_(1, at, -g)
    tG.add_(G.abs().mul_(STORE["bf16"] if dtype == "bf16" else 6 * U))
    for A, tA, B, n, got, what in ((G, tG, wd, V, dx, "dx"), (G.T, tG.T, xd, T, dw, "dw")):
        want, size, off = A @ B, A.abs() @ B.abs(), tA @ B.abs()
        within(got, want, off * 1.01 + size * chain(n, dtype, segment_out) + STORE[dtype] * 1.01 * want.abs() + 1e-30, what)


# Products that give a CTA pair several tiles, with a number of rows whose last tile has warps without any: rows of dw
# (vocabulary % 256 in 1 ... 224) in the first two, rows of G (rows % 256 in 1 ... 224) in the others.
@pytest.mark.parametrize("T,V,D,dtype", [(192, 50304, 2048, "bf16"), (64, 50257, 4096, "bf16"), (4000, 20000, 64, "bf16"),
                                         (4000, 20000, 64, "f32"), (700, 30000, 512, "f32")])
def test_many_tiles(T, V, D, dtype):
    segment_z = 256 if dtype == "f32" else max(D, 512)          # bf16 gradient: one sum over the width
    check(*case(T, V, D, dtype, T + V + D), dtype, segment_z, 256 if dtype == "f32" else 1 << 40)
