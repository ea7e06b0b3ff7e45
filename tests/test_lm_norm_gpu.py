"""The norm's 8-bit output at the ends of fp32's range."""
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def e4m3(v):
    _, e = torch.frexp(v)
    quantum = torch.ldexp(torch.ones_like(v), (e - 1).clamp(min=-6) - 3)
    return torch.round(v / quantum) * quantum


# |s w| of a group, whose reciprocal the quantisation takes, from 2^-120 to the largest that fp32 holds
@pytest.mark.parametrize("size", [2.0 ** -120, 2.0 ** -101, 2.0 ** -99, 1.0, 2.0 ** 99, 2.0 ** 101, 2.0 ** 125, 2.0 ** 126, 1.5 * 2.0 ** 126, 1.9 * 2.0 ** 127])
@pytest.mark.parametrize("D", [256, 250, 20000])
@pytest.mark.parametrize("group", [0, 128])
def test_groups_of_any_size(size, D, group):
    from paper_1810_10962_b200 import lm
    g = torch.Generator(device="cuda").manual_seed(9)
    # the rows' part is 2^40 for the large ones, so that their squares add up within fp32, and y = s rstd w is finite
    part = 2.0 ** 40 if size > 2.0 ** 60 else 1.0
    s = torch.randint(-64, 65, (3, D), device="cuda", generator=g) / 64.0
    s[:, ::100] = 1.0
    x = (s * part).float()
    w = torch.full((D,), size / part, device="cuda", dtype=torch.float64).float()
    assert bool(w.isfinite().all())
    q, scales, _, rstd = lm.rms_norm_forward_fp8(x, None, w, 1e-5, group=group)
    xd = x.double()
    y = xd / torch.sqrt((xd * xd).mean(1, keepdim=True) + 1e-5) * w.double()
    width = group or D
    n = -(-D // width)
    amax = torch.nn.functional.pad(y, (0, n * width - D)).view(3, n, width).abs().amax(2)
    # squares: at most ceil(D / 1024) + 16 in a row in a thread, ten joins; then the root, the scale's two products
    u = (D / 1024 + 16 + 10 + 8 + 6) * U
    assert bool(((scales.double() - amax / 448).abs() <= u * amax / 448).all())
    # half a step of the 8-bit grid; ties, of which 64ths of the largest value have some, may go either way by y's rounding
    want = y / (amax / 448).repeat_interleave(width, 1)[:, :D]
    got = q.double()
    assert bool(((got - want).abs() <= torch.maximum(want.abs() * 2.0 ** -4, torch.full_like(want, 2.0 ** -10)) * (1 + 1e-5)).all())
    assert float((got != e4m3(want)).double().mean()) < 0.1 and float(got.abs().max()) == 448
