"""The distillation's gradient takes q from the forward call's log-sum, which is rounded once: q is off by u |lse|, u = 2^-24, beside 2^x in
either call (two ulp), the exponents' roundings and the sum's."""
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.mark.parametrize("tau", [0.05, 0.7, 1.0, 1.2, 1.3, 1.7])
def test_probabilities_of_the_gradient_add_up(tau):
    """One entry a row: its share is 1, and the row of dlogits adds up to dloss tau (sum of q - 1)."""
    from paper_1810_10962_b200 import lm
    T, V = 4096, 100
    g = torch.Generator(device="cuda").manual_seed(7)
    z = (torch.randn(T, V, device="cuda", generator=g) * 2 + 100 + 145 * torch.rand(T, 1, device="cuda", generator=g)) * tau
    index, teacher = z.argmin(1, keepdim=True), torch.zeros(T, 1, device="cuda")
    loss, lse = lm.topk_distillation_forward(z, teacher, index, tau)
    exact = float(torch.tensor(tau, dtype=torch.float32))
    d = (z.double() - z.double().amax(1, keepdim=True)) / exact
    logq = d.log_softmax(1)
    want = (z.double() / exact).logsumexp(1)
    rho = U * z.double().abs().amax(1) * 1.4427 / exact
    distance = -(logq.exp() * d).sum(1) + rho
    of_sum = U * (24 + 2 * distance + V / 256)
    # c's own rounding is a temperature off by u, which moves the log-sum by u |z| / tau
    assert bool(((lse.double() - want).abs() <= of_sum + U * (want.abs() + 4 * distance + 1) + rho).all())
    dz = lm.topk_distillation_backward(z, teacher, index, lse, torch.full((T,), 1 / exact, device="cuda"), tau)
    off = dz.double().sum(1).abs()
    assert bool((off <= of_sum + U * (want.abs() + 12 + 2 * distance)).all()), float((off / (of_sum + U * (want.abs() + 12 + 2 * distance))).max())
    _, step = lm.topk_distillation_step(z, teacher, index, torch.full((T,), 1 / exact, device="cuda"), tau)
    assert bool((step.double().sum(1).abs() <= of_sum + U * (12 + 2 * distance)).all())
