"""Distillation: rows that go over the blocks of a cluster, against the definition in 64 bits."""
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def want_of(z, teacher, index, dloss, tau):
    zd = z.double() / tau
    lse = torch.logsumexp(zd, 1)
    logp = torch.log_softmax(teacher.double() / tau, 1)
    p, at = logp.exp(), index.long()
    logq = zd.gather(1, at) - lse[:, None]
    loss = tau * tau * (p * (logp - logq)).sum(1)
    size = tau * tau * (p * (logp.abs() + logq.abs() + 1)).sum(1)
    q = torch.softmax(zd, 1)
    share = torch.zeros_like(q).scatter_add_(1, at, p)
    scale = (dloss.double() * tau)[:, None]
    return loss, size, lse, (q - share) * scale, (q + share) * scale


# rows -> blocks a row on 148 SMs: 8, 8, 7, 5, 3, 2 (by the few rows), 2 (step, by the rows' length)
@pytest.mark.parametrize("T", [1, 37, 42, 57, 90, 140, 700])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_over_a_cluster(T, dtype):
    from paper_1810_10962_b200 import lm
    V, K, tau = 131072 + 5, 24, 2.0
    g = torch.Generator(device="cuda").manual_seed(500 + T)
    z = (torch.randn(T, V, device="cuda", generator=g) * 2).to(dtype)
    teacher = torch.randn(T, K, device="cuda", generator=g) * 2
    index = torch.randint(0, V, (T, K), device="cuda", generator=g)
    dloss = torch.rand(T, device="cuda", generator=g) + 0.5
    loss, lse = lm.topk_distillation_forward(z, teacher, index, tau)
    step_loss, dz = lm.topk_distillation_step(z, teacher, index, dloss, tau)
    for _ in range(10):
        again = (*lm.topk_distillation_forward(z, teacher, index, tau), *lm.topk_distillation_step(z, teacher, index, dloss, tau))
        assert all(torch.equal(a, b) for a, b in zip(again, (loss, lse, step_loss, dz)))
    want, size, want_lse, want_dz, size_dz = want_of(z, teacher, index, dloss, tau)
    # exponents of some 20: a multiply-add each, 2^x to 2 ulp; sums of V / 1024 exponentials in a row in a thread, then joins
    ue = 4 * U * 24 + U * (V / 1024 + 32)
    assert bool(((lse.double() - want_lse).abs() <= ue + 4 * U * want_lse.abs()).all())
    for got in (loss, step_loss):
        assert bool(((got.double() - want).abs() <= (2 * ue + 16 * U) * size).all())
    assert bool(((dz.double() - want_dz).abs() <= 2 * ue * size_dz + (2.0 ** -8 if dtype == torch.bfloat16 else 2 * U) * want_dz.abs() + 1e-37).all())
