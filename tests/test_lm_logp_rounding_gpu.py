"""Token log probabilities with bounds from the kernels' own roundings, whatever a row's common part is.

u = 2^-24 is fp32's rounding, L = log q, d = the distance to the largest logit over the temperature.  Exponents are
z c - m by one multiply-add, with c rounded once and m, the rounded reference, which is off its logit by rho = u |z| log2(e) / tau
at the most:
* a term 2^(z c - m) of either sum is good to 4 u (2^x, two ulp), the exponent's rounding u (d + rho), and as much again where the reference moves;
* a thread adds up V / 256 terms in a row at the most, some 20 joins follow: es = u (4 + 2 E[d] + 2 rho + V / 256 + 20) for the
  sum s, and as much relative to E[d] + rho for the weighted sum t;
* log2 s - t / s: two ulp of the first, which is H + rho at the most, a division, a difference and a product;
* c's own rounding is a temperature off by u, which moves the entropy by u Var L."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
STORE = {torch.float32: U, torch.bfloat16: 2.0 ** -8}
TYPES = [torch.bfloat16, torch.float32]


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


class Exact:
    """A row's values in 64 bits, differences to the largest logit first, and the allowances above."""

    def __init__(self, z, tau):
        tau = float(torch.tensor(tau, dtype=torch.float32))
        zd = z.double()
        most = zd.amax(1, keepdim=True)
        d = (most - zd) / tau
        logs = torch.logsumexp(-d, 1, keepdim=True)
        self.lse = (most / tau + logs)[:, 0]
        self.logq = -d - logs
        self.q = self.logq.exp()
        weighted = lambda x: torch.where(self.q > 0, self.q * x, 0.0).sum(1)  # noqa: E731
        self.entropy = -weighted(self.logq)
        self.rho = U * torch.where(d < 300, zd.abs(), 0.0).amax(1) * 1.4427 / tau       # of what counts
        distance = weighted(d) + self.rho
        self.of_sum = U * (24 + 2 * distance + z.shape[1] / 256)
        self.of_entropy = self.of_sum * (1 + 2 * distance) + U * (8 * distance + 4 * (self.entropy + self.rho) + weighted(self.logq.square()))


def within(got, want, tol, what):
    off = (got.double() - want).abs()
    bad = ~(off <= tol)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {float((off / tol).nan_to_num(math.inf).max()):.3g} times the bound"


# --------------------------------------------------------------------------------------------- entropy
@pytest.mark.parametrize("top", [0.0, 10.0, 1e3, -1e4, 1e5, 1e6, 1e7, -1e8, 1.5e8])
@pytest.mark.parametrize("V", [5, 37])
@pytest.mark.parametrize("dtype", TYPES)
def test_entropy_wherever_the_largest_logit_lies(dtype, V, top):
    """Each place of a row in turn, inside 16-byte vectors and outside, by itself far above the others and a little above."""
    from paper_1810_10962_b200 import lm
    below = (torch.arange(V, device="cuda") % 4).float()
    for others in (below - abs(top), top - 1 - below / 2):
        z = others.repeat(V, 1).fill_diagonal_(top).to(dtype)
        token = torch.zeros(V, dtype=torch.int64, device="cuda")
        want = Exact(z, 1.0)
        for got in (lm.token_log_probs_forward(z, token)[1], lm.token_log_probs_forward_top(z, token, 3)[1]):
            within(got, want.entropy, want.of_entropy, "entropy")


@pytest.mark.parametrize("tau", [1.0, 0.7])
@pytest.mark.parametrize("shift", [0.0, 300.0, -5000.0, 1e5, 1e7])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,V", [(40, 1003), (3, 9001), (2, 50257)])
def test_entropy_of_rows_with_a_common_part(T, V, dtype, shift, tau):
    from paper_1810_10962_b200 import lm
    z = (torch.randn(T, V, device="cuda", generator=gen(3 + V)) * 2 + shift).to(dtype)
    want = Exact(z, tau)
    entropy = lm.token_log_probs_forward(z, torch.zeros(T, dtype=torch.int64, device="cuda"), tau)[1]
    within(entropy, want.entropy, want.of_entropy, "entropy")


# --------------------------------------------------------------------------------------------- the gradient's probabilities
@pytest.mark.parametrize("tau", [0.05, 0.7, 1.0, 1.2, 1.3, 1.7])
def test_probabilities_of_the_gradient_add_up(tau):
    """With a gradient of -1 for one token's log probability the row of dlogits adds up to (sum of q - 1) / tau.  q comes from the
    log-sum, which is rounded once (u |lse|); 2^x, the exponent and the store take their roundings in either call."""
    from paper_1810_10962_b200 import lm
    T, V = 4096, 100
    g = gen(7)
    z = (torch.randn(T, V, device="cuda", generator=g) * 2 + 100 + 145 * torch.rand(T, 1, device="cuda", generator=g)) * tau
    token = z.argmin(1)
    want = Exact(z, tau)
    _, entropy, lse = lm.token_log_probs_forward(z, token, tau)
    assert float(lse.min()) > 64 and float(lse.max()) < 256
    dz = lm.token_log_probs_backward(z, token, lse, entropy, torch.full((T,), -1.0, device="cuda"), None, tau)
    distance = want.entropy - want.logq.amax(1)          # no less than E[d]
    within(dz.double().sum(1) * tau, torch.zeros_like(want.lse), want.of_sum + U * (want.lse.abs() + 12 + 2 * distance), "sum of q - 1")


KEPT = {torch.float32: 2.0 ** 8, torch.bfloat16: 2.0 ** 12}


def check_gradient(z, tau, seed, with_entropy=True):
    """The gradient in 64 bits.  q is off by the log-sum's errors, 2^x, and roundings of the exponent's size; beyond KEPT the sum is found again
    and the log-sum's rounding does not come in.  What multiplies q has the size of its terms and the entropy's error."""
    from paper_1810_10962_b200 import lm
    T, V = z.shape
    g = gen(seed)
    token = torch.randint(0, V, (T,), device="cuda", generator=g)
    token[::3] = z[::3].argmax(1)
    token[1::7] = -100
    dlogp, dentropy = torch.randn(T, device="cuda", generator=g), torch.randn(T, device="cuda", generator=g)
    logp, entropy, lse = lm.token_log_probs_forward(z, token, tau)
    got = lm.token_log_probs_backward(z, token, lse, entropy if with_entropy else None, dlogp, dentropy if with_entropy else None, tau)
    want, tau = Exact(z, tau), float(torch.tensor(tau, dtype=torch.float32))
    given = token >= 0
    one = torch.zeros(T, V, dtype=torch.bool, device="cuda")
    one[given, token[given]] = True
    a, b = (dlogp.double() * given)[:, None], dentropy.double()[:, None] * with_entropy
    L, H, q = torch.where(want.q > 0, want.logq, 0.0), want.entropy[:, None], want.q
    exact = (a * (one.double() - q) - b * q * (L + H)) / tau
    distance = want.entropy - want.logq.amax(1) + want.rho
    rounded = torch.where(want.lse.abs() < KEPT[z.dtype], want.lse.abs(), 0.0)
    of_q = (want.of_sum + U * (8 + 4 * distance + rounded))[:, None] + U * (4 * L.abs() + (L + H).abs())
    a, b = a.abs(), b.abs()
    size = a * (one.double() + q) + b * q * (L.abs() + H + 1)
    bound = (q * of_q * (a + b * (L + H).abs()) + b * q * (of_q + want.of_entropy[:, None]) + 6 * U * size) / tau
    lost = 2.0 ** -126 * (a + b * (want.logq.nan_to_num(0.0, 0.0, 0.0).abs() + H + 1)) / tau      # 2^x below 2^-126 is 0
    within(got, exact, bound + STORE[z.dtype] * exact.abs() + 2 * lost, "dlogits")


def normal_rows(T, V, seed, spread=2.0):
    return torch.randn(T, V, device="cuda", generator=gen(seed)) * spread


# a row's blocks all at once, and more of them than run at a time; rows at any phase, their tails in the first block or in another one
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,V", [(2, 131075), (300, 131075), (700, 70001), (650, 131072), (5, 300), (3, 9001)])
def test_gradient_of_rows_whose_sum_is_found_again(T, V, dtype):
    """Every other row has a log-sum beyond KEPT, in either direction."""
    z = normal_rows(T, V, 11 + V)
    z[::2] += KEPT[dtype] * 1.5
    z[::4] -= KEPT[dtype] * 3.5
    check_gradient(z.to(dtype), 1.0, 13)


def test_gradient_of_rows_whose_sum_is_found_again_takes_its_share_of_time():
    """Three passes over a row that is read once as a rule, whatever its length: not one for each of its blocks."""
    from paper_1810_10962_b200 import lm
    T, V = 600, 131072
    z, token, one = normal_rows(T, V, 15), torch.zeros(T, dtype=torch.int64, device="cuda"), torch.ones(T, device="cuda")
    times = []
    for shift in (0.0, 400.0):
        lse = lm.token_log_probs_forward(z + shift, token)[2]
        moved, best = z + shift, math.inf
        for _ in range(6):
            start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            start.record()
            lm.token_log_probs_backward(moved, token, lse, None, one)
            end.record()
            end.synchronize()
            best = min(best, start.elapsed_time(end))
        times.append(best)
    assert times[1] < 6 * times[0], times


# --------------------------------------------------------------------------------------------- all outputs
def check_forward(z, tau, K):
    """log q is (z c - m) - log2 s times ln 2: roundings of the size of both, the sum's error, and c's own rounding, which moves it by
    u |L + H|; the log-sum is rounded once, and c's rounding moves it by u |z| / tau."""
    from paper_1810_10962_b200 import lm
    T, V = z.shape
    token = torch.randint(0, V, (T,), device="cuda", generator=gen(V))
    token[::3] = z[::3].argmax(1)
    want = Exact(z, tau)
    distance = want.entropy - want.logq.amax(1) + want.rho
    of_log = lambda L: (want.of_sum + 4 * U * distance)[:, None] + U * (6 * L.abs() + (L + want.entropy[:, None]).abs())  # noqa: E731
    given = want.logq.gather(1, token[:, None])
    of_lse = want.of_sum + U * (want.lse.abs() + 4 * distance + 1) + want.rho
    *first, top, index = lm.token_log_probs_forward_top(z, token, K, tau)
    at = torch.sort(z.float(), dim=1, descending=True, stable=True).indices[:, :K]
    assert torch.equal(index.long(), at)
    within(top, want.logq.gather(1, at), of_log(want.logq.gather(1, at)), "alternatives")
    for got in (first, lm.token_log_probs_forward(z, token, tau)):
        within(got[0], given[:, 0], of_log(given)[:, 0], "logprob")
        within(got[1], want.entropy, want.of_entropy, "entropy")
        within(got[2], want.lse, of_lse, "lse")


# one to eight blocks a row, each number of threads, short rows and rows without a vector, odd lengths
@pytest.mark.parametrize("tau", [1.0, 0.6])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,V,K", [(1, 1, 1), (3, 7, 5), (4, 100, 64), (400, 1003, 7), (700, 130, 64), (3, 4099, 33), (37, 50257, 10), (140, 32768, 1),
                                   (320, 20001, 20), (310, 65537, 3), (1, 131072, 20), (2, 300001, 64), (1300, 9001, 5)])
def test_ordinary_rows(T, V, K, dtype, tau):
    z = normal_rows(T, V, 17 + T + V)
    z[:, V // 2] += 4
    check_forward(z.to(dtype), tau, K)
    check_gradient(z.to(dtype), tau, 19)
    check_gradient(z.to(dtype), tau, 19, with_entropy=False)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shift", [-3000.0, 300.0, 3700.0, 5000.0, 1e5, 3e6])
def test_a_common_part_costs_the_gradient_nothing(shift, dtype):
    """At a temperature of 16.  A log-sum's own rounding, 2^-12 for a shift of 1e5 and 2^-7 for one of 3e6, would be twenty times the bound and more."""
    z = (normal_rows(5, 9001, 23, 32.0) + shift).to(dtype)
    check_forward(z, 16.0, 4)
    check_gradient(z, 16.0, 29)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tau", [0.01, 0.1, 30.0])
def test_sharp_and_flat_distributions(tau, dtype):
    z = normal_rows(40, 9001, 31).to(dtype)
    check_forward(z, tau, 9)
    check_gradient(z, tau, 37)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("mask", [-math.inf, -1e30, -1e9])
def test_masked_places_beside_ordinary_ones(mask, dtype):
    from paper_1810_10962_b200 import lm
    z = normal_rows(30, 9001, 41)
    z[torch.rand(30, 9001, device="cuda", generator=gen(43)) < 0.9] = mask
    check_gradient(z.to(dtype), 0.7, 47)
    want, got = Exact(z.to(dtype), 0.7), lm.token_log_probs_forward(z.to(dtype), z.argmax(1), 0.7)
    within(got[1], want.entropy, want.of_entropy, "entropy")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T", [296, 297, 443, 444])
@pytest.mark.parametrize("V,K", [(32767, 3), (32768, 1), (65535, 20), (65536, 64), (98305, 2)])
def test_where_the_number_of_threads_changes(T, V, K, dtype):
    z = normal_rows(T, V, 53 + T + V).to(dtype)
    check_forward(z, 1.0, K)
