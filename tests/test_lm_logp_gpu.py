"""Log probabilities of given tokens, entropy, alternatives and the logits' gradient against their definitions in 64 bits.

u = 2^-24 is fp32's rounding.  Exponents are a multiply-add each of a constant rounded once (four roundings of their
magnitude at the most, the reference's among them), 2^x is good to two ulp, a thread adds up V / 1024 terms in each of two
sums in a row at the most, and some 64 joins follow."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
STORE = {torch.float32: U, torch.bfloat16: 2.0 ** -8}
TYPES = [torch.bfloat16, torch.float32]


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def case(T, V, dtype, seed, none=0.2):
    g = gen(seed)
    z = torch.randn(T, V, device="cuda", generator=g) * 2
    token = torch.randint(0, V, (T,), device="cuda", generator=g)
    z[torch.arange(T, device="cuda"), token] += 4
    token[torch.rand(T, device="cuda", generator=g) < none] = -100
    return z.to(dtype), token, torch.randn(T, device="cuda", generator=g), torch.randn(T, device="cuda", generator=g)


def want_of(z, token, tau):
    """(logprob, entropy, lse, log q) in 64 bits."""
    zd = z.double() / tau
    most = zd.amax(1, keepdim=True)
    rest = zd - torch.where(most == -math.inf, 0.0, most)      # first: 3e20 has a step of 65536 in 64 bits
    logs = torch.logsumexp(rest, 1)
    lse, logq = most[:, 0] + logs, rest - logs[:, None]
    q = logq.exp()
    entropy = -torch.where(q > 0, q * logq, torch.zeros_like(q)).sum(1)
    given = (token >= 0) & (token < z.shape[1])
    logp = torch.where(given, logq.gather(1, token.long().clamp(0, z.shape[1] - 1)[:, None])[:, 0], torch.zeros_like(lse))
    return logp, entropy, lse, logq


def gradient_of(z, token, dlogp, dentropy, tau):
    """(dlogits, the sum of its terms' magnitudes) in 64 bits."""
    _, entropy, _, logq = want_of(z, token, tau)
    q = logq.exp()
    one = torch.zeros_like(q)
    given = (token >= 0) & (token < z.shape[1])
    one[given, token.long()[given]] = 1
    g = (dlogp.double() * given)[:, None]
    h = 0 * g if dentropy is None else dentropy.double()[:, None]
    L = torch.where(q > 0, logq, torch.zeros_like(q))
    want = (g * (one - q) - h * q * (L + entropy[:, None])) / tau
    size = (g.abs() * (one + q) + h.abs() * q * (L.abs() + entropy[:, None] + 1)) / tau
    return want, size


def reach(z, tau):
    """Largest exponent of two that counts in a row, and the allowance for sums and exponents that goes with it."""
    counts = z.isfinite() & (z.float() > -1e9)              # masks are held to their own size
    finite = torch.where(counts, z.double().abs(), torch.zeros_like(z, dtype=torch.float64))
    r = finite.amax(1) * 1.4427 / tau + 40
    return r, U * (4 * r + z.shape[1] / 1024 + 64)


def within(got, want, tol, what):
    off = (got.double() - want).abs()
    # what lies outside fp32's range, a mask of -3.4e38 over a temperature of 0.5 say, is -inf in fp32
    bad = ~((off <= tol) | (got == want.float()))
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {float((off / tol).nan_to_num(math.inf).max()):.3g} times the bound"


def check(z, token, dlogp, dentropy, tau, K):
    from paper_1810_10962_b200 import lm
    logp, entropy, lse, logq = want_of(z, token, tau)
    r, ue = reach(z, tau)
    results = [lm.token_log_probs_forward(z, token, tau)]
    if K:
        *first, top, index = lm.token_log_probs_forward_top(z, token, K, tau)
        results.append(first)
        at = torch.sort(z.float(), dim=1, descending=True, stable=True).indices[:, :K]
        assert torch.equal(index.long(), at)
        assert index.dtype == torch.int32
        best = logq.gather(1, at)
        within(top, best, 2 * ue[:, None] + torch.where(best < -1e9, -4 * U * best, 0.0), "alternatives")
    for got in results:
        within(got[0], logp, 2 * ue + torch.where(logp < -1e9, -4 * U * logp, 0.0), "logprob")
        within(got[1], entropy, 2 * ue * (1 + r), "entropy")      # log s and t / s, each of a size up to r
        within(got[2], lse, 2 * ue, "lse")
    if dlogp is not None:
        dz = lm.token_log_probs_backward(z, token, results[0][2], results[0][1], dlogp, dentropy, tau)
        want, size = gradient_of(z, token, dlogp, dentropy, tau)
        assert dz.dtype == z.dtype and dz.shape == z.shape
        # the log-sum's and the entropy's own allowances come in once more
        # and 2^x below 2^-126 is 0: a probability that small is lost with all that multiplies it
        spread = torch.where(logq == -math.inf, 0.0, logq.abs()) + entropy[:, None] + 1
        lost = 2.0 ** -126 * (dlogp.abs()[:, None] + (0 if dentropy is None else dentropy.abs()[:, None]) * spread) / tau
        within(dz, want, 8 * ue[:, None] * (1 + r[:, None]) * size + STORE[z.dtype] * want.abs() + 2 * lost, "dlogits")


# one to eight blocks a row, short rows in small blocks, rows shorter than a vector, odd lengths
SIZES = [(1, 1, 1), (2, 2, 2), (3, 7, 5), (4, 100, 64), (5, 63, 63), (1, 1000, 20), (3, 4099, 33), (400, 1000, 7), (700, 130, 64), (1, 131072, 20),
         (1, 131077, 64), (37, 50257, 10), (90, 65537, 5), (140, 32768, 1), (320, 20001, 20), (2, 300001, 64), (1, 4096, 64), (2, 4104, 40)]


@pytest.mark.parametrize("tau", [1.0, 0.6])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,V,K", SIZES)
def test_log_probs(T, V, K, dtype, tau):
    z, token, dlogp, dentropy = case(T, V, dtype, 7 + T + V)
    check(z, token, dlogp, dentropy, tau, K)


@pytest.mark.parametrize("dtype", TYPES)
def test_without_entropy_gradient_and_narrow_tokens(dtype):
    from paper_1810_10962_b200 import lm
    z, token, dlogp, _ = case(9, 5003, dtype, 3)
    check(z, token.int(), dlogp, None, 1.0, 3)
    lse = lm.token_log_probs_forward(z, token)[2]
    a = lm.token_log_probs_backward(z, token, lse, None, dlogp)
    b = lm.token_log_probs_backward(z, token.int(), lse, None, dlogp, None, 1.0)
    assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pad,offset", [(0, 1), (1, 0), (8, 0), (3, 5)])
def test_strided_rows_and_odd_addresses(pad, offset, dtype):
    z, token, dlogp, dentropy = case(6, 9001, dtype, 5)
    room = torch.full((6 * (9001 + pad) + offset + 16,), 1e4, dtype=dtype, device="cuda")
    view = room[offset: offset + 6 * (9001 + pad)].view(6, 9001 + pad)[:, :9001]
    view.copy_(z)
    check(view, token, dlogp, dentropy, 1.0, 12)


def test_leading_dimensions():
    from paper_1810_10962_b200 import lm
    row, place = torch.randn(700, device="cuda", generator=gen(9)), torch.tensor(5, device="cuda")
    one = lm.token_log_probs_forward_top(row, place, 2)
    assert one[0].shape == () and one[3].shape == (2,)
    assert all(torch.equal(a, b[0]) for a, b in zip(one, lm.token_log_probs_forward_top(row[None], place[None], 2)))
    assert lm.token_log_probs_backward(row, place, one[2], one[1], one[0], one[1]).shape == (700,)
    z, token, _, _ = case(6, 500, torch.float32, 8)
    flat = lm.token_log_probs_forward_top(z, token, 4)
    for got, want in zip(lm.token_log_probs_forward_top(z.view(2, 3, 500), token.view(2, 3), 4), flat):
        assert got.shape[:2] == (2, 3) and torch.equal(got.reshape(want.shape), want)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,V", [(1, 131072), (300, 20000), (2, 700)])
def test_masked_vocabulary(T, V, dtype):
    """Fewer places left than alternatives: the masked ones follow, lowest place first, with log probability -inf."""
    z, token, dlogp, dentropy = case(T, V, dtype, 11)
    keep = torch.zeros(T, V, dtype=torch.bool, device="cuda")
    keep[:, [3, V // 2, V - 1]] = True
    token[token >= 0] = V // 2
    check(z.masked_fill(~keep, -math.inf), token, dlogp, dentropy, 1.0, 20)
    check(z.masked_fill(~keep, -1e30), token, dlogp, dentropy, 1.0, 20)
    check(z.masked_fill(~keep, torch.finfo(dtype).min), token, dlogp, dentropy, 0.5, 20)


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_at_the_types_lowest_value(dtype):
    """At a temperature below 1 the log-sum leaves fp32's range; the probabilities are all the same, and so is the gradient."""
    from paper_1810_10962_b200 import lm
    z = torch.full((2, 4000), torch.finfo(dtype).min, dtype=dtype, device="cuda")
    token, one = torch.tensor([7, -1], device="cuda"), torch.ones(2, device="cuda")
    logp, entropy, lse, top, index = lm.token_log_probs_forward_top(z, token, 3, 0.5)
    log = math.log(4000)
    assert abs(float(logp[0]) + log) < 1e-5 and logp[1] == 0 and bool(((entropy - log).abs() < 1e-5).all())
    assert index.tolist() == [[0, 1, 2]] * 2 and bool(((top + log).abs() < 1e-5).all())
    dz = lm.token_log_probs_backward(z, token, lse, entropy, one, one, 0.5)
    want = torch.full((2, 4000), -1 / 4000 / 0.5, device="cuda", dtype=torch.float64)
    want[0, 7] += 2
    want[1] = 0
    # log q + H is zero but for the rounding of both, some 2e-6
    assert bool(((dz.double() - want).abs() <= STORE[dtype] * want.abs() + 4e-6 / 4000).all())


def test_rows_of_which_nothing_is_left():
    from paper_1810_10962_b200 import lm
    z, token, dlogp, dentropy = case(5, 3000, torch.float32, 13, none=0)
    z[1] = -math.inf
    z[3] = -math.inf
    token[3] = -1
    logp, entropy, lse, top, index = lm.token_log_probs_forward_top(z, token, 3)
    assert logp[1] == -math.inf and logp[3] == 0 and bool((entropy[[1, 3]] == 0).all()) and bool((lse[[1, 3]] == -math.inf).all())
    assert bool((top[[1, 3]] == -math.inf).all()) and index[[1, 3]].tolist() == [[0, 1, 2]] * 2
    dz = lm.token_log_probs_backward(z, token, lse, entropy, dlogp * 0 + 1, dentropy)
    assert bool((dz[3] == 0).all()) and bool((dz[1][torch.arange(3000, device="cuda") != token[1]] == 0).all())
    assert dz[1, token[1]] == 0
    rest = torch.tensor([0, 2, 4], device="cuda")
    check(z[rest], token[rest], dlogp[rest], dentropy[rest], 1.0, 3)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T", [1, 50, 400])
def test_alternatives_of_difficult_rows(T, dtype):
    """Rows where far more values reach a bound than are asked for: one value throughout, two values, rising and falling
    values, the top ones next to one another or far apart, zeros of both signs."""
    from paper_1810_10962_b200 import lm
    V = 40000
    i = torch.arange(V, device="cuda")
    rows = [torch.ones(V, device="cuda"), (i % 2).float(), i.float() / 100, -i.float() / 100, torch.where((i >= 777) & (i < 5777), 5.0 + i / 1e4, 0.0),
            torch.where(i % 512 == 3, 2.0 + (i // 512) / 64, 0.0), torch.where(i % 3 == 0, -0.0, 0.0), torch.where(i < 39990, -math.inf, -5.0),
            torch.where(i % 4096 < 8, 3.0, 1.0), -torch.ones(V, device="cuda") * 3]
    z = torch.stack([rows[r % len(rows)] for r in range(max(T, len(rows)))]).to(dtype)
    token = torch.zeros(z.shape[0], dtype=torch.int64, device="cuda")
    for first in range(0, z.shape[0], T):
        for K in (1, 20, 64):
            _, _, _, top, index = lm.token_log_probs_forward_top(z[first: first + T], token[first: first + T], K)
            at = torch.sort(z[first: first + T].float(), dim=1, descending=True, stable=True).indices[:, :K]
            assert torch.equal(index.long(), at)


@pytest.mark.parametrize("mask", [-1e10, -3e20, 1e10, -1e38])
@pytest.mark.parametrize("tau", [0.5, 2.0])
def test_far_logits(mask, tau):
    """All of a row masked with a large finite value: differences to the largest one are what counts."""
    from paper_1810_10962_b200 import lm
    z, token, dlogp, dentropy = case(4, 6000, torch.float32, 17, none=0)
    z[0] = mask
    z[2, :3000] = mask
    logp, entropy, lse, top, index = lm.token_log_probs_forward_top(z, token, 9, tau)
    want, want_entropy, want_lse, _ = want_of(z, token, tau)
    size = want.abs() + 1
    assert bool(((logp.double() - want).abs() <= 2e-5 * size).all() or (logp.double() == want).all())
    assert bool(((entropy.double() - want_entropy).abs() <= 1e-4).all())
    assert bool(((lse.double() - want_lse).abs() <= 4 * U * want_lse.abs() + 1e-5).all())
    assert torch.equal(index.long(), torch.sort(z, dim=1, descending=True, stable=True).indices[:, :9])
    dz = lm.token_log_probs_backward(z, token, lse, entropy, dlogp, dentropy, tau)
    want_dz, size = gradient_of(z, token, dlogp, dentropy, tau)
    assert bool(((dz.double() - want_dz).abs() <= 1e-4 * size + 1e-30).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shift", [-3000.0, 300.0, 5000.0, 1e5])
def test_large_log_sums(shift, dtype):
    """A row's common part takes bits from its log-sum, not from its gradient."""
    z, token, dlogp, dentropy = case(5, 9001, torch.float32, 18)
    check((z * 16 + shift).to(dtype), token, dlogp, dentropy, 16.0, 4)


def test_nan_and_infinity_travel():
    from paper_1810_10962_b200 import lm
    for dtype in TYPES:
        for bad in (math.nan, math.inf):
            z, token, dlogp, dentropy = case(3, 2000, dtype, 19, none=0)
            z[1, 1234] = bad
            logp, entropy, lse, top, index = lm.token_log_probs_forward_top(z, token, 5)
            assert bool(logp[1].isnan()) and bool(entropy[1].isnan()) and bool((~logp[[0, 2]].isnan()).all())
            assert bool(((index >= 0) & (index < 2000)).all())
            if bad != bad:
                assert bool((index[1] != 1234).all())
            dz = lm.token_log_probs_backward(z, token, lse, entropy, dlogp, dentropy)
            assert bool(dz[1].isnan().any()) and bool((~dz[[0, 2]].isnan()).all())
        z = torch.full((2, 600), math.nan, dtype=dtype, device="cuda")
        z[1, 3] = 1.0
        logp, entropy, lse, top, index = lm.token_log_probs_forward_top(z, torch.zeros(2, dtype=torch.int64, device="cuda"), 2)
        assert bool(logp.isnan().all()) and index.tolist() == [[-1, -1], [3, -1]]


def test_tokens_outside_the_vocabulary_are_none():
    from paper_1810_10962_b200 import lm
    z, token, dlogp, dentropy = case(3, 700, torch.float32, 23, none=0)
    outside = torch.tensor([700, -1, 2 ** 40], device="cuda")
    got = lm.token_log_probs_forward(z, outside)
    assert bool((got[0] == 0).all())
    dz = lm.token_log_probs_backward(z, outside, got[2], got[1], dlogp, None)
    assert bool((dz == 0).all())


@pytest.mark.parametrize("dtype", TYPES)
def test_calls_of_the_c_interface(dtype):
    """Without an entropy, and a gradient whose rows lie apart: what is between them stays."""
    import ctypes
    from paper_1810_10962_b200 import bns, lm
    T, V, pad = 5, 4003, 13
    z, token, dlogp, _ = case(T, V, dtype, 25)
    want = lm.token_log_probs_forward(z, token)
    want_dz = lm.token_log_probs_backward(z, token, want[2], None, dlogp)
    shape = lm._LogProbs(T, V, 0, lm._CODES[dtype], V, 1, 1.0)
    logp, lse = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    room = torch.full((T * (V + pad) + 1,), 7.0, dtype=dtype, device="cuda")
    stream = torch.cuda.current_stream().cuda_stream
    assert lm._load().bns_token_log_probs_forward(ctypes.byref(shape), z.data_ptr(), token.data_ptr(), logp.data_ptr(), None, lse.data_ptr(),
                                                  None, None, stream) == bns.OK
    dz = room[1:].view(T, V + pad)
    assert lm._load().bns_token_log_probs_backward(ctypes.byref(shape), z.data_ptr(), token.data_ptr(), lse.data_ptr(), None, dlogp.data_ptr(),
                                                   None, dz.data_ptr(), V + pad, stream) == bns.OK
    assert torch.equal(logp, want[0]) and torch.equal(lse, want[2]) and torch.equal(dz[:, :V], want_dz)
    assert bool((dz[:, V:] == 7).all()) and room[0] == 7


def test_same_bits_every_time_and_no_rows():
    from paper_1810_10962_b200 import lm
    z, token, dlogp, dentropy = case(40, 50257, torch.bfloat16, 29)
    want = lm.token_log_probs_forward_top(z, token, 20)
    for _ in range(10):
        assert all(torch.equal(a, b) for a, b in zip(lm.token_log_probs_forward_top(z, token, 20), want))
    got = lm.token_log_probs_forward_top(z[:0], token[:0], 20)
    assert got[3].shape == (0, 20)
    assert lm.token_log_probs_backward(z[:0], token[:0], got[2], got[1], dlogp[:0]).shape == (0, 50257)


def test_gradient_against_differences():
    from paper_1810_10962_b200 import lm
    z, token, dlogp, dentropy = case(4, 50, torch.float32, 31, none=0)
    tau, step = 1.5, 2.0 ** -6

    def value(z):
        logp, entropy, _ = lm.token_log_probs_forward(z, token, tau)
        return float((logp.double() * dlogp.double() + entropy.double() * dentropy.double()).sum())

    _, entropy, lse = lm.token_log_probs_forward(z, token, tau)
    dz = lm.token_log_probs_backward(z, token, lse, entropy, dlogp, dentropy, tau)
    g = gen(37)
    for _ in range(4):
        e = torch.randn(4, 50, device="cuda", generator=g)
        e /= e.norm()
        want = (value(z + step * e) - value(z - step * e)) / (2 * step)
        # values of order 10 carry some 2e-5; third derivatives along a unit direction are below 100
        assert abs(float((dz.double() * e.double()).sum()) - want) < 2e-5 / step + 100 * step ** 2 / 6


def test_streams_and_graphs():
    from paper_1810_10962_b200 import lm
    z, token, dlogp, dentropy = case(20, 40001, torch.bfloat16, 41)

    def all_of():
        out = lm.token_log_probs_forward_top(z, token, 8)
        return (*out, lm.token_log_probs_backward(z, token, out[2], out[1], dlogp, dentropy))

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
    z.copy_(z.flip(0))
    graph.replay()
    torch.cuda.synchronize()
    again = all_of()
    assert all(torch.equal(a, b) for a, b in zip(got, again))


def test_past_32_bit_offsets():
    from paper_1810_10962_b200 import lm
    T, V = 17_000, 131072                                    # 2.2e9 elements
    z = torch.zeros(T, V, dtype=torch.bfloat16, device="cuda")
    tail, token, dlogp, dentropy = case(5, V, torch.bfloat16, 43)
    z[-5:] = tail
    full = lambda t: torch.cat([t[:1].expand(T - 5), t]).contiguous()  # noqa: E731
    got = lm.token_log_probs_forward(z, full(token))
    want = lm.token_log_probs_forward(tail, token)
    for a, b in zip(got, want):
        assert torch.allclose(a[-5:], b, rtol=1e-5, atol=1e-5)
    dz = lm.token_log_probs_backward(z, full(token), got[2], got[1], full(dlogp), full(dentropy))
    want_dz = lm.token_log_probs_backward(tail, token, want[2], want[1], dlogp, dentropy)
    assert torch.allclose(dz[-5:].float(), want_dz.float(), rtol=2 ** -7, atol=1e-6)
