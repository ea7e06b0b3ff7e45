"""Heads' norm + rotation on either side of the limits at which the vectors' width changes (bf16), against the 64-bit definition."""
import pytest
import torch

from test_lm_rotary_gpu import case, check

pytestmark = pytest.mark.gpu


# few heads at any number of positions; heads of queries and keys that fill some rounds of a warp, with few positions and with many; keys alone in number
@pytest.mark.parametrize("Hq,Hk,D,S", [(4, 1, 64, 40000), (8, 8, 64, 900), (8, 8, 64, 7000), (16, 16, 32, 900), (16, 16, 32, 7000), (32, 32, 32, 500), (32, 32, 32, 3000),
                                       (16, 16, 64, 500), (16, 16, 64, 3000), (16, 4, 64, 5000), (1, 32, 64, 300), (1, 32, 64, 3000), (2, 16, 128, 3000),
                                       (8, 1, 64, 9000)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_either_width(Hq, Hk, D, S, interleaved):
    check(*case(1, S, Hq, Hk, D, D, torch.bfloat16, 7 + S, P=S), interleaved)


def test_both_widths_agree_at_the_limit():
    """The same heads in a call of many positions and in calls of few: forward results have the same factors and sums of other orders."""
    from paper_1810_10962_b200 import lm
    q, k, qw, kw, cos, sin, position, grads = case(1, 8000, 16, 16, 64, 64, torch.bfloat16, 31, P=8000)
    whole = lm.head_norm_rotary_forward(q, k, qw, kw, cos, sin, position, 1e-6)
    for first in (0, 4000, 7800):
        part = slice(first, first + 200)
        few = lm.head_norm_rotary_forward(q[:, part], k[:, part], qw, kw, cos, sin, position[:, part].contiguous(), 1e-6)
        for a, b, w in zip(whole, few, (qw, kw)):
            # Each is 32 u (|n w cos| + |n w sin|) off before the store, n being sqrt(64) at the most; a cos - b sin may be much smaller than its
            # terms, so this does not go by the result.  The stores then differ by a step, 2^-7 of the value, at the most.
            size = 64 ** 0.5 * float(w.abs().max()) * 2 ** 0.5
            assert bool(((a[:, part].double() - b.double()).abs() <= 2.0 ** -7 * b.double().abs() + 64 * 2.0 ** -24 * size).all())
