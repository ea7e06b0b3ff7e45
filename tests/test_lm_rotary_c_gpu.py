"""Heads' gradient through the C interface, with weights' gradients that held something before: keys without heads and calls without positions
write zeros there, and nothing else is touched."""
import ctypes

import pytest
import torch

pytestmark = pytest.mark.gpu


def backward(batch, length, k_heads, dk_weight, dtype=torch.bfloat16):
    """(status, dq_weight, the values around both weights' gradients)."""
    from paper_1810_10962_b200 import lm
    H, D, R, P = 3, 64, 32, 9
    g = torch.Generator(device="cuda").manual_seed(3)
    normal = lambda *s, dtype=dtype: torch.randn(*s, device="cuda", generator=g).to(dtype)  # noqa: E731
    q, dy, dq = (normal(batch, length, H, D) for _ in range(3))
    k, dk_out, dk = (normal(batch, length, max(1, k_heads), D) for _ in range(3))
    table, weight = normal(P, R // 2, dtype=torch.float32), normal(D, dtype=torch.float32)
    position = torch.randint(0, P, (batch, length), device="cuda", generator=g)
    shape = lm._HeadNorm(batch, length, H, k_heads, D, R, lm._CODES[dtype], length * H * D, H * D, D, length * k_heads * D, k_heads * D, D, P, 1, 0, 1e-6)
    lib = lm._load()
    workspace = torch.empty(lib.bns_head_norm_rotary_workspace_bytes(ctypes.byref(shape)), dtype=torch.uint8, device="cuda")
    room = torch.full((3, D), 7.0, device="cuda")
    keys = (lambda t: t.data_ptr()) if k_heads else (lambda t: None)  # noqa: E731
    status = lib.bns_head_norm_rotary_backward(
        ctypes.byref(shape), dy.data_ptr(), keys(dk_out), q.data_ptr(), keys(k), weight.data_ptr(), keys(weight), table.data_ptr(), table.data_ptr(),
        position.data_ptr(), dq.data_ptr(), keys(dk), room[0].data_ptr(), room[1].data_ptr() if dk_weight else None, workspace.data_ptr(),
        workspace.nbytes, torch.cuda.current_stream().cuda_stream)
    return status, room


@pytest.mark.parametrize("batch,length", [(2, 5), (1, 1), (3, 700)])
def test_keys_without_heads(batch, length):
    status, room = backward(batch, length, 0, True)
    assert status == 0 and not room[1].any() and bool((room[2] == 7).all()) and bool((room[0] != 7).all())
    status, again = backward(batch, length, 0, False)
    assert status == 0 and bool((again[1:] == 7).all()) and torch.equal(again[0], room[0])


@pytest.mark.parametrize("k_heads", [0, 2])
@pytest.mark.parametrize("batch,length", [(0, 5), (4, 0), (0, 0)])
def test_without_positions(batch, length, k_heads):
    status, room = backward(batch, length, k_heads, True)
    assert status == 0 and not room[:2].any() and bool((room[2] == 7).all())


def test_keys_with_heads_write_both():
    status, room = backward(2, 5, 2, True)
    assert status == 0 and bool((room[:2] != 7).all()) and bool(room[:2].any(1).all()) and bool((room[2] == 7).all())
