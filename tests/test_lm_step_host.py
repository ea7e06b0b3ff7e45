"""CPU-side checks of token log probabilities, heads' norm + rotation and gradient clipping: everything that can be refused on
the host is refused before anything is launched, by the C ABI and by the binding."""
import ctypes

import pytest
import torch

from paper_1810_10962_b200 import bns, lm

P = 0x10000          # fake device addresses, never dereferenced: every call below is refused


@pytest.fixture
def lib():
    if torch.cuda.is_available():
        pytest.skip("fake device addresses are only used where no GPU can be reached")
    return lm._load()


def test_structures_match_the_header():
    """Field by field, as the C compiler lays them out."""
    import os
    import subprocess
    import tempfile
    fields = {"bns_token_log_probs": (lm._LogProbs, ["rows", "vocabulary", "entries", "dtype", "stride", "token_is_int64", "temperature"], None),
              "bns_head_norm": (lm._HeadNorm, ["batch", "length", "q_heads", "k_heads", "head_dim", "rotary", "dtype", "q_strides[0]", "q_strides[1]",
                                               "q_strides[2]", "k_strides[0]", "k_strides[1]", "k_strides[2]", "positions",
                                               "position_is_int64", "interleaved", "eps"], None),
              "bns_gradients": (lm._Gradients, ["count", "data", "out", "elements", "dtype"], None)}
    lines = ["#include <stdio.h>", "#include <stddef.h>", '#include "bns.h"', "int main(void) {"]
    for name, (_, members, _) in fields.items():
        lines.append(f'printf("%zu\\n", sizeof({name}));')
        lines += [f'printf("%zu\\n", offsetof({name}, {m}));' for m in members]
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    with tempfile.TemporaryDirectory() as d:
        with open(os.path.join(d, "a.c"), "w") as f:
            f.write("\n".join([*lines, "return 0; }"]))
        subprocess.run(["gcc", "-I", os.path.join(root, "include"), os.path.join(d, "a.c"), "-o", os.path.join(d, "a")], check=True)
        got = [int(v) for v in subprocess.run([os.path.join(d, "a")], check=True, capture_output=True, text=True).stdout.split()]
    want = []
    for struct, members, _ in fields.values():
        names = [n for n, _ in struct._fields_]
        assert len(names) == len(members)
        want += [ctypes.sizeof(struct), *(getattr(struct, n).offset for n in names)]
    assert got == want


def test_log_probs_refusals(lib):
    good = dict(rows=4, vocabulary=100, entries=8, dtype=bns.F32, stride=100, token_is_int64=0, temperature=1.0)

    def forward(z=P, token=P, logp=P, entropy=P, lse=P, top=P, index=P, **change):
        shape = lm._LogProbs(**{**good, **change})
        return lib.bns_token_log_probs_forward(ctypes.byref(shape), z, token, logp, entropy, lse, top, index, None)

    for change in (dict(rows=-1), dict(vocabulary=0), dict(entries=-1), dict(entries=65), dict(entries=60, vocabulary=59), dict(stride=99),
                   dict(vocabulary=(1 << 30) + 1, stride=1 << 31)):
        assert forward(**change) == -2
    for temperature in (0.0, -1.0, float("nan"), float("inf"), 1e-7, 1e7):
        assert forward(temperature=temperature) == -2
    assert forward(dtype=2) == -5
    for name in ("z", "token", "logp", "lse", "top", "index"):
        assert forward(**{name: None}) == -1
    for name in ("z", "token", "logp", "entropy", "lse", "top", "index"):
        assert forward(**{name: P + 2}) == -6
    assert forward(token=P + 4, token_is_int64=1) == -6
    assert forward(rows=0, z=None) == 0

    def backward(z=P, token=P, lse=P, entropy=P, dlogp=P, dentropy=P, dz=P, stride=100, **change):
        shape = lm._LogProbs(**{**good, **change})
        return lib.bns_token_log_probs_backward(ctypes.byref(shape), z, token, lse, entropy, dlogp, dentropy, dz, stride, None)

    for name in ("z", "token", "lse", "entropy", "dlogp", "dz"):
        assert backward(**{name: None}) == -1
        assert backward(**{name: P + 2}) == -6
    assert backward(stride=99) == -2 and backward(dentropy=P + 1) == -6 and backward(rows=0, dz=None) == 0


def test_head_norm_refusals(lib):
    good = dict(batch=2, length=3, q_heads=4, k_heads=2, head_dim=64, rotary=32, dtype=bns.BF16, q_batch=768, q_position=256, q_head=64,
                k_batch=384, k_position=128, k_head=64, positions=10, position_is_int64=1, interleaved=0, eps=1e-6)

    def forward(q=P, k=P, qw=P, kw=P, cos=P, sin=P, at=P, qo=P, ko=P, **change):
        return lib.bns_head_norm_rotary_forward(ctypes.byref(lm._HeadNorm(**{**good, **change})), q, k, qw, kw, cos, sin, at, qo, ko, None)

    for change in (dict(batch=-1), dict(length=-1), dict(batch=1 << 16, length=1 << 16), dict(q_heads=0), dict(k_heads=-1), dict(head_dim=1, rotary=1),
                   dict(head_dim=1025), dict(rotary=0), dict(rotary=33), dict(rotary=66), dict(positions=0), dict(eps=0.0), dict(eps=float("nan")),
                   dict(q_head=-1), dict(k_position=-5), dict(q_heads=40000)):
        assert forward(**change) == -2
    assert forward(dtype=7) == -5
    for name in ("q", "k", "qw", "kw", "cos", "sin", "at", "qo", "ko"):
        assert forward(**{name: None}) == -1
        assert forward(**{name: P + 1}) == -6
    assert forward(batch=0, q=None) == 0
    shape = lm._HeadNorm(**good)
    need = lib.bns_head_norm_rotary_workspace_bytes(ctypes.byref(shape))
    assert need >= 256 + 6 * 64 * 4 and need % 256 == 0
    assert lib.bns_head_norm_rotary_workspace_bytes(ctypes.byref(lm._HeadNorm(**{**good, "rotary": 1}))) == 0

    def backward(dqo=P, dko=P, q=P, k=P, qw=P, kw=P, cos=P, sin=P, at=P, dq=P, dk=P, dqw=P, dkw=P, ws=P, n=need):
        return lib.bns_head_norm_rotary_backward(ctypes.byref(shape), dqo, dko, q, k, qw, kw, cos, sin, at, dq, dk, dqw, dkw, ws, n, None)

    for name in ("dqo", "dko", "q", "k", "qw", "kw", "cos", "sin", "at", "dq", "dk", "dqw", "dkw"):
        assert backward(**{name: None}) == -1
        assert backward(**{name: P + 1}) == -6
    assert backward(ws=None) == -7 and backward(n=need - 1) == -7 and backward(ws=P + 64) == -7


def test_gradient_refusals(lib):
    def call(data=(P, P), out=(P, 2 * P), elements=(10, 20), dtype=(bns.F32, bns.BF16), max_norm=1.0, norm=P, ws=P, n=1 << 20, what="clip"):
        m = len(elements)
        arrays = ((ctypes.c_void_p * m)(*data), (ctypes.c_void_p * m)(*out), (ctypes.c_int64 * m)(*elements), (ctypes.c_int * m)(*dtype))
        shape = lm._Gradients(m, *(ctypes.addressof(a) for a in arrays))
        if what == "bytes":
            return lib.bns_gradient_norm_workspace_bytes(ctypes.byref(shape))
        if what == "norm":
            return lib.bns_gradient_norm(ctypes.byref(shape), norm, ws, n, None)
        return lib.bns_clip_gradients(ctypes.byref(shape), max_norm, norm, ws, n, None)

    for what in ("clip", "norm"):
        assert call(elements=(10, -1), what=what) == -2
        assert call(dtype=(0, 3), what=what) == -5
        assert call(data=(P, None), what=what) == -1 and call(norm=None, what=what) == -1
        assert call(data=(P + 2, P), what=what) == -6 and call(norm=P + 2, what=what) == -6
        assert call(ws=None, what=what) == -7 and call(n=16, what=what) == -7 and call(ws=P + 8, what=what) == -7
    assert call(out=(None, P)) == -1 and call(out=(P, P + 1)) == -6
    assert call(max_norm=-1.0) == -2 and call(max_norm=float("nan")) == -2
    assert call(what="bytes") >= 256 + 8 and call(elements=(1, -1), what="bytes") == 0
    none = lm._Gradients(3, None, None, None, None)
    assert lib.bns_gradient_norm(ctypes.byref(none), P, P, 1 << 20, None) == -1


def test_binding_refuses_what_is_not_a_cuda_tensor():
    z, token = torch.zeros(4, 64), torch.zeros(4, dtype=torch.int64)
    with pytest.raises(TypeError):
        lm.token_log_probs_forward(z, token)
    with pytest.raises(ValueError):
        lm.token_log_probs_forward_top(z, token, 0)
    with pytest.raises(TypeError):
        lm.token_log_probs_backward(z, token, torch.zeros(4), None, torch.zeros(4))
    q, w, table = torch.zeros(3, 2, 8), torch.ones(8), torch.zeros(5, 4)
    with pytest.raises(TypeError):
        lm.head_norm_rotary_forward(q, None, w, None, table, table, token[:3], 1e-6)
    with pytest.raises(TypeError):
        lm.head_norm_rotary_backward(q, None, q, None, w, None, table, table, token[:3], 1e-6)
    with pytest.raises(TypeError):
        lm.gradient_norm([z])
    with pytest.raises(TypeError):
        lm.clip_gradients([z], 1.0)


def test_which_tensors_are_dense():
    t = torch.zeros(4, 5, 6)
    for dense in (t, t.permute(2, 0, 1), t.transpose(0, 1), t[1:3], t[:, :, None], torch.zeros(0, 3), torch.zeros(())):
        assert lm._dense(dense)
    for not_dense in (t[:, 1:], t[:, :, ::2], t[:1].expand(4, 5, 6)):
        assert not lm._dense(not_dense)
