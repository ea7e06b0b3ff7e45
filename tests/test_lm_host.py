"""CPU-side checks of the language-model operators: everything that can be refused on the host is refused
before anything is launched, by the C ABI and by the binding."""
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


def norm_call(lib, shape=(8, 64, bns.BF16), x=P, xs=64, r=P, rs=64, w=P, eps=1e-5, y=P, h=P, rstd=P):
    return lib.bns_rms_norm_forward(ctypes.byref(lm._Rows(*shape)), x, xs, r, rs, w, eps, y, h, rstd, None)


def test_norm_refusals(lib):
    assert norm_call(lib, shape=(-1, 64, 0)) == -2 and norm_call(lib, shape=(8, 0, 0)) == -2
    assert norm_call(lib, shape=(8, 64, 2)) == -5
    for name in ("x", "w", "y", "rstd"):
        assert norm_call(lib, **{name: None}) == -1
    assert norm_call(lib, eps=0.0) == -2 and norm_call(lib, eps=float("nan")) == -2
    assert norm_call(lib, xs=63) == -2 and norm_call(lib, rs=63) == -2
    assert norm_call(lib, x=P + 1) == -6 and norm_call(lib, w=P + 2) == -6
    assert norm_call(lib, shape=(0, 64, 0), x=None) == 0            # no rows: nothing to do
    rows = lm._Rows(8, 64, bns.BF16)
    quantized = lib.bns_rms_norm_forward_quantized
    assert quantized(ctypes.byref(rows), P, 64, None, 0, P, 1e-5, 64, P, P, None, P, None) == -3
    assert quantized(ctypes.byref(rows), P, 64, None, 0, P, 1e-5, 128, P, None, None, P, None) == -1
    need = lib.bns_rms_norm_workspace_bytes(ctypes.byref(rows))
    assert need >= 256 + 8 * 64 * 4
    assert lib.bns_rms_norm_workspace_bytes(ctypes.byref(lm._Rows(8, -1, 0))) == 0
    backward = lambda ws=P, n=need, dh=None, dhs=64, dx=P, dw=P: lib.bns_rms_norm_backward(  # noqa: E731
        ctypes.byref(rows), P, 64, P, 64, P, P, dh, dhs, dx, dw, ws, n, None)
    assert backward(ws=None) == -7 and backward(ws=P + 16) == -7 and backward(n=need - 1) == -7
    assert backward(dx=None) == -1 and backward(dw=None) == -1 and backward(dh=P, dhs=10) == -2 and backward(dx=P + 1) == -6


def test_head_refusals(lib):
    good = dict(rows=10, vocabulary=100, width=64, dtype=bns.BF16, x_stride=64, w_stride=64, target_is_int64=1)

    def forward(x=P, w=P, target=P, loss=P, lse=P, ws=P, n=1 << 40, **change):
        shape = lm._Head(**{**good, **change})
        return lib.bns_linear_cross_entropy_forward(ctypes.byref(shape), x, w, target, loss, lse, ws, n, None)

    assert forward(vocabulary=0) == -2 and forward(width=0) == -2 and forward(rows=-1) == -2 and forward(x_stride=63) == -2
    assert forward(vocabulary=(1 << 28) + 1) == -2 and forward(width=(1 << 20) + 1, x_stride=1 << 21, w_stride=1 << 21) == -2
    assert forward(dtype=3) == -5
    for name in ("x", "w", "target", "loss", "lse"):
        assert forward(**{name: None}) == -1
    assert forward(x=P + 2) == -6 and forward(w=P + 8) == -6 and forward(target=P + 4) == -6
    assert forward(ws=None) == -7 and forward(n=16) == -7 and forward(ws=P + 128) == -7
    shape = lm._Head(**good)
    for backward in (0, 1):
        need = lib.bns_linear_cross_entropy_workspace_bytes(ctypes.byref(shape), backward)
        assert need > 256 and need % 256 == 0
    call = lambda dx=P, dw=P, lse=P, dloss=P, n=1 << 40: lib.bns_linear_cross_entropy_backward(  # noqa: E731
        ctypes.byref(shape), P, P, P, lse, dloss, dx, dw, P, n, None)
    assert call(dx=None) == -1 and call(dw=None) == -1 and call(lse=None) == -1 and call(dloss=None) == -1
    assert call(dx=P + 4) == -6 and call(n=0) == -7
    assert lib.bns_linear_cross_entropy_workspace_bytes(ctypes.byref(lm._Head(**{**good, "width": 0})), 0) == 0


def test_head_workspace_stays_near_its_aim(lib):
    """Neither the logits nor a second copy of a large weight is kept: the workspace of large products stays below a
    fixed part of what the logits would take."""
    for dtype, limit in ((bns.BF16, 0.45e9), (bns.F32, 1.6e9)):
        shape = lm._Head(8192, 131072, 4096, dtype, 4096, 4096, 1)
        assert lib.bns_linear_cross_entropy_workspace_bytes(ctypes.byref(shape), 1) < limit
        assert lib.bns_linear_cross_entropy_workspace_bytes(ctypes.byref(shape), 0) < limit


def test_distillation_refusals(lib):
    good = dict(rows=4, vocabulary=100, entries=8, dtype=bns.F32, stride=100, teacher_dtype=bns.F32, index_is_int64=0,
                temperature=1.0)

    def forward(z=P, a=P, i=P, loss=P, lse=P, **change):
        shape = lm._Distillation(**{**good, **change})
        return lib.bns_topk_distillation_forward(ctypes.byref(shape), z, a, i, loss, lse, None)

    assert forward(vocabulary=0) == -2 and forward(entries=0) == -2 and forward(entries=1025) == -2 and forward(stride=99) == -2
    for temperature in (0.0, -1.0, float("nan"), float("inf")):
        assert forward(temperature=temperature) == -2
    assert forward(dtype=9) == -5 and forward(teacher_dtype=9) == -5
    for name in ("z", "a", "i", "loss", "lse"):
        assert forward(**{name: None}) == -1
    assert forward(z=P + 2) == -6 and forward(i=P + 2) == -6 and forward(i=P + 4, index_is_int64=1) == -6
    assert forward(rows=0, z=None) == 0
    shape = lm._Distillation(**good)
    assert lib.bns_topk_distillation_backward(ctypes.byref(shape), P, P, P, P, P, P, 99, None) == -2
    assert lib.bns_topk_distillation_step(ctypes.byref(shape), P, P, P, None, P, P, 100, None) == -1


def test_distillation_temperature_range(lib):
    """Below some 4e-39 log2(e) / temperature is infinite, and every answer would be NaN."""
    call = lambda temperature: lib.bns_topk_distillation_forward(  # noqa: E731
        ctypes.byref(lm._Distillation(0, 100, 8, bns.F32, 100, bns.F32, 0, temperature)), P, P, P, P, P, None)
    for temperature in (1e-45, 1e-40, 4e-39, 1.1e30):
        assert call(temperature) == -2
    for temperature in (1.1e-38, 1e-30, 1.0, 0.9e30):
        assert call(temperature) == 0              # no rows: nothing is launched


def test_binding_refuses_what_is_not_a_cuda_tensor():
    x, w = torch.zeros(4, 64), torch.ones(64)
    with pytest.raises(TypeError):
        lm.rms_norm_forward(x, None, w, 1e-5)
    with pytest.raises(TypeError):
        lm.rms_norm_backward(x, x, w, torch.ones(4))
    with pytest.raises(TypeError):
        lm.linear_cross_entropy_forward(x, torch.zeros(10, 64), torch.zeros(4, dtype=torch.int64))
    with pytest.raises(TypeError):
        lm.topk_distillation_forward(x, torch.zeros(4, 2), torch.zeros(4, 2, dtype=torch.int32))


@pytest.mark.parametrize("D", [512, 1000, 4100])
def test_bound_of_fp32_products_sees_a_lost_term(D):
    """The bound that the GPU tests hold fp32 logits to, on sums made here: of all three products of terms they stay
    within it, without one of them nearly every row passes it."""
    from test_lm_head_gpu import chain
    g = torch.Generator().manual_seed(D)
    T, V = 40, 300
    x, w = torch.randn(T, D, generator=g), torch.randn(V, D, generator=g) * (2 / D ** 0.5)

    def terms(t):
        t = (t * 2.0 ** (13 - float(t.abs().max().log2().floor()))).float()
        high = t.half()
        return t.double(), high.double(), ((t - high.float()) * 2048).half().double() / 2048

    (xs, xh, xl), (ws, wh, wl) = terms(x), terms(w)
    scale = float((x.double() @ w.double().T).abs().max() / (xs @ ws.T).abs().max())
    target = torch.randint(0, V, (T, 1), generator=g)
    loss = lambda z: torch.logsumexp(z, 1) - z.gather(1, target)[:, 0]  # noqa: E731
    z = xs @ ws.T * scale
    tz = (xs.abs() @ ws.abs().T) * scale * chain(D, "f32", 256)
    bound = (torch.softmax(z, 1) * tz).sum(1) + tz.gather(1, target)[:, 0]
    off = lambda *products: ((loss(sum(products) * scale) - loss(z)).abs() / bound)  # noqa: E731
    assert float(off(xh @ wh.T, xh @ wl.T, xl @ wh.T).max()) < 1
    for lost in ((xh @ wh.T, xl @ wh.T), (xh @ wh.T, xh @ wl.T)):
        assert float(off(*lost).max()) > 1


@pytest.mark.gpu
def test_binding_refuses_tensors_that_do_not_fit():
    c = lambda *s, dtype=torch.bfloat16: torch.zeros(*s, dtype=dtype, device="cuda")  # noqa: E731
    x, w = c(4, 64), c(64, dtype=torch.float32)
    bad = [
        lambda: lm.rms_norm_forward(x, c(4, 32), w, 1e-5),
        lambda: lm.rms_norm_forward(x, c(4, 64, dtype=torch.float32), w, 1e-5),
        lambda: lm.rms_norm_forward(x, None, c(64), 1e-5),                           # weight must be fp32
        lambda: lm.rms_norm_forward(x, None, c(63, dtype=torch.float32), 1e-5),
        lambda: lm.rms_norm_forward(x.t(), None, c(4, dtype=torch.float32), 1e-5),   # rows that are not dense
        lambda: lm.rms_norm_forward(c(4, 64, dtype=torch.float16), None, w, 1e-5),
        lambda: lm.rms_norm_backward(x, x, w, c(3, dtype=torch.float32)),
        lambda: lm.linear_cross_entropy_forward(x, c(10, 32), c(4, dtype=torch.int64)),
        lambda: lm.linear_cross_entropy_forward(x, c(10, 64, dtype=torch.float32), c(4, dtype=torch.int64)),
        lambda: lm.linear_cross_entropy_forward(x, c(10, 64), c(5, dtype=torch.int64)),
        lambda: lm.linear_cross_entropy_forward(x, c(10, 64), c(4, dtype=torch.float32)),
        lambda: lm.linear_cross_entropy_backward(x, c(10, 64), c(4, dtype=torch.int64), c(4, dtype=torch.float32), c(4)),
        lambda: lm.topk_distillation_forward(x, c(4, 3), c(4, 2, dtype=torch.int32)),
        lambda: lm.topk_distillation_forward(x, c(5, 3), c(5, 3, dtype=torch.int32)),
        lambda: lm.topk_distillation_step(x, c(4, 3), c(4, 3, dtype=torch.int32), c(3, dtype=torch.float32)),
    ]
    for k, call in enumerate(bad):
        with pytest.raises(TypeError):
            call()
            pytest.fail(f"call {k} was not refused")
    with pytest.raises(bns.BnsError) as err:
        lm.rms_norm_forward(x, None, w, 0.0)
    assert err.value.status == -2
    with pytest.raises(bns.BnsError) as err:
        lm.rms_norm_forward_fp8(x, None, w, 1e-5, group=64)
    assert err.value.status == -3
    with pytest.raises(bns.BnsError) as err:
        lm.topk_distillation_forward(x, c(4, 3), c(4, 3, dtype=torch.int32), 0.0)
    assert err.value.status == -2
    with pytest.raises(bns.BnsError) as err:
        lm.linear_cross_entropy_forward(x, c(10, 64), c(4, dtype=torch.int64), workspace=c(16, dtype=torch.uint8))
    assert err.value.status == -7
