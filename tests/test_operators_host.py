"""Host-side checks of the operators of gated models that need no GPU: bad arguments are refused before anything is launched."""
import ctypes as C

import pytest
import torch

from paper_2411_18873_amd import eck

FAKE = C.c_void_p(0x1000)   # never dereferenced: every call below must fail validation first
ODD = C.c_void_p(0x1001)
HALF = C.c_void_p(0x1002)   # aligned for bf16, not for fp32
f = C.c_float


def test_layernorm_forward_validates_before_launch():
    F = eck.lib().layernorm_forward

    def call(x=FAKE, order=0, dtype=1, ld_x=64, n=16, width=64, gamma=FAKE, beta=FAKE, eps=1e-5, y=FAKE, ld_y=64, mean=None, rstd=None):
        return F(x, order, dtype, ld_x, n, width, gamma, beta, f(eps), y, ld_y, mean, rstd, None)

    assert call(x=None) == call(y=None) == call(n=0) == call(width=0) == eck.EINVAL
    assert call(order=2) == call(order=-1) == call(dtype=2) == call(dtype=-1) == eck.EINVAL
    assert call(eps=-1e-5) == call(eps=float("nan")) == call(eps=float("inf")) == eck.EINVAL
    assert call(mean=FAKE) == call(rstd=FAKE) == eck.EINVAL
    assert call(ld_x=63) == call(ld_y=63) == call(order=1, n=128) == eck.ESHAPE
    assert call(order=1, width=257, ld_x=512, ld_y=512) == eck.EUNSUPPORTED
    assert call(n=(1 << 31) + 1) == call(width=(1 << 24) + 1, ld_x=1 << 25, ld_y=1 << 25) == eck.EUNSUPPORTED
    assert call(x=ODD) == call(y=ODD) == call(dtype=0, x=HALF) == call(dtype=0, y=HALF) == eck.EALIGN
    assert call(gamma=HALF) == call(beta=HALF) == call(mean=HALF, rstd=FAKE) == call(mean=FAKE, rstd=HALF) == eck.EALIGN


def test_layernorm_backward_validates_before_launch():
    L = eck.lib()
    B, W = L.layernorm_backward, L.layernorm_backward_workspace_bytes
    assert W(0, 64, 1) == W(16, 0, 1) == W(16, 64, 2) == W((1 << 31) + 1, 64, 1) == W(16, (1 << 24) + 1, 1) == 0
    assert W(16, 64, 1) >= 2 * 64 * 4

    def call(x=FAKE, order=0, dtype=1, ld_x=64, dy=FAKE, ld_dy=64, n=16, width=64, gamma=FAKE, mean=FAKE, rstd=FAKE, dx=FAKE, ld_dx=64,
             dgamma=FAKE, dbeta=FAKE, ws=FAKE, ws_bytes=1 << 30):
        return B(x, order, dtype, ld_x, dy, ld_dy, n, width, gamma, mean, rstd, dx, ld_dx, dgamma, dbeta, ws, ws_bytes, None)

    assert call(x=None) == call(dy=None) == call(mean=None) == call(rstd=None) == call(n=0) == call(width=0) == eck.EINVAL
    assert call(dgamma=None) == call(dbeta=None) == call(dx=None, dgamma=None, dbeta=None) == eck.EINVAL
    assert call(order=2) == call(dtype=2) == eck.EINVAL
    assert call(ld_x=63) == call(ld_dy=63) == call(ld_dx=63) == call(order=1, n=128) == call(order=1, n=64, ld_dx=63) == eck.ESHAPE
    assert call(order=1, width=257, ld_x=512, ld_dy=512, ld_dx=512) == eck.EUNSUPPORTED
    assert call(ws=None) == call(ws_bytes=W(16, 64, 1) - 1) == eck.EWORKSPACE
    assert call(x=ODD) == call(dy=ODD) == call(dx=ODD) == call(gamma=HALF) == call(mean=HALF) == call(rstd=HALF) == eck.EALIGN
    assert call(dgamma=HALF) == call(dbeta=HALF) == call(ws=C.c_void_p(0x1010)) == eck.EALIGN


def test_dropout_validates_before_launch():
    D = eck.lib().dropout_apply

    def call(x=FAKE, dtype=1, ld_x=64, n=16, width=64, res=None, ld_res=0, out=FAKE, ld_out=64):
        return D(x, dtype, ld_x, n, width, 1 << 30, 7, 0, 0, res, ld_res, out, ld_out, None)

    assert call(x=None) == call(out=None) == call(n=0) == call(width=0) == call(dtype=2) == eck.EINVAL
    assert call(ld_x=63) == call(ld_out=63) == call(res=FAKE, ld_res=63) == eck.ESHAPE
    assert call(n=(1 << 31) + 1) == call(width=(1 << 24) + 1, ld_x=1 << 25, ld_out=1 << 25) == eck.EUNSUPPORTED
    assert call(x=ODD) == call(out=ODD) == call(res=ODD, ld_res=64) == call(dtype=0, x=HALF) == eck.EALIGN


def test_gatedffn_validates_before_launch():
    L = eck.lib()
    WF, WB = L.gatedffn_forward_workspace_bytes, L.gatedffn_backward_workspace_bytes
    for W in (WF, WB):
        assert W(0, 64, 64, 64, 1) == W(16, 0, 64, 64, 1) == W(16, 64, 0, 64, 1) == W(16, 64, 64, 0, 1) == W(16, 64, 64, 64, 2) == 0
        assert W((1 << 31) + 1, 64, 64, 64, 1) == W(16, (1 << 24) + 1, 64, 64, 1) == W(16, 64, (1 << 24) + 1, 64, 1) == 0
    assert WB(16, 64, 64, 64, 1) > 0

    def forward(x=FAKE, dtype=1, ld_x=64, n=16, n_in=64, n_hidden=64, n_out=64, wgu=FAKE, wd=FAKE, act=0, y=FAKE, ld_y=64, pre=None, ws=FAKE,
                ws_bytes=1 << 40):
        return L.gatedffn_forward(x, dtype, ld_x, n, n_in, n_hidden, n_out, wgu, wd, act, y, ld_y, pre, ws, ws_bytes, None)

    def backward(x=FAKE, dtype=1, ld_x=64, n=16, n_in=64, n_hidden=64, n_out=64, wgu=FAKE, wd=FAKE, act=0, pre=FAKE, dy=FAKE, ld_dy=64,
                 dx=FAKE, ld_dx=64, dwgu=FAKE, dwd=FAKE, ws=FAKE, ws_bytes=1 << 40):
        return L.gatedffn_backward(x, dtype, ld_x, n, n_in, n_hidden, n_out, wgu, wd, act, pre, dy, ld_dy, dx, ld_dx, dwgu, dwd, ws, ws_bytes,
                                   None)

    for call in (forward, backward):
        assert call(x=None) == call(wgu=None) == call(wd=None) == eck.EINVAL
        assert call(n=0) == call(n_in=0) == call(n_hidden=0) == call(n_out=0) == call(dtype=2) == call(act=3) == call(act=-1) == eck.EINVAL
        assert call(ld_x=63) == eck.ESHAPE
        assert call(n=(1 << 31) + 1) == call(n_hidden=(1 << 24) + 1) == eck.EUNSUPPORTED
        assert call(x=ODD) == call(wgu=ODD) == call(wd=ODD) == call(ws=C.c_void_p(0x1010)) == eck.EALIGN
        assert call(dtype=0, x=HALF) == call(dtype=0, wgu=HALF) == call(dtype=0, wd=HALF) == call(pre=HALF) == eck.EALIGN
    assert forward(y=None) == backward(pre=None) == backward(dy=None) == backward(dx=None, dwgu=None, dwd=None) == eck.EINVAL
    assert forward(ld_y=63) == backward(ld_dy=63) == backward(ld_dx=63) == eck.ESHAPE
    assert forward(y=ODD) == backward(dy=ODD) == backward(dx=ODD) == backward(dwgu=ODD) == backward(dwd=ODD) == eck.EALIGN
    need = WB(16, 64, 64, 64, 1)
    assert backward(ws=None) == backward(ws_bytes=need - 1) == eck.EWORKSPACE
    need = WF(1000, 64, 1000, 64, 1)
    if need:
        assert forward(n=1000, n_hidden=1000, ws=None) == forward(n=1000, n_hidden=1000, ws_bytes=need - 1) == eck.EWORKSPACE


def test_the_binding_refuses_tensors_that_are_not_what_they_should_be():
    x = torch.zeros(4, 8)
    for call in (lambda: eck.layernorm_forward(x, None, None, x), lambda: eck.dropout_apply(x, x, 1 << 30, 1),
                 lambda: eck.gatedffn_forward(x, torch.zeros(8, 32), torch.zeros(16, 8), x, None)):
        with pytest.raises(TypeError):   # not on a GPU
            call()
    for p in (-1, 1 << 32):
        with pytest.raises(ValueError):  # a probability that does not fit
            eck.dropout_apply(x, x, p, 1)


class OnGpu:
    """what the binding asks of a CUDA tensor, answered by a host one"""
    is_cuda = True

    def __init__(self, t):
        self.shape, self.dtype, self.stride = t.shape, t.dtype, t.stride


@pytest.mark.parametrize("n", [1, 2, 1000])
def test_the_binding_passes_the_row_distance_that_a_feature_matrix_has(n):
    """a distance below n, which the library refuses, must not be replaced by one that the memory behind the view does not have"""
    whole = torch.zeros(64, n + 3)
    for view, ld in ((whole, n + 3), (whole[:, :n], n + 3), (whole[:, 3:], n + 3), (torch.zeros(1, n).expand(64, n), 0),
                     (torch.zeros(64 * 8 + n).as_strided((64, n), (8, 1)), 8)):
        assert eck._feature_rows(OnGpu(view), n, 64, torch.float32, "x") == ld
    # a single feature's row has no next one, whatever torch says of its distance
    assert eck._feature_rows(OnGpu(torch.zeros(n).as_strided((1, n), (0, 1))), n, 1, torch.float32, "x") == n
    for shape in ((63, n), (64, n - 1)):
        with pytest.raises(ValueError):
            eck._feature_rows(OnGpu(torch.zeros(shape)), n, 64, torch.float32, "x")


def test_gatedffn_passes_are_refused_for_their_own_products_only():
    """2^22 tiles of 64 x 64 a product: dx and the weights' gradients are products of the backward pass, which a forward pass has not"""
    L = eck.lib()
    WF, WB = L.gatedffn_forward_workspace_bytes, L.gatedffn_backward_workspace_bytes
    for sizes in ((1 << 24, 2048, 64, 64, 1), (1 << 20, 1 << 18, 64, 64, 1), (16, 1 << 18, 1 << 16, 64, 1), (16, 64, 1 << 18, 1 << 17, 0)):
        assert WF(*sizes) > 0 and WB(*sizes) == 0, sizes
    for sizes in ((1 << 24, 64, 1024, 64, 1), (1 << 24, 64, 64, 2048, 1)):      # [g | u], y
        assert WF(*sizes) == WB(*sizes) == 0, sizes
    assert WF(1 << 24, 64, 64, 64, 1) > 0 and WB(1 << 24, 64, 64, 64, 1) > 0
