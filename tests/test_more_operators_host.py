"""Host-side checks that need no GPU: refits' and scoring's operators refuse bad arguments before anything is launched."""
import ctypes as C

import pytest
import torch

from paper_2411_18873_amd import eck

FAKE = 0x1000   # never dereferenced: every call below must fail validation first


def entry(**change):
    at = dict(param=FAKE, grad=FAKE, m=FAKE, v=FAKE, m_scale=FAKE, v_scale=FAKE, bf16_out=FAKE, n=100, grad_dtype=0, weight_decay=0.0)
    at.update(change)
    return eck.Parameter(**at)


def listed(*entries):
    return (eck.Parameter * len(entries))(*entries)


def test_adamw_validates_before_launch():
    F = eck.lib().adamw_step

    def call(*entries, p=0, count=None, state=0, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=1, more=None, scale=None):
        p = listed(*(entries or [entry()])) if p == 0 else p
        return F(p, len(p) if count is None else count, state, lr, beta1, beta2, eps, step, more, scale, 0, None)

    nan, inf = float("nan"), float("inf")
    assert call(p=None, count=1) == call(count=0) == call(state=2) == call(state=-1) == eck.EINVAL
    assert call(lr=-1.0) == call(lr=nan) == call(lr=inf) == call(eps=-1.0) == call(eps=nan) == call(step=0) == eck.EINVAL
    assert call(beta1=1.0) == call(beta1=-0.1) == call(beta2=1.0) == call(beta2=nan) == eck.EINVAL
    for field in ("param", "grad", "m", "v"):
        assert call(entry(), entry(**{field: None})) == eck.EINVAL
    assert call(entry(n=0, param=None)) == eck.EINVAL           # no element at all
    assert call(entry(n=0), entry(grad_dtype=2)) == call(entry(weight_decay=-1.0)) == call(entry(weight_decay=nan)) == eck.EINVAL
    assert call(entry(m_scale=None), state=1) == call(entry(v_scale=None), state=1) == eck.EINVAL
    assert call(entry(n=(1 << 40) + 1)) == eck.EUNSUPPORTED
    assert call(entry(param=FAKE + 2)) == call(entry(grad=FAKE + 2)) == call(entry(grad=FAKE + 1, grad_dtype=1)) == eck.EALIGN
    assert call(entry(m=FAKE + 1)) == call(entry(v=FAKE + 2)) == call(entry(bf16_out=FAKE + 1)) == eck.EALIGN
    assert call(more=C.c_void_p(FAKE + 2)) == call(scale=C.c_void_p(FAKE + 1)) == eck.EALIGN


def test_gradients_norm_validates_before_launch():
    L = eck.lib()

    def call(*entries, count=None, most=1.0, norm=FAKE, scale=FAKE, ws=FAKE, ws_bytes=1 << 20):
        p = listed(*(entries or [entry(param=None, m=None, v=None)]))
        vp = lambda x: None if x is None else C.c_void_p(x)  # noqa: E731
        return L.gradients_norm(p, len(p) if count is None else count, most, vp(norm), vp(scale), vp(ws), ws_bytes, None)

    assert L.gradients_norm_workspace_bytes(listed(entry(n=0)), 1) == L.gradients_norm_workspace_bytes(None, 1) == 0
    need = L.gradients_norm_workspace_bytes(listed(entry(n=1 << 30), entry(n=5)), 2)
    assert 0 < need <= 8 * 16500
    assert call(norm=None, scale=None) == call(most=0.0) == call(most=-1.0) == call(most=float("nan")) == call(count=0) == eck.EINVAL
    assert call(entry(grad=None)) == call(entry(n=0)) == call(entry(grad_dtype=7)) == eck.EINVAL
    assert call(entry(n=(1 << 40) + 1)) == eck.EUNSUPPORTED
    assert call(ws=None) == call(ws_bytes=7) == eck.EWORKSPACE
    assert call(ws=FAKE + 16) == call(norm=FAKE + 2) == call(scale=FAKE + 2) == call(entry(grad=FAKE + 2)) == eck.EALIGN


def test_parameters_are_checked_by_the_binding():
    cpu = torch.zeros(4)
    with pytest.raises(TypeError):
        eck.Parameters([cpu])
    with pytest.raises(ValueError):
        eck.Parameters([cpu], params=[cpu, cpu], m=[cpu], v=[cpu])
    with pytest.raises(ValueError):
        eck.Parameters([cpu], params=[cpu])
    with pytest.raises(ValueError):
        eck.Parameters([cpu], weight_decay=[0.1, 0.2])
    with pytest.raises(ValueError):
        eck.Parameters([cpu], [cpu], [torch.zeros(4, dtype=torch.uint8)], [torch.zeros(4, dtype=torch.uint8)])
