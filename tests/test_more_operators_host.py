"""Host-side checks that need no GPU: refits' and scoring's operators refuse bad arguments before anything is launched."""
import ctypes as C
import gc
import weakref

import pytest
import torch

from paper_2411_18873_amd import eck, gated

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
    assert call(entry(n=(1 << 40) + 1)) == call(entry(n=(1 << 34) + 1)) == eck.EUNSUPPORTED
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
    assert call(entry(n=(1 << 40) + 1)) == call(entry(n=(1 << 34) + 1)) == eck.EUNSUPPORTED
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


def test_quantise_rows_validates_before_launch():
    vp = C.c_void_p

    def call(x=FAKE, order=0, dtype=1, ld_x=64, n=16, width=64, q=FAKE, ld_q=64, scale=FAKE):
        of = lambda a: None if a is None else vp(a)  # noqa: E731
        return eck.lib().quantise_rows(of(x), order, dtype, ld_x, n, width, of(q), ld_q, of(scale), None)

    assert call(x=None) == call(q=None) == call(scale=None) == call(n=0) == call(width=0) == call(order=2) == call(dtype=2) == eck.EINVAL
    assert call(ld_x=63) == call(ld_q=48) == call(order=1, n=65) == eck.ESHAPE
    assert call(n=(1 << 31) + 1) == call(width=131072, ld_x=1 << 18, ld_q=1 << 18) == eck.EUNSUPPORTED
    assert call(x=FAKE + 1) == call(x=FAKE + 2, dtype=0) == call(q=FAKE + 8) == call(ld_q=72) == call(scale=FAKE + 2) == eck.EALIGN


def test_product_int8_validates_before_launch():
    vp = C.c_void_p
    W = eck.lib().product_int8_workspace_bytes

    def call(x=FAKE, ld_x=64, xs=FAKE, n=16, n_in=64, n_out=32, w=FAKE, ld_w=64, scale=FAKE, act=-1, dtype=1, y=FAKE, ld_y=32, ws=None, ws_bytes=0):
        of = lambda a: None if a is None else vp(a)  # noqa: E731
        return eck.lib().product_int8(of(x), ld_x, of(xs), n, n_in, n_out, of(w), ld_w, of(scale), act, dtype, of(y), ld_y, of(ws), ws_bytes, None)

    assert call(x=None) == call(xs=None) == call(w=None) == call(scale=None) == call(y=None) == eck.EINVAL
    assert call(n=0) == call(n_in=0) == call(n_out=0) == call(act=-2) == call(act=3) == call(dtype=2) == eck.EINVAL
    assert call(ld_x=48) == call(ld_w=48) == call(ld_y=31) == eck.ESHAPE
    assert call(n=(1 << 31) + 1) == call(n_in=131072, ld_x=1 << 18, ld_w=1 << 18) == call(n_out=(1 << 20) + 1, ld_y=1 << 21) == eck.EUNSUPPORTED
    assert call(n=1 << 24, n_out=2048, ld_y=2048) == call(ld_x=1 << 23) == call(ld_w=1 << 23) == eck.EUNSUPPORTED
    assert call(x=FAKE + 8) == call(w=FAKE + 4) == call(ld_x=72) == call(ld_w=72) == eck.EALIGN
    assert call(xs=FAKE + 1) == call(scale=FAKE + 2) == call(y=FAKE + 1) == call(y=FAKE + 2, dtype=0) == eck.EALIGN
    assert W(0, 64, 64, -1) == W(16, 0, 64, -1) == W(16, 64, 0, -1) == W(16, 64, 64, 3) == W(1, 4096, 4096, 0) == 0
    need = W(100, 8192, 130, -1)
    assert need >= 100 * 130 * 4 * 2
    big = dict(n=100, n_in=8192, n_out=130, ld_x=8192, ld_w=8192, ld_y=130)
    assert call(**big) == call(ws=FAKE, ws_bytes=need - 1, **big) == eck.EWORKSPACE
    assert call(ws=FAKE + 16, ws_bytes=need, **big) == eck.EALIGN


def test_sample_select_validates_before_launch():
    vp = C.c_void_p
    W = eck.lib().sample_select_workspace_bytes

    def call(energy=FAKE, legal=None, n=1 << 12, seg=4, uniform=FAKE, draws=8, t=0.5, k=0, top_p=0.9, min_p=0.1, idx=FAKE, logprob=FAKE, count=FAKE,
             ws=FAKE, ws_bytes=1 << 40):
        of = lambda a: None if a is None else vp(a)  # noqa: E731
        return eck.lib().sample_select(of(energy), of(legal), n, seg, of(uniform), draws, t, k, top_p, min_p, of(idx), of(logprob), of(count), of(ws),
                                       ws_bytes, None)

    nan, inf = float("nan"), float("inf")
    assert call(energy=None) == call(uniform=None) == call(idx=None) == call(n=0) == call(seg=0) == call(draws=0) == eck.EINVAL
    assert call(t=-0.1) == call(t=nan) == call(t=inf) == call(top_p=0.0) == call(top_p=1.01) == call(top_p=nan) == eck.EINVAL
    assert call(min_p=-0.1) == call(min_p=1.01) == call(min_p=nan) == eck.EINVAL
    assert call(seg=3) == eck.ESHAPE
    assert call(n=(1 << 31) + 1, seg=1) == call(n=(1 << 21) + 2, seg=(1 << 20) + 1) == eck.EUNSUPPORTED
    need = W(1 << 18, 1, 8)
    assert need > 0 == W(1 << 14, 1, 8) == W(1 << 20, 64, 8) and W((1 << 31) + 1, 1, 8) == W((1 << 21) + 2, (1 << 20) + 1, 8) == 0
    assert call(n=1 << 18, seg=1, ws=None) == call(n=1 << 18, seg=1, ws_bytes=need - 1) == eck.EWORKSPACE
    assert call(n=1 << 18, seg=1, ws=FAKE + 16) == eck.EALIGN
    assert call(energy=FAKE + 2) == call(uniform=FAKE + 1) == call(idx=FAKE + 2) == call(logprob=FAKE + 2) == call(count=FAKE + 1) == eck.EALIGN
    assert W(0, 1, 1) == W(10, 3, 1) == W(10, 0, 1) == W(10, 1, 0) == 0


def test_the_binding_refuses_what_it_cannot_pass_on():
    """tensors that are not on the GPU, of other shapes and types: refused before the library is called"""
    f, b, q = torch.zeros(4, 16), torch.zeros(4, 16, dtype=torch.bfloat16), torch.zeros(4, 16, dtype=torch.int8)
    for call in (lambda: eck.quantise_rows(f, q, torch.zeros(4)), lambda: eck.quantise_rows(f.double(), q, torch.zeros(4)),
                 lambda: eck.product_int8(q, torch.zeros(4), q, torch.zeros(4), torch.zeros(4, 4), None),
                 lambda: eck.product_int8(q, torch.zeros(4), q, torch.zeros(4), torch.zeros(4, 4).double(), None),
                 lambda: eck.sample_select(f.view(-1), None, 1, torch.zeros(1, 2), torch.zeros(2, dtype=torch.int32), None, None, None)):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: eck.quantise_rows(f, torch.zeros(4, 15, dtype=torch.int8), torch.zeros(4)),
                 lambda: eck.quantise_rows(b, torch.zeros(17, 4, dtype=torch.int8), torch.zeros(17), order=eck.COLUMNS),
                 lambda: eck.sample_select(f.view(-1), None, 2, torch.zeros(1, 2), torch.zeros(2, dtype=torch.int32), None, None, None),
                 lambda: eck.sample_select(f.view(-1), None, 1, torch.zeros(2), torch.zeros(2, dtype=torch.int32), None, None, None),
                 lambda: eck.sample_select(f.view(-1), None, 1, torch.zeros(1, 2), None, None, None, None)):
        with pytest.raises(ValueError):
            call()


def test_a_captured_pass_of_a_gated_model_has_a_workspace_of_its_own(monkeypatch):
    """what a graph writes to is neither lent to other calls nor given up when one of them wants more"""
    empty, capturing = torch.empty, [False]
    monkeypatch.setattr(torch, "empty", lambda *size, device=None, **kw: empty(*size, **kw))
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: capturing[0])
    model = object.__new__(gated.GatedModel)
    model._work = {}
    first = model._ws(100)
    assert model._ws(60) is first
    capturing[0] = True
    captured = [model._ws(100), model._ws(100), model._ws(500)]
    capturing[0] = False
    assert captured[2].numel() == 500 and model._ws(70) is first
    larger = model._ws(1000)
    assert larger.numel() == 1000 and model._ws(1) is larger
    assert len({t.data_ptr() for t in captured + [first, larger]}) == 5


def test_8_bit_weights_are_not_laid_out_by_a_pass_that_is_only_recorded(monkeypatch):
    capturing = [True]
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: capturing[0])
    model = object.__new__(gated.GatedModel)
    model.params, model.bf16, model.steps, model._int8, model._int8_steps = {}, {}, 3, None, None
    with pytest.raises(RuntimeError, match="laid out"):
        model._quantised()
    assert model._int8 is None
    capturing[0] = False
    model._quantised()
    capturing[0] = True
    model._quantised()
    model.steps = 4
    with pytest.raises(RuntimeError, match="laid out"):
        model._quantised()
    assert model._int8_steps == 3


@pytest.fixture
def on_the_cpu(monkeypatch):
    """plans of CPU tensors, which the library never sees"""
    def here(t, dtype, name):
        if t.dtype is not dtype or not t.is_contiguous():
            eck._refuse(t, dtype, name, "a contiguous CUDA tensor")
        return t

    monkeypatch.setattr(eck, "_here", here)
    monkeypatch.setattr(eck, "_device", lambda: 0)


def lists_of(count, n, eight=False):
    state = (lambda: torch.zeros(n, dtype=torch.uint8)) if eight else (lambda: torch.zeros(n))
    make = {"grads": lambda: torch.zeros(n), "params": lambda: torch.zeros(n), "m": state, "v": state, "copies": lambda: torch.zeros(n, dtype=torch.bfloat16)}
    if eight:
        make["m_scale"] = make["v_scale"] = lambda: torch.zeros(-(-n // eck.STATE_BLOCK), dtype=torch.uint8)
    return {name: [one() for _ in range(count)] for name, one in make.items()}


@pytest.mark.parametrize("eight", [False, True])
def test_a_plan_holds_its_tensors_whatever_becomes_of_the_lists(on_the_cpu, eight):
    lists = lists_of(3, 200, eight)
    seen = [weakref.ref(t) for tensors in lists.values() for t in tensors]
    plan = eck.Parameters(**lists)
    lists["m"][1] = None
    for tensors in lists.values():
        tensors.clear()
    gc.collect()
    assert all(r() is not None for r in seen)
    del plan
    gc.collect()
    assert all(r() is None for r in seen)


def test_gradients_that_are_refused_leave_a_plan_as_it_is(on_the_cpu):
    lists = lists_of(3, 50)
    plan = eck.Parameters(**lists)
    had = [(e.grad, e.grad_dtype, e.n) for e in plan._array]
    for bad in (torch.zeros(49), torch.zeros(50, dtype=torch.float64), torch.zeros(100)[::2]):
        with pytest.raises((ValueError, TypeError)):
            plan.set_grads([torch.zeros(50, dtype=torch.bfloat16), torch.zeros(50), bad])
        assert [(e.grad, e.grad_dtype, e.n) for e in plan._array] == had
        assert [t.data_ptr() for t in plan._kept["grads"]] == [address for address, _, _ in had]
    new = [torch.zeros(50, dtype=torch.bfloat16) for _ in range(3)]
    plan.set_grads(new)
    assert [(e.grad, e.grad_dtype) for e in plan._array] == [(t.data_ptr(), eck.BF16) for t in new]


def test_tensors_that_share_memory_are_refused(on_the_cpu):
    n = 64
    apart = lambda: torch.zeros(n)  # noqa: E731
    memory, bytes_ = torch.zeros(4 * n), torch.zeros(8 * n, dtype=torch.uint8)

    def written(*tensors, **kw):
        with pytest.raises(ValueError, match="of their own"):
            eck.Parameters([apart()], *[[t] for t in tensors], **{k: [t] for k, t in kw.items()})

    at = lambda first: memory[first:first + n]  # noqa: E731
    eck.Parameters([apart()], [at(0)], [at(n)], [at(2 * n)], copies=[at(3 * n).view(torch.bfloat16)[:n]])  # (neighbours)
    for first in (0, 1, n - 1):
        written(at(n), at(n + first), apart())
        written(apart(), at(n), at(n - first))
        written(at(n + first), apart(), at(n))
    written(apart(), apart(), at(n), copies=at(n + 5).view(torch.bfloat16)[n:])
    written(at(0), apart(), apart(), copies=at(0).view(torch.bfloat16)[:n])
    state = lambda first, size=n: bytes_[first:first + size]  # noqa: E731
    eck.Parameters([apart()], [apart()], [state(0)], [state(n)], [state(2 * n, 1)], [state(2 * n + 1, 1)])
    written(apart(), state(0), state(n - 1), state(2 * n, 1), state(2 * n + 1, 1))
    written(apart(), state(0), state(n), state(2 * n, 1), state(2 * n, 1))
    written(apart(), state(0), state(n), state(2 * n - 1, 1), state(2 * n, 1))

    # gradients: in memory of their own or, element for element, where their parameter or its states lie
    def grads(*of, **how):
        plan = eck.Parameters([apart(), apart()], [at(0), at(n)], [apart(), at(2 * n)], [apart(), apart()], **how)
        plan.set_grads([apart() if g is None else g for g in of])

    copy = torch.zeros(2 * n, dtype=torch.bfloat16)
    grads(at(0), at(n))
    grads(None, at(2 * n))
    grads(copy[:n], None, copies=[copy[:n], None])
    grads(at(3 * n), at(3 * n))  # (both the same, but only read)
    for first, second in ((at(1), None), (at(n), None), (None, at(n - 1)), (at(2 * n), None), (None, at(3 * n - 1)), (at(0).view(torch.bfloat16)[:n], None),
                          (None, at(n).view(torch.bfloat16)[n:])):
        with pytest.raises(ValueError, match="must not lie"):
            grads(first, second)
    for first, second in ((copy[1:n + 1], None), (None, copy[:n])):
        with pytest.raises(ValueError, match="must not lie"):
            grads(first, second, copies=[copy[:n], None])
    with pytest.raises(ValueError, match="must not lie"):  # (a state of bytes is no gradient's memory)
        eck.Parameters([memory[:n // 4]], [apart()[:n // 4]], [memory[:n // 4].view(torch.uint8)[:n // 4]], [state(0, n // 4)], [state(n, 1)], [state(n + 1, 1)])


class ElsewhereOnTheGPU:
    is_cuda = True

    def is_contiguous(self):
        return True

    def get_device(self):
        return 1

    def data_ptr(self):
        return FAKE

    def numel(self):
        return 1 << 30

    def element_size(self):
        return 1


def test_plans_and_workspaces_of_another_device_are_refused(on_the_cpu, monkeypatch):
    lists = lists_of(2, 50)
    plan, one = eck.Parameters(**lists), torch.zeros(1)
    need = eck.gradients_norm_workspace_bytes(plan)
    assert need > 0
    monkeypatch.setattr(eck, "lib", lambda: pytest.fail("the library was called"))
    q, f = torch.zeros(4, 16, dtype=torch.int8), torch.zeros(4)
    for call in (lambda ws: eck.gradients_norm(plan, one, one, ws), lambda ws: eck.product_int8(q, f, q, f, torch.zeros(4, 4), ws),
                 lambda ws: eck.sample_select(torch.zeros(64), None, 1, torch.zeros(1, 2), torch.zeros(2, dtype=torch.int32), None, None, ws)):
        with pytest.raises(ValueError, match="current device"):
            call(ElsewhereOnTheGPU())
    monkeypatch.setattr(eck, "_device", lambda: 1)
    for call in (lambda: eck.adamw_step(plan, 1e-3, 1), lambda: eck.gradients_norm(plan, one, one, None), lambda: plan.set_grads(lists["grads"])):
        with pytest.raises(ValueError, match="current device"):
            call()


@pytest.mark.parametrize("n", [1 << 12, 1 << 18])
@pytest.mark.parametrize("k,t", [(0, 0.5), (1, 0.5), (100, 0.5), (5000, 0.5), (0, 0.0)])
def test_more_draws_than_are_counted_are_refused(n, k, t):
    F, W = eck.lib().sample_select, eck.lib().sample_select_workspace_bytes
    vp = C.c_void_p
    assert W(1 << 18, 1, 1 << 31) == W(1 << 18, 1, 8)
    for draws in ((1 << 31) + 1, (1 << 32) - 1):
        assert W(n, 1, draws) == 0
        assert F(vp(FAKE), None, n, 1, vp(FAKE), draws, t, k, 0.9, 0.1, vp(FAKE), vp(FAKE), vp(FAKE), vp(FAKE), 1 << 40, None) == eck.EUNSUPPORTED


def test_sizes_past_32_bits_are_refused_and_not_cut_off(on_the_cpu, monkeypatch):
    monkeypatch.setattr(eck, "lib", lambda: pytest.fail("the library was called"))
    monkeypatch.setattr(eck, "_here_rows", lambda t, name, dtype, shape: t.stride(0))
    monkeypatch.setattr(eck, "_int8", lambda t, name, shape: t.stride(0))
    monkeypatch.setattr(eck, "_stream", lambda: None)
    empty = lambda *shape, dtype=torch.float32: torch.empty(*shape, dtype=dtype, device="meta")  # noqa: E731
    past, i8 = (1 << 32) + 16, torch.int8
    few = dict(energy=empty(64), legal=None, n_segments=1, uniform=empty(1, 2), idx_out=empty(2, dtype=torch.int32), logprob_out=None, count_out=None, ws=None)
    for call in (lambda: eck.quantise_rows(empty(2, past), empty(2, past, dtype=i8), empty(2)),
                 lambda: eck.product_int8(empty(2, past, dtype=i8), empty(2), empty(3, past, dtype=i8), empty(3), empty(2, 3), None),
                 lambda: eck.product_int8(empty(2, 16, dtype=i8), empty(2), empty(past, 16, dtype=i8), empty(past), empty(2, past), None),
                 lambda: eck.product_int8_workspace_bytes(2, past, 3), lambda: eck.product_int8_workspace_bytes(2, 3, -1),
                 lambda: eck.sample_select(**dict(few, uniform=empty(1, past), idx_out=empty(past, dtype=torch.int32))),
                 lambda: eck.sample_select(**few, k=past), lambda: eck.sample_select(**few, k=-1),
                 lambda: eck.sample_select_workspace_bytes(64, 1, past), lambda: eck.sample_select_workspace_bytes(64, past, 1)):
        with pytest.raises(ValueError, match="32 bits"):
            call()


def test_indices_and_counts_are_whole_numbers(on_the_cpu, monkeypatch):
    monkeypatch.setattr(eck, "_stream", lambda: None)
    called = []
    library = type("Library", (), {"sample_select": staticmethod(lambda *args: called.append(args) or eck.OK)})
    monkeypatch.setattr(eck, "lib", lambda: library)

    def call(idx, count):
        eck.sample_select(torch.zeros(64), None, 1, torch.zeros(1, 2), idx, None, count, None)

    whole = (torch.int32, torch.uint32)
    for idx in whole:
        call(torch.zeros(2, dtype=idx), None)
        for count in whole:
            call(torch.zeros(2, dtype=idx), torch.zeros(1, dtype=count))
    assert len(called) == 6
    for wrong in (torch.float32, torch.int64, torch.int16):
        with pytest.raises(TypeError):
            call(torch.zeros(2, dtype=wrong), None)
        with pytest.raises(TypeError):
            call(torch.zeros(2, dtype=torch.int32), torch.zeros(1, dtype=wrong))
    assert len(called) == 6
