"""GPU: AdamW over many tensors and the norm of their gradients.

32-bit states against the formula in 64 bits, e = 2^-24 a rounding: m is two products and a sum of rounded constants, v one more product.
8-bit states byte by byte against the definition worked out with numpy's IEEE arithmetic, and against the formats' own properties."""
import math

import numpy as np
import pytest
import torch

from paper_2411_18873_amd import eck

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
MARK = 77
SIZES = [1, 3, 4, 5, 127, 128, 129, 1000, 0, 2047, 2048, 2049, 70001]
GAMMA, MIX, MASK64 = 0x9E3779B97F4A7C15, (0xBF58476D1CE4E5B9, 0x94D049BB133111EB), (1 << 64) - 1


class Piece:
    """n elements in a buffer of marks, `offset` elements from its start"""

    def __init__(self, values, offset=0):
        self.n, self.offset = values.numel(), offset
        self.flat = torch.full((self.n + offset + 40,), MARK, dtype=values.dtype, device="cuda")
        self.t = self.flat[offset:offset + self.n]
        self.t.copy_(values)

    def untouched(self):
        return bool((self.flat[:self.offset] == MARK).all() and (self.flat[self.offset + self.n:] == MARK).all())


def make(sizes, kind, seed, offset=0, eight=False):
    g = torch.Generator().manual_seed(seed)
    rand = lambda n, size: torch.randn(n, generator=g) * size  # noqa: E731
    out = {k: [] for k in ("grads", "params", "m", "v", "m_scale", "v_scale", "copies")}
    for i, n in enumerate(sizes):
        dtype = torch.bfloat16 if kind == "bf16" or (kind == "both" and i % 2) else torch.float32
        size = torch.exp(rand(n, 1.5)) * 0.01
        out["grads"].append(Piece((rand(n, 1.0) * size).to(dtype), offset))
        out["params"].append(Piece(rand(n, 0.1), offset))
        if eight:
            blocks = -(-n // eck.STATE_BLOCK)
            m = torch.randint(0, 256, (n,), generator=g)
            v = torch.randint(0, 0x7C, (n,), generator=g)  # (0x7C: infinity)
            out["m"].append(Piece(torch.where(m % 128 == 127, 3, m).to(torch.uint8), offset))
            out["v"].append(Piece(v.to(torch.uint8), offset))
            out["m_scale"].append(Piece(torch.randint(100, 118, (blocks,), generator=g).to(torch.uint8), offset))
            out["v_scale"].append(Piece(torch.randint(85, 105, (blocks,), generator=g).to(torch.uint8), offset))
        else:
            out["m"].append(Piece(rand(n, 1.0) * size, offset))
            out["v"].append(Piece((size * rand(n, 1.0)) ** 2, offset))
        out["copies"].append(None if i % 3 == 2 else Piece(torch.zeros(n, dtype=torch.bfloat16), offset))
    return out


def plan(t, decay=0.0):
    lists = {k: [None if p is None else p.t for p in v] if v else None for k, v in t.items()}
    return eck.Parameters(**lists, weight_decay=decay)


def all_untouched(t):
    return all(p is None or p.untouched() for v in t.values() for p in v)


def check_step(sizes, kind, seed, offset=0, step=3, decay=0.01, scale=0.5, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8):
    t = make(sizes, kind, seed, offset)
    had = {k: [p.t.double().cpu() for p in t[k]] for k in ("grads", "params", "m", "v")}
    factor = torch.full((1,), scale, device="cuda") if scale is not None else None
    eck.adamw_step(plan(t, decay), lr=lr, step=step, beta1=beta1, beta2=beta2, eps=eps, grad_scale=factor)
    torch.cuda.synchronize()
    assert all_untouched(t)
    for i in range(len(sizes)):
        g = had["grads"][i] * (1.0 if scale is None else scale)
        m, v = beta1 * had["m"][i] + (1 - beta1) * g, beta2 * had["v"][i] + (1 - beta2) * g * g
        m_size = beta1 * had["m"][i].abs() + (1 - beta1) * g.abs()
        den = torch.sqrt(v / (1 - beta2 ** step)) + eps
        rate = lr / (1 - beta1 ** step)
        w = had["params"][i] * (1 - lr * decay) - rate * m / den
        assert ((t["m"][i].t.double().cpu() - m).abs() <= 5 * E * m_size + 1e-45).all()
        assert ((t["v"][i].t.double().cpu() - v).abs() <= 6 * E * v + 1e-45).all()
        # the step: m's error, and eight roundings (g, v's six halved by the root, the correction, root, eps, quotient, rate)
        bound = 3 * E * had["params"][i].abs() + 20 * E * rate * m_size / den
        assert ((t["params"][i].t.double().cpu() - w).abs() <= bound).all()
        if t["copies"][i] is not None:
            assert torch.equal(t["copies"][i].t, t["params"][i].t.bfloat16())


@pytest.mark.parametrize("kind", ["f32", "bf16", "both"])
@pytest.mark.parametrize("offset", [0, 1, 3])
def test_step_with_32_bit_states(kind, offset):
    check_step(SIZES, kind, 1 + offset, offset)


@pytest.mark.parametrize("count", [1, 12, 13, 48, 49, 200, 201, 450])
def test_as_many_tensors_as_there_are(count):
    check_step([1 + 37 * i % 301 for i in range(count)], "both", count)


@pytest.mark.parametrize("step,decay,scale,beta1,beta2", [(1, 0.0, None, 0.9, 0.999), (1, 0.1, 1.0, 0.0, 0.0), (100000, 0.0, 0.01, 0.95, 0.98),
                                                          (2 ** 32 - 1, 0.5, 2.0, 0.9, 0.999)])
def test_numbers_of_a_step(step, decay, scale, beta1, beta2):
    check_step([1000, 77], "f32", 9, step=step, decay=decay, scale=scale, beta1=beta1, beta2=beta2)


def test_a_large_tensor_and_its_decay_by_tensor():
    t = make([3_000_001, 50], "bf16", 5)
    before = [p.t.clone() for p in t["params"]]
    for p in t["grads"] + t["m"]:
        p.t.zero_()
    eck.adamw_step(plan(t, [0.0, 0.25]), lr=0.5, step=2)
    assert torch.equal(t["params"][0].t, before[0]) and torch.equal(t["params"][1].t, before[1] * 0.875)


def finalise(z):
    z = (z ^ (z >> np.uint64(30))) * np.uint64(MIX[0])
    z = (z ^ (z >> np.uint64(27))) * np.uint64(MIX[1])
    return z ^ (z >> np.uint64(31))


def draws(first, n, seed, step):
    """16-bit draws of m and v of elements first .. first + n - 1"""
    with np.errstate(over="ignore"):
        start = finalise(np.array([(seed + GAMMA * (step + 1)) & MASK64], dtype=np.uint64))
        e = np.arange(first, first + n, dtype=np.uint64)
        word = finalise(start + (e // np.uint64(2) + np.uint64(1)) * np.uint64(GAMMA))
    half = np.where(e % 2 == 0, word & np.uint64(0xFFFFFFFF), word >> np.uint64(32)).astype(np.int64)
    return half & 0xFFFF, half >> 16


def grid(fraction, low, top):
    """a format's numbers from 0 up, by their codes"""
    codes = np.arange((top - low + 2) << fraction)
    exponent, part = codes >> fraction, codes & ((1 << fraction) - 1)
    return np.where(exponent == 0, part * 2.0 ** (low - fraction), (1 + part / 2.0 ** fraction) * 2.0 ** (exponent - 1 + low))


GRIDS = {"m": grid(3, -6, 8), "v": grid(2, -14, 15)}


def decode(code, scale, which):
    values = GRIDS[which]
    power = np.exp2(scale.astype(np.float64) - 127)[np.arange(code.size) // eck.STATE_BLOCK]
    return np.where(code & 0x80, -1.0, 1.0) * values[code & 0x7F] * power


def encode(x, draw, which):
    """bytes and scales of float32 numbers, by looking for the grid's neighbours"""
    n, values, top = x.size, GRIDS[which], 7 if which == "m" else 14
    blocks = -(-n // eck.STATE_BLOCK)
    padded = np.zeros(blocks * eck.STATE_BLOCK)
    padded[:n] = np.abs(x.astype(np.float64))
    most = padded.reshape(blocks, -1).max(1)
    exponent = np.where(most > 0, np.frexp(np.where(most > 0, most, 1.0))[1] - 1, -127)
    power = np.clip(exponent - top, -100, 100)
    size = np.abs(x.astype(np.float64)) / np.exp2(power)[np.arange(n) // eck.STATE_BLOCK]
    below = np.searchsorted(values, size, side="right") - 1
    step = values[below + 1] - values[below]
    code = below + ((size - values[below]) / step * 65536 + draw >= 65536)
    # where the way to the lower number lies within a rounding of the draw either neighbour is right (numbers below the normal ones are
    # rounded once on the way, to 2^-20 of a step)
    near = np.abs((size - values[below]) / step * 65536 + draw - 65536) < 2.0 ** -3
    if which == "v":
        code = np.where(size > 0, np.maximum(code, 1), code)
    return code | np.where((x < 0) | ((x == 0) & np.signbit(x)), 0x80, 0) if which == "m" else code, power + 127, near


@pytest.mark.parametrize("kind,offset", [("both", 0), ("bf16", 1), ("f32", 3)])
def test_8_bit_states_byte_by_byte(kind, offset):
    t = make(SIZES, kind, 21 + offset, offset, eight=True)
    f = np.float32
    seed, step, beta1, beta2, scale = 0x123456789ABCDEF, 12, f(0.9), f(0.999), f(0.5)
    had = {k: [p.t.cpu() for p in t[k]] for k in ("grads", "params", "m", "v", "m_scale", "v_scale")}
    eck.adamw_step(plan(t, 0.01), lr=1e-3, step=step, grad_scale=torch.full((1,), 0.5, device="cuda"), seed=seed)
    torch.cuda.synchronize()
    assert all_untouched(t)
    first = unsure = 0
    for i, n in enumerate(SIZES):
        if n == 0:
            continue
        code = {k: had[k][i].numpy() for k in ("m", "v", "m_scale", "v_scale")}
        g = had["grads"][i].float().numpy() * scale
        m = decode(code["m"], code["m_scale"], "m").astype(f) * beta1 + g * f(1 - 0.9)
        v = decode(code["v"], code["v_scale"], "v").astype(f) * beta2 + g * f(1 - 0.999) * g
        for name, x, draw in (("m", m, draws(first, n, seed, step)[0]), ("v", v, draws(first, n, seed, step)[1])):
            want, want_scale, near = encode(x, draw, name)
            got, got_scale = t[name][i].t.cpu().numpy(), t[name + "_scale"][i].t.cpu().numpy()
            assert np.array_equal(got_scale, want_scale), (name, n)
            assert (near | (got == want)).all(), (name, n)
            unsure += (got != want).sum()
        den = np.sqrt(v.astype(np.float64) / (1 - 0.999 ** step)) + 1e-8
        rate = 1e-3 / (1 - 0.9 ** step)
        w = had["params"][i].double().numpy() * (1 - 1e-5) - rate * m / den
        bound = 3 * E * np.abs(w) + 12 * E * rate * np.abs(m) / den + 3 * E * np.abs(had["params"][i].numpy())
        assert (np.abs(t["params"][i].t.double().cpu().numpy() - w) <= bound).all()
        first += -(-n // eck.STATE_BLOCK) * eck.STATE_BLOCK
    assert unsure <= 4


def test_states_of_zero_bytes_are_zeros_and_no_v_becomes_zero():
    n = 5000
    g = torch.Generator().manual_seed(1)
    grads = torch.exp(torch.randn(n, generator=g) * 6).cuda() * 1e-3  # (1e-3 times e^-20 to e^20)
    grads[100:300] = 0.0
    grads[1000] = 0.0
    param, m, v = torch.zeros(n, device="cuda"), torch.zeros(n, dtype=torch.uint8, device="cuda"), torch.zeros(n, dtype=torch.uint8, device="cuda")
    scales = [torch.zeros(-(-n // eck.STATE_BLOCK), dtype=torch.uint8, device="cuda") for _ in range(2)]
    p = eck.Parameters([grads], [param], [m], [v], [scales[0]], [scales[1]])
    for step in range(1, 4):
        eck.adamw_step(p, lr=1e-3, step=step, seed=5)
        if step == 1:  # m / (sqrt(v) + eps) is the gradient by its size and eps
            assert torch.allclose(param, -1e-3 * grads / (grads + 1e-8), rtol=1e-4, atol=0)
        assert torch.equal(v == 0, grads == 0)
        assert (m[grads == 0] == 0).all()
    assert torch.isfinite(param).all()


@pytest.mark.parametrize("size", [1e15, 1e17, 1e18, 1e20, 2e20])
def test_8_bit_states_of_the_largest_gradients(size):
    """squares up to the end of fp32: a state is the format's number below or above, a quarter (v) or an eighth (m) off at most"""
    n = 300
    g = torch.linspace(0.3, 1.0, n).double() * size
    grads = torch.where(torch.arange(n) % 3 == 0, -g, g).float().cuda()
    param = torch.zeros(n, device="cuda")
    m, v = [torch.zeros(n, dtype=torch.uint8, device="cuda") for _ in range(2)]
    scales = [torch.zeros(-(-n // eck.STATE_BLOCK), dtype=torch.uint8, device="cuda") for _ in range(2)]
    p = eck.Parameters([grads], [param], [m], [v], [scales[0]], [scales[1]])
    for step in range(1, 4):
        eck.adamw_step(p, lr=1e-3, step=step, seed=5)
        got_m, got_v = [t.view(kind).double() * torch.exp2(s.double() - 127).repeat_interleave(eck.STATE_BLOCK)[:n]
                        for t, kind, s in ((m, torch.float8_e4m3fn, scales[0]), (v, torch.float8_e5m2, scales[1]))]
        # (each step's rounding is part of the next one's state)
        want_m, want_v = (1 - 0.9 ** step) * grads.double(), (1 - 0.999 ** step) * grads.double() ** 2
        assert ((got_m - want_m).abs() <= step * 0.126 * want_m.abs()).all()
        assert ((got_v - want_v).abs() <= step * 0.251 * want_v).all()
        assert (param * grads <= 0).all() and torch.isfinite(param).all()  # (0 where v / (1 - beta2^t) passes fp32's range)


def test_8_bit_roundings_are_right_on_average():
    """the same step from the same state under 4000 seeds: the mean of the new states is the state in 32 bits.  A rounding is off by f(1 - f)
    of a step squared at most a quarter, so the mean of k of them by half a step over root k, and six times that is not seen"""
    n, k = 256, 4000
    t = make([n], "f32", 3, eight=True)
    had = {name: [p.t.clone() for p in t[name]] for name in ("params", "m", "v", "m_scale", "v_scale")}
    p = plan(t)
    total = {"m": 0.0, "v": 0.0}
    for seed in range(k):
        for name, tensors in had.items():
            t[name][0].t.copy_(tensors[0])
        eck.adamw_step(p, lr=0.0, step=1, seed=seed)
        for name, kind in (("m", torch.float8_e4m3fn), ("v", torch.float8_e5m2)):
            power = torch.exp2(t[name + "_scale"][0].t.double() - 127).repeat_interleave(eck.STATE_BLOCK)
            total[name] = total[name] + t[name][0].t.view(kind).double() * power
    assert torch.equal(t["params"][0].t, had["params"][0])
    g = t["grads"][0].t.double().cpu().numpy()
    for name, beta, part in (("m", 0.9, 0.1 * g), ("v", 0.999, 0.001 * g * g)):
        want = beta * decode(had[name][0].cpu().numpy(), had[name + "_scale"][0].cpu().numpy(), name) + part
        power = np.exp2(t[name + "_scale"][0].t.cpu().numpy() - 127.0).repeat(eck.STATE_BLOCK)
        values = GRIDS[name] * 1.0
        size = np.abs(want) / power
        below = np.searchsorted(values, size, side="right") - 1
        step = (values[below + 1] - values[below]) * power
        fine = (below > 0) | (name == "m")  # (a v below the least number becomes that)
        off = np.abs(total[name].cpu().numpy() / k - want)
        assert (off[fine] <= (6 * 0.5 / math.sqrt(k) + 2.0 ** -16) * step[fine]).all()


def test_what_is_not_finite_stays_where_it_is():
    for eight in (False, True):
        t = make([1000], "f32", 8, eight=eight)
        t["grads"][0].t[5], t["grads"][0].t[700] = float("nan"), float("inf")
        eck.adamw_step(plan(t), lr=1e-3, step=4)
        bad = torch.zeros(1000, dtype=torch.bool, device="cuda")
        bad[5] = bad[700] = True
        m, v = t["m"][0].t, t["v"][0].t
        if eight:
            m, v = m.view(torch.float8_e4m3fn).float(), v.view(torch.float8_e5m2).float()
        assert torch.equal(torch.isfinite(m), ~bad) and torch.equal(torch.isfinite(v), ~bad)
        assert torch.equal(torch.isfinite(t["params"][0].t), ~bad)


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("scale", [float("nan"), float("inf"), float("-inf")])
def test_a_scale_that_is_not_finite_changes_nothing(eight, scale):
    t = make(SIZES, "both", 30, eight=eight)
    before = {k: [None if p is None else p.flat.clone() for p in v] for k, v in t.items()}
    eck.adamw_step(plan(t, 0.1), lr=1e-3, step=4, grad_scale=torch.full((1,), scale, device="cuda"))
    for k, v in t.items():
        assert all(p is None or torch.equal(p.flat, b) for p, b in zip(v, before[k]))


@pytest.mark.parametrize("sizes", [[1], [3, 0, 5], SIZES, [8191, 8192, 8193], [17 * i % 900 + 1 for i in range(500)], [3_000_001]])
@pytest.mark.parametrize("kind", ["f32", "bf16", "both"])
@pytest.mark.parametrize("offset", [0, 1])
def test_norm(sizes, kind, offset):
    t = make(sizes, kind, 3, offset)
    p = eck.Parameters([x.t for x in t["grads"]])
    norm, scale = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda")
    ws = torch.empty(eck.gradients_norm_workspace_bytes(p), dtype=torch.uint8, device="cuda")
    want = math.sqrt(sum(x.t.double().square().sum().item() for x in t["grads"]))
    for most in (want / 3, want * 3, float("inf")):
        eck.gradients_norm(p, norm, scale, ws, max_norm=most)
        most = float(np.float32(most))
        assert abs(norm.item() - want) <= E * want * 1.001
        assert abs(scale.item() - min(1.0, most / want)) <= 1.001 * E * min(1.0, most / want)
    assert all_untouched(t)


@pytest.mark.parametrize("kind,offset", [("both", 0), ("f32", 1), ("bf16", 3)])
@pytest.mark.parametrize("sizes", [[2048], [2047, 2049, 1], [0, 4096, 0, 5, 2048 * 17 + 3], [131072], [131073], [100] * 16, [100] * 17, [1] * 64,
                                   [1] * 65, [0] * 30 + [777] * 64 + [0] * 9, [262144], [262145], [5000] * 40])
def test_norm_of_short_lists(sizes, kind, offset):
    """lists of a few blocks of threads, of as many tensors as a launch takes and one more, and of empty ones between"""
    test_norm(sizes, kind, offset)


def test_norm_of_the_largest_the_smallest_and_none():
    norm, scale = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda")
    ws = torch.empty(1 << 16, dtype=torch.uint8, device="cuda")
    for value, n, want, factor in ((1e30, 100, 1e31, 1e-31), (1e-40, 10000, 1e-38, 1.0), (0.0, 77, 0.0, 1.0), (3e38, 4, float("inf"), None)):
        grad = torch.full((n,), value, device="cuda")
        exact = grad[0].item() * math.sqrt(n)
        eck.gradients_norm(eck.Parameters([grad]), norm, scale, ws, max_norm=1.0)
        if factor is None:  # a norm past fp32's range
            assert norm.item() == float("inf") and scale.item() == pytest.approx(1.0 / exact, rel=1e-6)
        else:
            assert norm.item() == pytest.approx(exact, rel=1e-6, abs=1e-44) and scale.item() == pytest.approx(factor, rel=1e-6)
    for value in (float("nan"), float("inf")):
        grad = torch.ones(3000, device="cuda")
        grad[2999] = value
        eck.gradients_norm(eck.Parameters([grad]), norm, scale, ws, max_norm=1.0)
        assert not math.isfinite(norm.item()) and math.isnan(scale.item())
        eck.gradients_norm(eck.Parameters([grad]), None, scale, ws, max_norm=1.0)
        eck.gradients_norm(eck.Parameters([grad]), norm, None, ws)


@pytest.mark.parametrize("eight", [False, True])
def test_a_clipped_step_on_a_stream_and_as_a_graph(eight):
    """norm and step captured together, the step's number counted on the device: replays equal calls one by one"""
    sizes = [4096, 77, 12345, 128]
    sides = [make(sizes, "both", 40, eight=eight) for _ in range(2)]
    norms, scales = [torch.zeros(1, device="cuda") for _ in range(2)], [torch.zeros(1, device="cuda") for _ in range(2)]
    plans = [plan(t, 0.01) for t in sides]
    ws = [torch.empty(eck.gradients_norm_workspace_bytes(p), dtype=torch.uint8, device="cuda") for p in plans]
    count = torch.zeros(1, dtype=torch.int32, device="cuda")
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        count.add_(1)
        eck.gradients_norm(plans[1], norms[1], scales[1], ws[1], max_norm=0.05)
        eck.adamw_step(plans[1], lr=1e-2, step=5, step_more=count, grad_scale=scales[1], seed=9)
    for step in range(1, 6):
        for a, b in zip(sides[0]["grads"], sides[1]["grads"]):
            a.t.mul_(-0.7)
            b.t.copy_(a.t)
        torch.cuda.synchronize()
        eck.gradients_norm(plans[0], norms[0], scales[0], ws[0], max_norm=0.05)
        eck.adamw_step(plans[0], lr=1e-2, step=5 + step, grad_scale=scales[0], seed=9)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(norms[0], norms[1]) and torch.equal(scales[0], scales[1])
        for k in ("m", "v", "m_scale", "v_scale"):
            assert all(torch.equal(a.flat, b.flat) for a, b in zip(sides[0][k], sides[1][k]))
        # (powers of the betas by squaring on one side: a unit of the correction's last place)
        for a, b in zip(sides[0]["params"], sides[1]["params"]):
            assert (a.t - b.t).abs().max().item() <= 8 * E * (1 + 1e-2)
            b.t.copy_(a.t)


def test_a_tensor_in_two_places_is_refused():
    a = [torch.zeros(8, device="cuda") for _ in range(6)]
    eck.Parameters(a[:2], a[:2], a[2:4], a[4:6])  # (gradients are only read)
    for params, m, v in (([a[0], a[0]], a[2:4], a[4:6]), (a[:2], [a[2], a[2]], a[4:6]), (a[:2], a[2:4], [a[4], a[2]])):
        with pytest.raises(ValueError, match="of their own"):
            eck.Parameters(a[:2], params, m, v)
    copy = torch.zeros(8, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError, match="of their own"):
        eck.Parameters(a[:2], a[:2], a[2:4], a[4:6], copies=[copy, copy])


@pytest.mark.parametrize("eps", [0.0, 1e-30, 1e-18, 1e-13, 2e-12, 1e-8])
@pytest.mark.parametrize("step", [1, 5])
def test_8_bit_steps_of_the_smallest_gradients(eps, step):
    """down to those whose square is a denormal number: from states of zeros, as the formula has them.  Errors in relative terms: g and 1 - beta1 of m,
    g twice and 1 - beta2 of v, each product of v (of which those below 2^-126 are rounded to 2^-149: by half of that), the correction's factor
    and product, halved by the root; root and quotient by instructions of a unit each, eps, their sum, rate, its product with the step: 20 e"""
    n = 400
    grads = torch.exp2(torch.linspace(-73.0, -40.0, n)).cuda()
    grads[::2] *= -1
    param = torch.zeros(n, device="cuda")
    m, v = [torch.zeros(n, dtype=torch.uint8, device="cuda") for _ in range(2)]
    scales = [torch.zeros(-(-n // eck.STATE_BLOCK), dtype=torch.uint8, device="cuda") for _ in range(2)]
    eck.adamw_step(eck.Parameters([grads], [param], [m], [v], [scales[0]], [scales[1]]), lr=1e-3, beta1=0.5, beta2=0.5, step=step, eps=eps)
    g = grads.double()
    wide = 0.5 * g * g
    den = torch.sqrt(wide / (1 - 0.5 ** step)) + eps
    want = -1e-3 / (1 - 0.5 ** step) * 0.5 * g / den
    off = 20 * E + 0.5 * 1.5 * 2.0 ** -149 / wide  # (two products of v and the corrected one; half for the root)
    assert torch.isfinite(param).all()
    assert ((param.double() - want).abs() <= off * want.abs() * 1.01).all()
