"""GPU: gated feed-forward blocks at sizes whose products take each of the library's tiles, undivided and in shares of k, or the kernels
for narrow blocks, against 64-bit evaluations on the device.  Every case names the kernels that it is there for and is checked to have launched them, so that another
choice of tiles cannot take a kernel out of the tests unnoticed."""
import math
import re

import pytest
import torch

from paper_2411_18873_amd import eck
from test_gpu_operators import DTYPES, E, act_of

pytestmark = pytest.mark.gpu

# sizes (n, n_in, n_hidden, n_out) -> kernels: product and side of its tiles, "/k" where its k's are divided
BF16 = {
    (7706, 329, 769, 186): ("gate 256",),
    (5174, 151, 341, 2375): ("y 256",),
    (3406, 109, 3619, 354): ("slope 256",),
    (387, 4163, 3622, 2393): ("gradients 256",),
    (3012, 4162, 1020, 334): ("gradients 256",),
    (3743, 3271, 1261, 3933): ("gradients 256", "join store"),
    (4160, 4096, 4096, 4104): ("gate 128", "y 128", "slope 128", "gradients 128"),
    (8192, 2048, 4096, 2048): ("gate 256",),
    (2592, 102, 585, 124): ("gate 128",),
    (326, 3247, 2769, 112): ("gate 128/k",),
    (856, 198, 105, 3715): ("y 128",),
    (1584, 105, 1994, 110): ("slope 128",),
    (8728, 168, 196, 2946): ("slope 128/k",),
    (5579, 262, 142, 2383): ("slope 128/k",),
    (1398, 152, 136, 2100): ("slope 64/k",),
    (204, 215, 101, 2979): ("slope 64/k",),
    (206, 1203, 2186, 120): ("gradients 128",),
    (3981, 1631, 103, 170): ("gradients 128", "join store"),
    (208, 2961, 108, 140): ("gate 64/k",),
    (213, 107, 100, 131): ("gate 64", "y 64", "slope 64", "gradients 64"),
}
F32 = {
    (2078, 104, 486, 114): ("gate 128",),
    (430, 4135, 129, 213): ("gate 128/k",),
    (614, 227, 104, 3357): ("y 128",),
    (7380, 104, 272, 112): ("slope 128",),
    (742, 312, 130, 3885): ("slope 128/k",),
    (466, 4125, 101, 579): ("gradients 128",),
    (8686, 135, 350, 117): ("gradients 128", "join store"),
    (2048, 1024, 2048, 1024): ("gate 128", "slope 128", "gradients 128"),
    (218, 3700, 100, 1082): ("gate 64/k",),
    (241, 122, 101, 3582): ("slope 64/k",),
    (211, 120, 107, 141): ("gate 64", "y 64", "slope 64", "gradients 64"),
}
CASES = [(s, kind, k) for kind, cases in (("bf16", BF16), ("f32", F32)) for s, k in cases.items()]
NAMES = [kind + "-" + "x".join(map(str, s)) for s, kind, _ in CASES]


def kernels_of(events):
    """the block's kernels among a profile's events, as the tables above name them"""
    found, joins = set(), set()
    for e in events:
        name = e.name
        join = re.search(r"product::join_kernel<(\d), \d>", name)
        if join:
            joins.add(("store", "gate", "slope")[int(join.group(1))])
    for e in events:
        product = re.search(r"product_kernel<eck::product::Shape<(\d+), [^>]*>, (true|false), (true|false), (\d)>", e.name)
        gradients = re.search(r"gradients_kernel<eck::product::Shape<(\d+),", e.name)
        if gradients:
            found.add("gradients " + gradients.group(1))
        elif product:
            side, b_fast, kind = product.group(1), product.group(3) == "true", int(product.group(4))
            if kind:
                found.add(("", "gate ", "slope ")[kind] + side)
            elif b_fast:
                found.add("slope %s/k" % side)
            else:
                found.update({"y " + side} | ({"gate %s/k" % side} if "gate" in joins else set()))
    return found | {"join " + j for j in joins}


def profiled(call):
    with torch.profiler.profile(activities=[torch.profiler.ProfilerActivity.CUDA], acc_events=True) as profile:
        call()
        torch.cuda.synchronize()
    return kernels_of(profile.events())


class Block:
    """a block's operands, results and calls"""

    def __init__(self, x, wgu, wd, dy, kind, act):
        dtype, code, _ = DTYPES[kind]
        self.inputs = [t.to(dtype).cuda() for t in (x, wgu, wd, dy)]
        x, wgu, wd, dy = self.inputs
        (n, n_in), (n_hidden, n_out) = x.shape, wd.shape
        sizes = (n, n_in, n_hidden, n_out, code)
        nan = lambda *s, d=dtype: torch.full(s, math.nan, dtype=d, device="cuda")  # noqa: E731
        self.pre, self.y = nan(n, 2 * n_hidden, d=torch.float32), nan(n, n_out)
        self.grads = nan(n, n_in), nan(n_in, 2 * n_hidden), nan(n_hidden, n_out)
        self.ws = torch.full((max(eck.gatedffn_forward_workspace_bytes(*sizes), eck.gatedffn_backward_workspace_bytes(*sizes)),), 0xFF,
                             dtype=torch.uint8, device="cuda")
        self.act = act

    def forward(self):
        x, wgu, wd, _ = self.inputs
        eck.gatedffn_forward(x, wgu, wd, self.y, self.ws, pre_out=self.pre, act=self.act)

    def backward(self):
        x, wgu, wd, dy = self.inputs
        eck.gatedffn_backward(x, wgu, wd, self.pre, dy, *self.grads, self.ws, act=self.act)

    def both(self):
        self.forward()
        self.backward()


def hold(got, want, bound, what):
    worst = ((got.double() - want).abs() / (bound + 1e-300)).max().item()
    assert worst <= 1.0, "%s: %.3g times the bound" % (what, worst)     # (NaN is no less than anything)


@pytest.mark.parametrize("sizes,kind,kernels", CASES, ids=NAMES)
def test_results_of_every_tile(sizes, kind, kernels):
    n, n_in, n_hidden, n_out = sizes
    u, act = DTYPES[kind][2], eck.ACT_SILU if n % 2 else eck.ACT_GELU
    g = torch.Generator(device="cuda").manual_seed(n)
    normal = lambda *s, scale=1.0: torch.randn(*s, generator=g, device="cuda", dtype=torch.float64) * scale  # noqa: E731
    b = Block(normal(n, n_in), normal(n_in, 2 * n_hidden, scale=n_in ** -0.5), normal(n_hidden, n_out, scale=n_hidden ** -0.5), normal(n, n_out),
              kind, act)
    launched = profiled(b.both)
    assert set(kernels) <= launched, launched
    # the bounds of test_gpu_operators.ffn_case: sums of K terms off by K e of the sum of their magnitudes, stored values rounded once
    x, wgu, wd, dy = (t.double() for t in b.inputs)
    want_pre = x @ wgu
    off_pre = (n_in + 2) * E * (x.abs() @ wgu.abs())
    hold(b.pre, want_pre, off_pre, "pre")
    gate, up = want_pre.chunk(2, 1)
    off_g, off_u = off_pre.chunk(2, 1)
    a = act_of(act, gate)[0]
    h = a * up
    off_a = 1.13 * off_g + 8 * E * gate.abs()
    off_h = off_a * up.abs() + (a.abs() + off_a) * off_u
    off_h += u * (h.abs() + off_h)
    want = h @ wd
    hold(b.y, want, off_h @ wd.abs() + (n_hidden + 2) * E * (h.abs() @ wd.abs()) * 1.01 + u * want.abs() * 1.01, "y")

    gate, up = b.pre.double().chunk(2, 1)      # (the backward pass starts from the stored sums)
    a, slope = act_of(act, gate)
    h = a * up
    dh = dy @ wd.t()
    off_dh = (n_out + 2) * E * (dy.abs() @ wd.abs().t())
    off_a, off_s = 8 * E * gate.abs(), 16 * E * (1 + gate.abs())
    dg, du = dh * up * slope, dh * a
    off_dg = off_dh * (up * slope).abs() + (dh.abs() + off_dh) * up.abs() * off_s + 4 * E * dg.abs()
    off_du = off_dh * a.abs() + (dh.abs() + off_dh) * off_a + 4 * E * du.abs()
    d, off = torch.cat((dg, du), 1), torch.cat((off_dg, off_du), 1)
    off += u * (d.abs() + off)
    off_h = off_a * up.abs() + u * h.abs() + 4 * E * h.abs()
    for got, A, off_A, B, off_B, K, what in ((b.grads[0], d, off, wgu.t(), None, 2 * n_hidden, "dx"), (b.grads[1], x.t(), None, d, off, n, "dw_gate_up"),
                                             (b.grads[2], h.t(), off_h.t(), dy, None, n, "dw_down")):
        want = A @ B
        bound = (K + 2) * E * (A.abs() @ B.abs()) + u * want.abs()
        if off_A is not None:
            bound += off_A @ B.abs()
        if off_B is not None:
            bound += A.abs() @ off_B
        hold(got, want, 1.01 * bound, what)


@pytest.mark.parametrize("sizes,kind,kernels", CASES, ids=NAMES)
def test_whole_numbers_are_exact_in_every_tile(sizes, kind, kernels):
    """sums of a few small whole numbers, none of which loses anything: one right value per element"""
    n, n_in, n_hidden, n_out = sizes
    g = torch.Generator(device="cuda").manual_seed(n + 1)

    def whole(rows, columns, most, chance):
        t = torch.randint(-most, most + 1, (rows, columns), generator=g, device="cuda").double()
        return t * (torch.rand(rows, columns, generator=g, device="cuda") < chance)

    # about 24 terms a sum over the inputs, 4 over the outputs
    b = Block(whole(n, n_in, 1, 1.0), whole(n_in, 2 * n_hidden, 1, min(1.0, 24 / n_in)), whole(n_hidden, n_out, 1, min(1.0, 24 / n_hidden)),
              whole(n, n_out, 1, min(1.0, 4 / n_out)), kind, eck.ACT_RELU)
    b.both()
    x, wgu, wd, dy = (t.double() for t in b.inputs)
    pre = x @ wgu
    gate, up = pre.chunk(2, 1)
    a, slope = act_of(eck.ACT_RELU, gate)
    h, dh = a * up, dy @ wd.t()
    d = torch.cat((dh * up * slope, dh * a), 1)
    most = 256 if kind == "bf16" else 1 << 24          # whole numbers that the type holds, h and d being rounded to it
    assert h.abs().max() <= most and d.abs().max() <= most
    for got, want, what in ((b.pre, pre, "pre"), (b.y, h @ wd, "y"), (b.grads[0], d @ wgu.t(), "dx"), (b.grads[1], x.t() @ d, "dw_gate_up"),
                            (b.grads[2], h.t() @ dy, "dw_down")):
        assert want.abs().max() < 1 << 24              # (and the sums in fp32; results are rounded once)
        assert torch.equal(got, want.to(got.dtype)), what


ACTS = {"silu": eck.ACT_SILU, "gelu": eck.ACT_GELU, "relu": eck.ACT_RELU}
# rows that a narrow block of so many hidden units is one kernel for, by widths: inputs to 64 or 128, outputs to 64, 128 or 256
NARROW = [(n_in, n_out, n_hidden, n, act) for act in ACTS for n_in, n_out, rows in
          ((64, 64, 20011), (40, 128, 32700), (64, 200, 32768), (128, 57, 32700), (96, 100, 32000), (128, 256, 32767))
          for n_hidden, n in ((64, rows), (128, rows), (100, rows), (33, 70000 if n_in + n_out < 300 else 32767))]


@pytest.mark.parametrize("n_in,n_out,n_hidden,n,act", NARROW)
def test_narrow_blocks(n_in, n_out, n_hidden, n, act):
    u = DTYPES["bf16"][2]
    g = torch.Generator(device="cuda").manual_seed(n + n_hidden)
    normal = lambda *s, scale=1.0: torch.randn(*s, generator=g, device="cuda", dtype=torch.float64) * scale  # noqa: E731
    x, wgu, wd = (t.bfloat16() for t in (normal(n, n_in), normal(n_in, 2 * n_hidden, scale=n_in ** -0.5), normal(n_hidden, n_out, scale=n_hidden ** -0.5)))
    y = torch.full((n, n_out), math.nan, dtype=torch.bfloat16, device="cuda")
    ws = torch.full((eck.gatedffn_forward_workspace_bytes(n, n_in, n_hidden, n_out, eck.BF16),), 0xFF, dtype=torch.uint8, device="cuda")
    with torch.profiler.profile(activities=[torch.profiler.ProfilerActivity.CUDA], acc_events=True) as profile:
        eck.gatedffn_forward(x, wgu, wd, y, ws, act=ACTS[act])
        torch.cuda.synchronize()
    name = "narrow_kernel<%d, %d, %d, %s>" % (2 if n_in <= 64 else 4, 4 if n_out <= 64 else 8 if n_out <= 128 else 16, ACTS[act],
                                              "true" if n_hidden % 64 else "false")
    assert any(name in e.name for e in profile.events()), [e.name for e in profile.events()]
    x, wgu, wd = x.double(), wgu.double(), wd.double()
    pre = x @ wgu
    off_g, off_u = ((n_in + 2) * E * (x.abs() @ wgu.abs())).chunk(2, 1)
    gate, up = pre.chunk(2, 1)
    a = act_of(ACTS[act], gate)[0]
    h = a * up
    off_a = 1.13 * off_g + 8 * E * gate.abs()
    off_h = off_a * up.abs() + (a.abs() + off_a) * off_u
    off_h += u * (h.abs() + off_h)
    want = h @ wd
    hold(y, want, off_h @ wd.abs() + (n_hidden + 2) * E * (h.abs() @ wd.abs()) * 1.01 + u * want.abs() * 1.01, "y")
