"""GPU: rows in 8-bit integers and their products.  Scales and integers are those that IEEE arithmetic gives, to the bit; sums are exact, so
a product's result is off by the roundings behind them: of the sum to fp32, of two scales and of the result, e = 2^-24 and u each (u: half
a step of the result's type, 2^-8 bf16, 2^-24 fp32)."""
import math

import pytest
import torch

from paper_2411_18873_amd import eck

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
DTYPES = {"bf16": (torch.bfloat16, 2.0 ** -8), "f32": (torch.float32, E)}
MARK = 77


def marked(n, width, extra=0):
    """an int8 matrix amid marks: rows of whole sixteens and `extra` sixteens more, a row in front and one behind"""
    ld = -(-width // 16) * 16 + 16 * extra
    flat = torch.full(((n + 2) * ld,), MARK, dtype=torch.int8, device="cuda")
    return flat, flat[ld:(n + 1) * ld].view(n, ld)[:, :width]


def check_marks(flat, n, width, extra=0):
    """nothing but the rows' whole sixteens was written, and zeros behind the width"""
    whole = -(-width // 16) * 16
    m = flat.view(n + 2, whole + 16 * extra)
    assert (m[0] == MARK).all() and (m[n + 1] == MARK).all() and (m[:, whole:] == MARK).all()
    assert (m[1:n + 1, width:whole] == 0).all()


def expected(x):
    """x: float32 rows, on the host"""
    most = x.abs().amax(1)
    full = torch.full_like(most, 127.0)
    bad, none = ~torch.isfinite(most), most < 2.0 ** -100
    scale = torch.where(bad, math.nan, torch.where(none, 0.0, most / full))
    inverse = torch.where(bad | none, 0.0, full / most)
    q = torch.where((bad | none)[:, None], 0.0, torch.round(x * inverse[:, None]))
    return q.to(torch.int8), scale


def check_quantise(x, order, extra=0):
    """x: [n][width] on the host, of the type in question"""
    n, width = x.shape
    flat, q = marked(n, width, extra)
    scale = torch.full((n + 2,), -7.0, device="cuda")
    given = x.cuda()
    if order == eck.COLUMNS:
        given = torch.nn.functional.pad(given.t(), (0, 3), value=1e30).contiguous()
    elif extra:
        given = torch.nn.functional.pad(given, (0, extra), value=1e30)[:, :width]
    eck.quantise_rows(given, q, scale[1:n + 1], order=order)
    torch.cuda.synchronize()
    want_q, want_scale = expected(x.float())
    assert torch.equal(scale[1:n + 1].cpu().nan_to_num(nan=-3.0), want_scale.nan_to_num(nan=-3.0)) and (scale[[0, n + 1]] == -7.0).all()
    assert torch.equal(q.cpu(), want_q)
    check_marks(flat, n, width, extra)


@pytest.mark.parametrize("order", [eck.ROWS, eck.COLUMNS])
@pytest.mark.parametrize("kind", sorted(DTYPES))
@pytest.mark.parametrize("n,width", [(1, 1), (3, 2), (200, 15), (64, 16), (65, 17), (1000, 64), (129, 65), (70, 250), (33, 256), (300, 257), (9, 1000),
                                     (5, 1025), (130, 4096), (3, 4099), (40, 8192), (3, 8193), (2, 20000), (2, 131071), (20000, 64)])
def test_quantise(n, width, kind, order):
    g = torch.Generator().manual_seed(n * 7 + width)
    x = torch.randn(n, width, generator=g) * torch.exp(3 * torch.randn(n, 1, generator=g))
    check_quantise(x.to(DTYPES[kind][0]), order, extra=n % 3)


@pytest.mark.parametrize("order", [eck.ROWS, eck.COLUMNS])
@pytest.mark.parametrize("kind", sorted(DTYPES))
@pytest.mark.parametrize("width", [5, 64, 300, 20001])
def test_quantise_rows_that_are_zero_tiny_or_not_finite(width, kind, order):
    g = torch.Generator().manual_seed(3)
    x = torch.randn(80, width, generator=g)
    x[0], x[1], x[2], x[3] = 0.0, -0.0, x[2] * 1e-32, x[3] * 1e-25
    x[4], x[5], x[6] = 1e-44, 3.0e38, -1e-38
    x[10, 0], x[11, width // 2], x[12, width - 1], x[13, 1] = math.nan, math.inf, -math.inf, math.nan
    x[13, 2] = math.inf
    x[20] = 0.0
    x[20, 3] = -5.0
    check_quantise(x.to(DTYPES[kind][0]), order)


def test_quantise_halves_go_to_even():
    x = torch.arange(-127, 128).float() / 2
    x = torch.cat((x, torch.tensor([127.0, -126.5, 0.5, 1.5, 2.5])))[None]
    check_quantise(x, eck.ROWS)
    check_quantise(x, eck.COLUMNS)


def activation(g, act):
    if act == eck.ACT_SILU:
        return g / (1 + torch.exp(-g))
    return g * torch.special.ndtr(g) if act == eck.ACT_GELU else g.clamp(min=0)


def check_product(n, n_in, n_out, act, kind, seed, extra=0, ld_extra=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dtype, u = DTYPES[kind]
    rows = n_out * (1 if act == eck.ACT_NONE else 2)
    mats, scales = [], []
    for count in (n, rows):
        flat, m = marked(count, n_in, extra)
        whole = torch.as_strided(flat, (count, -(-n_in // 16) * 16), (m.stride(0) if count > 1 else -(-n_in // 16) * 16, 1), m.storage_offset())
        whole[:, n_in:] = 0 if count == rows and len(mats) else 99  # zeros are wanted in one of the two
        m.copy_(torch.randint(-128, 128, (count, n_in), generator=g, device="cuda"))
        mats.append(m)
        scales.append(torch.exp(torch.randn(count, generator=g, device="cuda")) * (0.014 * n_in ** -0.25))
    y = torch.full((n + 2, n_out + ld_extra), -7.0, dtype=dtype, device="cuda")
    ws = torch.empty(max(1, eck.product_int8_workspace_bytes(n, n_in, n_out, act)), dtype=torch.uint8, device="cuda")
    x, w = mats
    eck.product_int8(x, scales[0], w, scales[1], y[1:n + 1, :n_out], ws, act=act)
    torch.cuda.synchronize()
    assert (y[0] == -7).all() and (y[n + 1] == -7).all() and (y[:, n_out:] == -7).all()
    got = y[1:n + 1, :n_out].double()
    sums = x.double() @ w.double().t().contiguous()  # (whole numbers below 2^31: exact)
    p = sums * scales[0].double()[:, None] * scales[1].double()
    if act == eck.ACT_NONE:
        bound = (3.01 * E + 1.01 * u) * p.abs()
        want = p
    else:
        gate, up = p[:, :n_out], p[:, n_out:]
        want = activation(gate, act) * up
        # g and u three roundings each, passed on by slopes of 1.13 at most; the activation within 2^-21 of itself, SiLU in bf16 with another
        # |g| 2^-24 for its exponential's rounded argument, GELU the same for erfc's argument's square
        a = activation(gate, act).abs()
        own = a * (8 + 2 * gate.abs() * (1 + gate.abs())) * E
        bound = ((1.13 * 3.01 * E * gate.abs() + own) * up.abs() + 3.01 * E * want.abs()) + 1.01 * u * want.abs() + 1e-37
    worst = ((got - want).abs() / (bound + 1e-300)).max().item()
    assert worst <= 1.0, "%.3g times the bound" % worst


@pytest.mark.parametrize("kind", sorted(DTYPES))
@pytest.mark.parametrize("act", [eck.ACT_NONE, eck.ACT_SILU, eck.ACT_GELU, eck.ACT_RELU])
@pytest.mark.parametrize("n,n_in,n_out", [(1, 1, 1), (1, 4096, 333), (2, 15, 7), (15, 16, 8), (16, 17, 9), (17, 127, 16), (32, 128, 17), (33, 129, 64),
                                          (64, 300, 65), (65, 64, 130), (100, 1000, 40), (130, 255, 333), (257, 513, 100), (1000, 33, 1)])
def test_product(n, n_in, n_out, act, kind):
    check_product(n, n_in, n_out, act, kind, n + n_in, extra=n % 2, ld_extra=n_out % 4)


# few rows of many columns; tiles of 64 undivided and in shares of k, of 128, of 256
@pytest.mark.parametrize("act", [eck.ACT_NONE, eck.ACT_SILU])
@pytest.mark.parametrize("n,n_in,n_out", [(3, 700, 9000), (40, 1000, 5000), (100, 8192, 130), (70, 16000, 16), (70, 131071, 200), (500, 2000, 2050),
                                          (2100, 300, 2060), (4200, 400, 4100), (100000, 64, 70), (1 << 18, 40, 9), (20000, 128, 130),
                                          (140000, 250, 256), (9000, 130, 4000), (50000, 1, 1)])
def test_product_by_every_kernel(n, n_in, n_out, act):
    check_product(n, n_in, n_out, act, "bf16", n, extra=1, ld_extra=3)


def test_sums_of_the_largest_magnitude_do_not_overflow():
    for n in (2, 70, 300):
        x = eck.int8_rows(n, 131071)
        w = eck.int8_rows(40, 131071)
        x.fill_(-128)
        w.fill_(-128)
        w[1] = 127
        one, y = (lambda k: torch.ones(k, device="cuda")), torch.empty(n, 40, device="cuda")
        ws = torch.empty(max(1, eck.product_int8_workspace_bytes(n, 131071, 40)), dtype=torch.uint8, device="cuda")
        eck.product_int8(x, one(n), w, one(40), y, ws)
        assert (y[:, 0] == float(131071 * 16384)).all() and (y[:, 1] == float(torch.tensor(-131071.0 * 128 * 127))).all() and (y[:, 2:] == y[:, :1]).all()


def test_rows_that_are_not_finite_stay_by_themselves():
    for n in (9, 300):
        x = torch.randn(n, 100, device="cuda")
        x[3, 5], x[7, 99] = math.nan, math.inf
        q, scale, w, y = eck.int8_rows(n, 100), torch.empty(n, device="cuda"), eck.int8_rows(50, 100), torch.empty(n, 50, device="cuda")
        w.copy_(torch.randint(-127, 128, (50, 100)))
        eck.quantise_rows(x, q, scale)
        eck.product_int8(q, scale, w, torch.ones(50, device="cuda"), y, None)
        bad = torch.zeros(n, dtype=torch.bool, device="cuda")
        bad[3] = bad[7] = True
        assert torch.equal(torch.isnan(y).all(1), bad) and torch.equal(torch.isnan(y).any(1), bad)


def test_rows_far_apart_in_memory():
    """gates more than 2^32 bytes in front of their ups"""
    n_out, n_in, ld = 1100, 70, 1 << 22
    memory = torch.zeros(2 * n_out * ld, dtype=torch.int8, device="cuda")
    w = memory.view(2 * n_out, ld)[:, :n_in]
    w.copy_(torch.randint(-127, 128, (2 * n_out, n_in), generator=torch.Generator().manual_seed(1)))
    w_scale = torch.rand(2 * n_out, device="cuda") * 0.01
    for n in (5, 200):
        x, x_scale = eck.int8_rows(n, n_in), torch.rand(n, device="cuda") * 0.01
        x.copy_(torch.randint(-127, 128, (n, n_in)))
        near = eck.int8_rows(2 * n_out, n_in)
        near.copy_(w)
        y = [torch.empty(n, n_out, device="cuda") for _ in range(2)]
        for to, m in zip(y, (w, near)):
            eck.product_int8(x, x_scale, m, w_scale, to, None, act=eck.ACT_SILU)
        assert torch.equal(*y) and y[0].abs().max() > 0


@pytest.mark.parametrize("n", [5, 300, 3000])
def test_a_gated_block_in_8_bits_on_a_stream_and_as_a_graph(n):
    """quantise, gate, quantise, product: replays equal the calls one by one, and both the block in 64 bits, whose rows and weights are rounded
    to 1 / 254 of their largest: three such roundings (of x, h and of weights twice), each a root of a third of half a step, are about 1 %"""
    f, h = 96, 160
    g = torch.Generator(device="cuda").manual_seed(n)
    x = torch.randn(n, f, generator=g, device="cuda").bfloat16()
    weights = [torch.randn(f, 2 * h, generator=g, device="cuda") * f ** -0.5, torch.randn(h, f, generator=g, device="cuda") * h ** -0.5]
    w = []
    for t in weights:  # columns become rows
        q, s = eck.int8_rows(t.shape[1], t.shape[0]), torch.empty(t.shape[1], device="cuda")
        eck.quantise_rows(t, q, s, order=eck.COLUMNS)
        w.append((q, s))
    need = max(eck.product_int8_workspace_bytes(n, f, h, eck.ACT_SILU), eck.product_int8_workspace_bytes(n, h, f), 1)

    def buffers():
        return dict(xq=eck.int8_rows(n, f), xs=torch.empty(n, device="cuda"), h=torch.empty(n, h, dtype=torch.bfloat16, device="cuda"),
                    hq=eck.int8_rows(n, h), hs=torch.empty(n, device="cuda"), y=torch.empty(n, f, dtype=torch.bfloat16, device="cuda"),
                    ws=torch.empty(need, dtype=torch.uint8, device="cuda"))

    def block(b):
        eck.quantise_rows(x, b["xq"], b["xs"])
        eck.product_int8(b["xq"], b["xs"], *w[0], b["h"], b["ws"], act=eck.ACT_SILU)
        eck.quantise_rows(b["h"], b["hq"], b["hs"])
        eck.product_int8(b["hq"], b["hs"], *w[1], b["y"], b["ws"])

    eager, captured = buffers(), buffers()
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        block(captured)
    for _ in range(3):
        x.copy_(torch.randn(n, f, generator=g, device="cuda"))
        torch.cuda.synchronize()
        block(eager)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(eager["y"], captured["y"])
        gate, up = (x.double() @ weights[0].double()).chunk(2, 1)
        want = (gate * torch.sigmoid(gate) * up) @ weights[1].double()
        assert (eager["y"].double() - want).norm() <= 0.03 * want.norm()


def test_candidates_past_2e29_columns():
    """more columns than one launch takes: the last ones, those at the border of two launches, and offsets past 2^32 bytes"""
    n = (1 << 29) + 1000
    x = torch.zeros(1, n, dtype=torch.bfloat16, device="cuda")
    some = torch.tensor([0, 1, 127, 128, (1 << 29) - 1, 1 << 29, (1 << 29) + 1, n - 1], device="cuda")
    values = torch.tensor([1.0, -2.0, 0.5, 3.0, -4.0, 5.0, -0.25, 6.0], device="cuda")
    x[0, some] = values.bfloat16()
    q, scale = torch.full((n, 16), 7, dtype=torch.int8, device="cuda"), torch.full((n,), 7.0, device="cuda")
    eck.quantise_rows(x, q[:, :1], scale, order=eck.COLUMNS)
    assert torch.equal(q[some, 0].float(), 127 * values.sign()) and torch.allclose(scale[some], values.abs() / 127, rtol=2.0 ** -23, atol=0)
    assert (q[some, 1:] == 0).all()
    assert torch.count_nonzero(scale) == some.numel() and torch.count_nonzero(q[:, 0]) == some.numel()


@pytest.mark.parametrize("n,n_in,n_out", [(1, 15, 40), (20, 100, 40), (300, 33, 70), (300, 100, 64), (300, 300, 70), (40, 4099, 33), (1, 4099, 9000)])
@pytest.mark.parametrize("act", [eck.ACT_NONE, eck.ACT_SILU])
def test_what_lies_behind_the_width_counts_nothing_where_one_side_is_zero(n, n_in, n_out, act):
    g = torch.Generator(device="cuda").manual_seed(n + n_in)
    rows, whole, got = n_out * (1 if act == eck.ACT_NONE else 2), -(-n_in // 16) * 16, []
    full = [torch.randint(-128, 128, (count, whole), generator=g, device="cuda").to(torch.int8) for count in (n, rows)]
    scales = [torch.rand(count, generator=g, device="cuda") for count in (n, rows)]
    ws = torch.empty(max(1, eck.product_int8_workspace_bytes(n, n_in, n_out, act)), dtype=torch.uint8, device="cuda")
    for zeros in ((True, True), (True, False), (False, True)):
        x, w = [m.clone() for m in full]
        for m, zero in zip((x, w), zeros):
            if zero:
                m[:, n_in:] = 0
        got.append(torch.empty(n, n_out, device="cuda"))
        eck.product_int8(x[:, :n_in], scales[0], w[:, :n_in], scales[1], got[-1], ws, act=act)
    assert torch.equal(got[0], got[1]) and torch.equal(got[0], got[2])
