"""The operators that gated cost models are made of, at the sizes they are used at, for timing and comparison.

A gated cost model normalises the candidates' features, passes them through residual blocks
x + dropout(feedforward(layernorm(x))), and is refitted on measured kernels.  Every case is one such operator as a program
calls it: layer norm (over feature matrices, or over rows of activations, with its backward pass), dropout from the
counter-based generator with the residual's sum (and its backward pass), and the gated feed-forward block (forward, or
forward and backward).  Where `own` is true run() calls the library; elsewhere it computes the same in plain torch in 32 bits.

exact() restates each operator in 64 bits, with gradients by differentiation rather than by formula.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-5
GAMMA = 0x9E3779B97F4A7C15
MIX = (0xBF58476D1CE4E5B9, 0x94D049BB133111EB)
MASK64 = (1 << 64) - 1

# The most that a drawn case may cost: elements of the elementwise operators, multiplications of the products
MOST_ELEMENTS = 1 << 25
MOST_PRODUCTS = 8192 * 8192 * 3 * 4096


def listed():
    return [
        # one candidate's features on their way into a model that answers a single question: latency
        dict(name="layernorm_one_row", do="layernorm", order="rows", train=False, n=1, width=512, dtype="bf16"),
        # a generation's feature matrix, as features_compute leaves it, into rows of a model's input
        dict(name="layernorm_features_2e20", do="layernorm", order="columns", train=False, n=1 << 20, width=64, dtype="bf16"),
        # a training step of a wide model: forward and backward
        dict(name="layernorm_train_8192x4096", do="layernorm", order="rows", train=True, n=8192, width=4096, dtype="bf16"),
        # a model kept in 32 bits, neither size a power of two
        dict(name="layernorm_train_f32_50003x250", do="layernorm", order="rows", train=True, n=50003, width=250, dtype="f32"),
        # a refit's minibatch of a small model
        dict(name="dropout_train_512x256", do="dropout", train=True, residual=True, n=512, width=256, dtype="bf16", p=0.1),
        # a training step of a wide model, with the residual's sum
        dict(name="dropout_train_8192x4096", do="dropout", train=True, residual=True, n=8192, width=4096, dtype="bf16", p=0.1),
        # predictions with dropout left on, for their spread; odd sizes
        dict(name="dropout_f32_40961x333", do="dropout", train=False, residual=False, n=40961, width=333, dtype="f32", p=0.25),
        # one row through a wide block: the weights' bytes
        dict(name="ffn_one_row_4096", do="ffn", train=False, n=1, n_in=4096, n_hidden=8192, n_out=4096, dtype="bf16", act="silu"),
        # a generation scored by a small block
        dict(name="ffn_score_2e18x64", do="ffn", train=False, n=1 << 18, n_in=64, n_hidden=256, n_out=64, dtype="bf16", act="silu"),
        # a refit's minibatch of a small model
        dict(name="ffn_train_512x256", do="ffn", train=True, n=512, n_in=256, n_hidden=1024, n_out=256, dtype="bf16", act="gelu"),
        # a training step of a wide block: the largest
        dict(name="ffn_train_8192x4096", do="ffn", train=True, n=8192, n_in=4096, n_hidden=8192, n_out=4096, dtype="bf16", act="silu"),
        # a block kept in 32 bits, odd sizes
        dict(name="ffn_train_f32_1000x200", do="ffn", train=True, n=1000, n_in=200, n_hidden=777, n_out=200, dtype="f32", act="silu"),
    ]


def _between(rng, lo, hi):
    """a whole number between lo and hi, uniform over the logarithm"""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    """a width: mostly a multiple of 64 or of 8, as models have them, sometimes any number"""
    w = _between(rng, lo, hi)
    step = rng.choice([64, 64, 64, 8, 1])
    return w if w < step else w - w % step


def draw(rng):
    do = rng.choice(["layernorm", "layernorm", "dropout", "ffn", "ffn", "ffn"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if do == "layernorm":
        order = rng.choice(["rows", "rows", "columns"])
        width = rng.choice([32, 64]) if order == "columns" else _width(rng, 16, 16384)
        train = order == "rows" and rng.random() < 0.6
        return dict(do=do, order=order, train=train, n=_between(rng, 1, min(1 << 20, MOST_ELEMENTS // width)), width=width, dtype=dtype)
    if do == "dropout":
        width = _width(rng, 16, 16384)
        return dict(do=do, train=rng.random() < 0.6, residual=rng.random() < 0.6, n=_between(rng, 1, min(1 << 20, MOST_ELEMENTS // width)),
                    width=width, dtype=dtype, p=rng.choice([0.05, 0.1, 0.25, 0.5]))
    train = rng.random() < 0.5
    n_in = _width(rng, 16, 4096)
    n_hidden = _width(rng, 32, 16384)
    n_out = n_in if rng.random() < 0.7 else _width(rng, 1, 4096)
    # (a training pass has three times the products of a forward pass)
    most = MOST_PRODUCTS // (n_hidden * (2 * n_in + n_out)) * (1 if train else 3)
    n = _between(rng, 1, max(1, min(1 << 16 if train else 1 << 18, most if dtype == "bf16" else most // 8, (1 << 28) // n_hidden)))
    return dict(do=do, train=train, n=n, n_in=n_in, n_hidden=n_hidden, n_out=n_out, dtype=dtype, act=rng.choice(["silu", "gelu"]))


# ------------------------------------------------------------------------------------------------- inputs


def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed((seed * 1000003 + 7919) & 0x7FFFFFFF)
    return g


def _normal(g, *shape, dtype, scale=1.0, shift=0.0):
    return torch.randn(*shape, generator=g, device=DEV).mul_(scale).add_(shift).to(dtype)


def _seed64(seed):
    """a stream of the generator, as a program names it"""
    return (seed * 0xD1342543DE82EF95 + 0x2545F4914F6CDD1D) & MASK64


def _drop_q32(p):
    return int(round(p * (1 << 32)))


def prepare(case, seed):
    """Inputs, parameters and result buffers on the GPU, and the workspaces that the library asks for"""
    g, dtype = _generator(seed), TORCH[case["dtype"]]
    s = {"case": case}
    empty = lambda *shape, dtype=dtype: torch.empty(*shape, dtype=dtype, device=DEV)  # noqa: E731
    n = case["n"]
    if case["do"] == "layernorm":
        w, columns = case["width"], case["order"] == "columns"
        if columns:  # fixed-point logarithms: a level and a spread for every feature, ten bits behind the point
            level = 2.0 + 22.0 * torch.rand(w, 1, generator=g, device=DEV)
            spread = 0.5 + 2.5 * torch.rand(w, 1, generator=g, device=DEV)
            ld = n + (n & 1)
            x = torch.randn(w, ld, generator=g, device=DEV).mul_(spread).add_(level)
            s["x"] = x.clamp_(0.0, 47.0).mul_(1024.0).floor_().div_(1024.0).to(dtype)
        else:  # activations of a residual trunk: rows of different mean and size
            size = 0.5 + 2.0 * torch.rand(n, 1, generator=g, device=DEV)
            shift = 0.5 + torch.rand(n, 1, generator=g, device=DEV)
            s["x"] = torch.randn(n, w, generator=g, device=DEV).mul_(size).add_(shift).to(dtype)
        s["gamma"] = _normal(g, w, dtype=torch.float32, scale=0.1, shift=1.0)
        s["beta"] = _normal(g, w, dtype=torch.float32, scale=0.1)
        s["y"] = empty(n, w)
        s["mean"], s["rstd"] = (empty(n, dtype=torch.float32) for _ in range(2)) if case["train"] else (None, None)
        if case["train"]:
            s["dy"] = _normal(g, n, w, dtype=dtype)
            s["dx"], s["dgamma"], s["dbeta"] = empty(n, w), empty(w, dtype=torch.float32), empty(w, dtype=torch.float32)
    elif case["do"] == "dropout":
        w = case["width"]
        s["x"] = _normal(g, n, w, dtype=dtype)
        s["residual"] = _normal(g, n, w, dtype=dtype) if case["residual"] else None
        s["out"], s["seed"], s["round"], s["p"] = empty(n, w), _seed64(seed), seed & 0xFFFF, _drop_q32(case["p"])
        if case["train"]:
            s["dy"], s["dx"] = _normal(g, n, w, dtype=dtype), empty(n, w)
    else:
        n_in, n_hidden, n_out = case["n_in"], case["n_hidden"], case["n_out"]
        s["x"] = _normal(g, n, n_in, dtype=dtype)
        s["w_gate_up"] = _normal(g, n_in, 2 * n_hidden, dtype=dtype, scale=n_in ** -0.5)
        s["w_down"] = _normal(g, n_hidden, n_out, dtype=dtype, scale=n_hidden ** -0.5)
        s["y"] = empty(n, n_out)
        s["pre"] = empty(n, 2 * n_hidden, dtype=torch.float32) if case["train"] else None
        if case["train"]:
            s["dy"] = _normal(g, n, n_out, dtype=dtype)
            s["dx"] = empty(n, n_in)
            s["dw_gate_up"], s["dw_down"] = empty(n_in, 2 * n_hidden), empty(n_hidden, n_out)
    if own:  # what a program that calls the library keeps beside its buffers
        from paper_2411_18873_amd import eck
        s["act"] = {"silu": eck.ACT_SILU, "gelu": eck.ACT_GELU}.get(case.get("act"))
        code = eck.F32 if case["dtype"] == "f32" else eck.BF16
        need = 0
        if case["do"] == "layernorm" and case["train"]:
            need = eck.layernorm_backward_workspace_bytes(n, case["width"], code)
        elif case["do"] == "ffn":
            sizes = (n, case["n_in"], case["n_hidden"], case["n_out"], code)
            need = eck.gatedffn_forward_workspace_bytes(*sizes)
            if case["train"]:
                need = max(need, eck.gatedffn_backward_workspace_bytes(*sizes))
        s["ws"] = empty(need, dtype=torch.uint8) if need else None
    return s


# ------------------------------------------------------------------------------------------------- one pass


def run(s):
    return _own(s) if own else _plain(s)


def _own(s):
    from paper_2411_18873_amd import eck
    case = s["case"]
    if case["do"] == "layernorm":
        eck.layernorm_forward(s["x"], s["gamma"], s["beta"], s["y"], s["mean"], s["rstd"], eps=EPS,
                              order=eck.COLUMNS if case["order"] == "columns" else eck.ROWS)
        if not case["train"]:
            return s["y"]
        eck.layernorm_backward(s["x"], s["dy"], s["gamma"], s["mean"], s["rstd"], s["dx"], s["dgamma"], s["dbeta"], s["ws"])
        return {k: s[k] for k in ("y", "mean", "rstd", "dx", "dgamma", "dbeta")}
    if case["do"] == "dropout":
        eck.dropout_apply(s["x"], s["out"], s["p"], s["seed"], round=s["round"], residual=s["residual"])
        if not case["train"]:
            return s["out"]
        eck.dropout_apply(s["dy"], s["dx"], s["p"], s["seed"], round=s["round"])
        return {k: s[k] for k in ("out", "dx")}
    eck.gatedffn_forward(s["x"], s["w_gate_up"], s["w_down"], s["y"], s["ws"], pre_out=s["pre"], act=s["act"])
    if not case["train"]:
        return s["y"]
    eck.gatedffn_backward(s["x"], s["w_gate_up"], s["w_down"], s["pre"], s["dy"], s["dx"], s["dw_gate_up"], s["dw_down"], s["ws"],
                          act=s["act"])
    return {k: s[k] for k in ("y", "dx", "dw_gate_up", "dw_down")}


def _plain(s):
    case, dtype = s["case"], TORCH[s["case"]["dtype"]]
    if case["do"] == "layernorm":
        x = s["x"].float()
        if case["order"] == "columns":
            x = x[:, :case["n"]].t()
        mean = x.mean(1)
        away = x - mean[:, None]
        rstd = (away.square().mean(1) + EPS).rsqrt()
        unit = away * rstd[:, None]
        y = (unit * s["gamma"] + s["beta"]).to(dtype)
        if not case["train"]:
            return y.contiguous()
        dy = s["dy"].float()
        g = dy * s["gamma"]
        dx = rstd[:, None] * (g - g.mean(1, keepdim=True) - unit * (g * unit).mean(1, keepdim=True))
        return {"y": y, "mean": mean, "rstd": rstd, "dx": dx.to(dtype), "dgamma": (dy * unit).sum(0), "dbeta": dy.sum(0)}
    if case["do"] == "dropout":
        kept = _kept(case["n"], case["width"], s["p"], s["seed"], s["round"])
        scale = (1 << 32) / ((1 << 32) - s["p"])
        out = torch.where(kept, s["x"].float() * scale, 0.0)
        if s["residual"] is not None:
            out = out + s["residual"].float()
        if not case["train"]:
            return out.to(dtype)
        return {"out": out.to(dtype), "dx": torch.where(kept, s["dy"].float() * scale, 0.0).to(dtype)}
    x, w_gate_up, w_down = s["x"].float(), s["w_gate_up"].float(), s["w_down"].float()
    pre = x @ w_gate_up
    gate, up = pre.chunk(2, 1)
    if case["act"] == "silu":
        part = torch.sigmoid(gate)
        slope = part * (1.0 + gate * (1.0 - part))
    else:
        part = 0.5 * (1.0 + torch.erf(gate * math.sqrt(0.5)))
        slope = part + gate * torch.exp(-0.5 * gate * gate) * (1.0 / math.sqrt(2.0 * math.pi))
    acted = gate * part
    hidden = acted * up
    y = (hidden @ w_down).to(dtype)
    if not case["train"]:
        return y
    dy = s["dy"].float()
    d_hidden = dy @ w_down.t()
    d_pre = torch.cat((d_hidden * up * slope, d_hidden * acted), 1)
    return {"y": y, "dx": (d_pre @ w_gate_up.t()).to(dtype), "dw_gate_up": (x.t() @ d_pre).to(dtype),
            "dw_down": (hidden.t() @ dy).to(dtype)}


def _signed(v):
    return v - (1 << 64) if v >> 63 else v


def _mix(z):
    """SplitMix64's output function on 64-bit words held as signed ones (host whole numbers or a tensor)"""
    for shift, factor in ((30, MIX[0]), (27, MIX[1])):
        z = (z ^ ((z >> shift) & ((1 << (64 - shift)) - 1))) * _signed(factor)
    return z ^ ((z >> 31) & ((1 << 33) - 1))


def _kept(n, width, p, seed, round):
    """which elements stay: half (column's parity) of word (row, column / 2) of the stream (seed, round) is p or more"""
    start = _mix(torch.tensor(_signed((seed + GAMMA * (round + 1)) & MASK64), device=DEV))
    words = (width + 1) // 2
    word = _mix(start + torch.arange(1, n * words + 1, device=DEV) * _signed(GAMMA))
    halves = torch.stack((word & 0xFFFFFFFF, (word >> 32) & 0xFFFFFFFF), 1).view(n, 2 * words)
    return halves[:, :width] >= p


# ------------------------------------------------------------------------------------------------- costs


def work(case):
    n, size = case["n"], 4 if case["dtype"] == "f32" else 2
    if case["do"] == "layernorm":
        # x in, y out; training: dy in and dx out as well, the statistics and the parameters' gradients
        elements = n * case["width"]
        extra = 2 * elements * size + 8 * n + 8 * case["width"] if case["train"] else 0
        return {"bytes": 2 * elements * size + 8 * case["width"] + extra, "flops": elements * (20 if case["train"] else 8)}
    if case["do"] == "dropout":
        elements = n * case["width"]
        arrays = 2 + (1 if case["residual"] else 0) + (2 if case["train"] else 0)
        return {"bytes": arrays * elements * size, "flops": elements * (4 if case["train"] else 2)}
    n_in, n_hidden, n_out = case["n_in"], case["n_hidden"], case["n_out"]
    weights = n_hidden * (2 * n_in + n_out)
    rows = n * (n_in + n_out)
    return {"bytes": (weights + rows) * size * (2 if case["train"] else 1), "flops": 2 * n * weights * (3 if case["train"] else 1)}


# ------------------------------------------------------------------------------------------------- in 64 bits


def exact(case, seed):
    s = prepare(case, seed)
    n = case["n"]
    if case["do"] == "dropout":
        kept = torch.from_numpy(_kept_on_host(n, case["width"], s["p"], s["seed"], s["round"])).to(DEV)
        factor = kept.double() / (1.0 - s["p"] / 2.0 ** 32)
        out = s["x"].double() * factor
        if s["residual"] is not None:
            out += s["residual"].double()
        return {"out": out, "dx": s["dy"].double() * factor} if case["train"] else out
    if case["do"] == "layernorm":
        x = s["x"].double()
        if case["order"] == "columns":
            x = x.t()[:n].contiguous()
        leaves = [x, s["gamma"].double(), s["beta"].double()]
        for t in leaves:
            t.requires_grad_(case["train"])
        x, gamma, beta = leaves
        mean = x.sum(1) / case["width"]
        variance = ((x - mean[:, None]) ** 2).sum(1) / case["width"]
        rstd = 1.0 / torch.sqrt(variance + EPS)
        y = (x - mean[:, None]) * rstd[:, None] * gamma + beta
        if not case["train"]:
            return y
        dx, dgamma, dbeta = torch.autograd.grad(y, leaves, s["dy"].double())
        return {"y": y.detach(), "mean": mean.detach(), "rstd": rstd.detach(), "dx": dx, "dgamma": dgamma, "dbeta": dbeta}
    leaves = [s[k].double().requires_grad_(case["train"]) for k in ("x", "w_gate_up", "w_down")]
    x, w_gate_up, w_down = leaves
    gate, up = x @ w_gate_up[:, :case["n_hidden"]], x @ w_gate_up[:, case["n_hidden"]:]
    if case["act"] == "silu":
        acted = gate / (1.0 + torch.exp(-gate))
    else:
        acted = gate * (1.0 + torch.erf(gate / math.sqrt(2.0))) / 2.0
    y = (acted * up) @ w_down
    if not case["train"]:
        return y
    dx, dw_gate_up, dw_down = torch.autograd.grad(y, leaves, s["dy"].double())
    return {"y": y.detach(), "dx": dx, "dw_gate_up": dw_gate_up, "dw_down": dw_down}


def _kept_on_host(n, width, p, seed, round):
    """the generator's definition in unsigned words: a state that grows by GAMMA, and its finaliser"""
    def finalise(z):
        z = (z ^ (z >> np.uint64(30))) * np.uint64(MIX[0])
        z = (z ^ (z >> np.uint64(27))) * np.uint64(MIX[1])
        return z ^ (z >> np.uint64(31))

    with np.errstate(over="ignore"):
        state = finalise(np.array([(seed + GAMMA * (round + 1)) & MASK64], dtype=np.uint64))
        words = (width + 1) // 2
        number = np.arange(1, n * words + 1, dtype=np.uint64)
        word = finalise(state + number * np.uint64(GAMMA))
    kept = np.empty((n, 2 * words), dtype=bool)
    kept[:, 0::2] = ((word & np.uint64(0xFFFFFFFF)) >= p).reshape(n, words)
    kept[:, 1::2] = ((word >> np.uint64(32)) >= p).reshape(n, words)
    return kept[:, :width].copy()
