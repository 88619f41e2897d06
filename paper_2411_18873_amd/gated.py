"""A gated cost model: residual blocks of the library's layer norm, gated feed-forward block and dropout over the candidates'
features, with a gated head that predicts the normalised energy (Sec. 5.4: the model outputs a normalised score, lower is better;
Eq. (1) is the loss of a refit).

    x  = layernorm(features)                                 feature matrix [n_feat][ld] -> rows [n][n_feat]
    x <- x + dropout(feedforward(layernorm(x)))              `blocks` times, in bf16
    score = feedforward(layernorm(x))                        one output, in fp32

The operators run in the library.  torch holds the memory, and does what lies between them: changes of type before the first block
and the head (and, in a refit, of their gradients), the sum of the residual's two gradients, the loss on vectors of scores, and
Adam's arithmetic on the fp32 master parameters.  A model's calls share one workspace, so they belong on one stream.
`python -m paper_2411_18873_amd.gated` fits one on simulated measurements and picks candidates with it."""
import numpy as np
import torch

from . import eck, synth

EPS = 1e-5


class GatedModel:
    def __init__(self, n_feat=64, hidden=256, blocks=2, head=64, p_drop=0.05, seed=1):
        self.n_feat, self.hidden, self.blocks, self.head = int(n_feat), int(hidden), int(blocks), int(head)
        self.p_drop_q32, self.seed, self.steps = int(p_drop * 2 ** 32), int(seed), 0
        g = torch.Generator().manual_seed(self.seed)
        f, h = self.n_feat, self.hidden

        def weights(fan_in, fan_out):
            return (torch.randn(fan_in, fan_out, generator=g) * fan_in ** -0.5).cuda()

        ones, zeros = (lambda: torch.ones(f, device="cuda")), (lambda: torch.zeros(f, device="cuda"))
        self.params = {"in.gamma": ones(), "in.beta": zeros(), "head.gamma": ones(), "head.beta": zeros(),
                       "head.gate_up": weights(f, 2 * self.head), "head.down": weights(self.head, 1)}
        for b in range(self.blocks):
            self.params.update({"%d.gamma" % b: ones(), "%d.beta" % b: zeros(), "%d.gate_up" % b: weights(f, 2 * h), "%d.down" % b: weights(h, f)})
        self.moments = {k: (torch.zeros_like(p), torch.zeros_like(p)) for k, p in self.params.items()}
        self._work = {}
        self._copy()

    def _copy(self):
        """bf16 copies of the blocks' weights, which their products are made with"""
        self.bf16 = {k: p.bfloat16() for k, p in self.params.items() if k[0].isdigit() and p.dim() == 2}

    def _ws(self, need):
        """one workspace for all calls: they follow each other on one stream"""
        if self._work.get("ws") is None or self._work["ws"].numel() < need:
            self._work["ws"] = torch.empty(need, dtype=torch.uint8, device="cuda")
        return self._work["ws"]

    def _forward(self, feat, n, train):
        """scores float [n]; train: with dropout, and what the backward pass needs of every layer, of which a scoring pass keeps none"""
        f, p = self.n_feat, self.params
        kept = {} if train else None
        rows = lambda width=f, dtype=torch.bfloat16: torch.empty(n, width, dtype=dtype, device="cuda")  # noqa: E731
        stats = lambda: [torch.empty(n, device="cuda") for _ in range(2)] if train else [None, None]  # noqa: E731
        x, s = rows(dtype=feat.dtype), stats()
        eck.layernorm_forward(feat, p["in.gamma"], p["in.beta"], x, *s, eps=EPS, order=eck.COLUMNS)
        if train:
            kept["in"] = s
        x = x.bfloat16()
        ws = self._ws(max(eck.gatedffn_forward_workspace_bytes(n, f, self.hidden, f, eck.BF16),
                          eck.gatedffn_forward_workspace_bytes(n, f, self.head, 1, eck.F32)))
        for b in range(self.blocks):
            xn, out, s = rows(), rows(), stats()
            pre = rows(2 * self.hidden, torch.float32) if train else None
            eck.layernorm_forward(x, p["%d.gamma" % b], p["%d.beta" % b], xn, *s, eps=EPS)
            eck.gatedffn_forward(xn, self.bf16["%d.gate_up" % b], self.bf16["%d.down" % b], out, ws, pre_out=pre)
            if train:
                kept[b] = x, xn, pre, s
            nxt = rows()
            eck.dropout_apply(out, nxt, self.p_drop_q32 if train else 0, self.seed + b, round=self.steps, residual=x)
            x = nxt
        x, xn, s = x.float(), rows(dtype=torch.float32), stats()
        pre = rows(2 * self.head, torch.float32) if train else None
        score = rows(1, torch.float32)
        eck.layernorm_forward(x, p["head.gamma"], p["head.beta"], xn, *s, eps=EPS)
        eck.gatedffn_forward(xn, p["head.gate_up"], p["head.down"], score, ws, pre_out=pre)
        if train:
            kept["head"] = x, xn, pre, s
        return score.view(n), kept

    def score(self, feat, n, score_out):
        """predicted scores of candidates 0 .. n - 1 of a feature matrix [n_feat][ld], as costmodel_score writes them"""
        score_out[:n].copy_(self._forward(feat, n, False)[0])

    def _backward(self, feat, n, kept, d_score):
        """gradients of all parameters from dL/d score"""
        f, p, grads = self.n_feat, self.params, {}
        ws = self._ws(max(eck.gatedffn_backward_workspace_bytes(n, f, self.hidden, f, eck.BF16),
                          eck.gatedffn_backward_workspace_bytes(n, f, self.head, 1, eck.F32),
                          *(eck.layernorm_backward_workspace_bytes(n, f, t) for t in (eck.F32, eck.BF16))))

        def ffn(name, xn, pre, dy, gate_up, down):
            d_xn, d_gate_up, d_down = torch.empty_like(xn), torch.empty_like(gate_up), torch.empty_like(down)
            eck.gatedffn_backward(xn, gate_up, down, pre, dy, d_xn, d_gate_up, d_down, ws)
            grads[name + ".gate_up"], grads[name + ".down"] = d_gate_up.float(), d_down.float()
            return d_xn

        def norm(name, x, dy, stats, dx, order=eck.ROWS):
            grads[name + ".gamma"], grads[name + ".beta"] = torch.empty(f, device="cuda"), torch.empty(f, device="cuda")
            eck.layernorm_backward(x, dy, p[name + ".gamma"], *stats, dx, grads[name + ".gamma"], grads[name + ".beta"], ws, order=order)
            return dx

        x, xn, pre, s = kept["head"]
        d_xn = ffn("head", xn, pre, d_score.view(n, 1), p["head.gate_up"], p["head.down"])
        dx = norm("head", x, d_xn, s, d_xn).bfloat16()
        for b in reversed(range(self.blocks)):
            x, xn, pre, s = kept[b]
            d_out = torch.empty_like(dx)
            eck.dropout_apply(dx, d_out, self.p_drop_q32, self.seed + b, round=self.steps)
            d_xn = ffn("%d" % b, xn, pre, d_out, self.bf16["%d.gate_up" % b], self.bf16["%d.down" % b])
            dx = dx + norm("%d" % b, x, d_xn, s, d_xn)
        norm("in", feat, dx.to(feat.dtype), kept["in"], None, order=eck.COLUMNS)
        return grads

    def refit(self, feat, energy_measured, n_steps, minibatch, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8):
        """Adam on Eq. (1) over minibatches of measured kernels, as costmodel_update goes over them; the losses of all steps.  As there,
        minibatches have to divide the pairs, and with an energy that is not positive and finite losses are NaN and the model is left
        unchanged (which the host waits for, once a refit)."""
        n, pairs, losses = int(minibatch), energy_measured.numel(), []
        if n <= 0 or n_steps <= 0 or pairs == 0 or pairs % n:
            raise ValueError("pairs must be a whole number of minibatches, steps one or more")
        if feat.shape[1] < pairs:
            raise ValueError("feat must have a candidate per energy")
        if not bool(((energy_measured > 0) & torch.isfinite(energy_measured)).all()):
            return torch.full((n_steps,), float("nan"), device="cuda")
        y_all = energy_measured / energy_measured.max()
        for step in range(n_steps):
            first = step % (pairs // n) * n
            x, y = feat[:, first:first + n], y_all[first:first + n]
            pred, kept = self._forward(x, n, True)
            losses.append(((pred - y) ** 2 / y).mean())
            grads = self._backward(x, n, kept, 2.0 * (pred - y) / y / n)
            self.steps += 1
            for k, param in self.params.items():
                m, v = self.moments[k]
                m.mul_(beta1).add_(grads[k], alpha=1 - beta1)
                v.mul_(beta2).addcmul_(grads[k], grads[k], value=1 - beta2)
                param.addcdiv_(m, (v / (1 - beta2 ** self.steps)).sqrt_().add_(eps), value=-lr / (1 - beta1 ** self.steps))
            self._copy()
        return torch.stack(losses)


def main(pairs=4096, n=1 << 18, steps=200, k=32):
    cfg = synth.CONFIGS["c2"]
    space = eck.Space(cfg["problem"], eck.SPACE_SPLIT)
    feats = []
    for count, seed in ((pairs, 11), (n, 12)):
        genes = torch.zeros((space.n_genes, count), dtype=torch.int16, device="cuda")
        feat = torch.zeros((64, count), dtype=torch.float32, device="cuda")
        legal = torch.zeros(count, dtype=torch.uint8, device="cuda")
        eck.candidate_enumerate(space, eck.MODE_SAMPLE, count, genes, seed=seed)
        eck.features_compute(space, genes, count, 64, eck.F32, feat_out=feat, legal_out=legal)
        feats.append(feat)
    energy = torch.from_numpy(np.ascontiguousarray(synth.measured_energy(feats[0].cpu().numpy(), 5), dtype=np.float32)).cuda()
    model = GatedModel()
    losses = model.refit(feats[0], energy, steps, 512)
    score = torch.empty(n, device="cuda")
    model.score(feats[1].bfloat16(), n, score)
    idx, best = torch.zeros((1, k), dtype=torch.int32, device="cuda"), torch.zeros((1, k), device="cuda")
    count = torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = torch.empty(eck.topk_select_workspace_bytes(n, 1, k), dtype=torch.uint8, device="cuda")
    eck.topk_select(score, None, legal, 1, k, idx, best, count, ws)
    print("Eq. (1) loss %.4f -> %.4f in %d steps; least of %d predicted scores: %s" % (losses[0], losses[-8:].mean(), steps, n, best[0, :4].tolist()))


if __name__ == "__main__":
    main()
