"""A gated cost model: residual blocks of the library's layer norm, gated feed-forward block and dropout over the candidates'
features, with a gated head that predicts the normalised energy (Sec. 5.4: the model outputs a normalised score, lower is better;
Eq. (1) is the loss of a refit).

    x  = layernorm(features)                                 feature matrix [n_feat][ld] -> rows [n][n_feat]
    x <- x + dropout(feedforward(layernorm(x)))              `blocks` times, in bf16
    score = feedforward(layernorm(x))                        one output, in fp32

The operators run in the library, a refit's norm of all gradients and its steps of AdamW on the fp32 master parameters among them (states in
32 or in 8 bits), and scoring with the blocks' products in 8-bit integers.  torch holds the memory, and does what lies between them:
changes of type before the first block and the head (and, in a refit, of their rows' gradients), the sum of the residual's two gradients and
the loss on vectors of scores.  A model's calls share one workspace, so they belong on one stream.
`python -m paper_2411_18873_amd.gated` fits one on simulated measurements, picks candidates with it and draws parents for the next ones."""
import numpy as np
import torch

from . import eck, synth

EPS = 1e-5


class GatedModel:
    def __init__(self, n_feat=64, hidden=256, blocks=2, head=64, p_drop=0.05, seed=1, state_bits=32):
        if state_bits not in (8, 32):
            raise ValueError("state_bits must be 8 or 32")
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
        # of each parameter m and v, and, in 8 bits, the powers of two of their blocks
        if state_bits == 32:
            self.moments = {k: (torch.zeros_like(p), torch.zeros_like(p)) for k, p in self.params.items()}
        else:
            self.moments = {k: tuple(torch.zeros(m, dtype=torch.uint8, device="cuda")
                                     for m in (p.numel(), p.numel(), *[-(-p.numel() // eck.STATE_BLOCK)] * 2)) for k, p in self.params.items()}
        self._work, self._left_out = {}, None  # (minus the number of steps that a norm that is not finite left out, on the device; None: none can be)
        self._copy()

    def _copy(self):
        """bf16 copies of the blocks' weights, which their products are made with"""
        self.bf16 = {k: p.bfloat16() for k, p in self.params.items() if k[0].isdigit() and p.dim() == 2}
        self._int8, self._int8_steps = None, None  # (of which step they are)

    def _quantised(self):
        """the blocks' weights in 8-bit integers, a row and a scale for each column, laid out when a scoring pass first wants them.  Not by one that
        is captured, which would only record it: other passes would take what has not been written yet for the weights"""
        if (self._int8 is None or self._int8_steps != self.steps) and torch.cuda.is_current_stream_capturing():
            raise RuntimeError("the weights in 8-bit integers have to be laid out before a pass is captured: score(int8=True) once")
        if self._int8 is None:
            self._int8 = {k: (eck.int8_rows(w.shape[1], w.shape[0]), torch.empty(w.shape[1], device="cuda"))
                          for k, w in self.params.items() if k in self.bf16}
        if self._int8_steps != self.steps:
            self._lay_out_int8()
        return self._int8

    def _lay_out_int8(self):
        """the 8-bit weights of the parameters as they are, where they have lain before: a captured scoring pass reads them there"""
        if self._int8 is not None:
            for k, (q, scale) in self._int8.items():
                eck.quantise_rows(self.params[k], q, scale, order=eck.COLUMNS)
            self._int8_steps = self.steps

    def _block_int8(self, b, w, xn, out, ws):
        """out = feedforward(xn) of block b in 8-bit integers: rows of xn and of h by their largest; w: _quantised()"""
        n, f, h = xn.shape[0], self.n_feat, self.hidden
        q, scale, hidden = eck.int8_rows(n, f), torch.empty(n, device="cuda"), torch.empty(n, h, dtype=torch.bfloat16, device="cuda")
        eck.quantise_rows(xn, q, scale)
        eck.product_int8(q, scale, *w["%d.gate_up" % b], hidden, ws, act=eck.ACT_SILU)
        q = eck.int8_rows(n, h)
        eck.quantise_rows(hidden, q, scale)
        eck.product_int8(q, scale, *w["%d.down" % b], out, ws)

    def _ws(self, need):
        """one workspace for all calls, which follow each other on one stream; for one that is captured its own, out of the graph's memory: the
        shared one goes back to the allocator when a later call wants a larger one, and replays would still write there"""
        if torch.cuda.is_current_stream_capturing():
            return torch.empty(need, dtype=torch.uint8, device="cuda")
        if self._work.get("ws") is None or self._work["ws"].numel() < need:
            self._work["ws"] = torch.empty(need, dtype=torch.uint8, device="cuda")
        return self._work["ws"]

    def _forward(self, feat, n, train, int8=False):
        """scores float [n]; train: with dropout, and what the backward pass needs of every layer, of which a scoring pass keeps none;
        int8: the blocks' products in 8-bit integers (scoring alone)"""
        f, p = self.n_feat, self.params
        w = self._quantised() if int8 else None
        kept = {} if train else None
        rows = lambda width=f, dtype=torch.bfloat16: torch.empty(n, width, dtype=dtype, device="cuda")  # noqa: E731
        stats = lambda: [torch.empty(n, device="cuda") for _ in range(2)] if train else [None, None]  # noqa: E731
        x, s = rows(dtype=feat.dtype), stats()
        eck.layernorm_forward(feat, p["in.gamma"], p["in.beta"], x, *s, eps=EPS, order=eck.COLUMNS)
        if train:
            kept["in"] = s
        x = x.bfloat16()
        need = max(eck.gatedffn_forward_workspace_bytes(n, f, self.hidden, f, eck.BF16),
                   eck.gatedffn_forward_workspace_bytes(n, f, self.head, 1, eck.F32))
        if int8:
            need = max(need, eck.product_int8_workspace_bytes(n, f, self.hidden, eck.ACT_SILU), eck.product_int8_workspace_bytes(n, self.hidden, f))
        ws = self._ws(need)
        for b in range(self.blocks):
            xn, out, s = rows(), rows(), stats()
            pre = rows(2 * self.hidden, torch.float32) if train else None
            eck.layernorm_forward(x, p["%d.gamma" % b], p["%d.beta" % b], xn, *s, eps=EPS)
            if int8:
                self._block_int8(b, w, xn, out, ws)
            else:
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

    def score(self, feat, n, score_out, int8=False):
        """predicted scores of candidates 0 .. n - 1 of a feature matrix [n_feat][ld], as costmodel_score writes them; int8: the blocks'
        products in 8-bit integers (which has to have been called once before it is captured).  That is for models as wide as features may be,
        and many candidates: two blocks of 256-4096 take 1436 us for 65 536 of them and 1496 in bf16, of 256-8192 725 and 789 for 16 384.  Narrow
        blocks, which are one kernel in bf16, take longer (64-256 on 2^18 candidates 531 and 360 us), as do few candidates"""
        score_out[:n].copy_(self._forward(feat, n, False, int8)[0])

    def _backward(self, feat, n, kept, d_score):
        """gradients of all parameters from dL/d score"""
        f, p, grads = self.n_feat, self.params, {}
        ws = self._ws(max(eck.gatedffn_backward_workspace_bytes(n, f, self.hidden, f, eck.BF16),
                          eck.gatedffn_backward_workspace_bytes(n, f, self.head, 1, eck.F32),
                          *(eck.layernorm_backward_workspace_bytes(n, f, t) for t in (eck.F32, eck.BF16))))

        def ffn(name, xn, pre, dy, gate_up, down):
            d_xn, d_gate_up, d_down = torch.empty_like(xn), torch.empty_like(gate_up), torch.empty_like(down)
            eck.gatedffn_backward(xn, gate_up, down, pre, dy, d_xn, d_gate_up, d_down, ws)
            grads[name + ".gate_up"], grads[name + ".down"] = d_gate_up, d_down
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

    def refit(self, feat, energy_measured, n_steps, minibatch, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, max_norm=None):
        """Adam on Eq. (1) over minibatches of measured kernels, as costmodel_update goes over them; the losses of all steps.  As there,
        minibatches have to divide the pairs, and with an energy that is not positive and finite losses are NaN and the model is left
        unchanged (which the host waits for, once a refit).  weight_decay: AdamW's, of the matrices; max_norm: what the norm of all gradients
        is brought down to (a step whose norm is not finite changes nothing, and Adam does not count it; `steps`, which numbers the masks of the
        dropout, does)."""
        n, pairs, losses = int(minibatch), energy_measured.numel(), []
        if n <= 0 or n_steps <= 0 or pairs == 0 or pairs % n:
            raise ValueError("pairs must be a whole number of minibatches, steps one or more")
        if feat.shape[1] < pairs:
            raise ValueError("feat must have a candidate per energy")
        if not bool(((energy_measured > 0) & torch.isfinite(energy_measured)).all()):
            return torch.full((n_steps,), float("nan"), device="cuda")
        y_all = energy_measured / energy_measured.max()
        names = list(self.params)
        params = [self.params[k] for k in names]
        states = list(zip(*(self.moments[k] for k in names)))
        plan = None
        scale = torch.ones(1, device="cuda") if max_norm is not None else None
        left_out = torch.zeros(1, dtype=torch.bool, device="cuda") if max_norm is not None else None
        if max_norm is not None and self._left_out is None:
            self._left_out = torch.zeros(1, dtype=torch.int32, device="cuda")
        for step in range(n_steps):
            first = step % (pairs // n) * n
            x, y = feat[:, first:first + n], y_all[first:first + n]
            pred, kept = self._forward(x, n, True)
            losses.append(((pred - y) ** 2 / y).mean())
            grads = self._backward(x, n, kept, 2.0 * (pred - y) / y / n)
            self.steps += 1
            of = [grads[k] for k in names]
            if plan is None:
                plan = eck.Parameters(of, params, *states, copies=[self.bf16.get(k) for k in names],
                                      weight_decay=[weight_decay if p.dim() == 2 else 0.0 for p in params])
            else:
                plan.set_grads(of)
            if max_norm is not None:
                eck.gradients_norm(plan, None, scale, self._ws(eck.gradients_norm_workspace_bytes(plan)), max_norm=max_norm)
                self._left_out.add_(torch.ne(scale, scale, out=left_out), alpha=-1)  # (a norm that is not finite: NaN)
            eck.adamw_step(plan, lr, self.steps, beta1, beta2, eps, grad_scale=scale, seed=self.seed, step_more=self._left_out)
        self._lay_out_int8()
        return torch.stack(losses)


def main(pairs=4096, n=1 << 18, steps=200, k=32, parents=256):
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
    # the next generation's parents: drawn from the better ones, by scores whose products are made in 8-bit integers
    quick = torch.empty(n, device="cuda")
    model.score(feats[1].bfloat16(), n, quick, int8=True)
    drawn, logprob = torch.zeros((1, parents), dtype=torch.int32, device="cuda"), torch.zeros((1, parents), device="cuda")
    uniform = torch.rand((1, parents), generator=torch.Generator().manual_seed(model.seed)).cuda()
    ws = torch.empty(eck.sample_select_workspace_bytes(n, 1, parents), dtype=torch.uint8, device="cuda")
    eck.sample_select(quick, legal, 1, uniform, drawn, logprob, count, ws, temperature=0.02, k=4096, top_p=0.95)
    bred = torch.empty((space.n_genes, parents), dtype=torch.int16, device="cuda")
    eck.candidates_gather(genes, n, drawn.view(-1), parents, bred)
    print("8-bit scores %.4f off on average; %d parents, %d of them different, drawn from the best %d" % (
        (quick - score).abs().mean(), parents, bred.unique(dim=1).shape[1], int(count)))


if __name__ == "__main__":
    main()
