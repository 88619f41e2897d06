"""GPU: the gated cost model against a plain 64-bit evaluation of the same network, its gradients against differentiation of that,
and its refit and selection as a search uses them."""
import numpy as np
import pytest
import torch

from paper_2411_18873_amd import eck, gated
from test_gpu_operators import draws

pytestmark = pytest.mark.gpu


def features(n_feat, n, seed, dtype):
    g = torch.Generator().manual_seed(seed)
    level, spread = 2 + 22 * torch.rand(n_feat, 1, generator=g), 0.5 + 2.5 * torch.rand(n_feat, 1, generator=g)
    return ((level + spread * torch.randn(n_feat, n, generator=g)).clamp(0, 47) * 1024).floor().div(1024).to(dtype).cuda()


def plain(model, feat, params):
    """the network in 64 bits, without dropout"""
    def norm(x, name):
        m = x.mean(1, keepdim=True)
        return (x - m) / torch.sqrt(((x - m) ** 2).mean(1, keepdim=True) + gated.EPS) * params[name + ".gamma"] + params[name + ".beta"]

    def ffn(x, name):
        g, u = (x @ params[name + ".gate_up"]).chunk(2, 1)
        return (g * torch.sigmoid(g) * u) @ params[name + ".down"]

    x = norm(feat.double().t(), "in")
    for b in range(model.blocks):
        x = x + ffn(norm(x, str(b)), str(b))
    return ffn(norm(x, "head"), "head").view(-1)


@pytest.mark.parametrize("n", [1, 3, 200, 1001, 20000])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_scores(n, dtype):
    model = gated.GatedModel(hidden=96, blocks=2, head=40, seed=n)
    feat = features(64, n + 1, 3, dtype)
    got = torch.full((n + 2,), -7.0, device="cuda")
    model.score(feat[:, :n], n, got)
    assert (got[n:] == -7.0).all()
    want = plain(model, feat[:, :n], {k: p.double() for k, p in model.params.items()})
    # bf16 rounds x, the normed rows, the weights, h and the block's result: about five roundings of 2^-9 (a third of half a unit each,
    # root mean square) in each of two blocks, 6e-3 of the size of x, and the head passes that on with a slope of about one
    size = plain_size(model)
    assert (got[:n].double() - want).abs().max().item() <= 8 * 6e-3 * size
    assert (got[:n].double() - want).square().mean().sqrt().item() <= 2 * 6e-3 * size


def plain_size(model):
    """the size of scores: of the head's sum of `head` products of two numbers of about 0.6 and 1 and weights of head^-0.5"""
    return 1.0


def test_gradients_and_refit():
    n = 512
    model = gated.GatedModel(hidden=128, blocks=2, head=64, p_drop=0.0, seed=4)
    feat = features(64, n, 5, torch.float32)
    params = {k: p.double().requires_grad_(True) for k, p in model.params.items()}
    d = torch.randn(n, generator=torch.Generator().manual_seed(6)).cuda() / n
    (plain(model, feat, params) * d.double()).sum().backward()
    score, kept = model._forward(feat, n, True)
    grads = model._backward(feat, n, kept, d)
    for k, p in params.items():
        rel = ((grads[k].double() - p.grad).norm() / p.grad.norm()).item()
        assert rel <= 0.04, (k, rel)     # the roundings of the pass above forward and as many backward, 1.2e-2, three times over
    # a refit lowers the loss on what it learns from; the labels depend on four features
    y = 0.2 + torch.sigmoid((feat[3] - feat[3].mean()) / feat[3].std() + 0.5 * (feat[8] - feat[8].mean()) / feat[8].std())
    model = gated.GatedModel(hidden=128, blocks=2, head=64, p_drop=0.05, seed=4)
    losses = model.refit(feat, y, 120, 256, lr=3e-3)
    assert torch.isfinite(losses).all() and losses[-10:].mean() < 0.2 * losses[:4].mean()


def test_selection_by_a_gated_model():
    n, k = 30000, 16
    model = gated.GatedModel(seed=9)
    feat = features(64, n, 10, torch.bfloat16)
    score = torch.empty(n, device="cuda")
    model.score(feat, n, score)
    idx, best = torch.zeros((1, k), dtype=torch.int32, device="cuda"), torch.zeros((1, k), device="cuda")
    count = torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = torch.empty(eck.topk_select_workspace_bytes(n, 1, k), dtype=torch.uint8, device="cuda")
    eck.topk_select(score, None, None, 1, k, idx, best, count, ws)
    order = np.argsort(score.cpu().numpy(), kind="stable")[:k]
    assert idx[0].cpu().numpy().tolist() == order.tolist()


def normed(x, params, name):
    m = x.mean(1, keepdim=True)
    return (x - m) / torch.sqrt(((x - m) ** 2).mean(1, keepdim=True) + gated.EPS) * params[name + ".gamma"] + params[name + ".beta"]


def fed(x, params, name):
    g, u = (x @ params[name + ".gate_up"]).chunk(2, 1)
    return (g * torch.sigmoid(g) * u) @ params[name + ".down"]


def plain_with_dropout(model, feat, params, round):
    """the network in 64 bits as a refit's step number `round` runs it: masks from the generator's definition"""
    n, p = feat.shape[1], model.p_drop_q32

    def branch(y, b):
        kept = torch.from_numpy(draws(n, model.n_feat, model.seed + b, round, 0) >= p).cuda()
        return torch.where(kept, y * (2.0 ** 32 / (2.0 ** 32 - p)), 0.0)

    x = normed(feat.double().t(), params, "in")
    for b in range(model.blocks):
        x = x + branch(fed(normed(x, params, str(b)), params, str(b)), b)
    return fed(normed(x, params, "head"), params, "head").view(-1)


@pytest.mark.parametrize("step", [0, 3])
def test_gradients_with_dropout(step):
    """forward and backward pass drop the same elements, those of this step"""
    n = 384
    model = gated.GatedModel(hidden=128, blocks=2, head=64, p_drop=0.25, seed=14)
    model.steps = step
    feat = features(64, n, 15, torch.float32)
    params = {k: p.double().requires_grad_(True) for k, p in model.params.items()}
    d = torch.randn(n, generator=torch.Generator().manual_seed(16)).cuda() / n
    want = plain_with_dropout(model, feat, params, step)
    (want * d.double()).sum().backward()
    score, kept = model._forward(feat, n, True)
    grads = model._backward(feat, n, kept, d)
    # as in test_scores and test_gradients_and_refit, the branches and their errors being up to 4 / 3 larger
    assert (score.double() - want.detach()).square().mean().sqrt().item() <= 2 * 8e-3
    for k, p in params.items():
        assert ((grads[k].double() - p.grad).norm() / p.grad.norm()).item() <= 0.054, k
    # masks of another step, or of the other block, would be seen
    for round, swap in ((step + 1, False), (step, True)):
        other = gated.GatedModel(hidden=128, blocks=2, head=64, p_drop=0.25, seed=14 + swap)
        params = {k: p.detach().requires_grad_(True) for k, p in params.items()}
        (plain_with_dropout(other, feat, params, round) * d.double()).sum().backward()
        assert any(((grads[k].double() - p.grad).norm() / p.grad.norm()).item() > 0.2 for k, p in params.items())


def test_scoring_keeps_no_layers():
    """memory of a scoring pass does not grow with the number of blocks: nothing of a layer is kept that no backward pass will read"""
    n, peaks = 1 << 16, []
    feat = features(64, n, 17, torch.bfloat16)
    score = torch.empty(n, device="cuda")
    for blocks in (2, 8):
        model = gated.GatedModel(hidden=64, blocks=blocks, head=64, seed=18)
        model.score(feat, n, score)      # (the workspace)
        torch.cuda.synchronize()
        before = torch.cuda.memory_allocated()
        torch.cuda.reset_peak_memory_stats()
        model.score(feat, n, score)
        torch.cuda.synchronize()
        peaks.append(torch.cuda.max_memory_allocated() - before)
    assert peaks[1] <= peaks[0] + (1 << 20), peaks      # (a layer's rows alone are 8 MB)


def test_refit_refuses_what_costmodel_update_refuses():
    feat = features(64, 300, 19, torch.float32)
    energy = 0.5 + torch.rand(300, generator=torch.Generator().manual_seed(20)).cuda()
    model = gated.GatedModel(hidden=32, blocks=1, head=16, seed=21)
    before = {k: p.clone() for k, p in model.params.items()}

    def unchanged():
        return (model.steps == 0 and all(torch.equal(model.params[k], p) for k, p in before.items())
                and all((m == 0).all() and (v == 0).all() for m, v in model.moments.values()))

    for pairs, minibatch, steps in ((300, 256, 4), (300, 301, 4), (300, 0, 4), (300, -100, 4), (300, 100, 0)):
        with pytest.raises(ValueError):      # pairs that are no whole number of minibatches; nothing to do
            model.refit(feat, energy[:pairs], steps, minibatch)
    with pytest.raises(ValueError):          # fewer candidates than energies
        model.refit(feat[:, :200], energy, 4, 100)
    assert unchanged()
    # a data error: losses of NaN, and the model is as it was
    for bad in (0.0, -1.0, float("nan"), float("inf")):
        wrong = energy.clone()
        wrong[250] = bad
        losses = model.refit(feat, wrong, 4, 100)
        assert losses.shape == (4,) and torch.isnan(losses).all() and unchanged()
    assert torch.isfinite(model.refit(feat, energy, 4, 100)).all() and not unchanged()
