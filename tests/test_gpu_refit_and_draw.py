"""GPU: the operators of a search round as models and loops use them together: a gated model refitted by AdamW (in 32 and 8 bits, with and
without a bound on the norm), scored in 8-bit integers, and parents drawn from its scores."""
import numpy as np
import pytest
import torch

from paper_2411_18873_amd import eck, gated, search, synth
from test_gpu_gated import features, plain
from test_gpu_sample import check_segment, sample

pytestmark = pytest.mark.gpu


def labels(feat):
    return 0.2 + torch.sigmoid((feat[3] - feat[3].mean()) / feat[3].std() + 0.5 * (feat[8] - feat[8].mean()) / feat[8].std())


def refitted_by_torch(model, feat, energy, n_steps, minibatch, lr, beta1=0.9, beta2=0.999, eps=1e-8):
    """a refit whose Adam is torch's elementwise operations"""
    n, pairs, losses = minibatch, energy.numel(), []
    y_all = energy / energy.max()
    for step in range(n_steps):
        first = step % (pairs // n) * n
        x, y = feat[:, first:first + n], y_all[first:first + n]
        pred, kept = model._forward(x, n, True)
        losses.append(((pred - y) ** 2 / y).mean())
        grads = model._backward(x, n, kept, 2.0 * (pred - y) / y / n)
        model.steps += 1
        for k, param in model.params.items():
            m, v = model.moments[k]
            g = grads[k].float()
            m.mul_(beta1).add_(g, alpha=1 - beta1)
            v.mul_(beta2).addcmul_(g, g, value=1 - beta2)
            param.addcdiv_(m, (v / (1 - beta2 ** model.steps)).sqrt_().add_(eps), value=-lr / (1 - beta1 ** model.steps))
        model._copy()
    return torch.stack(losses)


def test_a_refit_is_the_one_of_torchs_operations_to_the_bit():
    feat = features(64, 512, 5, torch.float32)
    models = [gated.GatedModel(hidden=96, blocks=2, head=40, p_drop=0.05, seed=4) for _ in range(2)]
    losses = [models[0].refit(feat, labels(feat), 12, 128, lr=3e-3), refitted_by_torch(models[1], feat, labels(feat), 12, 128, 3e-3)]
    assert torch.equal(*losses)
    for k, p in models[0].params.items():
        assert torch.equal(p, models[1].params[k]), k
        assert all(torch.equal(a, b) for a, b in zip(models[0].moments[k], models[1].moments[k])), k
    assert all(torch.equal(models[0].bf16[k], models[1].bf16[k]) for k in models[0].bf16)


@pytest.mark.parametrize("bits", [8, 32])
def test_refits_with_decay_and_a_bound_on_the_norm(bits):
    feat = features(64, 512, 5, torch.float32)
    y = labels(feat)
    model = gated.GatedModel(hidden=128, blocks=2, head=64, p_drop=0.05, seed=4, state_bits=bits)
    losses = model.refit(feat, y, 120, 256, lr=3e-3, weight_decay=0.01, max_norm=1.0)
    assert torch.isfinite(losses).all()
    again = gated.GatedModel(hidden=128, blocks=2, head=64, p_drop=0.05, seed=4, state_bits=bits)
    assert torch.equal(again.refit(feat, y, 120, 256, lr=3e-3, weight_decay=0.01, max_norm=1.0), losses)
    # a second refit goes on from the states as they are, and a norm that is not finite leaves all of them alone
    held = [p.clone() for p in model.params.values()] + [t.clone() for m in model.moments.values() for t in m]
    poisoned = feat.clone()
    poisoned[5, 7] = float("nan")
    model.refit(poisoned[:, :256], y[:256], 1, 256, max_norm=1.0)
    now = list(model.params.values()) + [t for m in model.moments.values() for t in m]
    assert all(torch.equal(a, b) for a, b in zip(held, now))


def test_8_bit_states_learn_as_32_bit_ones_do():
    """a state of e4m3 or e5m2 is off by some 4 and 9 % (a step of an eighth or a quarter at most, root mean square), so an update by 15 %
    (m's errors last ten steps), the next one's by others: sixty updates of one direction by 2 % of the way, of random ones by 15 %, and
    gradients that answer to it by as much again.  Half of the way is past all of that and far from what a wrong state gives"""
    feat = features(64, 512, 5, torch.float32)
    models = [gated.GatedModel(hidden=128, blocks=2, head=64, p_drop=0.0, seed=4, state_bits=b) for b in (8, 32)]
    start = {k: p.clone() for k, p in models[0].params.items()}
    for model in models:
        model.refit(feat, labels(feat), 60, 256, lr=1e-3)
    for k, p in models[0].params.items():
        way = (models[1].params[k] - start[k]).norm()
        assert (p - models[1].params[k]).norm() <= 0.5 * way, k


@pytest.mark.parametrize("n", [1, 33, 5000, 70000])
@pytest.mark.parametrize("refit", [False, True])
def test_scores_in_8_bit_integers(n, refit):
    model = gated.GatedModel(hidden=96, blocks=2, head=40, seed=3)
    if refit:  # (the weights' 8-bit layout has to follow)
        feat = features(64, 512, 5, torch.float32)
        model.score(feat, 512, torch.empty(512, device="cuda"), int8=True)
        model.refit(feat, labels(feat), 4, 128, lr=1e-2)
    feat = features(64, n + 1, 3, torch.bfloat16)
    got = torch.full((n + 2,), -7.0, device="cuda")
    model.score(feat[:, :n], n, got, int8=True)
    assert (got[n:] == -7.0).all()
    want = plain(model, feat[:, :n], {k: p.double() for k, p in model.params.items()})
    # rows' largest are some three times their size, so a rounding to 1 / 254 of it is off by 3 / 254 / sqrt(3), 0.7 %, of an element; four of
    # them (rows, h, both weights) in each of two blocks, and bf16's as ever: 2 % of the size of x, with which the head goes on as it is
    assert (got[:n].double() - want).square().mean().sqrt().item() <= 3 * 0.02
    assert (got[:n].double() - want).abs().max().item() <= 8 * 0.02


@pytest.mark.parametrize("before", [False, True])
def test_8_bit_weights_are_those_of_the_parameters(before):
    """whether a scoring pass has laid them out before the refit or not"""
    feat, got = features(64, 512, 5, torch.float32), torch.empty(512, device="cuda")
    model = gated.GatedModel(hidden=96, blocks=2, head=40, seed=3)
    for _ in range(2):
        if before:
            model.score(feat, 512, got, int8=True)
        model.refit(feat, labels(feat), 2, 128, lr=1e-2)
        model.score(feat, 512, got, int8=True)
        for k, (q, scale) in model._int8.items():
            w = model.params[k].t()
            most = w.abs().amax(1)
            all127 = torch.full_like(most, 127.0)  # (quotients by a number are products with its reciprocal in torch)
            assert torch.equal(scale, most / all127) and torch.equal(q.float(), torch.round(w * (all127 / most)[:, None])), k


def test_a_captured_score_in_8_bit_integers_follows_refits():
    feat = features(64, 512, 5, torch.float32)
    model = gated.GatedModel(hidden=96, blocks=2, head=40, seed=3)
    model.refit(feat, labels(feat), 2, 128)  # (the workspace has its size)
    got, want = torch.zeros(512, device="cuda"), torch.zeros(512, device="cuda")
    model.score(feat, 512, got, int8=True)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        model.score(feat, 512, got, int8=True)
    for _ in range(3):
        model.refit(feat, labels(feat), 4, 128, lr=1e-2)
        got.zero_()
        graph.replay()
        model.score(feat, 512, want, int8=True)
        torch.cuda.synchronize()
        assert torch.equal(got, want)


def test_parents_drawn_from_a_refitted_models_scores():
    """the whole round: refit, lay out, score, draw; and each draw is a launchable candidate among the best"""
    n, k = 30000, 512
    model = gated.GatedModel(seed=9, state_bits=8)
    small = features(64, 512, 10, torch.float32)
    model.refit(small, labels(small), 40, 256, lr=3e-3, max_norm=1.0)
    feat = features(64, n, 11, torch.bfloat16)
    score = torch.empty(n, device="cuda")
    model.score(feat, n, score, int8=True)
    g = np.random.default_rng(2)
    legal, u = (g.random(n) < 0.8).astype(np.uint8), g.random((1, 300)).astype(np.float32)
    how = dict(temperature=0.02, k=k, top_p=0.9)
    got = sample(score.cpu().numpy(), legal, u, **how)
    check_segment(score.cpu().numpy(), legal, u[0], [x[0] for x in got], **how)


@pytest.mark.parametrize("temperature", [0.0, 0.02])
def test_a_search_that_draws_its_parents(temperature):
    cfg = synth.CONFIGS["c2"]
    runs = []
    for _ in range(2):
        s = search.EnergySearch(cfg["problem"], eck.SPACE_SPLIT, lambda x, batch: synth.simulated_kernel_metrics(x, 7, batch), population=4096, M=32,
                                parents="sampled", temperature=temperature, seed=3)
        s.initialise()
        runs.append([s.step() for _ in range(3)])
    for a, b in zip(*runs):
        assert a["parents"].size == 16 and (a["parents"] < 4096).all() and np.array_equal(a["parents"], b["parents"]) and a["best"] == b["best"]
        assert len(np.unique(a["parents"])) == 1 if temperature == 0 else len(np.unique(a["parents"])) > 1


@pytest.mark.parametrize("int8", [False, True])
def test_a_captured_score_outlives_calls_that_want_more_memory(int8):
    """captured after a small pass; then a refit and a score whose workspace is larger, memory that they gave up handed out again, and replays
    that neither write there nor read it"""
    small, feat = features(64, 512, 5, torch.float32), features(64, 70000, 6, torch.float32)
    model = gated.GatedModel(hidden=96, blocks=2, head=40, seed=3)
    got, want, many = torch.zeros(512, device="cuda"), torch.zeros(512, device="cuda"), torch.zeros(70000, device="cuda")
    model.score(small, 512, got, int8=int8)
    before = model._work["ws"].numel()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        model.score(small, 512, got, int8=int8)
    for step in range(3):
        model.refit(small, labels(small), 4, 256, lr=1e-2)
        model.score(feat, 70000, many, int8=int8)
        assert model._work["ws"].numel() > before
        others = [torch.full((size,), 0x5A, dtype=torch.uint8, device="cuda") for size in (before, before // 2, 2 * before) for _ in range(20)]
        got.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(bool((t == 0x5A).all()) for t in others)
        model.score(small, 512, want, int8=int8)
        assert torch.equal(got, want)


def test_a_first_score_in_8_bit_integers_is_not_captured():
    feat = features(64, 512, 5, torch.float32)
    model, other = [gated.GatedModel(hidden=96, blocks=2, head=40, seed=3) for _ in range(2)]
    got, want = torch.zeros(512, device="cuda"), torch.zeros(512, device="cuda")
    other.score(feat, 512, want, int8=True)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with pytest.raises(RuntimeError, match="laid out"):
        with torch.cuda.graph(graph):
            got.add_(1.0)
            model.score(feat, 512, got, int8=True)
    for _ in range(2):  # eager ones, before any replay
        model.score(feat, 512, got.zero_(), int8=True)
        assert torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        model.score(feat, 512, got, int8=True)
    for _ in range(3):
        got.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want)
        other.score(feat, 512, want, int8=True)


@pytest.mark.parametrize("bits", [8, 32])
def test_a_step_that_is_left_out_does_not_count(bits):
    """two poisoned minibatches, then good ones with and without a bound: as the good ones alone"""
    feat = features(64, 512, 5, torch.float32)
    poisoned, y = feat.clone(), labels(feat)
    poisoned[5, 7] = float("nan")
    models = [gated.GatedModel(hidden=96, blocks=2, head=40, p_drop=0.0, seed=4, state_bits=bits) for _ in range(2)]
    models[0].refit(poisoned[:, :128], y[:128], 2, 128, max_norm=1.0)
    assert models[0].steps == 2
    losses = [[m.refit(feat, y, 3, 128, lr=1e-2, max_norm=1.0) for m in models]]
    models[0].refit(poisoned[:, :128], y[:128], 1, 128, max_norm=1.0)
    losses += [[m.refit(feat, y, 3, 128, lr=1e-2, max_norm=1.0) for m in models], [m.refit(feat, y, 3, 128, lr=1e-2) for m in models]]
    assert all(torch.equal(*two) and torch.isfinite(two[0]).all() for two in losses)
    for k, p in models[0].params.items():
        assert torch.equal(p, models[1].params[k]), k
        assert all(torch.equal(a, b) for a, b in zip(models[0].moments[k], models[1].moments[k])), k


def test_a_bound_that_is_never_reached_changes_no_refit():
    """but by Adam's corrections, whose powers are made by squaring on the device: within a unit of their last place, so a step's size within two"""
    feat = features(64, 512, 5, torch.float32)
    models = [gated.GatedModel(hidden=96, blocks=2, head=40, p_drop=0.0, seed=4) for _ in range(2)]
    start = {k: p.clone() for k, p in models[0].params.items()}
    for model, most in zip(models, (None, 1e30)):
        model.refit(feat, labels(feat), 1, 128, lr=1e-3, max_norm=most)
    for k, p in models[0].params.items():
        # (w is rounded once more: by half a unit of its own last place on either side)
        bound = 3 * 2.0 ** -24 * (p - start[k]).abs() + 2 * 2.0 ** -24 * torch.maximum(p.abs(), start[k].abs())
        assert ((p - models[1].params[k]).abs() <= bound).all(), k
