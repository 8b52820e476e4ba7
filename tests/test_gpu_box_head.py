"""The dense layers and class log probabilities in autograd, the box head on them, the relation head with
its dense layers in these kernels, and a memory that forgets by weight.

Tolerances: binary32 results are off by some 2^-23 for each of the square roots of the lengths of the
sums that lead to them (largest 2048 here, a few in a row): 1e-5 of the largest value of a tensor, and
through the relation head's layers the 1.6e-4 and 5e-4 of its own tests.
"""
import numpy as np
import pytest
import torch
from torch.nn import functional as F

import paper_1906_07155_amd as rex
from test_gpu_relation_attn import draw_boxes

pytestmark = pytest.mark.gpu


def near(got, want, tol, what):
    size = float(want.abs().max()) + 1e-30
    err = float((got.double() - want).abs().max())
    assert got.shape == want.shape and err <= tol * size, (what, err / size)


def randn(seed, *shape, dtype=torch.float32):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return torch.randn(shape, generator=gen, device="cuda").to(dtype)


ACT = {"none": lambda t: t, "relu": F.relu, "gelu": F.gelu, "silu": F.silu}


@pytest.mark.parametrize("act", sorted(ACT))
@pytest.mark.parametrize("wants", [(1, 1, 1, 1), (1, 0, 0, 0), (0, 1, 0, 0), (0, 0, 1, 0), (0, 0, 0, 1)])
def test_linear_act_gradients(act, wants):
    given = [randn(1, 3, 7, 40), randn(2, 24, 40) * 0.2, randn(3, 24), randn(4, 3, 7, 24)]
    g = randn(5, 3, 7, 24)
    leaves = [t.clone().requires_grad_(bool(w)) for t, w in zip(given, wants)]
    y = rex.linear_act(*leaves[:3], act=act, residual=leaves[3])
    y.backward(g)
    ref = [t.double().requires_grad_(bool(w)) for t, w in zip(given, wants)]
    z = ACT[act](F.linear(*ref[:3])) + ref[3]
    z.backward(g.double())
    near(y.detach(), z.detach(), 1e-5, "y")
    for t, r, w in zip(leaves, ref, wants):
        assert (t.grad is not None) == bool(w)
        if w:
            near(t.grad, r.grad, 1e-5, "grad")


def test_gradients_against_differences():
    """Central differences of the kernels' own results, along random directions."""
    x, w, b = randn(1, 5, 16), randn(2, 12, 16) * 0.3, randn(3, 12)
    labels = torch.tensor([0, 11, 3, -1, 5], device="cuda")

    def value(x, w, b):
        logp, entropy, _, _ = rex.class_logprob(rex.linear_act(x, w, b, act="silu"), labels, scale=1.3)
        return logp.double().sum() + 0.5 * entropy.double().sum()
    leaves = [t.clone().requires_grad_() for t in (x, w, b)]
    value(*leaves).backward()
    for i, t in enumerate((x, w, b)):
        d = randn(10 + i, *t.shape)
        d = d / d.norm()
        step = 2.0 ** -6
        with torch.no_grad():
            up, down = [], []
            for sign, out in ((1, up), (-1, down)):
                args = [x, w, b]
                args[i] = t + sign * step * d
                out.append(value(*args))
        slope = float((up[0] - down[0]) / (2 * step))
        # ten results of size 10 off by 32 * 2^-23 each, third derivatives along a unit direction below 50
        tol = 10 * 10 * 32 * 2.0 ** -23 / step + 50 * step * step
        assert abs(slope - float((leaves[i].grad.double() * d.double()).sum())) <= tol


def test_results_may_be_written_to():
    x, labels = randn(1, 6, 9), torch.tensor([0, 8, 3, -1, 5, 2], device="cuda")
    keep = torch.tensor([1, 0, 1, 1, 0, 1], device="cuda")
    for grad in (True, False):
        leaf = x.clone().requires_grad_(grad)
        weight = torch.ones(6, device="cuda", requires_grad=True)
        logp, entropy, _, _ = rex.class_logprob(leaf, labels)
        logp.masked_fill_(keep == 0, 0.0)
        logp *= weight
        (logp.sum() + 0.5 * entropy.sum()).backward()
        ref = x.double().requires_grad_(grad)
        full = torch.log_softmax(ref, 1)
        picked = full.gather(1, labels.clamp(min=0)[:, None])[:, 0] * ((labels >= 0) & (keep == 1))
        near(weight.grad, picked.detach(), 1e-5, "weight")
        if grad:
            (picked.sum() - 0.5 * (full.exp() * full).sum()).backward()
            near(leaf.grad, ref.grad, 1e-5, "grad")
    out = (torch.empty(6, device="cuda"), torch.empty(6, device="cuda"), torch.empty(6, 2, device="cuda"))
    want = rex.class_logprob_fwd(x, labels)
    got = rex.class_logprob_fwd(x, labels, out=out)
    assert all(a is b and torch.equal(a, w) for a, b, w in zip(got, out, want))
    with pytest.raises(ValueError):
        rex.class_logprob_fwd(x, labels, out=(out[0], out[1][:5], out[2]))


def test_second_derivatives_are_refused():
    x, w = randn(1, 4, 8).requires_grad_(), randn(2, 6, 8).requires_grad_()
    g, = torch.autograd.grad(rex.linear_act(x, w, act="gelu").sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        g.sum().backward()
    g, = torch.autograd.grad(rex.class_logprob(x, torch.zeros(4, dtype=torch.int64, device="cuda"))[0].sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        g.sum().backward()


def test_views_and_broadcasts():
    """Transposed and expanded operands, a gradient that is one number everywhere."""
    x, w = randn(1, 30, 9).t(), randn(2, 30, 14).t()
    leaf = x.clone().requires_grad_()
    y = rex.linear_act(leaf, w, act="relu")
    y.sum().backward()
    ref = x.double().clone().requires_grad_()
    z = F.relu(F.linear(ref, w.double()))
    z.sum().backward()
    near(y.detach(), z.detach(), 1e-5, "y")
    near(leaf.grad, ref.grad, 1e-5, "grad")
    one = randn(3, 30)
    near(rex.linear_act(one.expand(9, 30), w), F.linear(one.double().expand(9, 30), w.double()), 1e-5, "expanded")


@pytest.mark.parametrize("dtype,tol", [(torch.float32, 1e-5), (torch.bfloat16, 0.05)])
def test_box_head_and_its_gradients(dtype, tol):
    """RoI features to a loss and back, against the same in 64 bits.  (bf16: five roundings of 2^-8 on the
    way to a gradient, and again as many on the way back.)"""
    torch.manual_seed(0)
    head = rex.BoxHead(8 * 7 * 7, classes=11, hidden=64).cuda().to(dtype)
    feats = randn(1, 90, 8, 7, 7, dtype=dtype).requires_grad_()
    labels = torch.randint(-1, 12, (90,), generator=torch.Generator().manual_seed(1)).cuda()
    goal = randn(2, 90, 44, dtype=dtype)
    scores, deltas = head(feats)
    loss = head.loss(scores, labels) + (deltas * goal).float().mean()
    loss.backward()
    p = {k: v.detach().double().requires_grad_() for k, v in head.named_parameters()}
    ref = feats.detach().double().requires_grad_()
    x = ref.flatten(1)
    on = []
    for fc, mine in (("fc1", head.fc1), ("fc2", head.fc2)):
        x = F.linear(x, p[fc + ".weight"], p[fc + ".bias"]).clamp(min=0)
    s, d = (F.linear(x, p[n + ".weight"], p[n + ".bias"]) for n in ("score", "delta"))
    keep = labels >= 0
    want = F.cross_entropy(s[keep], labels[keep]) + (d * goal.double()).mean()
    want.backward()
    assert abs(float(loss.detach()) - float(want.detach())) <= tol * 5
    near(scores.detach(), s.detach(), tol, "scores")
    if dtype == torch.float32:
        near(feats.grad, ref.grad, 1e-4, "features")
        for k, v in head.named_parameters():
            near(v.grad, p[k].grad, 1e-4, k)
    else:
        assert all(v.grad is not None and v.grad.dtype == dtype and bool(v.grad.isfinite().all()) for v in head.parameters())
    logp, classes = head.best(scores.detach(), 3)
    top = torch.log_softmax(scores.detach().double(), -1).sort(dim=-1, descending=True, stable=True)
    assert torch.equal(classes, top[1][:, :3])
    near(logp, top[0][:, :3], 1e-5, "best")
    empty = head(feats.detach()[:0])
    assert [tuple(t.shape) for t in empty] == [(0, 12), (0, 44)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_captured_training_step(dtype):
    torch.manual_seed(3)
    head = rex.BoxHead(64 * 9, classes=5, hidden=48).cuda().to(dtype)
    weights = list(head.parameters())
    x, labels = randn(1, 70, 64, 3, 3, dtype=dtype), torch.arange(70, device="cuda") % 8 - 1

    def step():
        scores, deltas = head(x)
        loss = head.loss(scores, labels) + 0.1 * (deltas * deltas).sum(1).mean()
        return (loss.detach(), *torch.autograd.grad(loss, weights))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for seed in range(2, 6):
        x.copy_(randn(seed, 70, 64, 3, 3, dtype=dtype))
        graph.replay()
        got = [t.clone() for t in held]
        want = step()                                   # eager, between replays
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, want)), seed


def test_box_head_on_extracted_features():
    """roi_extract's results through the head: one path from a pyramid to scores."""
    torch.manual_seed(0)
    feats = [randn(i, 1, 16, 64 >> i, 64 >> i).contiguous(memory_format=torch.channels_last) for i in range(2)]
    rois = torch.tensor([[0, 4.0, 8.0, 100.0, 90.0], [0, 30.0, 10.0, 200.0, 220.0], [0, 0.0, 0.0, 30.0, 30.0]], device="cuda")
    pooled = rex.roi_extract(feats, [0.25, 0.125], rois)
    head = rex.BoxHead(16 * 49, classes=4, hidden=32).cuda()
    scores, deltas = head(pooled)
    want = pooled.double().flatten(1)
    for fc in (head.fc1, head.fc2):
        want = F.linear(want, fc.weight.double(), fc.bias.double()).clamp(min=0)
    near(scores.detach(), F.linear(want, head.score.weight.double(), head.score.bias.double()).detach(), 1e-5, "scores")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_relation_head_in_these_kernels(dtype):
    """The same head with its dense layers in torch's kernels and in these: results and gradients."""
    def make(fused):
        torch.manual_seed(3)
        return rex.RelationHead(64, heads=4, kv_heads=2, fused=fused).cuda().to(dtype)
    rng = np.random.default_rng(1)
    boxes = torch.from_numpy(draw_boxes(rng, (2, 50))).cuda()
    found = []
    for fused in (False, True):
        head, x = make(fused), randn(1, 2, 50, 64, dtype=dtype).requires_grad_()
        y = head(x, boxes, [50, 33])
        (y * randn(2, 2, 50, 64, dtype=dtype)).float().sum().backward()
        found.append((y.detach(), x.grad, {k: v.grad for k, v in head.named_parameters()}))
    tol = 1.6e-4 if dtype == torch.float32 else 20 * 2.0 ** -8
    near(found[1][0], found[0][0].double(), tol, "y")
    if dtype == torch.float32:
        near(found[1][1], found[0][1].double(), 5e-4, "grad x")
        for k, v in found[1][2].items():
            if not k.endswith("qkv.bias"):          # (a key's bias has gradient 0, but for rounding)
                near(v, found[0][2][k].double(), 5e-4, k)


def test_video_that_forgets_by_weight():
    """Frames of two streams through a memory that is soon full: what is kept has had the most attention,
    and the next frame attends to exactly what the memory says it holds."""
    torch.manual_seed(5)
    head = rex.RelationHead(64, heads=4, kv_heads=2).cuda()
    memory = head.memory(num_pages=8, streams=2, max_pages=3, evict="weight", decay=0.5)
    rng = np.random.default_rng(2)
    weights = torch.zeros(2, 96, dtype=torch.float64)
    for frame, counts in enumerate(([40, 17], [30, 40], [40, 40], [33, 1], [0, 40], [40, 0])):
        boxes = torch.from_numpy(draw_boxes(rng, (2, 40))).cuda()
        x = randn(20 + frame, 2, 40, 64)
        used = list(memory.used)
        before = [[t.clone() for t in layer] for layer in memory.layers]
        table = [list(p) for p in memory.table]
        with torch.no_grad():
            y = head(x, boxes, counts, memory)
        assert bool(y.isfinite().all())
        assert memory.used == [min(u, 96 - c) + c for u, c in zip(used, counts)]
        for s in range(2):
            room = min(used[s], 96 - counts[s])
            got = memory.weight[s].double().cpu()
            assert not got[room:].any() and bool((got[:room] >= 0).all())
            # shares of the softmax: a frame gives at most a row's whole weight, in each layer and head
            assert float(got.sum()) <= 0.5 * float(weights[s].sum()) + 2 * 4 * counts[s] + 1e-3
            weights[s] = got
            # every box that is there was there before, or is one of this frame's
            old = {tuple(b) for b in before[0][4][table[s]].reshape(-1, 4)[:used[s]].tolist()} if used[s] else set()
            new = {tuple(b) for b in boxes[s, :counts[s]].tolist()}
            held = memory.layers[0][4][memory.table[s]].reshape(-1, 4)[:memory.used[s]].tolist() if memory.used[s] else []
            held = [tuple(b) for b in held]
            assert len(set(held)) == memory.used[s] and set(held) <= old | new and new <= set(held)
            if memory.used[s]:                      # and its box is the same in both layers
                assert torch.equal(memory.layers[0][4][memory.table[s]].reshape(-1, 4)[:memory.used[s]],
                                   memory.layers[1][4][memory.table[s]].reshape(-1, 4)[:memory.used[s]])


def test_memories_agree_until_they_are_full():
    """Both ways of forgetting give the same results as long as there is room."""
    torch.manual_seed(6)
    head = rex.RelationHead(64, heads=4).cuda()
    rng = np.random.default_rng(3)
    memories = [head.memory(num_pages=12, streams=1, max_pages=6, evict=e) for e in ("oldest", "weight")]
    for frame in range(3):
        boxes, x = torch.from_numpy(draw_boxes(rng, (1, 40))).cuda(), randn(frame, 1, 40, 64)
        with torch.no_grad():
            a, b = (head(x, boxes, [40], m) for m in memories)
        assert torch.equal(a, b)
