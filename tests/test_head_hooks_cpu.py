"""Hooks of the dense layers of BoxHead and of RelationHead(fused=True): they run, see what those of torch's
layers see, and what they do to weights, inputs and results counts (host code; the kernels' part is played by
plain ones)."""
import pytest
import torch
from torch import nn
from torch.nn import functional as F
from torch.nn.utils import parametrize, prune

from paper_1906_07155_amd import box_head, relation_head

CALLS = []


@pytest.fixture(autouse=True)
def plain(monkeypatch):
    CALLS.clear()

    def linear(x, weight, bias=None, *, act="none", residual=None, save=False):
        CALLS.append(act)
        y = F.linear(x, weight, bias).detach()
        return (y.relu() if act == "relu" else y), None

    def attention(q, k, v, **kw):
        return q.detach().clone(), torch.zeros(q.shape[0], q.shape[2], q.shape[1]), None

    def norm(x, branch=None, **kw):
        y = x.detach() if branch is None else (x + branch * kw["gate"]).detach()
        return y.clone(), y.clone(), None
    monkeypatch.setattr(box_head.ops, "linear_act_fwd", linear)
    monkeypatch.setattr(relation_head.relation, "box_attn_fwd", attention)
    monkeypatch.setattr(relation_head.relation, "gated_norm_fwd", norm)


def box(names):
    torch.manual_seed(0)
    head = box_head.BoxHead(6, classes=2, hidden=5)
    x = torch.randn(4, 6)

    def run():
        with torch.no_grad():
            return torch.cat(head(x), 1)

    def want(layers):
        with torch.no_grad():
            t = layers["fc2"](layers["fc1"](x).relu()).relu()
            return torch.cat([layers["score"](t), layers["delta"](t)], 1)
    return head, run, want


def relation(names):
    torch.manual_seed(1)
    head = relation_head.RelationHead(16, heads=2, layers=1, fused=True)
    torch.manual_seed(1)
    other = relation_head.RelationHead(16, heads=2, layers=1)       # torch's layers
    x, boxes = torch.randn(1, 3, 16), torch.rand(1, 3, 4)

    def run():
        with torch.no_grad():
            return head(x, boxes)

    def want(layers):
        for n in names:
            setattr(other.layers[0], n, layers[n])
        with torch.no_grad():
            return other(x, boxes)
    return head.layers[0], run, want


HEADS = {"box": (box, ("fc1", "fc2", "score", "delta")), "relation": (relation, ("qkv", "proj", "gate", "fc1", "fc2"))}
EACH = [(h, n) for h, (_, names) in HEADS.items() for n in names]


def plain_layers(owner, names):
    """torch's layers of the same weights."""
    out = {}
    for n in names:
        layer = getattr(owner, n)
        out[n] = nn.Linear(layer.in_features, layer.out_features)
        with torch.no_grad():
            out[n].weight.copy_(layer.weight)
            out[n].bias.copy_(layer.bias)
    return out


def near(a, b):
    return torch.allclose(a, b, rtol=1e-5, atol=1e-6)


@pytest.mark.parametrize("which,name", EACH)
def test_hooks_see_and_change_what_those_of_torch_do(which, name):
    make, names = HEADS[which]
    owner, run, want = make(names)
    layers = plain_layers(owner, names)
    assert near(run(), want(layers))
    seen = {"here": [], "there": []}
    for at, layer in (("here", getattr(owner, name)), ("there", layers[name])):
        layer.register_forward_pre_hook(lambda m, args, at=at: (seen[at].append(args[0].clone()), (args[0] + 0.25,))[1])
        layer.register_forward_hook(lambda m, args, y, at=at: (seen[at].append(y.clone()), y - 0.5)[1])
    a, b = run(), want(layers)
    assert near(a, b) and len(seen["here"]) == 2 and all(near(p, q) for p, q in zip(seen["here"], seen["there"]))


@pytest.mark.parametrize("which,name", EACH)
def test_weights_that_a_hook_makes(which, name):
    make, names = HEADS[which]
    owner, run, want = make(names)
    layer = getattr(owner, name)
    prune.l1_unstructured(layer, "weight", amount=0.5)
    with torch.no_grad():
        layer.weight_orig += 1.0                        # made anew from it before each call
    layers = plain_layers(owner, names)
    with torch.no_grad():
        layers[name].weight.copy_(layer.weight_orig * layer.weight_mask)
    assert near(run(), want(layers))
    prune.remove(layer, "weight")
    assert near(run(), want(layers))


def test_parametrized_weights():
    class Twice(nn.Module):
        def forward(self, w):
            return 2 * w
    owner, run, want = box(HEADS["box"][1])
    layers = plain_layers(owner, HEADS["box"][1])
    parametrize.register_parametrization(owner.fc1, "weight", Twice())
    with torch.no_grad():
        layers["fc1"].weight *= 2
    assert near(run(), want(layers))


@pytest.mark.parametrize("which", sorted(HEADS))
def test_without_hooks_an_activation_is_in_the_kernel(which):
    make, names = HEADS[which]
    owner, run, want = make(names)
    run()
    assert sorted(CALLS) == sorted(["relu"] * (2 if which == "box" else 1) + ["none"] * (2 if which == "box" else 4))


def test_a_backward_hook_sees_the_gradient_before_the_activation(monkeypatch):
    def backward(g, x, w, saved, *, bias, act, want_x, want_weight, want_bias):
        g = g * (saved > 0) if act == "relu" else g
        return g @ w, g.t() @ x, g.sum(0)

    def forward(x, weight, bias=None, *, act="none", residual=None, save=False):
        y = F.linear(x, weight, bias).detach()
        y = y.relu() if act == "relu" else y
        return y, (y if save and act == "relu" else None)
    monkeypatch.setattr(box_head.ops, "linear_act_fwd", forward)
    monkeypatch.setattr(box_head.ops, "linear_act_bwd", backward)
    torch.manual_seed(0)
    head = box_head.BoxHead(6, classes=2, hidden=5)
    x, seen = torch.randn(4, 6, requires_grad=True), []
    head.fc1.register_full_backward_hook(lambda m, gx, gy: seen.append(gy[0].clone()))
    sum(t.sum() for t in head(x)).backward()
    t = F.linear(x, head.fc1.weight, head.fc1.bias).detach().requires_grad_()
    y = F.linear(t.relu(), head.fc2.weight, head.fc2.bias).relu()
    sum(F.linear(y, layer.weight, layer.bias).sum() for layer in (head.score, head.delta)).backward()
    assert len(seen) == 1 and near(seen[0], t.grad) and bool((seen[0] == 0).any())


def test_another_layer_in_its_place():
    owner, run, want = box(HEADS["box"][1])
    owner.fc2 = nn.Sequential(nn.Linear(5, 7), nn.Linear(7, 5))
    layers = plain_layers(owner, ("fc1", "score", "delta"))
    layers["fc2"] = owner.fc2
    assert near(run(), want(layers))


def test_state_is_that_of_torchs_layers():
    head = box_head.BoxHead(6, classes=2, hidden=5)
    assert set(head.state_dict()) == {"%s.%s" % (n, p) for n in HEADS["box"][1] for p in ("weight", "bias")}
    assert all(isinstance(getattr(head, n), nn.Linear) for n in HEADS["box"][1])
    one, other = (relation_head.RelationHead(16, heads=2, layers=2, fused=f) for f in (False, True))
    assert list(one.state_dict()) == list(other.state_dict())
    other.load_state_dict(one.state_dict())
