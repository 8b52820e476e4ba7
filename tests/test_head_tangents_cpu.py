"""Forward-mode tangents are refused where there are none to give, not dropped (host code; the kernels'
part is played by plain ones)."""
import pytest
import torch
from torch.autograd import forward_ad as fw

from paper_1906_07155_amd import box_head, relation_head


@pytest.fixture(autouse=True)
def plain(monkeypatch):
    def linear(x, weight, bias=None, *, act="none", residual=None, save=False):
        y = x @ weight.t() + (0 if bias is None else bias) + (0 if residual is None else residual)
        return y.detach().clone(), None

    def logprob(logits, labels, *, scale=1.0, top=0):
        logp = torch.log_softmax(logits.detach(), 1)
        some = logp[:, :top].clone() if top else None
        return logp[:, 0].clone(), -(logp.exp() * logp).sum(1), torch.zeros(len(logits), 2), some, some

    def attention(q, k, v, **kw):
        return q.detach().clone(), torch.zeros(q.shape[0], q.shape[2], q.shape[1]), None

    def norm(x, branch=None, **kw):
        return x.detach().clone(), x.detach().clone(), torch.zeros(len(x), 2)
    monkeypatch.setattr(box_head.ops, "linear_act_fwd", linear)
    monkeypatch.setattr(box_head.ops, "class_logprob_fwd", logprob)
    monkeypatch.setattr(relation_head.relation, "box_attn_fwd", attention)
    monkeypatch.setattr(relation_head.relation, "gated_norm_fwd", norm)


LABELS = torch.zeros(3, dtype=torch.int64)
CALLS = {
    "linear_act": (lambda x, w, b, r: box_head.linear_act(x, w, b, act="gelu", residual=r), [(3, 4), (5, 4), (5,), (3, 5)]),
    "class_logprob": (lambda x: box_head.class_logprob(x, LABELS, top=2)[0], [(3, 4)]),
    "box_attention": (lambda q, k, v: relation_head.box_attention(q, k, v)[0], [(1, 3, 2, 8)] * 3),
    "gated_norm": (lambda x, y, g, w: relation_head.gated_norm(x, y, gate=g, post_weight=w)[0], [(3, 4), (3, 4), (1, 4), (4,)]),
}


@pytest.mark.parametrize("name", sorted(CALLS))
@pytest.mark.parametrize("requires_grad", [False, True])
@pytest.mark.parametrize("grad_mode", [False, True])
def test_a_tangent_is_refused(name, requires_grad, grad_mode):
    call, shapes = CALLS[name]
    for i in range(len(shapes)):
        with fw.dual_level(), torch.set_grad_enabled(grad_mode):
            given = [torch.ones(s, requires_grad=requires_grad) for s in shapes]
            call(*given)                                # a level alone changes nothing
            given[i] = fw.make_dual(given[i], torch.ones(shapes[i]))
            with pytest.raises(NotImplementedError, match="jvp"):
                call(*given)


def test_the_likeliest_classes_have_no_derivative():
    head = box_head.BoxHead(4, classes=3, hidden=4)
    with fw.dual_level():
        scores = fw.make_dual(torch.ones(3, 4), torch.ones(3, 4))
        assert all(fw.unpack_dual(t).tangent is None for t in head.best(scores, 2))


def test_a_memory_refuses_tangents(monkeypatch):
    """Also where they come with a layer's weights alone."""
    monkeypatch.setattr(relation_head.relation, "box_memory_attn_fwd",
                        lambda q, *a, **kw: (q.detach().clone(), torch.zeros(q.shape[0], q.shape[2], q.shape[1])))
    monkeypatch.setattr(relation_head.relation, "box_memory_append", lambda *a: None)
    head = relation_head.RelationHead(16, heads=2)
    memory = relation_head.BoxMemory(8, 1, 3, 2, 8, layers=2, device="cpu")
    x, boxes = torch.ones(1, 3, 16), torch.rand(1, 3, 4)
    with torch.no_grad():
        head(x, boxes, [3], memory)
        with fw.dual_level():
            weight = head.layers[0].qkv.weight
            del head.layers[0].qkv.weight
            head.layers[0].qkv.weight = fw.make_dual(weight.detach(), torch.ones_like(weight))
            with pytest.raises(RuntimeError, match="memory"):
                head(x, boxes, [3], memory)
    assert memory.used == [3]
