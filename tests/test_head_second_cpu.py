"""What fails where a gradient is differentiated again names the operator (host code)."""
import pytest
import torch

from paper_1906_07155_amd import box_head, relation_head


@pytest.mark.parametrize("name", ["linear_act", "class_logprob", "box_attention", "gated_norm"])
def test_second_derivatives_name_their_operator(name, monkeypatch):
    monkeypatch.setattr(box_head.ops, "linear_act_fwd", lambda x, w, b, **kw: (x.detach() @ w.detach().t(), None))
    monkeypatch.setattr(box_head.ops, "linear_act_bwd", lambda g, x, w, *a, **kw: (g @ w, g.t() @ x, None))
    monkeypatch.setattr(box_head.ops, "class_logprob_fwd",
                        lambda x, *a, **kw: (x.sum(1), x.sum(1), x[:, :2].clone(), None, None))
    monkeypatch.setattr(box_head.ops, "class_logprob_bwd", lambda g, *a, **kw: g[:, None].expand(3, 4).clone())
    monkeypatch.setattr(relation_head.relation, "box_attn_fwd", lambda q, *a, **kw: (q.detach().clone(), q[..., 0].detach(), None))
    monkeypatch.setattr(relation_head.relation, "box_attn_bwd", lambda g, *a, **kw: (g.clone(), g.clone(), g.clone(), None))
    monkeypatch.setattr(relation_head.relation, "gated_norm_fwd", lambda x, *a, **kw: (x.clone(), x.clone(), x[:, :2].clone()))
    monkeypatch.setattr(relation_head.relation, "gated_norm_bwd", lambda gy, gu, x, *a, **kw: (gu.clone(),) + (None,) * 6)
    x = torch.ones(3, 4, requires_grad=True)
    y = {"linear_act": lambda: box_head.linear_act(x, torch.ones(5, 4)),
         "class_logprob": lambda: box_head.class_logprob(x, torch.zeros(3, dtype=torch.int64))[0],
         "box_attention": lambda: relation_head.box_attention(*(x.view(1, 3, 1, 4),) * 3)[0],
         "gated_norm": lambda: relation_head.gated_norm(x)[1]}[name]()
    g, = torch.autograd.grad(y.sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="^%s is once_differentiable" % name):
        g.sum().backward()
