"""The kernels' parameters keep their binary32 values and gradients when the head's type changes (host
code; nothing here runs on a GPU)."""
import pytest
import torch

from paper_1906_07155_amd.relation_head import RelationHead

OWN = ("bias", "post.0", "post.1", "pre.0", "pre.1")


def make():
    torch.manual_seed(1)
    head = RelationHead(64, 4, layers=2)
    with torch.no_grad():
        for layer in head.layers:
            layer.bias.normal_()
            layer.bias[0, 0, 0] = -1e30             # half has no such number
            for p in (*layer.post, *layer.pre):
                p.uniform_(0.5, 1.5)
    return head


def own(head):
    return {k: p for k, p in head.named_parameters() if k.split(".", 2)[2] in OWN}


@pytest.mark.parametrize("change", [lambda h: h.bfloat16(), lambda h: h.half(), lambda h: h.double(),
                                    lambda h: h.to(torch.bfloat16), lambda h: h.bfloat16().float().half(),
                                    lambda h: h.to("cpu"), lambda h: h.float()])
def test_values_are_kept_to_the_last_bit(change):
    head = make()
    before = {k: p.detach().clone() for k, p in own(head).items()}
    params = dict(own(head))
    assert len(before) == 10
    change(head)
    for k, p in own(head).items():
        assert p is params[k] and p.dtype == torch.float32 and p.requires_grad
        assert torch.equal(p.detach(), before[k]), k


def test_gradients_are_kept_and_an_optimizer_steps():
    head = make()
    optimizer = torch.optim.Adam(head.parameters(), lr=1e-3)
    for p in head.parameters():
        p.grad = torch.randn_like(p)
    grads = {k: p.grad.clone() for k, p in own(head).items()}
    head.bfloat16()
    assert head.layers[0].qkv.weight.dtype == torch.bfloat16
    for k, p in own(head).items():
        assert p.grad.dtype == torch.float32 and torch.equal(p.grad, grads[k])
    optimizer.step()
    assert all(bool(torch.isfinite(p).all()) for p in head.parameters())
