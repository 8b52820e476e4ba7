"""What the autograd functions keep for the backward is what torch knows about."""
import pytest

import paper_1906_07155_amd as rex
from gpu_helpers import log
from test_gpu_relation_attn import Case

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    rex.lib()


@pytest.mark.parametrize("name", ["q_boxes", "k_boxes", "q_len", "k_len", "k_mask"])
def test_inputs_written_before_the_backward_are_noticed(name):
    log("autograd %s" % name)
    c = Case("f32", 2, 20, 30, 4, 2, 16, 7, q_len=[20, 9], k_len=[30, 11], masked=0.2)
    q = c.q.clone().requires_grad_()
    args = c.args()
    out, _ = rex.box_attention(q, c.k, c.v, **args)
    out.backward(c.g)
    want = q.grad.clone()
    assert torch.equal(want, c.both()["grad_q"])
    out, _ = rex.box_attention(q, c.k, c.v, **args)
    args[name].copy_(torch.zeros_like(args[name]))          # the next batch's, say
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        out.backward(c.g)


def test_second_derivatives_are_refused():
    """The kernels have none; a gradient asked for with create_graph is no constant."""
    log("autograd twice")
    c = Case("f32", 1, 5, 6, 2, 2, 8, 3)
    q = c.q.clone().requires_grad_()
    out, _ = rex.box_attention(q, c.k, c.v, **c.args())
    first, = torch.autograd.grad((out * c.g).sum(), q, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        ((first * first).sum() + (q * q).sum()).backward()
    x = torch.randn(6, 16, device="cuda", requires_grad=True)
    for branch in (None, torch.randn(6, 16, device="cuda")):
        y, u = rex.gated_norm(x, branch)
        first, = torch.autograd.grad((u * u).sum(), x, create_graph=True)
        with pytest.raises(RuntimeError, match="once_differentiable"):
            ((first * first).sum() + (x * x).sum()).backward()


def test_nothing_is_kept_where_no_gradient_is_asked_for(monkeypatch):
    log("autograd inference")
    from paper_1906_07155_amd import relation
    c = Case("bf16", 1, 20, 90, 2, 2, 16, 3)
    x, w = torch.randn(30, 64, device="cuda"), torch.ones(64, device="cuda", requires_grad=True)
    want = rex.box_attention(c.q, c.k, c.v, **c.args()), rex.gated_norm(x, x, pre_weight=w), rex.gated_norm(x, pre_weight=w)
    kept = []
    for name in ("box_attn_fwd", "gated_norm_fwd"):
        def call(*args, name=name, real=getattr(relation, name), **kw):
            found = real(*args, **kw)
            kept.append(found[2])
            return found
        monkeypatch.setattr(relation, name, call)
    with torch.no_grad():
        got = rex.box_attention(c.q, c.k, c.v, **c.args()), rex.gated_norm(x, x, pre_weight=w), rex.gated_norm(x, pre_weight=w)
    assert kept == [None] * 3
    for a, b in zip(got, want):
        assert all(torch.equal(s, t.detach()) and not s.requires_grad for s, t in zip(a, b))
    y, _ = rex.gated_norm(x, second=True, pre_weight=w.detach())
    assert y is x and rex.gated_norm(x, x, second=False)[1] is None
