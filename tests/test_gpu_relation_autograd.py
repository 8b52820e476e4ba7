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
