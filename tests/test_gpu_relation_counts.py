"""The numbers of boxes that RelationHead is given: tensors, and no images at all."""
import numpy as np
import pytest

import paper_1906_07155_amd as rex
from gpu_helpers import log
from test_gpu_relation_attn import draw_boxes
from test_gpu_relation_head import make

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    rex.lib()


def test_counts_on_the_device_are_read_at_once(monkeypatch):
    log("counts device")
    rng = np.random.default_rng(1)
    head = make(1)
    boxes = torch.from_numpy(draw_boxes(rng, (3, 20))).cuda()
    x = torch.randn(3, 20, 64, device="cuda")
    counts = torch.tensor([20, 0, 7], dtype=torch.int32, device="cuda")
    with torch.no_grad():
        want = head(x, boxes, [20, 0, 7])

        def one_by_one(self):
            raise AssertionError("a tensor read element by element")
        monkeypatch.setattr(torch.Tensor, "__iter__", one_by_one)
        assert torch.equal(head(x, boxes, counts), want)
        with pytest.raises(ValueError, match="counts"):
            head(x, boxes, counts + 1)


@pytest.mark.parametrize("shape", [(0, 20), (2, 0), (0, 0)], ids=str)
def test_no_images_and_no_boxes(shape):
    """A batch that nothing is left of: empty results and gradients of 0."""
    log("counts empty %s" % (shape,))
    head = make(2, 2)
    x = torch.randn(*shape, 64, device="cuda", requires_grad=True)
    boxes = torch.rand(*shape, 4, device="cuda")
    for counts in (None, [0] * shape[0]):
        head.zero_grad()
        y = head(x, boxes, counts)
        assert y.shape == x.shape
        y.sum().backward()
        assert x.grad.shape == x.shape
        assert all(float(p.grad.abs().sum()) == 0.0 for p in head.parameters() if p.grad is not None)


def test_gates_of_no_rows():
    log("counts gates")
    x, gate = torch.zeros(0, 16, device="cuda"), torch.zeros(0, 16, device="cuda")
    y, u, stats = rex.gated_norm_fwd(x, x, gate=gate, save=True)
    assert y.shape == u.shape == (0, 16)
    grads = rex.gated_norm_bwd(y, u, x, x, stats, gate=gate, pre_weight=torch.ones(16, device="cuda"))
    assert grads[2].shape == (0, 16) and float(grads[5].abs().sum()) == 0.0
    with pytest.raises(ValueError, match="gate"):
        rex.gated_norm_fwd(torch.zeros(3, 16, device="cuda"), torch.zeros(3, 16, device="cuda"), gate=gate)
